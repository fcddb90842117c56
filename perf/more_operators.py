"""Operators around the paged 4-bit key / value cache, case by case: rotary positions with several axes (with the append that
stores the rotated keys), attention with a sliding window and first tokens that stay visible, attention of a tree of drafted
tokens, and keeping the accepted path of such a tree.

They stand where ``essa_apply_block`` leaves q, k and v of every candidate's tokens: q and k are rotated by their tokens'
positions, k and v are appended to the candidate's sequence, q attends over it.  Where a small model drafts several
continuations at once they form a tree; one pass computes them all, and the path that is accepted stays.

A page holds 64 tokens of one layer.  For each kv head it is one run of 72 * head_dim bytes:

* the codes of K, then those of V: [head_dim / 32][64 tokens][16 bytes], two codes per byte, low nibble = even channel;
* (scale, minimum) of K, then those of V: [head_dim / 64][64 tokens][2] fp16, one pair per group of 64 channels.

A value is ``code * scale + minimum``.  With ``own`` false `run` computes the operators from elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

PAGE = 64     # tokens per page
GROUP = 64    # channels that share a scale and a minimum
DEV = "cuda"


# ---------------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # One decode step of 256 candidates (3584 = 28 heads of 128, 512 = 4 kv heads): one axis, the position in the sequence.
        {"name": "rotary-step-256", "op": "store", "n": 256, "heads": 28, "kv_heads": 4, "dim": 128, "axes": 1, "adjacent": False, "interleaved": False,
         "ctx_lo": 0, "ctx_hi": 1023, "new_lo": 1, "new_hi": 1},
        # Prompts of text and images for 64 candidates (5120 = 40 heads, 1024 = 8 kv heads): time, height and width.
        {"name": "rotary-prompts-64", "op": "store", "n": 64, "heads": 40, "kv_heads": 8, "dim": 128, "axes": 3, "adjacent": False, "interleaved": False,
         "ctx_lo": 0, "ctx_hi": 0, "new_lo": 1, "new_hi": 1024},
        # The patches of a short video, queries alone (14 heads of 64, neighbouring channels are pairs, the axes take turns).
        {"name": "rotary-video", "op": "rotate", "T": 9001, "heads": 14, "dim": 64, "axes": 3, "adjacent": True, "interleaved": True},
        # One decode step of 256 candidates with ragged histories, some of them shorter than the window.
        {"name": "window-step-256", "op": "window", "n": 256, "heads": 28, "kv_heads": 4, "dim": 128, "ctx_lo": 0, "ctx_hi": 1023, "new_lo": 1, "new_hi": 1,
         "window": 512, "sinks": 4},
        # One decode step of 128 candidates (8192 = 64 heads, 1024 = 8 kv heads) far into long answers: most of the cache is out of sight.
        {"name": "window-step-128-long", "op": "window", "n": 128, "heads": 64, "kv_heads": 8, "dim": 128, "ctx_lo": 4093, "ctx_hi": 8191, "new_lo": 1, "new_hi": 1,
         "window": 1024, "sinks": 4},
        # Long prompts from an empty cache: the window moves with every row.
        {"name": "window-prompts-6", "op": "window", "n": 6, "heads": 40, "kv_heads": 8, "dim": 128, "ctx_lo": 0, "ctx_hi": 0, "new_lo": 777, "new_hi": 2801,
         "window": 1000, "sinks": 16},
        # A chunk of two long prompts whose first 16 thousand tokens are in the cache already.
        {"name": "window-chunk-2", "op": "window", "n": 2, "heads": 64, "kv_heads": 8, "dim": 128, "ctx_lo": 15001, "ctx_hi": 16385, "new_lo": 383, "new_hi": 509,
         "window": 4096, "sinks": 64},
        # A few drafted tokens of a small model (896 = 14 heads of 64) for four candidates: latency is all there is.
        {"name": "tree-4-small", "op": "tree", "n": 4, "heads": 14, "kv_heads": 2, "dim": 64, "ctx_lo": 16, "ctx_hi": 99, "new_lo": 3, "new_hi": 8},
        # Trees of 26 tokens and fewer for 64 candidates with ragged histories.
        {"name": "tree-64", "op": "tree", "n": 64, "heads": 28, "kv_heads": 4, "dim": 128, "ctx_lo": 100, "ctx_hi": 2047, "new_lo": 11, "new_hi": 26},
        # Large trees behind long histories.
        {"name": "tree-12-long", "op": "tree", "n": 12, "heads": 64, "kv_heads": 8, "dim": 128, "ctx_lo": 8001, "ctx_hi": 20011, "new_lo": 31, "new_hi": 61},
        # Accepting a few drafted tokens of four candidates.
        {"name": "keep-4-small", "op": "keep", "layers": 4, "n": 4, "kv_heads": 2, "dim": 64, "ctx_lo": 16, "ctx_hi": 99, "new_lo": 3, "new_hi": 8},
        # Accepting the paths of 128 candidates in a model of 28 layers.
        {"name": "keep-128", "op": "keep", "layers": 28, "n": 128, "kv_heads": 4, "dim": 128, "ctx_lo": 100, "ctx_hi": 901, "new_lo": 17, "new_hi": 61},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["store", "store", "rotate", "step", "step", "prompts", "chunk", "tree", "tree", "tree", "keep"])
    kv_heads, dim = rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 128])
    heads = kv_heads * rng.choice([1, 2, 4, 5, 7, 8])
    shape = {"heads": heads, "kv_heads": kv_heads, "dim": dim}
    turn = {"axes": rng.choice([1, 2, 3, 4]), "adjacent": rng.random() < 0.4, "interleaved": rng.random() < 0.4}
    if op == "store":
        n = _log(rng, 1, 256)
        new = _log(rng, 1, max(1, 32768 // n))
        return {"op": "store", "n": n, **shape, **turn, "ctx_lo": 0, "ctx_hi": _log(rng, 1, 2000), "new_lo": rng.randint(1, new), "new_hi": new}
    if op == "rotate":
        return {"op": "rotate", "T": _log(rng, 1, 32768), "heads": heads, "dim": dim, **turn}
    if op == "step":
        n = _log(rng, 1, 256)
        hi = _log(rng, 1, max(2, min(100000, 128 * 8192 // n)))
        return {"op": "window", "n": n, **shape, "ctx_lo": rng.randint(0, hi), "ctx_hi": hi, "new_lo": 1, "new_hi": 1,
                "window": _log(rng, 1, 4096), "sinks": rng.choice([0, 1, 4, 64, 130])}
    if op == "prompts":
        hi = _log(rng, 2, 2800)
        return {"op": "window", "n": _log(rng, 1, max(1, min(64, 16000 // hi))), **shape, "ctx_lo": 0, "ctx_hi": 0, "new_lo": rng.randint(1, hi), "new_hi": hi,
                "window": _log(rng, 1, 2000), "sinks": rng.choice([0, 1, 4, 64, 130])}
    if op == "chunk":
        ctx, new = _log(rng, 64, 16000), _log(rng, 2, 500)
        return {"op": "window", "n": rng.choice([1, 2]), **shape, "ctx_lo": ctx // 2, "ctx_hi": ctx, "new_lo": rng.randint(1, new), "new_hi": new,
                "window": _log(rng, 16, 8000), "sinks": rng.choice([0, 1, 4, 64, 130])}
    n, new = _log(rng, 1, 128), _log(rng, 2, 64)
    if op == "tree":
        return {"op": "tree", "n": n, **shape, "ctx_lo": 1, "ctx_hi": _log(rng, 2, max(3, min(20000, 200000 // n))), "new_lo": rng.randint(1, new), "new_hi": new}
    return {"op": "keep", "layers": rng.randint(1, 28), "n": n, "kv_heads": kv_heads, "dim": dim, "ctx_lo": 0, "ctx_hi": _log(rng, 2, 900),
            "new_lo": rng.randint(1, new), "new_hi": new}


def _spread(lo, hi, n):
    """n lengths spread evenly over lo .. hi (the seed only shuffles them, so that work() knows their sum)."""
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _mixed(case):
    """New tokens and history of every sequence.  (Which history meets which number of new tokens is fixed.)"""
    n = case["n"]
    rng = np.random.default_rng(n)
    return np.array(_spread(case["new_lo"], case["new_hi"], n))[rng.permutation(n)], np.array(_spread(case["ctx_lo"], case["ctx_hi"], n))[rng.permutation(n)]


def _pages_of(tokens):
    return -(-tokens // PAGE)


def _page_bytes(case):
    return case["kv_heads"] * 72 * case["dim"]


def _accepted(case, new):
    """Length of the accepted path of each tree (what the seed draws lies around it)."""
    return np.minimum(new, 1 + np.arange(case["n"]) % 6)


def work(case):
    op, dim = case["op"], case["dim"]
    if op == "rotate":
        return {"bytes": case["T"] * (4 * case["heads"] * dim + 4 * case["axes"]), "flops": 3 * case["T"] * case["heads"] * dim}
    new, ctx = _mixed(case)
    token, T = _page_bytes(case) // PAGE, int(new.sum())
    if op == "store":  # q in and out; k and v in, cache rows out; cache rows in, k and v out
        return {"bytes": T * (4 * case["heads"] * dim + 8 * case["kv_heads"] * dim + 2 * token), "flops": T * dim * (3 * case["heads"] + 11 * case["kv_heads"])}
    if op == "keep":  # the accepted tokens of every layer move to the front
        return {"bytes": 2 * int(_accepted(case, new).sum()) * token * case["layers"] + 12 * int(sum(_pages_of(int(c)) for c in ctx + new)), "flops": 0}
    if op == "tree":  # every cached token once, q and out once; the products of a draft with the history and (about half of) its tree
        seen = int((new * ctx + new * (new + 1) // 2).sum())
        return {"bytes": T * case["heads"] * dim * 4 + int((new + ctx).sum()) * token, "flops": 4 * seen * case["heads"] * dim}
    window, sinks = case["window"], case["sinks"]
    seen, read = 0, 0
    for n, c in zip(new.tolist(), ctx.tolist()):
        pos = np.arange(c, c + n)
        seen += int((np.minimum(pos + 1, window) + np.minimum(sinks, np.maximum(pos + 1 - window, 0))).sum())
        start = max(0, c - window + 1)
        read += c + n - start + min(sinks, start)
    return {"bytes": T * case["heads"] * dim * 4 + read * token, "flops": 4 * seen * case["heads"] * dim}


# --------------------------------------------------------------------------------------------------------- the inputs
def _ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


def _cached(case, layers, pages, g):
    """A pool with the values that N(0, 1) keys and values leave: bell-shaped codes, a step of about a third, a minimum near -2.4."""
    raw = torch.empty((layers, pages, case["kv_heads"], 72 * case["dim"]), dtype=torch.uint8, device=DEV)
    codes, dim = 64 * case["dim"], case["dim"]
    a = torch.randint(0, 256, raw[..., :codes].shape, dtype=torch.uint8, device=DEV, generator=g)
    b = torch.randint(0, 256, raw[..., :codes].shape, dtype=torch.uint8, device=DEV, generator=g)
    raw[..., :codes] = (((a & 15) + (b & 15)) >> 1) | ((((a >> 4) + (b >> 4)) >> 1) << 4)
    meta = torch.rand((layers, pages, case["kv_heads"], 2 * PAGE * dim // GROUP, 2), device=DEV, generator=g)
    meta[..., 0] = 0.28 + 0.08 * meta[..., 0]
    meta[..., 1] = -2.1 - 0.6 * meta[..., 1]
    raw[..., codes:] = meta.half().flatten(-2).view(torch.uint8)
    return raw.view(layers, pages, -1)


def _table(lengths, seqs, max_pages, order):
    table, at = np.full((seqs, max_pages), -1, np.int32), 0
    for s, n in enumerate(lengths):
        k = _pages_of(n)
        table[s, :k] = order[at:at + k]
        at += k
    return table


def _turns(case):
    """Frequencies (radians per position) and axes of the pairs of channels: sections for the axes, one after another or in turns."""
    half, axes = case["dim"] // 2, case["axes"]
    sections = [half] if axes == 1 else [half - (axes - 1) * (3 * half // (4 * axes))] + [3 * half // (4 * axes)] * (axes - 1)
    axis, left = [], list(sections)
    while len(axis) < half:
        for a in range(axes):
            take = min(1, left[a]) if case["interleaved"] else left[a]
            axis += [a] * take
            left[a] -= take
    return 1000000.0 ** (-np.arange(half) / half), np.array(axis), sections


def _grid(tokens, axes, start, rng):
    """Positions [axes, tokens] of text with an image in it: text moves all axes, an image's rows and columns count from where it begins."""
    at = np.tile(np.arange(start, start + tokens), (axes, 1))
    side = int(math.isqrt(tokens // 2))
    if axes > 1 and side > 1:
        first = int(rng.integers(0, tokens - side * side + 1))
        rows, cols = np.divmod(np.arange(side * side), side)
        at[:, first:first + side * side] = start + first
        at[1, first:first + side * side] += rows
        at[-1, first:first + side * side] += cols
        at[:, first + side * side:] = start + first + side + np.arange(tokens - first - side * side)
    return at


def _tree(n, rng):
    """Parents of n drafted tokens (-1: the last token before them): mostly short branches off a main line."""
    parents = np.full(n, -1, np.int32)
    for j in range(1, n):
        parents[j] = j - 1 if rng.random() < 0.4 else int(rng.integers(-1, j))
    return parents


def _path(parents, length, rng):
    """A chain of at most `length` tokens from a child of the history on."""
    path, at = [], -1
    while len(path) < length:
        below = np.flatnonzero(parents == at)
        if not len(below):
            break
        at = int(rng.choice(below))
        path.append(at)
    return path


def prepare(case, seed):
    rng, g = np.random.default_rng([seed, 1]), torch.Generator(device=DEV).manual_seed(int(seed))
    op, dim = case["op"], case["dim"]
    s = {"case": dict(case), "op": op, "dim": dim, "start": {}}
    if op in ("store", "rotate"):
        freq, axis, sections = _turns(case)
        s |= {"freq": torch.tensor(freq, dtype=torch.float64, device=DEV), "axis": _ints(axis), "sections": sections}
    if op == "rotate":
        T = case["T"]
        s |= {"T": T, "positions": _ints(_grid(T, case["axes"], int(rng.integers(0, 100000)), rng)),
              "q": torch.randn((T, case["heads"], dim), device=DEV, generator=g).bfloat16()}
        return s
    n, kvh = case["n"], case["kv_heads"]
    new, ctx = _mixed(case)
    mix = rng.permutation(n)
    new, ctx = new[mix], ctx[mix]
    total, T = new + ctx, int(new.sum())
    pool = int(sum(_pages_of(int(t)) for t in total)) + 3
    table = _table(total.tolist(), n, _pages_of(int(total.max())), rng.permutation(pool))
    refs = np.zeros(pool, np.int32)
    refs[table[table >= 0]] = 1
    s |= {"n": n, "T": T, "kv_heads": kvh, "max_new": int(new.max()), "lengths": _ints(total), "table": _ints(table), "refs": _ints(refs), "new": _ints(new),
          "tok_offsets": _ints(np.concatenate([[0], np.cumsum(new)])), "slots": _ints(np.arange(n)), "pages": _cached(case, case.get("layers", 1), pool, g)}
    if op in ("store", "window", "tree"):
        s["q"] = torch.randn((T, case["heads"], dim), device=DEV, generator=g).bfloat16()
    if op == "store":
        s["k"] = torch.randn((T, kvh, dim), device=DEV, generator=g).bfloat16()
        s["v"] = torch.randn((T, kvh, dim), device=DEV, generator=g).bfloat16()
        s["positions"] = None if case["axes"] == 1 else _ints(np.concatenate([_grid(int(a), case["axes"], int(c), rng) for a, c in zip(new, ctx)], 1))
    if op in ("tree", "keep"):
        trees = [_tree(int(a), rng) for a in new]
        s["parents"] = _ints(np.concatenate(trees))
    if op == "keep":
        want = _accepted(case, _mixed(case)[0])[mix]
        paths = [_path(p, int(w), rng) for p, w in zip(trees, want)]
        picks = np.zeros((n, int(new.max())), np.int32)
        for i, p in enumerate(paths):
            picks[i, :len(p)] = p
        s |= {"picks": _ints(picks), "counts": _ints([len(p) for p in paths])}
        # A pass begins from the same page table: these are what it is set back to.
        s["start"] = {k: s[k].clone() for k in ("lengths", "table", "refs")}
    return s


# ------------------------------------------------------------------------------------------------- the plain operators
def _unpack(blocks, dim):
    """Pages [..., kv_heads * 72 * dim] as fp32 values: K and V, each [..., kv_heads, 64, dim]."""
    b = blocks.reshape(*blocks.shape[:-1], -1, 72 * dim)
    lead = b.shape[:-1]
    c = b[..., :64 * dim].reshape(*lead, 2, dim // 32, PAGE, 16)
    c = torch.stack((c & 15, c >> 4), -1).reshape(*lead, 2, dim // 32, PAGE, 32).transpose(-3, -2)   # [2, 64, dim/32, 32]
    meta = b[..., 64 * dim:].contiguous().view(torch.float16).float().reshape(*lead, 2, dim // GROUP, PAGE, 1, 2).transpose(-4, -3)  # [2, 64, groups, 1, 2]
    x = c.reshape(*lead, 2, PAGE, dim // GROUP, GROUP).float() * meta[..., 0] + meta[..., 1]
    x = x.reshape(*lead, 2, PAGE, dim)
    return x[..., 0, :, :], x[..., 1, :, :]


def _pack(x):
    """x [T, kv_heads, dim] bf16: codes [T, kv_heads, dim] and (scale, minimum) [T, kv_heads, dim / 64] fp16."""
    g = x.float().unflatten(-1, (-1, GROUP))
    low = g.amin(-1).half()
    scale = ((g.amax(-1) - low.float()) / torch.full((), 15.0, device=DEV)).half()
    codes = torch.round((g - low.float()[..., None]) / scale.float()[..., None]).nan_to_num(0.0).clamp(0, 15).to(torch.uint8)
    return codes.flatten(-2), scale, low


def _gathered(pages, table, dim):
    """All tokens of the sequences of `table` in order: K and V [seqs, kv_heads, max_pages * 64, dim] fp32."""
    k, v = _unpack(pages[table.clamp(min=0).long()], dim)
    return k.transpose(1, 2).flatten(2, 3), v.transpose(1, 2).flatten(2, 3)


def _own_rows(s):
    """Of every row: its entry, and its position in the sequence."""
    t = torch.arange(s["T"], device=DEV)
    i = torch.searchsorted(s["tok_offsets"].long(), t, right=True) - 1
    return i, s["lengths"][i].long() - s["new"][i] + t - s["tok_offsets"][i]


def _rotated(s, x, positions):
    """x [T, heads, dim] turned by positions [axes, T]; angles in 64 bits."""
    angle = positions.double()[s["axis"].long()].T * s["freq"]         # [T, dim / 2]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    y = x.float()
    a, b = (y[..., 0::2], y[..., 1::2]) if s["case"]["adjacent"] else y.chunk(2, -1)
    y = (a * cos - b * sin, b * cos + a * sin)
    return (torch.stack(y, -1).flatten(-2) if s["case"]["adjacent"] else torch.cat(y, -1)).to(x.dtype)


def _store(s):
    i, pos = _own_rows(s)
    at = pos[None] if s["positions"] is None else s["positions"]
    page, off = s["table"][i, pos // PAGE].long(), pos % PAGE
    dim, kvh = s["dim"], s["kv_heads"]
    pool = s["pages"][0].view(-1, kvh, 72 * dim)
    codes = pool[..., :64 * dim].unflatten(-1, (2, dim // 32, PAGE, 16))
    meta = pool[..., 64 * dim:].view(torch.float16).unflatten(-1, (2, dim // GROUP, PAGE, 2))
    packed = [_pack(_rotated(s, s["k"], at)), _pack(s["v"])]
    c = torch.stack([p[0] for p in packed], 2)                         # [T, kv_heads, 2, dim]
    c = (c[..., 0::2] | (c[..., 1::2] << 4)).unflatten(-1, (dim // 32, 16))
    codes[page, :, :, :, off] = c
    meta[page, :, :, :, off] = torch.stack([torch.stack(p[1:], -1) for p in packed], 2)
    c, m = codes[page, :, :, :, off], meta[page, :, :, :, off].float()  # read back: the new tokens' values
    x = torch.stack((c & 15, c >> 4), -1).reshape(*c.shape[:3], dim // GROUP, GROUP) * m[..., :1] + m[..., 1:]
    k, v = x.flatten(-2).to(s["k"].dtype).unbind(2)
    return {"q": _rotated(s, s["q"], at), "k": k, "v": v}


def _attend(s, seen):
    """softmax(q k / sqrt(dim)) v; seen [n, L, keys]: what the j-th new token of a sequence sees."""
    q, n, L, dim, kvh = s["q"], s["n"], s["max_new"], s["dim"], s["kv_heads"]
    k, v = _gathered(s["pages"][0], s["table"], dim)
    j = torch.arange(L, device=DEV)
    row = s["tok_offsets"][:-1, None].long() + j                       # [n, L] rows of q
    real = j < s["new"][:, None]
    x = q[row.clamp(max=s["T"] - 1)].float()                           # [n, L, heads, dim]
    x = x.unflatten(2, (kvh, -1)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [n, kv_heads, L * group, dim]
    score = (x @ k.transpose(-1, -2)) * (1.0 / math.sqrt(dim))
    score = score.unflatten(2, (L, -1)).masked_fill_(~seen[:, None, :, None], -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    o = (p.flatten(2, 3) @ v).unflatten(2, (L, -1)) / p.sum(-1, keepdim=True)
    return o.permute(0, 2, 1, 3, 4).flatten(2, 3)[real].to(q.dtype)    # [T, heads, dim]


def _window(s):
    j, key = torch.arange(s["max_new"], device=DEV), torch.arange(s["table"].shape[1] * PAGE, device=DEV)
    pos = (s["lengths"] - s["new"])[:, None, None] + j[:, None]
    return _attend(s, (key <= pos) & ((key > pos - s["case"]["window"]) | (key < s["case"]["sinks"])))


def _ancestors(s):
    """[n, L, L]: whether a drafted token of a sequence has another one above it, or is it."""
    L = s["max_new"]
    j = torch.arange(L, device=DEV)
    row = s["tok_offsets"][:-1, None].long() + j
    real = j < s["new"][:, None]
    parent = torch.where(real, s["parents"][row.clamp(max=s["T"] - 1)].long(), -1)
    up = (parent[..., None] == j).double() + torch.eye(L, dtype=torch.float64, device=DEV)
    return (torch.matrix_power(up, L) > 0) & real[..., None] & real[:, None]


def _drafts(s):
    above = _ancestors(s)
    base = (s["lengths"] - s["new"]).long()
    key = torch.arange(s["table"].shape[1] * PAGE, device=DEV)
    at = (key - base[:, None])                                         # [n, keys]: which draft a key is
    drafted = torch.gather(above, 2, at.clamp(0, s["max_new"] - 1)[:, None].expand(-1, s["max_new"], -1)) & (at < s["new"][:, None])[:, None]
    seen = torch.where((at < 0)[:, None], True, drafted)
    i, _ = _own_rows(s)
    depth = above.sum(-1)[i, torch.arange(s["T"], device=DEV) - s["tok_offsets"][i]] - 1
    return {"out": _attend(s, seen), "positions": (base[i] + depth).int()}


def _keep(s):
    n, dim, kvh, width = s["n"], s["dim"], s["kv_heads"], s["picks"].shape[1]
    base = (s["lengths"] - s["new"]).long()
    m = torch.arange(width, device=DEV)
    i, m = (m < s["counts"][:, None]).nonzero().unbind(1)
    old, to = base[i] + s["picks"][i, m], base[i] + m
    pool = s["pages"].view(s["pages"].shape[0], -1, kvh, 72 * dim)
    codes = pool[..., :64 * dim].unflatten(-1, (2, dim // 32, PAGE, 16))
    meta = pool[..., 64 * dim:].view(torch.float16).unflatten(-1, (2, dim // GROUP, PAGE, 2))
    page_from, page_to = s["table"][i, old // PAGE].long(), s["table"][i, to // PAGE].long()
    for x in (codes, meta):
        x[:, page_to, :, :, :, to % PAGE] = x[:, page_from, :, :, :, old % PAGE]
    length = base + s["counts"]
    col = torch.arange(s["table"].shape[1], device=DEV)
    gone = (col >= ((length + PAGE - 1) // PAGE)[:, None]) & (s["table"] >= 0)
    s["refs"][s["table"][gone].long()] -= 1
    s["table"][gone] = -1
    s["lengths"].copy_(length)


# --------------------------------------------------------------------------------------------------------------- a pass
_ctx = None


def _context():
    global _ctx
    if _ctx is None:
        from paper_2507_04453_b200 import binding
        _ctx = binding.Context(0)
    return _ctx


def _rotary(s):
    """The library's table of turns, made once as a program would."""
    if "rotary" not in s:
        from paper_2507_04453_b200 import binding
        c = s["case"]
        s["rotary"] = binding.Rotary(c["dim"], base=1000000.0, sections=s["sections"], interleaved=c["interleaved"], adjacent=c["adjacent"])
    return s["rotary"]


def _cache(s):
    """The library's view of the state's buffers, made once as a program would."""
    if "cache" not in s:
        s["cache"] = _context().kv_cache(s["pages"].shape[0], s["pages"].shape[1], s["kv_heads"], s["dim"], s["table"].shape[0], s["table"].shape[1],
                                         pages=s["pages"], table=s["table"], lengths=s["lengths"], refs=s["refs"])
    return s["cache"]


def run(state):
    s = state
    for k, v in s["start"].items():
        s[k].copy_(v)
    if s["op"] == "rotate":
        return _context().rotary(_rotary(s), s["q"], s["positions"]) if own else _rotated(s, s["q"], s["positions"])
    if s["op"] == "store":
        if own:
            c = _cache(s)
            q = c.append_rotary(0, _rotary(s), s["q"], s["k"], s["v"], s["positions"], s["tok_offsets"], slots=s["slots"])
            k, v = c.read(0, s["tok_offsets"], s["T"], slots=s["slots"])
            return {"q": q, "k": k, "v": v}
        return _store(s)
    if s["op"] == "window":
        if own:
            return _cache(s).attend(0, s["q"], s["tok_offsets"], slots=s["slots"], max_new=s["max_new"], window=s["case"]["window"], sinks=s["case"]["sinks"])
        return _window(s)
    if s["op"] == "tree":
        if own:
            c = _cache(s)
            tree, positions = c.tree(s["parents"], s["tok_offsets"], s["max_new"], slots=s["slots"])
            return {"out": c.attend(0, s["q"], s["tok_offsets"], slots=s["slots"], max_new=s["max_new"], tree=tree), "positions": positions}
        return _drafts(s)
    if own:
        _cache(s).keep(s["counts"], s["tok_offsets"], s["picks"], slots=s["slots"])
    else:
        _keep(s)
    # tokens are moved as they are: their bytes are the result
    return {"pages": s["pages"], "lengths": s["lengths"], "table": s["table"], "refs": s["refs"]}


# ------------------------------------------------------------------------------------------------------------- in 64 bits
def _exact_values(blocks, dim):
    """Pages [n, kv_heads, 72 * dim] -> (K, V) [kv_heads, n * 64, dim] float64, channel by channel from the layout's description."""
    n, kvh, half = blocks.shape[0], blocks.shape[1], 32 * dim
    out = []
    for part in range(2):
        code = blocks[..., part * half:(part + 1) * half].reshape(n, kvh, dim // 32, PAGE, 16)
        meta = blocks[..., 2 * half + part * 4 * dim:2 * half + (part + 1) * 4 * dim].contiguous().view(torch.float16).double()
        meta = meta.reshape(n, kvh, dim // GROUP, PAGE, 2)
        x = torch.empty((n, kvh, PAGE, dim), dtype=torch.float64, device=DEV)
        for c in range(dim):
            x[..., c] = ((code[:, :, c // 32, :, (c % 32) // 2] >> (4 * (c % 2))) & 15) * meta[:, :, c // GROUP, :, 0] + meta[:, :, c // GROUP, :, 1]
        out.append(x.transpose(0, 1).reshape(kvh, n * PAGE, dim))
    return out


def _exact_seen(case, parents, length, new):
    """[new, length] on the host: what each new token sees."""
    base = length - new
    seen = np.zeros((new, length), bool)
    for j in range(new):
        if case["op"] == "tree":
            seen[j, :base] = True
            at = j
            while at >= 0:
                seen[j, base + at] = True
                at = int(parents[at])
        else:
            pos = base + j
            seen[j, max(0, pos - case["window"] + 1):pos + 1] = True
            seen[j, :min(case["sinks"], pos + 1)] = True
    return torch.from_numpy(seen).to(DEV)


def _exact_attend(case, s):
    dim, kvh, heads = case["dim"], case["kv_heads"], case["heads"]
    group = heads // kvh
    out = torch.empty((s["T"], heads, dim), dtype=torch.float64, device=DEV)
    offs, lens, table = s["tok_offsets"].tolist(), s["lengths"].tolist(), s["table"].tolist()
    parents = s["parents"].tolist() if case["op"] == "tree" else None
    for i in range(case["n"]):
        ids = [p for p in table[i] if p >= 0]
        k, v = _exact_values(s["pages"][0][ids].reshape(len(ids), kvh, 72 * dim), dim)
        lo, hi = offs[i], offs[i + 1]
        seen = _exact_seen(case, parents and parents[lo:hi], lens[i], hi - lo)
        for h in range(heads):
            w = s["q"][lo:hi, h].double() @ k[h // group, :lens[i]].T / math.sqrt(dim)
            out[lo:hi, h] = torch.softmax(w.masked_fill(~seen, -math.inf), -1) @ v[h // group, :lens[i]]
    return out


def _exact_rotated(case, s, x, positions):
    """Channel pair by channel pair, as complex numbers of 64-bit parts."""
    freq, axis, _ = _turns(case)
    y, half = x.double(), case["dim"] // 2
    out = torch.empty_like(y)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if case["adjacent"] else (i, i + half)
        turn = torch.polar(torch.ones(x.shape[0], dtype=torch.float64, device=DEV), positions[int(axis[i])].double() * float(freq[i]))
        z = torch.complex(y[..., a], y[..., b]) * turn[:, None]
        out[..., a], out[..., b] = z.real, z.imag
    return out


def _exact_stored(x):
    """What is read back of x (bf16) after 4-bit storage, in 64 bits (the scale and the minimum are stored as fp16)."""
    g = x.double().cpu().numpy().reshape(*x.shape[:-1], -1, GROUP)
    low = g.min(-1).astype(np.float16).astype(np.float64)
    scale = ((g.max(-1) - low) / 15).astype(np.float16).astype(np.float64)
    code = np.divide(g - low[..., None], scale[..., None], out=np.zeros_like(g), where=scale[..., None] > 0)
    return torch.from_numpy((np.clip(np.rint(code), 0, 15) * scale[..., None] + low[..., None]).reshape(x.shape))


def exact(case, seed):
    if case["op"] == "keep":
        return None  # whole numbers and bytes
    s = prepare(case, seed)
    if case["op"] == "rotate":
        return _exact_rotated(case, s, s["q"], s["positions"])
    if case["op"] == "store":
        at = s["positions"]
        if at is None:
            at = torch.cat([torch.arange(n - a, n, device=DEV) for n, a in zip(s["lengths"].tolist(), s["new"].tolist())])[None]
        # keys are stored from what the rotation rounds them to, bf16
        k = _exact_rotated(case, s, s["k"], at).bfloat16()
        return {"q": _exact_rotated(case, s, s["q"], at), "k": _exact_stored(k), "v": _exact_stored(s["v"])}
    out = _exact_attend(case, s)
    return {"out": out, "positions": None} if case["op"] == "tree" else out
