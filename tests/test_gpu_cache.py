"""GPU tests of the paged 4-bit key / value cache: storing, reading, attention and page management against the fp64 / integer
model (oracle/cache_oracle.py), the refusals that only the device can see, graphs, streams, and the use beside the projections."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from oracle import essa_oracle as orc
from paper_2507_04453_b200 import binding, workloads as wl
from tests.cache_utils import Pair, attend_bound, bf16
from tests.parity_utils import Case, to_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("CUDA device required for -m gpu tests")
    return torch


@pytest.fixture(scope="module")
def ctx(torch):
    c = binding.Context(0)
    yield c
    assert c.get_status() == 0
    c.close()


# ------------------------------------------------------------------------------------------------ pages
def test_grow_free_fork_compact_follow_the_model(torch, ctx):
    """A few hundred random page operations, state compared after each; contents after the copying ones."""
    rng = np.random.default_rng(5)
    p = Pair(torch, ctx, 2, 40, 1, 64, 12, 7)
    layers, pages, heads, d = p.cpu.shape
    stamp = rng.integers(0, 16, p.cpu.codes.shape).astype(np.uint8)  # every page recognisable
    p.cpu.codes[:] = stamp
    p.cpu.scale[:], p.cpu.low[:] = 1, 0
    p.push()
    refused = 0
    for step in range(200):
        op = rng.choice(["grow", "grow", "grow", "free", "fork", "fork", "compact"])
        try:
            if op == "grow":
                n = int(rng.integers(1, 8))
                slots, counts = rng.permutation(12)[:n], rng.integers(0, 130, n)
                p.gpu.grow(p.ints(slots), p.ints(counts))
                p.cpu.grow(slots, counts)
            elif op == "free":
                slots = rng.permutation(12)[:int(rng.integers(1, 5))]
                p.gpu.free(p.ints(slots))
                p.cpu.free(slots)
            elif op == "fork":
                n = int(rng.integers(1, 6))
                mix = rng.permutation(12)
                dst, src = mix[:n], rng.choice(mix[n:], n)
                lens = None if rng.random() < 0.5 else [int(rng.integers(0, p.cpu.lengths[s] + 1)) for s in src]
                p.gpu.fork(p.ints(src), p.ints(dst), p.ints(lens))
                p.cpu.fork(src, dst, lens)
            else:
                used = torch.zeros(1, dtype=torch.int32, device="cuda")
                p.gpu.compact(used)
                assert int(used) == p.cpu.compact()
            assert ctx.get_status() == 0
        except co.Refused:
            refused += 1
            assert ctx.get_status() == binding.ESSA_ERR_CACHE
        p.assert_same(pages=op in ("fork", "compact"))
    assert 5 < refused < 150  # both kinds have been met


@pytest.mark.parametrize("what", ["grow-slot-twice", "grow-slot-outside", "grow-negative", "grow-too-long", "grow-no-pages", "free-twice", "free-outside",
                                  "fork-dst-twice", "fork-dst-is-src", "fork-too-long", "fork-src-outside", "fork-no-pages", "fork-bad-page"])
def test_page_operations_that_are_refused_change_nothing(torch, ctx, what):
    # five pages in use, a sixth free; without the sixth, a fork that frees one page and wants two finds too few
    p = Pair(torch, ctx, 1, 5 if what == "fork-no-pages" else 6, 1, 64, 5, 3)
    p.place([70, 0, 64, 10, 1], np.random.default_rng(1))
    if what == "fork-bad-page":
        p.cpu.table[0, 0] = 6
        p.push()
    call = {"grow-slot-twice": lambda g, i: g.grow(i([1, 1]), i([1, 1])), "grow-slot-outside": lambda g, i: g.grow(i([0, 5]), i([1, 1])),
            "grow-negative": lambda g, i: g.grow(i([0, 1]), i([1, -1])), "grow-too-long": lambda g, i: g.grow(i([0]), i([200])),
            "grow-no-pages": lambda g, i: g.grow(i([1, 3]), i([100, 1])), "free-twice": lambda g, i: g.free(i([0, 2, 0])),
            "free-outside": lambda g, i: g.free(i([0, -1])), "fork-dst-twice": lambda g, i: g.fork(i([0, 0]), i([1, 1])),
            "fork-dst-is-src": lambda g, i: g.fork(i([0, 1]), i([1, 3])), "fork-too-long": lambda g, i: g.fork(i([0]), i([1]), i([71])),
            "fork-src-outside": lambda g, i: g.fork(i([5]), i([1])), "fork-no-pages": lambda g, i: g.fork(i([0, 3]), i([1, 4])),
            "fork-bad-page": lambda g, i: g.fork(i([0]), i([1]))}[what]
    call(p.gpu, p.ints)
    assert ctx.get_status() == binding.ESSA_ERR_CACHE
    p.assert_same()


def test_pool_of_many_pages_and_sequences(torch, ctx):
    """More sequences than a thread block has threads, more pages than one round of its scans, one table row of many pages."""
    rng = np.random.default_rng(8)
    p = Pair(torch, ctx, 1, 9000, 1, 64, 1500, 40)
    counts = rng.integers(0, 300, 1500)
    p.gpu.grow(None, p.ints(counts))
    p.cpu.grow(range(1500), counts)
    gone = rng.permutation(1500)[:700]
    p.gpu.free(p.ints(gone))
    p.cpu.free(gone)
    rest = np.setdiff1d(np.arange(1500), gone)
    src = rng.choice(rest, 600)
    p.gpu.fork(p.ints(src), p.ints(gone[:600]))
    p.cpu.fork(src, gone[:600])
    p.gpu.compact()
    p.cpu.compact()
    assert ctx.get_status() == 0
    p.assert_same()


def test_long_table_with_offsets_beyond_32_bits(torch, ctx):
    """A pool of more than 2^32 bytes: the last pages are written, forked, read and attended to at their own addresses."""
    kv_heads, d = 8, 128
    page_bytes = 72 * kv_heads * d
    pages = (1 << 32) // page_bytes + 40
    g = ctx.kv_cache(1, pages, kv_heads, d, 3, 4)
    rng = np.random.default_rng(3)
    ints = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    g.refs[:pages - 6] = 1  # (all but the last six pages taken)
    g.grow(ints([0]), ints([150]))
    assert g.table[0].tolist() == [pages - 6, pages - 5, pages - 4, -1]
    k, v = (to_dev(torch, bf16(rng, (150, kv_heads, d)), torch.bfloat16) for _ in range(2))
    off = ints([0, 150])
    g.append(0, k, v, off, slots=ints([0]))
    g.fork(ints([0]), ints([2]))
    rk, rv = g.read(0, off, 150, slots=ints([2]))
    kk, vv = (x.float().cpu().numpy() for x in (k, v))
    for got, x in ((rk, kk), (rv, vv)):
        want = co.dequantize(*co.quantize(x))
        np.testing.assert_array_equal(got.float().cpu().numpy(), wl.round_to_bf16(want.astype(np.float32)))
    q = to_dev(torch, bf16(rng, (1, 16, d)), torch.bfloat16)
    out = g.attend(0, q, slots=ints([2]))
    vals = [np.moveaxis(co.dequantize(*co.quantize(x)), 0, 1) for x in (kk, vv)]
    want, w = co.attend(q.float().cpu().numpy(), vals[0], vals[1], 150, d ** -0.5)
    assert ctx.get_status() == 0
    assert np.max(np.abs(out.float().cpu().numpy() - want)) < 0.05 * np.max(np.abs(want))


# ------------------------------------------------------------------------------------------------ append and read
@pytest.mark.parametrize("kv_heads,d", [(1, 64), (2, 128), (5, 64), (8, 128)])
@pytest.mark.parametrize("rows,history", [([1, 1, 1, 1], [0, 63, 64, 200]), ([70, 1, 0, 129], [1, 0, 5, 62])])
def test_append_stores_and_read_returns_the_models_values(torch, ctx, kv_heads, d, rows, history):
    rng = np.random.default_rng(kv_heads * 100 + d + len(rows))
    p = Pair(torch, ctx, 2, 24, kv_heads, d, 6, 5)
    slots = [4, 0, 5, 2]
    p.place([history[slots.index(s)] if s in slots else 0 for s in range(6)], rng)
    p.gpu.grow(p.ints(slots), p.ints(rows))
    p.cpu.grow(slots, rows)
    off = np.concatenate([[0], np.cumsum(rows)])
    T = int(off[-1])
    # k is a strided view (a slice of a fused projection's output), with large constant channels; v has tiny and huge groups
    k = bf16(rng, (T, kv_heads, d)) + wl.round_to_bf16(np.where(rng.random((kv_heads, d)) < 0.1, 32.0, 0.0).astype(np.float32))
    k = wl.round_to_bf16(k)
    v = wl.round_to_bf16(bf16(rng, (T, kv_heads, d)) * 10.0 ** rng.integers(-6, 4, (T, kv_heads, 1)).astype(np.float32))
    v[:, :, :64] = np.where(rng.random((T, kv_heads, 1)) < 0.2, np.float32(0.75), v[:, :, :64])  # groups of one value: scale 0
    wide = torch.full((T, (kv_heads + 3) * d), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:, d:(kv_heads + 1) * d] = p.bf(k).reshape(T, -1)
    for layer in (1, 0):
        p.gpu.append(layer, wide[:, d:(kv_heads + 1) * d], p.bf(v), p.ints(off), slots=p.ints(slots))
        p.cpu.append(layer, k, v, off, slots)
    assert ctx.get_status() == 0
    p.assert_same()
    rk, rv = p.gpu.read(1, p.ints(off), T, slots=p.ints(slots))
    for got, x in ((rk, k), (rv, v)):
        # the sum of product and minimum is rounded to fp32, then to bf16: at most one bf16 step from the fp64 value's rounding
        want = co.dequantize(*co.quantize(x))
        err = np.abs(got.float().cpu().numpy().astype(np.float64) - want)
        assert np.all(err <= 2.0 ** -8 * np.abs(want) + 2.0 ** -22 * (np.abs(want) + 64))
        # and half a quantisation step (plus the fp16 roundings of minimum and scale) from what was stored
        g = x.reshape(T, kv_heads, -1, 64).astype(np.float64)
        step = (g.max(-1) - g.min(-1)) / 15
        lim = 0.5 * step + 2.0 ** -11 * (np.abs(g.min(-1)) + 15 * step) * 1.01 + 2.0 ** -8 * np.abs(g).max(-1) + 16 * 2.0 ** -24
        assert np.all(np.abs(got.float().cpu().numpy().reshape(g.shape) - g) <= lim[..., None])


def test_append_of_values_that_do_not_fit_reads_as_nan(torch, ctx):
    rng = np.random.default_rng(2)
    p = Pair(torch, ctx, 1, 4, 2, 128, 1, 4)
    T = 8
    k, v = bf16(rng, (T, 2, 128)), bf16(rng, (T, 2, 128))
    k[1, 0, 5], k[2, 1, 127], v[3, 0, 64], v[4, 1, 0] = np.nan, np.inf, -np.inf, np.nan
    k[5, 0, 3] = -1e5   # the minimum does not fit fp16
    v[6, 1, 3] = 60000  # fits: the scale is 4000
    p.gpu.grow(None, p.ints([T]))
    p.cpu.grow([0], [T])
    p.gpu.append(0, p.bf(k), p.bf(v), p.ints([0, T]))
    p.cpu.append(0, wl.round_to_bf16(k), wl.round_to_bf16(v), [0, T], [0])
    p.assert_same()
    rk, rv = (x.float().cpu().numpy() for x in p.gpu.read(0, p.ints([0, T]), T))
    bad = np.zeros((T, 2), bool)
    bad[[1, 2, 3, 4, 5], [0, 1, 0, 1, 0]] = True
    np.testing.assert_array_equal(np.isnan(rk).all(-1), bad)
    np.testing.assert_array_equal(np.isnan(rv).all(-1), bad)
    assert np.isfinite(rk[~bad]).all() and np.isfinite(rv[~bad]).all()
    # attention: rows that see a bad token are NaN in its kv head, the others are as if it were not there
    for rows in (T, 3):
        q = p.bf(bf16(rng, (rows, 4, 128)))
        for hint in (1, rows, 100):
            out = p.gpu.attend(0, q, p.ints([0, rows]), max_new=hint).float().cpu().numpy()
            for j in range(rows):
                see = T - rows + j + 1
                for h in range(4):
                    assert np.isnan(out[j, h]).all() == bad[:see, h // 2].any() and np.isnan(out[j, h]).any() == bad[:see, h // 2].any()
    assert ctx.get_status() == 0


def test_append_and_read_leave_what_is_not_theirs(torch, ctx):
    """Rows outside the entries, tokens that are not in the cache, pages shared with another sequence."""
    rng = np.random.default_rng(4)
    p = Pair(torch, ctx, 1, 10, 1, 64, 4, 3)
    p.place([64, 100, 3, 0], rng, shared=0)
    p.gpu.fork(p.ints([1]), p.ints([3]))
    p.cpu.fork([1], [3])
    T = 90
    k, v = bf16(rng, (T, 1, 64)), bf16(rng, (T, 1, 64))
    # entry 0 wants 40 rows of sequence 3, of which the first four are on the page that it shares with sequence 1; entry 1 has
    # five rows for a sequence of three tokens; entry 2 names no sequence
    off, slots = [2, 42, 47, 50], [3, 2, 9]
    p.gpu.append(0, p.bf(k), p.bf(v), p.ints(off), slots=p.ints(slots))
    assert ctx.get_status() == binding.ESSA_ERR_CACHE
    p.cpu.append(0, k[6:42], v[6:42], [0, 36], [3])
    p.cpu.append(0, k[44:47], v[44:47], [0, 3], [2])
    p.assert_same()
    ko, vo = (torch.full((T, 1, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    p.gpu.read(0, p.ints(off), T, slots=p.ints(slots), k_out=ko, v_out=vo)
    assert ctx.get_status() == binding.ESSA_ERR_CACHE
    for got in (ko, vo):
        got = got.float().cpu().numpy()
        assert (got[:2] == 9).all() and (got[50:] == 9).all()      # rows of no entry
        assert (got[42:44] == 0).all() and (got[47:50] == 0).all()  # tokens that are nowhere
    assert np.abs(ko.float().cpu().numpy()[44:47, 0] - k[44:47, 0]).max() < 0.3


# ------------------------------------------------------------------------------------------------ attention
def run_attend(torch, ctx, p, rows, slots, heads, rng, hint, layer=0, scale=None, pad=0, strided=False):
    """Attention of `rows[i]` new tokens on sequence slots[i], checked row by row; returns the output."""
    d = p.cpu.shape[3]
    off = pad + np.concatenate([[0], np.cumsum(rows)])
    T = int(off[-1]) + pad
    q = bf16(rng, (T, heads, d))
    dq = p.bf(q)
    out = torch.full((T, heads * d + (64 if strided else 0)), 5.0, dtype=torch.bfloat16, device="cuda")[:, :heads * d]
    if strided:
        wide = torch.zeros((T, heads * d + 128), dtype=torch.bfloat16, device="cuda")
        wide[:, 64:64 + heads * d] = dq.reshape(T, -1)
        dq = wide[:, 64:64 + heads * d]
    else:
        dq = dq.reshape(T, -1)
    p.gpu.attend(layer, dq, p.ints(off), slots=p.ints(slots), max_new=hint, out=out, scale=scale)
    assert ctx.get_status() == 0
    got = out.float().cpu().numpy().reshape(T, heads, d)
    assert (got[:off[0]] == 5).all() and (got[off[-1]:] == 5).all()  # rows of no entry
    for i, s in enumerate(slots):
        if rows[i] == 0:
            continue
        k, v, codes, sc = p.cpu.sequence(layer, s)
        mine = q[off[i]:off[i + 1]]
        c = d ** -0.5 if scale is None else scale
        want, w = co.attend(mine, k, v, int(p.cpu.lengths[s]), c)
        tol = attend_bound(mine, v, codes, sc, want, w, c, k)
        err = np.abs(got[off[i]:off[i + 1]] - want)
        assert np.isfinite(got[off[i]:off[i + 1]]).all()
        assert (err <= tol).all(), (i, s, rows[i], float(np.max(err / tol)))
    return got


HEADS = [(1, 1, 64), (7, 1, 64), (14, 2, 64), (28, 4, 128), (5, 5, 128), (24, 2, 128), (20, 1, 128)]


@pytest.mark.parametrize("heads,kv_heads,d", HEADS)
def test_decode_step_of_ragged_sequences(torch, ctx, heads, kv_heads, d):
    lengths = [1, 0, 2, 15, 16, 17, 63, 64, 65, 128, 300, 1000]
    rng = np.random.default_rng(heads * 7 + d)
    p = Pair(torch, ctx, 2, 60, kv_heads, d, len(lengths), 17)
    p.place(lengths, rng)
    slots = [int(s) for s in rng.permutation(len(lengths))]
    slots.remove(1)  # the empty sequence has a test of its own
    for strided in (False, True):
        run_attend(torch, ctx, p, [1] * len(slots), slots, heads, rng, 1, layer=1, strided=strided)


@pytest.mark.parametrize("heads,kv_heads,d", HEADS)
@pytest.mark.parametrize("hint", [1, 2, 1000])
def test_rows_of_several_tokens_see_their_own_past(torch, ctx, heads, kv_heads, d, hint):
    """Prompts and chunks of odd sizes, from an empty and a filled cache; the hint only chooses the schedule."""
    lengths, rows = [1, 5, 64, 130, 200, 257, 300, 90], [1, 5, 64, 3, 77, 257, 0, 90]
    rng = np.random.default_rng(heads + d + hint)
    p = Pair(torch, ctx, 1, 40, kv_heads, d, len(lengths), 6)
    p.place(lengths, rng, shared=0)
    run_attend(torch, ctx, p, rows, list(range(8)), heads, rng, hint, pad=3)


@pytest.mark.parametrize("rows,hint", [(1, 1), (2, 2), (37, 64)])
def test_long_sequence_is_split_and_joined(torch, ctx, rows, hint):
    """One long sequence: its keys are shared by every thread block of the grid; twice the same call gives the same bits."""
    rng = np.random.default_rng(rows)
    p = Pair(torch, ctx, 1, 400, 2, 128, 2, 390)
    p.place([24901, 77], rng)
    a = run_attend(torch, ctx, p, [rows, 1], [0, 1], 14, rng, hint)
    assert np.isfinite(a).all()
    q = p.bf(bf16(rng, (rows, 14, 128)))
    outs = [p.gpu.attend(0, q, p.ints([0, rows]), max_new=hint) for _ in range(3)]
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("hint", [1, 100])
def test_rows_that_see_nothing_are_zero(torch, ctx, hint):
    """An empty sequence, and entries with more rows than their sequence has tokens."""
    rng = np.random.default_rng(6)
    p = Pair(torch, ctx, 1, 8, 2, 64, 3, 2)
    p.place([0, 3, 70], rng)
    got = run_attend(torch, ctx, p, [2, 40, 100], [0, 1, 2], 8, rng, hint)
    assert (got[:2] == 0).all() and (got[2:39] == 0).all() and (got[39:42] != 0).any() and (got[42:72] == 0).all()


@pytest.mark.parametrize("hint", [1, 100])
def test_bad_pages_and_slots_are_hidden_and_reported(torch, ctx, hint):
    """A table that names pages outside the pool: their tokens are hidden, nothing outside the pool is read."""
    rng = np.random.default_rng(7)
    p = Pair(torch, ctx, 1, 8, 1, 128, 3, 4)
    p.place([200, 64, 10], rng)
    q = p.bf(bf16(rng, (3, 4, 128)))
    p.gpu.table[0, 1] = 8
    p.gpu.table[0, 2] = -5
    p.gpu.table[1, 0] = 1 << 30
    out = p.gpu.attend(0, q, p.ints([0, 1, 2, 3]), slots=p.ints([0, 1, 99]), max_new=hint).float().cpu().numpy()
    assert ctx.get_status() == binding.ESSA_ERR_CACHE
    k, v, codes, sc = p.cpu.sequence(0, 0)
    keep = np.r_[0:64, 192:200]
    want, w = co.attend(q[:1].float().cpu().numpy(), k[:, keep], v[:, keep], len(keep), 128 ** -0.5)
    tol = attend_bound(q[:1].float().cpu().numpy(), v[:, keep], codes[:, :, keep], sc[:, :, keep], want, w, 128 ** -0.5, k[:, keep])
    assert (np.abs(out[:1] - want) <= tol).all()
    assert (out[1:] == 0).all()


@pytest.mark.parametrize("hint", [1, 100])
def test_large_scores_and_uneven_weights(torch, ctx, hint):
    """Scores of hundreds that rise along the sequence (the running maximum moves at almost every page) or peak at its start."""
    rng = np.random.default_rng(9)
    p = Pair(torch, ctx, 1, 20, 1, 64, 2, 8)
    p.place([450, 450], rng)
    for s, ramp in ((0, np.linspace(0, 40, 450)), (1, np.linspace(40, 0, 450))):
        k = wl.round_to_bf16(bf16(rng, (450, 1, 64)) * 0.05 + ramp[:, None, None].astype(np.float32))
        p.cpu.append(0, k, bf16(rng, (450, 1, 64)), [0, 450], [s])
    p.push()
    for rows in (1, 20):
        run_attend(torch, ctx, p, [rows, rows], [0, 1], 4, rng, hint, scale=2.0)


# ------------------------------------------------------------------------------------------------ streams, graphs, together
def test_calls_on_two_streams_overlap_safely(torch, ctx):
    rng = np.random.default_rng(10)
    p = Pair(torch, ctx, 1, 80, 2, 128, 4, 40)
    p.place([2000, 300, 700, 1], rng)
    q = [p.bf(bf16(rng, (4, 16, 128))) for _ in range(2)]
    want = [p.gpu.attend(0, x) for x in q]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[], []]
    for rep in range(20):
        for i, s in enumerate(streams):
            outs[i].append(p.gpu.attend(0, q[i], stream=s))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i in range(2) for o in outs[i]) and ctx.get_status() == 0


def test_decode_step_captured_into_a_graph_follows_the_growing_sequences(torch, ctx):
    """grow, append and attend in one graph, replayed over page borders: each replay is the model's next step."""
    rng = np.random.default_rng(11)
    p = Pair(torch, ctx, 1, 30, 2, 64, 5, 6)
    p.place([62, 0, 127, 5, 64], rng)
    one, slots = p.ints([1] * 5), p.ints(range(5))
    k, v, q = (p.bf(bf16(rng, (5, h, 64))) for h in (2, 2, 6))
    out = torch.empty_like(q)

    def step():
        p.gpu.grow(slots, one)
        p.gpu.append(0, k, v)
        p.gpu.attend(0, q, out=out)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    p.push()
    for _ in range(4):
        new = [bf16(rng, (5, h, 64)) for h in (2, 2, 6)]
        for t, a in zip((k, v, q), new):
            t.copy_(p.bf(a))
        graph.replay()
        p.cpu.grow(range(5), [1] * 5)
        p.cpu.append(0, new[0], new[1], list(range(6)), range(5))
        p.assert_same()
        got = out.float().cpu().numpy()
        for s in range(5):
            kk, vv, codes, sc = p.cpu.sequence(0, s)
            want, w = co.attend(new[2][s:s + 1], kk, vv, int(p.cpu.lengths[s]), 64 ** -0.5)
            assert (np.abs(got[s:s + 1] - want) <= attend_bound(new[2][s:s + 1], vv, codes, sc, want, w, 64 ** -0.5, kk)).all()
    assert ctx.get_status() == 0


def test_population_evaluates_prompts_forks_and_decodes(torch, ctx):
    """The operators as they are used: the candidates' q, k, v projections, the cache between them and the o projection, a prompt
    of ragged lengths, two rollouts of every candidate, and a decode step of all of them; against the oracles chained in fp64."""
    cfg = wl.scaled_config("3", d_model=256, d_kv=128, rank=8, P=3, seg_len=40)
    heads, kv_heads, d = 4, 2, 64
    rng = np.random.default_rng(12)
    case = Case(torch, ctx, cfg)
    cols = [cfg.sigma_cols(i) for i in range(4)]
    cache = ctx.kv_cache(1, 40, kv_heads, d, 9, 4)
    ints = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")

    def block(x, seg, slots, rows):
        dseg = ints(seg)
        tok = ints(np.concatenate([[0], np.cumsum(rows)]))
        dx = to_dev(torch, x, torch.bfloat16)
        q, k, v = ctx.apply_block(case.handles_list[:3], [dx] * 3, dseg, case.d_sigma, cols[:3])
        cache.grow(ints(slots), ints(rows))
        cache.append(0, k, v, tok, slots=ints(slots))
        a = cache.attend(0, q, tok, slots=ints(slots), max_new=int(max(rows)))
        y = ctx.apply_projection(case.handles_list[3], a, dseg, case.d_sigma, *cols[3])
        return [t.float().cpu().numpy() for t in (q, k, v, a, y)]

    case.handles_list = [case.handles[i] for i in range(4)]
    model = co.Cache(1, 40, kv_heads, d, 9, 4)

    def check(x, seg, slots, rows, got):
        q, k, v, a, y = got
        off = np.concatenate([[0], np.cumsum(rows)])
        for i in range(3):  # projections against their oracle
            ad = case.adapters[i]
            want = orc.apply_projection(ad.W0, ad.U_A, ad.V_A, ad.U_B, ad.V_B, x, np.asarray(seg, np.int32), case.sigma32, *cols[i], cfg.rank)
            assert orc.relative_error(got[i], want) <= 2e-2
        model.grow(slots, rows)
        model.append(0, k.reshape(-1, kv_heads, d), v.reshape(-1, kv_heads, d), off, slots)
        for i, s in enumerate(slots):
            kk, vv, codes, sc = model.sequence(0, s)
            mine = q[off[i]:off[i + 1]].reshape(-1, heads, d)
            want, w = co.attend(mine, kk, vv, int(model.lengths[s]), d ** -0.5)
            assert (np.abs(a[off[i]:off[i + 1]].reshape(want.shape) - want) <= attend_bound(mine, vv, codes, sc, want, w, d ** -0.5, kk)).all()
        ad = case.adapters[3]
        want = orc.apply_projection(ad.W0, ad.U_A, ad.V_A, ad.U_B, ad.V_B, a, np.asarray(seg, np.int32), case.sigma32, *cols[3], cfg.rank)
        assert orc.relative_error(y, want) <= 2e-2

    rows = [70, 1, 64]
    x = bf16(rng, (sum(rows), 256))
    seg = np.concatenate([[0], np.cumsum(rows)])
    check(x, seg, [0, 1, 2], rows, block(x, seg, [0, 1, 2], rows))
    cache.fork(ints([0, 0, 1, 1, 2, 2]), ints([3, 4, 5, 6, 7, 8]))
    model.fork([0, 0, 1, 1, 2, 2], [3, 4, 5, 6, 7, 8])
    cache.free(ints([0, 1, 2]))
    model.free([0, 1, 2])
    for step in range(3):
        x = bf16(rng, (6, 256))
        check(x, [0, 2, 4, 6], [3, 4, 5, 6, 7, 8], [1] * 6, block(x, [0, 2, 4, 6], [3, 4, 5, 6, 7, 8], [1] * 6))
        if step == 1:
            cache.compact()
            model.compact()
    np.testing.assert_array_equal(cache.table.cpu().numpy(), model.table)
    assert ctx.get_status() == 0
    case.close()


def test_host_side_refusals(torch, ctx):
    g = ctx.kv_cache(1, 4, 2, 64, 2, 2)
    ints = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    bad = [lambda: g.attend(0, bf(1, 3, 64)), lambda: g.attend(1, bf(1, 4, 64)), lambda: g.attend(0, bf(1, 4, 64), max_new=0), lambda: g.attend(0, bf(1, 4, 64), scale=0.0),
           lambda: g.attend(0, bf(1, 4, 64), scale=float("nan")), lambda: g.attend(0, bf(1, 4, 64).float()), lambda: g.attend(0, bf(1, 4, 32)),
           lambda: g.attend(0, bf(2, 4, 64), ints([0, 2]), slots=ints([0, 1])), lambda: g.attend(0, bf(1, 4, 65)[:, :, 1:]),
           lambda: g.attend(0, bf(2, 4 * 64 + 4)[:, :256]), lambda: g.attend(0, bf(1, 4, 64).cpu()), lambda: g.attend(0, bf(1, 4, 64), out=bf(1, 2, 64)),
           lambda: g.append(0, bf(1, 2, 64), bf(2, 2, 64)), lambda: g.append(0, bf(1, 3, 64), bf(1, 3, 64)), lambda: g.append(-1, bf(1, 2, 64), bf(1, 2, 64)),
           lambda: g.grow(None, ints([1, 1, 1])), lambda: g.grow(ints([0, 1]).long(), ints([1, 1])), lambda: g.free(ints([0, 0, 0])), lambda: g.fork(ints([0, 1]), ints([1])),
           lambda: g.read(0, ints([0, 2]), 2, k_out=bf(1, 2, 64)), lambda: ctx.kv_cache(1, 4, 2, 96, 2, 2), lambda: ctx.kv_cache(1, 0, 2, 64, 2, 2),
           lambda: ctx.kv_cache(1, 4, 2, 64, 2, 2, pages=g.pages), lambda: ctx.kv_cache(1, 5, 2, 64, 2, 2, pages=g.pages, table=g.table, lengths=g.lengths, refs=g.refs)]
    for i, call in enumerate(bad):
        with pytest.raises((binding.EssaError, RuntimeError)):
            call()
            print("not refused:", i)
    # calls with nothing to do
    g.grow(ints([]), ints([]))
    g.append(0, bf(0, 2, 64), bf(0, 2, 64), ints([0, 0]))
    assert g.attend(0, bf(0, 4, 64), ints([0, 0])).shape == (0, 4, 64)
    assert g.attend(0, bf(0, 4, 64)).shape == (0, 4, 64)
    g.fork(ints([]), ints([]))
    g.free(ints([]))
    assert ctx.get_status() == 0


# ------------------------------------------------------------------------------------------------ sizes, extremes, ways of calling
def check_rows(p, got, q, slot, scale, extra=0.0, length=None):
    """Rows `got` for the queries `q` of the last tokens of a sequence against the model; `extra` is added to the bound."""
    k, v, codes, sc = p.cpu.sequence(0, slot)
    want, w = co.attend(q, k, v, int(p.cpu.lengths[slot]), scale)
    with np.errstate(over="ignore"):  # (a bound may be infinite where scores are large)
        tol = attend_bound(q, v, codes, sc, want, w, scale, k) + extra
    err = np.abs(got - want)
    assert np.isfinite(got).all() and (err <= tol).all(), (slot, float(np.max(err / tol)))


def test_one_sequence_grows_by_many_pages_beside_short_ones(torch, ctx):
    """A prompt of thousands of pages in the same call as sequences that get one, none, or two."""
    p = Pair(torch, ctx, 1, 3000, 1, 64, 70, 2100)
    counts = np.random.default_rng(1).integers(0, 130, 70)
    counts[[3, 40]] = 64 * 2000 + 5, 64 * 600
    for _ in range(2):
        p.gpu.grow(None, p.ints(counts))
        p.cpu.grow(range(70), counts)
        assert ctx.get_status() == 0
        p.assert_same(pages=False)
        counts = np.minimum(counts, 70)


def test_more_entries_than_a_thread_block_has_offsets_for(torch, ctx):
    rng = np.random.default_rng(14)
    n = 2600
    p = Pair(torch, ctx, 1, 4000, 1, 64, n, 3)
    p.place(rng.integers(0, 100, n), rng)
    rows = np.minimum(rng.integers(0, 4, n), p.cpu.lengths)
    slots = rng.permutation(n)
    off = np.concatenate([[0], np.cumsum(rows[slots])])
    T = int(off[-1])
    k, v = (bf16(rng, (T, 1, 64)) for _ in range(2))
    p.gpu.append(0, p.bf(k), p.bf(v), p.ints(off), slots=p.ints(slots))
    p.cpu.append(0, k, v, off, slots)
    p.assert_same()
    ko, vo = p.gpu.read(0, p.ints(off), T, slots=p.ints(slots))
    for got, x in ((ko, k), (vo, v)):
        want = co.dequantize(*co.quantize(x))
        np.testing.assert_array_equal(got.float().cpu().numpy(), wl.round_to_bf16(want.astype(np.float32)))
    q = bf16(rng, (T, 3, 64))
    for hint in (1, 100):
        got = p.gpu.attend(0, p.bf(q), p.ints(off), slots=p.ints(slots), max_new=hint).float().cpu().numpy()
        for i in rng.permutation(n)[:200]:
            if rows[slots[i]]:
                check_rows(p, got[off[i]:off[i + 1]], q[off[i]:off[i + 1]], slots[i], 64 ** -0.5)
    assert ctx.get_status() == 0


@pytest.mark.parametrize("hint", [1, 100])
@pytest.mark.parametrize("d", [64, 128])
def test_queries_of_very_different_size(torch, ctx, hint, d):
    """Rows between 2^-110 and 2^6 side by side, rows of zeros, rows whose channels lie far apart, and a scale that takes them below fp32's range."""
    rng = np.random.default_rng(15)
    p = Pair(torch, ctx, 1, 30, 2, d, 3, 6)
    p.place([300, 64, 7], rng)
    rows = [40, 30, 7]
    off = np.concatenate([[0], np.cumsum(rows)])
    T = int(off[-1])
    q = bf16(rng, (T, 6, d))
    q *= np.float32(2.0) ** rng.integers(-110, 7, (T, 6, 1)).astype(np.float32)
    q[::7] = 0
    q[1::7, :, ::2] *= np.float32(2.0 ** -20)
    for scale in (d ** -0.5, 1e-12, 1e-38):
        got = p.gpu.attend(0, p.bf(q), p.ints(off), max_new=hint, scale=scale).float().cpu().numpy()
        for i in range(3):
            check_rows(p, got[off[i]:off[i + 1]], q[off[i]:off[i + 1]], i, scale)
    assert ctx.get_status() == 0


@pytest.mark.parametrize("hint", [1, 100])
@pytest.mark.parametrize("size_k,size_v", [(1.0, 14000.0), (14000.0, 1.0), (1.0, 1e-6), (1.0, 0.0)])
def test_keys_and_values_of_extreme_size(torch, ctx, hint, size_k, size_v):
    """Up to fp16's end, and down to values that its subnormal numbers hold."""
    rng = np.random.default_rng(16)
    p = Pair(torch, ctx, 1, 30, 1, 128, 2, 6)
    p.place([300, 65], rng)
    for s in range(2):
        n = int(p.cpu.lengths[s])
        k, v = (np.clip(bf16(rng, (n, 1, 128)), -4, 4) * np.float32(size) for size in (size_k, size_v))
        p.cpu.append(0, wl.round_to_bf16(k), wl.round_to_bf16(v), [0, n], [s])
    p.push()
    off, q = [0, 30, 60], bf16(rng, (60, 5, 128))
    scale = 128 ** -0.5 / size_k
    got = p.gpu.attend(0, p.bf(q), p.ints(off), max_new=hint, scale=scale).float().cpu().numpy()
    assert ctx.get_status() == 0
    # many rows: a value's offset and the value itself are rounded to fp16, below its normal range to 2^-25 absolutely each; weights sum to 1
    for s in range(2):
        check_rows(p, got[off[s]:off[s + 1]], q[off[s]:off[s + 1]], s, scale, extra=2.0 ** -24)


@pytest.mark.parametrize("hint", [1, 100])
def test_a_token_that_did_not_fit_reaches_only_the_rows_that_see_it(torch, ctx, hint):
    rng = np.random.default_rng(17)
    p = Pair(torch, ctx, 1, 8, 1, 64, 2, 4)
    p.place([200, 60], rng)
    k, v = bf16(rng, (40, 1, 64)), bf16(rng, (40, 1, 64))
    v[25, 0, 3] = np.inf
    k[33, 0, 60] = np.nan
    p.gpu.append(0, p.bf(k), p.bf(v), p.ints([0, 40]), slots=p.ints([0]))
    p.cpu.append(0, k, v, [0, 40], [0])
    p.assert_same()
    q = bf16(rng, (60, 4, 64))
    got = p.gpu.attend(0, p.bf(q), p.ints([0, 40, 60]), max_new=hint).float().cpu().numpy()
    assert ctx.get_status() == 0
    assert np.isnan(got[25:40]).all()
    p.cpu.lengths[0] = 160 + 25  # what the rows before it see
    check_rows(p, got[:25], q[:25], 0, 64 ** -0.5)
    check_rows(p, got[40:], q[40:], 1, 64 ** -0.5)


@pytest.mark.parametrize("hint", [1, 100])
def test_two_entries_on_one_sequence(torch, ctx, hint):
    """attend and read may name a sequence as often as they like."""
    rng = np.random.default_rng(18)
    p = Pair(torch, ctx, 1, 8, 2, 64, 2, 4)
    p.place([130, 60], rng)
    q = bf16(rng, (5, 4, 64))
    off, slots = p.ints([0, 2, 5]), p.ints([0, 0])
    got = p.gpu.attend(0, p.bf(q), off, slots=slots, max_new=hint).float().cpu().numpy()
    check_rows(p, got[:2], q[:2], 0, 64 ** -0.5)
    check_rows(p, got[2:], q[2:], 0, 64 ** -0.5)
    ko, _ = p.gpu.read(0, off, 5, slots=slots)
    assert torch.equal(ko[:2], ko[3:]) and ctx.get_status() == 0


def test_graphs_of_two_calls_replayed_beside_one_another(torch, ctx):
    """Two captured calls of each kernel hold workspaces of their own: replays that overlap give what the calls alone give."""
    rng = np.random.default_rng(19)
    p = Pair(torch, ctx, 1, 200, 2, 128, 3, 180)
    p.place([11000, 300, 64], rng)
    for hint in (1, 100):
        q = [p.bf(bf16(rng, (3, 8, 128))) for _ in range(2)]
        want = [p.gpu.attend(0, x, max_new=hint) for x in q]
        outs, graphs = [torch.empty_like(x) for x in q], [torch.cuda.CUDAGraph() for _ in q]
        torch.cuda.synchronize()
        for x, out, graph in zip(q, outs, graphs):
            with torch.cuda.graph(graph):
                p.gpu.attend(0, x, max_new=hint, out=out)
        streams = [torch.cuda.Stream() for _ in q]
        for _ in range(20):
            for out in outs:
                out.fill_(7.0)
            torch.cuda.synchronize()
            for _ in range(3):
                for graph, s in zip(graphs, streams):
                    with torch.cuda.stream(s):
                        graph.replay()
                eager = p.gpu.attend(0, q[0], max_new=hint)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want)) and torch.equal(eager, want[0])
    assert ctx.get_status() == 0


def test_a_step_on_a_stream_of_its_own(torch, ctx):
    """Every call with `stream`: nothing of it depends on the current stream, which is busy with other work."""
    rng = np.random.default_rng(20)
    p = Pair(torch, ctx, 1, 20, 2, 64, 4, 4)
    p.place([62, 0, 127, 64], rng)
    k, v = (bf16(rng, (4, 2, 64)) for _ in range(2))
    q = bf16(rng, (2, 4, 64))
    dk, dv, dq, one, src, dst, off = p.bf(k), p.bf(v), p.bf(q), p.ints([1] * 4), p.ints([0]), p.ints([1]), p.ints([0, 1])
    pair = p.ints([0, 2])
    busy = torch.zeros(64 << 20, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(20):
        busy += 1
    p.gpu.grow(None, one, stream=s)
    p.gpu.append(0, dk, dv, stream=s)
    out = p.gpu.attend(0, dq, slots=pair, stream=s)
    p.gpu.fork(src, dst, stream=s)
    ko, vo = p.gpu.read(0, off, 1, slots=dst, stream=s)
    p.gpu.compact(stream=s)
    s.synchronize()
    p.cpu.grow(range(4), [1] * 4)
    p.cpu.append(0, k, v, [0, 1, 2, 3, 4], range(4))
    for i, slot in enumerate((0, 2)):
        check_rows(p, out[i:i + 1].float().cpu().numpy(), q[i:i + 1], slot, 64 ** -0.5)
    p.cpu.fork([0], [1])
    p.cpu.compact()
    p.assert_same()
    want = co.dequantize(*co.quantize(k[:1]))
    np.testing.assert_array_equal(ko.float().cpu().numpy(), wl.round_to_bf16(want.astype(np.float32)))
    assert ctx.get_status() == 0


def test_scales_out_of_range_empty_offsets_and_a_closed_context_are_refused(torch):
    c = binding.Context(0)
    g = c.kv_cache(1, 4, 2, 64, 2, 2)
    q = torch.zeros((1, 4, 64), dtype=torch.bfloat16, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    for call in (lambda: g.attend(0, q, scale=float("inf")), lambda: g.attend(0, q, scale=3e38), lambda: g.attend(0, q, scale=-1.0), lambda: g.attend(0, q, none),
                 lambda: g.attend(0, q[0]), lambda: g.attend(0, q.expand(2, 4, 64))):
        with pytest.raises((binding.EssaError, RuntimeError)):
            call()
    assert c.get_status() == 0
    g.attend(0, q)
    torch.cuda.synchronize()
    c.close()
    for call in (lambda: g.attend(0, q), lambda: g.reset(), lambda: g.append(0, q[:, :2], q[:, :2]), lambda: c.kv_cache(1, 4, 2, 64, 2, 2)):
        with pytest.raises(binding.EssaError):
            call()


@pytest.mark.parametrize("d", [64, 128])
def test_codes_of_offset_tied_and_flat_groups(torch, ctx, d):
    """Codes, scales and minima bit by bit where the quotient is hard: ties, minima hundreds of steps away, groups of one or two values, huge and
    tiny steps; enough tokens for the schedule of long prompts too."""
    rng = np.random.default_rng(21)
    for T in (40, 5000):
        p = Pair(torch, ctx, 1, 90, 2, d, 1, 90)
        k, v = bf16(rng, (T, 2, d)), bf16(rng, (T, 2, d))
        kind = np.arange(T) % 8
        k[kind == 1] += 300
        k[kind == 2] = rng.integers(0, 31, k[kind == 2].shape) / 2          # minimum 0 and maximum 15 in nearly every group: halves tie
        k[kind == 2, :, ::64], k[kind == 2, :, 1::64] = 0, 15
        k[kind == 3] = 1.7
        k[kind == 4] = rng.choice([-3.0, 5.0], k[kind == 4].shape)
        k[kind == 5] = k[kind == 5] * 0.02 + 2.5                            # 2.5 / (0.1 / 15): some 300 steps
        k[kind == 6] *= 9000
        k[kind == 7] *= 1e-5
        v[kind < 4] = rng.integers(-15, 16, v[kind < 4].shape) / 2 + 0.25   # quotients at many fractions
        v[kind >= 4] -= 40
        k, v = wl.round_to_bf16(k.astype(np.float32)), wl.round_to_bf16(v.astype(np.float32))
        p.gpu.grow(None, p.ints([T]))
        p.cpu.grow([0], [T])
        p.gpu.append(0, p.bf(k), p.bf(v), p.ints([0, T]))
        p.cpu.append(0, k, v, [0, T], [0])
        assert ctx.get_status() == 0
        p.assert_same()


@pytest.mark.parametrize("heads,kv_heads,d", [(300, 1, 64), (33, 3, 128), (32, 2, 64), (17, 17, 64)])
def test_groups_of_unusual_size(torch, ctx, heads, kv_heads, d):
    """More heads in a group than a row block has rows, groups of 11 and 16 heads, and 17 kv heads of one head each."""
    rng = np.random.default_rng(heads)
    p = Pair(torch, ctx, 1, 20, kv_heads, d, 3, 5)
    p.place([300, 65, 2], rng)
    for rows, hint in (([1, 1, 1], 1), ([3, 2, 2], 3), ([40, 65, 2], 65)):
        run_attend(torch, ctx, p, rows, [0, 1, 2], heads, rng, hint)


def test_second_cache_object_on_the_same_buffers(torch, ctx):
    """A second cache object on the buffers of the first sees the same sequences."""
    rng = np.random.default_rng(23)
    p = Pair(torch, ctx, 2, 10, 2, 64, 3, 4)
    p.place([100, 3, 64], rng)
    g = p.gpu
    other = ctx.kv_cache(2, 10, 2, 64, 3, 4, pages=g.pages, table=g.table, lengths=g.lengths, refs=g.refs)
    q = p.bf(bf16(rng, (3, 4, 64)))
    for layer in range(2):
        assert torch.equal(other.attend(layer, q), g.attend(layer, q))
    other.grow(None, p.ints([1, 1, 1]))
    p.cpu.grow(range(3), [1, 1, 1])
    assert ctx.get_status() == 0
    p.assert_same(pages=False)


def test_projections_of_several_layers_right_behind_an_attention(torch, ctx):
    """apply_layers chains its launches loosely; what stands before it on the stream (an attention without a join, one with, a fork) has ended
    all the same when they read its output."""
    cfg = wl.scaled_config("3", d_model=256, d_kv=128, rank=8, P=3, seg_len=40)
    rng = np.random.default_rng(24)
    case = Case(torch, ctx, cfg)
    seg = torch.tensor([0, 40, 80, 120], dtype=torch.int32, device="cuda")
    for pages in (20, 60):
        p = Pair(torch, ctx, 1, 120 * pages, 2, 64, 120, pages)
        p.gpu.pages.random_(0, 60)  # (small scales and minima, whatever they are)
        p.gpu.grow(None, p.ints([pages * 64 - 3] * 120))
        outs = [torch.empty((120, 256), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
        a = torch.empty((120, 256), dtype=torch.bfloat16, device="cuda")

        def step(q, wait):
            a.fill_(3.0)
            p.gpu.attend(0, q, out=a)
            if wait:
                torch.cuda.synchronize()
            ctx.apply_layers([[(case.handles[3], a, cfg.sigma_cols(3), o)] for o in outs], seg, case.d_sigma)
            torch.cuda.synchronize()
            return [o.clone() for o in outs]

        for _ in range(10):
            q = p.bf(bf16(rng, (120, 256)))
            for x, y in zip(step(q, False), step(q, True)):
                assert torch.equal(x, y)
    assert ctx.get_status() == 0
    case.close()
