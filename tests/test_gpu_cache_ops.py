"""GPU tests of the operators around the key / value cache: rotary positions, windowed attention, trees of drafted tokens, keeping a path, against the fp64 /
integer model (oracle/cache_oracle.py); their refusals, streams and graphs, and a run of them as a program would make it."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from paper_2507_04453_b200 import binding, workloads as wl
from tests.cache_utils import NORM_LIMIT, Pair, attend_bound, bf16, norm_error
from tests.parity_utils import to_dev

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


def f32(t):
    return t.float().cpu().numpy()


# ------------------------------------------------------------------------------------------------ rotation
# Of a pair (a, b): cosine and sine are wrong by 2^-22 at most (the fraction of a turn by 2^-32 and by its rounding to fp32, 2^-25 of half a turn, times
# pi; the function by 2^-23), the products and their sum are rounded to fp32 (2^-24 each), and the result to bf16 (2^-8 of it, or 2^-134 absolutely).
def rotate_bound(x, want, adjacent, magnitude):
    y = np.abs(x.astype(np.float64))
    d = x.shape[-1]
    both = (y[..., 0::2] + y[..., 1::2]) if adjacent else (y[..., :d // 2] + y[..., d // 2:])
    both = np.repeat(both, 2, -1) if adjacent else np.concatenate([both, both], -1)
    return 2.0 ** -8 * np.abs(want) + (2.0 ** -21 * (1 + 2.0 ** -8)) * abs(magnitude) * both + 2.0 ** -133


@pytest.mark.parametrize("d", [16, 48, 64, 80, 128, 256])
@pytest.mark.parametrize("T,heads", [(1, 1), (7, 3), (33, 17)])
@pytest.mark.parametrize("adjacent", [False, True])
def test_rotation_of_any_rows(torch, ctx, d, T, heads, adjacent):
    rng = np.random.default_rng(d + T)
    axes = 1 + (d // 16 + T) % 4
    axis = rng.integers(0, axes, d // 2)
    axis[0] = axes - 1
    freq = 10.0 ** -rng.uniform(0, 6, d // 2)
    freq[-1] = 0.0
    rot = binding.Rotary(d, frequencies=freq, axis=axis, adjacent=adjacent, magnitude=1.25)
    x = bf16(rng, (T, heads, d))
    pos = rng.integers(-70000, 1 << 20, (axes, T)).astype(np.int32)
    pos[:, 0] = [0, -1, 2147483647, -2147483648][:axes]
    want = co.rotate(x, pos, freq, axis, adjacent, 1.25)
    dx, dp = to_dev(torch, x, torch.bfloat16), torch.from_numpy(pos).cuda()
    got = ctx.rotary(rot, dx, dp)
    assert (np.abs(f32(got) - want) <= rotate_bound(x, want, adjacent, 1.25)).all()
    # strided rows (a slice of a fused projection's output, positions of a longer buffer), and in place: the same bits
    wide = torch.full((T, (heads + 2) * d), 3.0, dtype=torch.bfloat16, device="cuda")
    view = wide[:, d:(heads + 1) * d].unflatten(1, (heads, d))
    view.copy_(dx)
    long = torch.zeros((axes, T + 5), dtype=torch.int32, device="cuda")
    long[:, :T] = dp
    out = ctx.rotary(rot, view, long[:, :T], out=view)
    assert out is view and torch.equal(view, got) and (wide[:, :d] == 3).all() and (wide[:, (heads + 1) * d:] == 3).all()
    assert ctx.get_status() == 0


def test_rotation_turns_back_and_far_positions_are_exact(torch, ctx):
    """Positions beyond 2^31 - 200 at a radian per position: the angle's fraction is what counts, and fp32 has none left."""
    rng = np.random.default_rng(1)
    rot = binding.Rotary(128, base=1e4)
    x = bf16(rng, (100, 2, 128))
    pos = (2 ** 31 - 1 - np.arange(100)).astype(np.int32)[None]
    want = co.rotate(x, pos, 1e4 ** (-np.arange(64) / 64), [0] * 64)
    dx, dp = to_dev(torch, x, torch.bfloat16), torch.from_numpy(pos).cuda()
    got = ctx.rotary(rot, dx, dp[0])
    # (the frequency itself is rounded to fp64: 2^31 2^-53 radians)
    assert (np.abs(f32(got) - want) <= rotate_bound(x, want, False, 1.0) + 2.0 ** -21 * np.abs(x).max()).all()
    back = ctx.rotary(rot, got, -dp[0])
    # two roundings to bf16, the first one's turned: 2^-8 of a pair's length each
    pair = np.hypot(x[..., :64], x[..., 64:])
    assert (np.abs(f32(back) - x) <= 2.0 ** -7 * 1.01 * np.concatenate([pair, pair], -1) + 1e-30).all()


def test_rotation_of_infinities_and_nan_stays_in_its_pair(torch, ctx):
    rot = binding.Rotary(64, base=100.0)
    x = torch.ones((2, 3, 64), dtype=torch.bfloat16, device="cuda")
    x[0, 1, 5], x[1, 2, 40] = float("nan"), float("inf")
    got = ctx.rotary(rot, x, torch.tensor([3, 4], dtype=torch.int32, device="cuda"))
    bad = ~torch.isfinite(got)
    want = torch.zeros_like(bad)
    want[0, 1, 5] = want[0, 1, 37] = want[1, 2, 8] = want[1, 2, 40] = True
    assert torch.equal(bad, want)


@pytest.mark.parametrize("T", [0, 1])
def test_rotary_refuses(torch, ctx, T):
    rot = binding.Rotary(64, sections=[16, 16])
    x, pos = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 1), dtype=torch.int32, device="cuda")
    x, pos = x[:T], pos[:, :T]
    ctx.rotary(rot, x, pos)
    for bad_x, bad_pos, out in ((x.half(), pos, None), (x.cpu(), pos, None), (x.reshape(T, 1, 128), pos, None), (x, pos[:1], None), (x, pos.long(), None), (x, pos.cpu(), None),
                                (x, pos, x.half()), (x, pos, torch.zeros((T + 1, 2, 64), dtype=torch.bfloat16, device="cuda"))):
        with pytest.raises(binding.EssaError):
            ctx.rotary(rot, bad_x, bad_pos, out=out)
    if T:
        wide = torch.zeros((3, 140), dtype=torch.bfloat16, device="cuda")
        for view in (wide[:, 1:129], wide[:, :128:1].unflatten(1, (2, 64)).transpose(1, 2)):
            with pytest.raises(binding.EssaError):
                ctx.rotary(rot, view.unflatten(1, (2, 64)) if view.dim() == 2 else view, torch.zeros((2, 3), dtype=torch.int32, device="cuda"))
        p = lambda t: t.data_ptr()
        call = lambda **kw: ctx.lib.essa_rotary_apply(ctx.handle, rot._ref, kw.get("x", p(x)), kw.get("ld", 128), kw.get("heads", 2), kw.get("T", 1), kw.get("pos", p(pos)),
                                                      kw.get("ldp", 1), kw.get("out", p(x)), kw.get("ldo", 128), None)
        for kw in (dict(x=None), dict(ld=120), dict(ld=129), dict(heads=0), dict(T=-1), dict(pos=None), dict(pos=p(pos) + 2), dict(ldp=0), dict(out=None), dict(out=p(x) + 2),
                   dict(ldo=136)):
            assert call(**kw) == binding.ESSA_ERR_INVALID_ARG, kw
        assert call() == 0
    assert ctx.get_status() == 0


# ------------------------------------------------------------------------------------------------ rotation and append
@pytest.mark.parametrize("heads,kv_heads,d", [(1, 1, 64), (14, 2, 64), (10, 5, 64), (28, 4, 128), (8, 8, 128), (40, 1, 128)])
@pytest.mark.parametrize("adjacent,axes", [(False, 1), (True, 3), (False, 3)])
@pytest.mark.parametrize("rows,history", [([1, 1, 1, 1], [0, 63, 64, 200]), ([70, 1, 0, 129], [1, 0, 5, 62])])
def test_append_rotary_is_rotation_and_append(torch, ctx, heads, kv_heads, d, adjacent, axes, rows, history):
    """The same bits as essa_rotary_apply on q and k and essa_cache_append, strided and in place too; and the model's values."""
    rng = np.random.default_rng(heads + d + len(rows) + axes)
    p, other = (Pair(torch, ctx, 2, 24, kv_heads, d, 6, 5) for _ in range(2))
    slots = [4, 0, 5, 2]
    at = [history[slots.index(s)] if s in slots else 0 for s in range(6)]
    for c in (p, other):
        c.place(at, np.random.default_rng(3))
        c.gpu.grow(c.ints(slots), c.ints(rows))
    p.cpu.grow(slots, rows)
    off = np.concatenate([[0], np.cumsum(rows)])
    T = int(off[-1])
    sections = [d // 2] if axes == 1 else [d // 2 - 2 * (d // 8), d // 8, d // 8]
    rot = binding.Rotary(d, base=1e4, sections=sections, adjacent=adjacent)
    freq, axis = 1e4 ** (-np.arange(d // 2) * 2 / d), list(rot.desc.axis)[:d // 2]
    q, k, v = bf16(rng, (T, heads, d)), bf16(rng, (T, kv_heads, d)), bf16(rng, (T, kv_heads, d))
    own = np.concatenate([np.arange(p.cpu.lengths[s] - r, p.cpu.lengths[s]) for s, r in zip(slots, rows)]).astype(np.int32)
    pos = own[None] if axes == 1 else rng.integers(0, 100000, (axes, T)).astype(np.int32)
    dp = torch.from_numpy(pos).cuda()
    given = None if axes == 1 else dp
    wide = torch.full((T, (heads + 2 * kv_heads) * d), 7.0, dtype=torch.bfloat16, device="cuda")  # q, k, v of one fused projection
    dq, dk, dv = (wide[:, a * d:(a + n) * d] for a, n in ((0, heads), (heads, kv_heads), (heads + kv_heads, kv_heads)))
    for view, x in ((dq, q), (dk, k), (dv, v)):
        view.copy_(p.bf(x).reshape(T, -1))
    got = p.gpu.append_rotary(1, rot, dq.unflatten(1, (heads, d)), dk, dv, given, p.ints(off), slots=p.ints(slots))
    turned = [ctx.rotary(rot, p.bf(x), dp) for x in (q, k)]
    other.gpu.append(1, turned[1], p.bf(v), p.ints(off), slots=p.ints(slots))
    assert torch.equal(got, turned[0]) and torch.equal(p.gpu.pages, other.gpu.pages) and ctx.get_status() == 0
    want = co.rotate(q, pos, freq, axis, adjacent)
    assert (np.abs(f32(got) - want) <= rotate_bound(q, want, adjacent, 1.0)).all()
    p.cpu.append(1, f32(turned[1]), v, off, slots)
    p.assert_same()
    out = p.gpu.append_rotary(1, rot, dq, dk, dv, given, p.ints(off), slots=p.ints(slots), q_out=dq)  # in place, 2-d
    assert out is dq and torch.equal(dq.unflatten(1, (heads, d)), got) and torch.equal(dv.unflatten(1, (kv_heads, d)), p.bf(v))
    p.assert_same()


def test_append_rotary_of_values_that_do_not_fit(torch, ctx):
    rng = np.random.default_rng(2)
    p, other = (Pair(torch, ctx, 1, 4, 2, 128, 1, 4) for _ in range(2))
    T = 8
    q, k, v = bf16(rng, (T, 4, 128)), bf16(rng, (T, 2, 128)), bf16(rng, (T, 2, 128))
    k[1, 0, 5], k[2, 1, 127], v[3, 0, 64], k[5, 0, 3] = np.nan, np.inf, -np.inf, -1e5
    k[6, 1, :] = 0
    rot = binding.Rotary(128)
    for c in (p, other):
        c.gpu.grow(None, c.ints([T]))
    p.gpu.append_rotary(0, rot, p.bf(q), p.bf(k), p.bf(v), tok_offsets=p.ints([0, T]))
    other.gpu.append(0, ctx.rotary(rot, p.bf(k), torch.arange(T, dtype=torch.int32, device="cuda")), p.bf(v), p.ints([0, T]))
    assert torch.equal(p.gpu.pages, other.gpu.pages)
    bad = np.isnan(f32(p.gpu.read(0, p.ints([0, T]), T)[0])).all(-1)
    # (-1e5 is turned by 5 * 10000 ** (-3 / 64) = 3.25 radians: 9.9e4, and 1.1e4 in channel 67, are largest values, with scales that fit)
    want = np.zeros((T, 2), bool)
    want[[1, 2, 3], [0, 1, 0]] = True
    np.testing.assert_array_equal(bad, want)
    assert ctx.get_status() == 0


def test_append_rotary_leaves_what_is_not_its(torch, ctx):
    """Rows outside the entries, a slot that is none, tokens before a sequence's first, pages shared with another sequence."""
    rng = np.random.default_rng(4)
    for given in (False, True):
        p = Pair(torch, ctx, 1, 10, 1, 64, 4, 3)
        p.place([64, 100, 3, 0], rng)
        p.gpu.fork(p.ints([1]), p.ints([3]))
        p.cpu.fork([1], [3])
        T = 90
        q, k, v = bf16(rng, (T, 2, 64)), bf16(rng, (T, 1, 64)), bf16(rng, (T, 1, 64))
        off, slots = [2, 42, 47, 50], [3, 2, 9]
        rot, q_out = binding.Rotary(64), torch.full((T, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda")
        pos = np.zeros(T, np.int64)
        pos[2:42], pos[42:47], pos[47:50] = np.arange(60, 100), np.arange(-2, 3), [7, 8, 9]
        dp = torch.from_numpy(pos.astype(np.int32)).cuda()
        p.gpu.append_rotary(0, rot, p.bf(q), p.bf(k), p.bf(v), dp if given else None, p.ints(off), slots=p.ints(slots), q_out=q_out)
        assert ctx.get_status() == binding.ESSA_ERR_CACHE
        turned_q, turned_k = (ctx.rotary(rot, p.bf(x), dp) for x in (q, k))
        p.cpu.append(0, f32(turned_k)[6:42], v[6:42], [0, 36], [3])
        p.cpu.append(0, f32(turned_k)[44:47], v[44:47], [0, 3], [2])
        p.assert_same()
        wrote = np.zeros(T, bool)
        wrote[2:50] = True
        if not given:
            wrote[[42, 43, 47, 48, 49]] = False  # rows whose position nobody knows
        assert torch.equal(q_out[wrote], turned_q[wrote]) and (q_out[~wrote] == 9).all()


def test_append_rotary_with_many_entries_and_without_offsets(torch, ctx):
    """More entries than a thread block keeps offsets of; one row per entry without offsets."""
    n, d = 2500, 64
    rng = np.random.default_rng(6)
    p, other = (Pair(torch, ctx, 1, n + 2, 1, d, n, 1) for _ in range(2))
    rows = rng.integers(0, 3, n)
    T = int(rows.sum())
    rot = binding.Rotary(d)
    for c in (p, other):
        c.gpu.grow(None, c.ints(rows))
    q, k, v = (p.bf(bf16(rng, (T, h, d))) for h in (2, 1, 1))
    off = p.ints(np.concatenate([[0], np.cumsum(rows)]))
    pos = torch.from_numpy(np.concatenate([np.arange(r) for r in rows]).astype(np.int32)).cuda()
    got = p.gpu.append_rotary(0, rot, q, k, v, None, off)
    other.gpu.append(0, ctx.rotary(rot, k, pos), v, off)
    assert torch.equal(got, ctx.rotary(rot, q, pos)) and torch.equal(p.gpu.pages, other.gpu.pages)
    q, k, v = (p.bf(bf16(rng, (n, h, d))) for h in (2, 1, 1))
    one = torch.ones(n, dtype=torch.int32, device="cuda")
    for c in (p, other):
        c.gpu.grow(None, one)
    got = p.gpu.append_rotary(0, rot, q, k, v)
    last = p.gpu.lengths - 1
    other.gpu.append(0, ctx.rotary(rot, k, last), v)
    assert torch.equal(got, ctx.rotary(rot, q, last)) and torch.equal(p.gpu.pages, other.gpu.pages) and ctx.get_status() == 0


def test_append_rotary_refuses(torch, ctx):
    p = Pair(torch, ctx, 1, 2, 2, 64, 2, 1)
    p.place([3, 3], np.random.default_rng(0))
    rot, z = binding.Rotary(64, sections=[16, 16]), lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    q, k, v, pos = z(2, 4, 64), z(2, 2, 64), z(2, 2, 64), torch.zeros((2, 2), dtype=torch.int32, device="cuda")
    g = p.gpu
    for call in (lambda: g.append_rotary(0, rot, z(3, 4, 64), k, v, pos), lambda: g.append_rotary(0, rot, q, z(2, 3, 64), v, pos), lambda: g.append_rotary(0, rot, q, k, v.half(), pos),
                 lambda: g.append_rotary(0, rot, q, k, v, pos[:1]), lambda: g.append_rotary(1, rot, q, k, v, pos), lambda: g.append_rotary(0, binding.Rotary(128), q, k, v),
                 lambda: g.append_rotary(0, rot, q, k, v, pos, q_out=z(2, 3, 64)), lambda: g.append_rotary(0, rot, q, k, v, pos, slots=p.ints([0])),
                 lambda: g.append_rotary(0, rot, z(2, 0), k, v, pos), lambda: g.append_rotary(0, rot, q, k, v, pos.long())):
        with pytest.raises(binding.EssaError):
            call()
    p.assert_same()
    g.append_rotary(0, rot, q[:0], k[:0], v[:0], pos[:, :0])  # nothing to do
    assert ctx.get_status() == 0


# ------------------------------------------------------------------------------------------------ attention
def check_attend(torch, ctx, p, rows, slots, heads, rng, hint, seen, pad=0, layer=0, scale=None, norms=False, **mask):
    """Attention of `rows[i]` new tokens on slots[i], row i of entry e seeing seen[e]; every row checked, rows of no entry untouched."""
    d = p.cpu.shape[3]
    off = pad + np.concatenate([[0], np.cumsum(rows)]).astype(int)
    T = int(off[-1]) + pad
    q = bf16(rng, (T, heads, d))
    out = torch.full((T, heads, d), 5.0, dtype=torch.bfloat16, device="cuda")
    if "tree" in mask:
        full = torch.full((T, mask["tree"].shape[1]), -1, dtype=torch.int32, device="cuda")
        full[pad:T - pad] = mask["tree"]
        mask["tree"] = full
    p.gpu.attend(layer, p.bf(q), p.ints(off), slots=p.ints(slots), max_new=hint, out=out, scale=scale, **mask)
    assert ctx.get_status() == 0
    got = f32(out)
    assert (got[:off[0]] == 5).all() and (got[off[-1]:] == 5).all()
    c = d ** -0.5 if scale is None else scale
    for i, s in enumerate(slots):
        if rows[i] == 0:
            continue
        k, v, codes, sc = p.cpu.sequence(layer, s)
        mine, here = q[off[i]:off[i + 1]], got[off[i]:off[i + 1]]
        assert np.isfinite(here).all()
        want, w = co.attend_seen(mine, k, v, seen[i], c)
        assert (here[~seen[i].any(-1)] == 0).all()
        if norms:
            assert norm_error(here, want).max() <= NORM_LIMIT, (i, s)
        else:
            tol = attend_bound(mine, v, codes, sc, want, w, c, k)
            err = np.abs(here - want)
            assert (err <= tol).all(), (i, s, rows[i], float(np.max(err / tol)))
    return got


SHAPES = [(1, 1, 64), (14, 2, 64), (28, 4, 128), (5, 5, 128), (20, 1, 128)]
LENGTHS, ROWS = [1, 5, 64, 130, 200, 257, 300, 90, 513], [1, 5, 64, 3, 77, 257, 0, 90, 2]


@pytest.mark.parametrize("heads,kv_heads,d", SHAPES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (63, 1), (64, 64), (65, 0), (100, 130), (10 ** 6, 4), (200, 2 ** 31 - 1), (2 ** 31 - 1, 0)])
def test_window_of_decode_steps(torch, ctx, heads, kv_heads, d, window, sinks):
    lengths = [1, 2, 63, 64, 65, 128, 129, 300, 1000]
    rng = np.random.default_rng(heads * 7 + d + window % 1000)
    p = Pair(torch, ctx, 2, 60, kv_heads, d, len(lengths), 17)
    p.place(lengths, rng)
    seen = [co.seen_mask(n, 1, window, sinks) for n in lengths]
    check_attend(torch, ctx, p, [1] * len(lengths), range(len(lengths)), heads, rng, 1, seen, layer=1, window=window, sinks=sinks)


@pytest.mark.parametrize("heads,kv_heads,d", SHAPES)
@pytest.mark.parametrize("hint", [1, 2, 1000])
@pytest.mark.parametrize("window,sinks", [(1, 0), (30, 5), (64, 0), (70, 65)])
def test_window_of_prompts_and_chunks(torch, ctx, heads, kv_heads, d, hint, window, sinks):
    rng = np.random.default_rng(heads + d + hint + window)
    p = Pair(torch, ctx, 1, 45, kv_heads, d, len(LENGTHS), 9)
    p.place(LENGTHS, rng)
    seen = [co.seen_mask(n, r, window, sinks) for n, r in zip(LENGTHS, ROWS)]
    check_attend(torch, ctx, p, ROWS, range(len(LENGTHS)), heads, rng, hint, seen, pad=3, window=window, sinks=sinks)


@pytest.mark.parametrize("hint", [1, 100])
def test_a_window_that_reaches_everything_gives_the_same_bits(torch, ctx, hint):
    """(Where the work is divided alike: one run per row block.)"""
    rng = np.random.default_rng(3)
    p = Pair(torch, ctx, 1, 45, 2, 128, len(LENGTHS), 9)
    p.place(LENGTHS, rng)
    T = sum(ROWS)
    q, off = p.bf(bf16(rng, (T, 14, 128))), p.ints(np.concatenate([[0], np.cumsum(ROWS)]))
    a = p.gpu.attend(0, q, off, max_new=hint)
    b = p.gpu.attend(0, q, off, max_new=hint, window=2 ** 31 - 1, sinks=7)
    assert norm_error(f32(a), f32(b).astype(np.float64)).max() <= NORM_LIMIT


@pytest.mark.parametrize("window,sinks,like", [(2 ** 32 + 5, 0, None), (2 ** 63, 3, None), (5, 2 ** 32 + 1, None), (5, 2 ** 40, None), (5, 0, 5)])
def test_windows_and_first_tokens_beyond_32_bits_are_all_of_them(torch, ctx, window, sinks, like):
    rng = np.random.default_rng(41)
    p = Pair(torch, ctx, 1, 9, 2, 64, 2, 9)
    p.place([70, 200], rng)
    q = p.bf(bf16(rng, (2, 6, 64)))
    a, b = p.gpu.attend(0, q, window=like), p.gpu.attend(0, q, window=window, sinks=sinks)
    assert norm_error(f32(a), f32(b).astype(np.float64)).max() <= NORM_LIMIT
    with pytest.raises(binding.EssaError):
        p.gpu.attend(0, q, window=5, sinks=-2 ** 32)


def test_rotary_refuses_more_heads_than_a_row_has(torch, ctx):
    """Refused on the host: nothing of this size is read."""
    rot, x, pos = binding.Rotary(16), torch.zeros((1, 1, 16), dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    for heads in (2 ** 20 + 1, 2 ** 31 - 1):
        assert ctx.lib.essa_rotary_apply(ctx.handle, rot._ref, x.data_ptr(), 16 * heads, heads, 1, pos.data_ptr(), 1, x.data_ptr(), 16 * heads,
                                         None) == binding.ESSA_ERR_UNSUPPORTED_SHAPE
    p = Pair(torch, ctx, 1, 2, 1, 64, 1, 1)
    p.place([3], np.random.default_rng(0))
    rot, x = binding.Rotary(64), torch.zeros((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    for heads in (2 ** 20 + 1, 2 ** 31 - 1):
        assert ctx.lib.essa_cache_append_rotary(ctx.handle, p.gpu._ref, 0, rot._ref, x.data_ptr(), 64 * heads, heads, x.data_ptr(), 64, x.data_ptr(), 64, 1, None, 0, None, None, 1,
                                                x.data_ptr(), 64 * heads, None) == binding.ESSA_ERR_UNSUPPORTED_SHAPE
    p.assert_same()
    assert ctx.get_status() == 0


@pytest.mark.parametrize("rows,hint", [(1, 1), (37, 64)])
@pytest.mark.parametrize("window,sinks", [(20000, 0), (5000, 1000)])
def test_long_window_is_split_and_joined(torch, ctx, rows, hint, window, sinks):
    rng = np.random.default_rng(rows + sinks)
    p = Pair(torch, ctx, 1, 400, 2, 128, 2, 390)
    p.place([24901, 77], rng)
    seen = [co.seen_mask(24901, rows, window, sinks), co.seen_mask(77, 1, window, sinks)]
    check_attend(torch, ctx, p, [rows, 1], [0, 1], 14, rng, hint, seen, norms=True, window=window, sinks=sinks)
    q = p.bf(bf16(rng, (rows, 14, 128)))
    outs = [p.gpu.attend(0, q, p.ints([0, rows]), max_new=hint, window=window, sinks=sinks) for _ in range(3)]
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("hint", [1, 100])
@pytest.mark.parametrize("window,sinks", [(1, 0), (40, 3), (300, 0)])
def test_rows_that_see_nothing_through_a_window_are_zero(torch, ctx, hint, window, sinks):
    """Empty sequences, and entries with more rows than their sequence has tokens."""
    rng = np.random.default_rng(6)
    p = Pair(torch, ctx, 1, 8, 2, 64, 3, 2)
    p.place([0, 3, 70], rng)
    rows = [2, 40, 100]
    seen = [np.zeros((r, max(n, 0)), bool) for n, r in zip([0, 3, 70], rows)]
    for n, r, s in zip([0, 3, 70], rows, seen):
        s[max(0, r - n):] = co.seen_mask(n, min(n, r), window, sinks)
    got = check_attend(torch, ctx, p, rows, range(3), 8, rng, hint, seen, window=window, sinks=sinks)
    assert (got[:2] == 0).all() and (got[2:39] == 0).all() and (got[39:42] != 0).any()


@pytest.mark.parametrize("hint", [1, 100])
def test_pages_out_of_every_window_may_be_missing(torch, ctx, hint):
    """... and hold anything: their tokens are not read.  A page that a row can see and that is missing is reported."""
    rng = np.random.default_rng(5)
    p = Pair(torch, ctx, 1, 20, 2, 64, 2, 16)
    p.place([1000, 10], rng)
    q, off = p.bf(bf16(rng, (21, 4, 64))), p.ints([0, 20, 21])
    want = p.gpu.attend(0, q, off, max_new=hint, window=100, sinks=70)
    assert ctx.get_status() == 0
    p.gpu.table[0, 2:13] = torch.tensor([-1, 99, -7] + [-1] * 8, dtype=torch.int32)  # the first window begins at 1000 - 20 - 99 = 881, in page 13
    assert torch.equal(p.gpu.attend(0, q, off, max_new=hint, window=100, sinks=70), want) and ctx.get_status() == 0
    p.gpu.attend(0, q, off, max_new=hint, window=150, sinks=70)
    assert ctx.get_status() == binding.ESSA_ERR_CACHE


@pytest.mark.parametrize("hint", [1, 100])
def test_hidden_tokens_of_nan_do_not_matter(torch, ctx, hint):
    """Tokens that do not fit (keys of NaN) before the window, among the other drafts and behind the row."""
    rng = np.random.default_rng(6)
    p = Pair(torch, ctx, 1, 6, 1, 64, 2, 3)
    rows, n = 6, 150
    k, v = bf16(rng, (n, 1, 64)), bf16(rng, (n, 1, 64))
    p.gpu.grow(None, p.ints([n, n]))
    p.cpu.grow([0, 1], [n, n])
    k[[4, 70, 100, 145, 147], 0, 3] = np.nan
    for s in (0, 1):
        p.gpu.append(0, p.bf(k), p.bf(v), p.ints([0, n]), slots=p.ints([s]))
    q = p.bf(bf16(rng, (rows, 4, 64)))
    bad = np.isnan(k[:, 0, 3])
    for window, sinks in ((5, 4), (30, 0), (60, 5), (2, 0), (50, 71)):
        out = np.isnan(f32(p.gpu.attend(0, q, p.ints([0, rows]), max_new=hint, window=window, sinks=sinks)))
        want = (co.seen_mask(n, rows, window, sinks) & bad).any(-1)
        assert (out == want[:, None, None]).all()
    bits, _ = co.ancestors([-1, 0, 0, 2, 1, 3])
    good = p.gpu.tree(p.ints([-1, 0, 0, 2, 1, 3]), p.ints([0, rows]), rows)[0]
    k[[4, 70, 100], 0, 3] = 1.0
    p.gpu.append(0, p.bf(k), p.bf(v), p.ints([0, n]), slots=p.ints([1]))
    out = np.isnan(f32(p.gpu.attend(0, q, p.ints([0, rows]), slots=p.ints([1]), max_new=hint, tree=good)))
    want = (co.seen_mask(n, rows, drafts=bits) & np.isnan(k[:, 0, 3])).any(-1)
    assert want.any() and not want.all() and (out == want[:, None, None]).all() and ctx.get_status() == 0


# ------------------------------------------------------------------------------------------------ trees
def random_tree(rng, n):
    return [-1] + [int(rng.integers(-1, j)) if rng.random() < 0.6 else j - 1 for j in range(1, n)] if n else []


@pytest.mark.parametrize("sizes,words", [([1], 1), ([5, 0, 32, 3], 1), ([33, 64, 1], 2), ([100, 7], 4), ([256, 200, 31], 8)])
def test_tree_bits_and_positions(torch, ctx, sizes, words):
    rng = np.random.default_rng(sum(sizes))
    p = Pair(torch, ctx, 1, 40, 1, 64, len(sizes) + 1, 9)
    lengths = [s + 40 * i for i, s in enumerate(sizes)] + [3]
    p.place(lengths, rng)
    slots = [int(s) for s in rng.permutation(len(sizes))]
    trees = [random_tree(rng, n) for n in sizes]
    pad = 2
    off = pad + np.concatenate([[0], np.cumsum(sizes)])
    T = int(off[-1]) + pad
    parents = p.ints(sum(trees, [99] * pad) + [-9] * pad)
    drafts, positions = (torch.full(s, 7, dtype=torch.int32, device="cuda") for s in ((T, words), (T,)))
    dslots, doff = p.ints(slots), p.ints(off)
    st = ctx.lib.essa_cache_tree(ctx.handle, p.gpu._ref, parents.data_ptr(), T, dslots.data_ptr(), doff.data_ptr(), len(sizes), drafts.data_ptr(), words,
                                 positions.data_ptr(), None)
    assert st == 0 and ctx.get_status() == 0
    got, pos = drafts.cpu().numpy().view(np.uint32), positions.cpu().numpy()
    assert (got[:pad] == 7).all() and (got[T - pad:] == 7).all() and (pos[:pad] == 7).all() and (pos[T - pad:] == 7).all()
    for i, (tree, s) in enumerate(zip(trees, slots)):
        bits, depth = co.ancestors(tree)
        np.testing.assert_array_equal(got[off[i]:off[i + 1]], co.pack_bits(bits, words))
        np.testing.assert_array_equal(pos[off[i]:off[i + 1]], lengths[s] - sizes[i] + depth)
    if max(sizes) > 32 * (words - 1):
        a, b = p.gpu.tree(parents, p.ints(off), max(sizes), slots=p.ints(slots))
        assert torch.equal(a[pad:T - pad], drafts[pad:T - pad]) and torch.equal(b[pad:T - pad], positions[pad:T - pad])
        assert p.gpu.tree(parents, p.ints(off), max(sizes), slots=p.ints(slots), positions=False)[1] is None


def test_trees_that_are_none(torch, ctx):
    """Parents that are not before their children, more rows than bits, a slot outside the cache: reported, nothing else touched."""
    p = Pair(torch, ctx, 1, 4, 1, 64, 2, 2)
    p.place([10, 40], np.random.default_rng(0))
    for tree, as_if in (([-1, 1, 0], [-1, -1, 0]), ([2, 0, 1], [-1, 0, 1]), ([-2, 0, -1], [-1, 0, -1]), ([1 << 30, -(1 << 30), 0], [-1, -1, 0])):
        drafts, pos = p.gpu.tree(p.ints(tree), p.ints([0, 3]), 3)
        assert ctx.get_status() == binding.ESSA_ERR_CACHE
        bits, depth = co.ancestors(as_if)
        np.testing.assert_array_equal(drafts.cpu().numpy().view(np.uint32), co.pack_bits(bits, 1))
        np.testing.assert_array_equal(pos.cpu().numpy(), 7 + depth)
    drafts, pos = p.gpu.tree(p.ints(list(range(-1, 39))), p.ints([0, 40]), 32, slots=p.ints([1]))
    assert ctx.get_status() == binding.ESSA_ERR_CACHE
    assert (drafts[32:] == 0).all() and pos[31] == 31 and (pos[32:] == 0).all() and int(drafts[31, 0]) == -1
    pos = torch.full((2,), 9, dtype=torch.int32, device="cuda")
    one, offs, two, none = p.ints([0]), p.ints([0, 2]), p.ints([-1, 0]), p.ints([5])
    st = ctx.lib.essa_cache_tree(ctx.handle, p.gpu._ref, two.data_ptr(), 2, none.data_ptr(), offs.data_ptr(), 1, drafts.data_ptr(), 1, pos.data_ptr(), None)
    assert st == 0 and ctx.get_status() == binding.ESSA_ERR_CACHE and pos.tolist() == [9, 9] and drafts[:2, 0].tolist() == [1, 3]
    for words, d in ((0, drafts.data_ptr()), (9, drafts.data_ptr()), (1, None), (1, drafts.data_ptr() + 2)):
        assert ctx.lib.essa_cache_tree(ctx.handle, p.gpu._ref, one.data_ptr(), 1, None, None, 1, d, words, None, None) in (binding.ESSA_ERR_INVALID_ARG, binding.ESSA_ERR_UNSUPPORTED_SHAPE)
    for size in (0, 257):
        with pytest.raises(binding.EssaError):
            p.gpu.tree(p.ints([-1]), None, size)
    assert ctx.get_status() == 0


@pytest.mark.parametrize("heads,kv_heads,d", SHAPES)
@pytest.mark.parametrize("hint", [1, 2, 300])
def test_attention_of_trees(torch, ctx, heads, kv_heads, d, hint):
    """Trees behind histories of no token, part of a page, whole pages; as long as their sequence; across pages."""
    sizes, lengths = [1, 5, 30, 33, 64, 7, 150], [1, 5, 94, 200, 128, 71, 190]
    rng = np.random.default_rng(heads + d + hint)
    p = Pair(torch, ctx, 1, 40, kv_heads, d, len(sizes), 4)
    p.place(lengths, rng)
    trees = [random_tree(rng, n) for n in sizes]
    off = p.ints(np.concatenate([[0], np.cumsum(sizes)]))
    drafts, _ = p.gpu.tree(p.ints(sum(trees, [])), off, max(sizes))
    seen = [co.seen_mask(n, r, drafts=co.ancestors(t)[0]) for n, r, t in zip(lengths, sizes, trees)]
    check_attend(torch, ctx, p, sizes, range(len(sizes)), heads, rng, hint, seen, pad=2, tree=drafts)


@pytest.mark.parametrize("hint", [1, 100])
def test_attention_of_any_draft_bits(torch, ctx, hint):
    """Bits that are no tree: drafts that see later ones, or nothing (a row of zeros if there is no history either); bits of drafts that do not exist."""
    rng = np.random.default_rng(9)
    sizes, lengths, words = [40, 6, 20], [40, 200, 21], 3
    p = Pair(torch, ctx, 1, 10, 2, 64, 3, 4)
    p.place(lengths, rng)
    bits = [rng.random((n, n)) < 0.4 for n in sizes]
    bits[0][3] = bits[0][39] = bits[1][2] = False
    packed = np.concatenate([co.pack_bits(np.pad(b, ((0, 0), (0, 96 - len(b)))), words) for b in bits])
    packed[40:46, 1:] = 0xffffffff  # (drafts that the entry does not have)
    packed[46:, 2] = 0x80000001
    seen = [co.seen_mask(n, r, drafts=b) for n, r, b in zip(lengths, sizes, bits)]
    tree = torch.from_numpy(packed.view(np.int32)).cuda()
    got = check_attend(torch, ctx, p, sizes, range(3), 6, rng, hint, seen, pad=1, tree=tree)
    assert (got[[4, 40]] == 0).all()


@pytest.mark.parametrize("hint", [1, 100])
def test_drafts_beyond_the_bits_are_seen_by_nobody(torch, ctx, hint):
    rng = np.random.default_rng(10)
    p = Pair(torch, ctx, 1, 4, 1, 128, 1, 2)
    p.place([50], rng)
    bits = np.tril(np.ones((40, 40), bool))
    seen = co.seen_mask(50, 40, drafts=bits)
    seen[:, 10 + 32:] = False
    check_attend(torch, ctx, p, [40], [0], 4, rng, hint, [seen], tree=torch.from_numpy(co.pack_bits(bits, 1).view(np.int32)).cuda())
    # more rows than the sequence has tokens: drafts before the first token do not exist
    p.place([0], rng)
    p.cpu.lengths[0] = 30
    p.cpu.table[0, 0], p.cpu.refs[:] = 1, [0, 1, 0, 0]
    p.cpu.codes[0, 1], p.cpu.scale[0, 1], p.cpu.low[0, 1] = rng.integers(0, 16, p.cpu.codes[0, 1].shape), 0.3, -2
    p.push()
    wide = co.seen_mask(40, 40, drafts=bits)[:, 10:]  # (draft j is token j - 10)
    wide[:, 22:] = False
    check_attend(torch, ctx, p, [40], [0], 4, rng, hint, [wide], tree=torch.from_numpy(co.pack_bits(bits, 1).view(np.int32)).cuda())


@pytest.mark.parametrize("heads,kv_heads,d", [(14, 2, 64), (20, 1, 128)])
@pytest.mark.parametrize("hint", [1, 100])
@pytest.mark.parametrize("window,sinks", [(64, 0), (64, 3), (100, 64), (250, 1)])
def test_trees_through_a_window(torch, ctx, heads, kv_heads, d, hint, window, sinks):
    sizes, lengths = [1, 5, 30, 64, 7], [1, 300, 94, 500, 71]
    rng = np.random.default_rng(window + d)
    p = Pair(torch, ctx, 1, 40, kv_heads, d, len(sizes), 9)
    p.place(lengths, rng)
    trees = [random_tree(rng, n) for n in sizes]
    drafts, _ = p.gpu.tree(p.ints(sum(trees, [])), p.ints(np.concatenate([[0], np.cumsum(sizes)])), max(sizes))
    seen = [co.seen_mask(n, r, window, sinks, co.ancestors(t)[0]) for n, r, t in zip(lengths, sizes, trees)]
    check_attend(torch, ctx, p, sizes, range(len(sizes)), heads, rng, hint, seen, tree=drafts, window=window, sinks=sinks)


@pytest.mark.parametrize("hint", [1, 100])
def test_bits_of_drafts_that_do_not_exist_do_not_move_a_window(torch, ctx, hint):
    """A row's position counts the drafts that it sees; set bits behind its entry's rows are not among them."""
    rng = np.random.default_rng(40)
    sizes, lengths, words = [5, 40], [300, 500], 2
    p = Pair(torch, ctx, 1, 20, 2, 64, 2, 9)
    p.place(lengths, rng)
    trees = [random_tree(rng, n) for n in sizes]
    bits = [co.ancestors(t)[0] for t in trees]
    packed = np.concatenate([co.pack_bits(b, words) for b in bits])
    packed[:5, 0] |= np.uint32(0xffffffe0)
    packed[:5, 1] = 0xffffffff
    packed[5:, 1] |= np.uint32(0xffffff00)
    for window, sinks in ((64, 0), (100, 70)):
        seen = [co.seen_mask(n, r, window, sinks, b) for n, r, b in zip(lengths, sizes, bits)]
        check_attend(torch, ctx, p, sizes, range(2), 6, rng, hint, seen, tree=torch.from_numpy(packed.view(np.int32)).cuda(), window=window, sinks=sinks)


def test_long_history_of_a_tree_is_split_and_joined(torch, ctx):
    rng = np.random.default_rng(11)
    p = Pair(torch, ctx, 1, 400, 1, 128, 1, 390)
    p.place([24901], rng)
    for size, hint in ((2, 2), (61, 64)):
        tree = random_tree(rng, size)
        drafts, _ = p.gpu.tree(p.ints(tree), p.ints([0, size]), size)
        seen = [co.seen_mask(24901, size, drafts=co.ancestors(tree)[0])]
        check_attend(torch, ctx, p, [size], [0], 7, rng, hint, seen, norms=True, tree=drafts)


def test_masked_attention_refuses(torch, ctx):
    p = Pair(torch, ctx, 1, 2, 1, 64, 1, 1)
    p.place([5], np.random.default_rng(0))
    q, tree = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((3, 1), dtype=torch.int32, device="cuda")
    off = p.ints([0, 3])
    for kw in (dict(window=0), dict(window=-1), dict(window=4, sinks=-1), dict(sinks=-1), dict(tree=tree[:2]), dict(tree=tree.long()), dict(tree=tree.cpu()), dict(tree=tree[:, 0]),
               dict(tree=torch.zeros((3, 9), dtype=torch.int32, device="cuda")), dict(tree=torch.zeros((3, 2), dtype=torch.int32, device="cuda")[:, :1]),
               dict(tree=tree, window=31)):
        with pytest.raises(binding.EssaError):
            p.gpu.attend(0, q, off, max_new=3, **kw)
    p.gpu.attend(0, q, off, max_new=3, tree=tree, window=32)
    assert p.gpu.attend(0, q[:0], p.ints([0]), max_new=3, tree=tree[:0]).shape[0] == 0
    assert ctx.get_status() == 0


# ------------------------------------------------------------------------------------------------ keeping a path
def sorted_picks(rng, rows, count):
    return sorted(int(x) for x in rng.permutation(rows)[:count])


@pytest.mark.parametrize("kv_heads,d,layers", [(1, 64, 1), (3, 128, 2)])
def test_keep_follows_the_model(torch, ctx, kv_heads, d, layers):
    """Random keeps of several sequences among grows, every byte compared."""
    rng = np.random.default_rng(d)
    p = Pair(torch, ctx, layers, 40, kv_heads, d, 6, 8)
    p.place([300, 64, 1, 130, 0, 65], rng)
    p.cpu.codes[:] = rng.integers(0, 16, p.cpu.codes.shape)
    p.cpu.scale[:], p.cpu.low[:] = rng.random(p.cpu.scale.shape), rng.random(p.cpu.scale.shape)
    p.push()
    for step in range(40):
        n = int(rng.integers(1, 7))
        slots = rng.permutation(6)[:n]
        rows = [int(rng.integers(0, min(p.cpu.lengths[s], 256) + 1)) for s in slots]
        counts = [int(rng.integers(0, r + 1)) for r in rows]
        picks = [sorted_picks(rng, r, c) for r, c in zip(rows, counts)] if step % 3 else None
        width = max(counts) + int(rng.integers(0, 3))
        table = None if picks is None else torch.full((n, width), 77, dtype=torch.int32, device="cuda")
        for i, x in enumerate(picks or []):
            table[i, :len(x)] = p.ints(x)
        p.gpu.keep(p.ints(counts), p.ints(np.concatenate([[0], np.cumsum(rows)])), table, slots=p.ints(slots))
        co.keep(p.cpu, slots, rows, counts, None if picks is None else [list(x) + [77] * (width - len(x)) for x in picks])
        assert ctx.get_status() == 0
        p.assert_same()
        more = rng.integers(0, 120, 6)
        try:
            p.cpu.grow(range(6), more)
            p.gpu.grow(None, p.ints(more))
        except co.Refused:
            pass


def test_keep_of_whole_trees_and_without_offsets(torch, ctx):
    """256 drafts over five pages; everything kept, nothing kept; a step taken back without offsets; a long end cut off."""
    rng = np.random.default_rng(2)
    p = Pair(torch, ctx, 1, 20, 1, 64, 3, 8)
    p.place([319, 500, 256], rng)
    picks = [list(range(256)), list(range(1, 256)), [255]]
    t = torch.zeros((3, 256), dtype=torch.int32, device="cuda")
    for i, x in enumerate(picks):
        t[i, :len(x)] = p.ints(x)
    p.gpu.keep(p.ints([256, 255, 1]), p.ints([0, 256, 512, 768]), t)
    co.keep(p.cpu, [0, 1, 2], [256] * 3, [256, 255, 1], picks)
    p.assert_same()
    p.gpu.keep(p.ints([0, 1]), slots=p.ints([0, 1]))  # the last token of sequence 0 goes
    co.keep(p.cpu, [0, 1], [1, 1], [0, 1])
    p.assert_same()
    p.gpu.keep(p.ints([5]), p.ints([0, 499]), slots=p.ints([1]))
    co.keep(p.cpu, [1], [499], [5])
    p.assert_same()
    p.gpu.keep(p.ints([0]), p.ints([3, 4]), torch.zeros((1, 0), dtype=torch.int32, device="cuda"), slots=p.ints([2]))
    co.keep(p.cpu, [2], [1], [0], [[]])
    p.assert_same()
    p.gpu.keep(p.ints([]), p.ints([0]), slots=p.ints([]))
    assert ctx.get_status() == 0


def test_keep_gives_up_its_share_of_shared_pages(torch, ctx):
    """A fork shares full pages: an end that lies on them is given up, the other sequence keeps it; tokens are not moved onto them."""
    rng = np.random.default_rng(3)
    p = Pair(torch, ctx, 2, 12, 1, 64, 3, 4)
    p.place([200, 0, 10], rng)
    for c in (p.gpu, ):
        c.fork(p.ints([0]), p.ints([1]))
    p.cpu.fork([0], [1])
    p.gpu.keep(p.ints([2]), p.ints([0, 190]), slots=p.ints([1]))
    co.keep(p.cpu, [1], [190], [2])
    p.assert_same()
    assert ctx.get_status() == 0
    before = p.gpu.pages.clone()
    p.gpu.keep(p.ints([1]), p.ints([0, 5]), p.ints([2]).reshape(1, 1), slots=p.ints([1]))  # would write token 7 of a page that sequence 0 shares
    assert ctx.get_status() == binding.ESSA_ERR_CACHE
    with pytest.raises(co.Refused):
        co.keep(p.cpu, [1], [5], [1], [[2]])
    p.assert_same()
    assert torch.equal(before, p.gpu.pages)
    p.gpu.keep(p.ints([2]), p.ints([0, 5]), p.ints([0, 1]).reshape(1, 2), slots=p.ints([1]))  # nothing moves
    co.keep(p.cpu, [1], [5], [2], [[0, 1]])
    p.assert_same()


@pytest.mark.parametrize("what", ["slot-twice", "slot-outside", "too-many-rows", "negative-rows", "count-negative", "count-above-rows", "picks-equal", "picks-descend", "picks-outside",
                                  "picks-negative", "count-above-width", "too-many-drafts", "bad-page", "free-page", "bad-length"])
def test_keeps_that_are_refused_change_nothing(torch, ctx, what):
    rng = np.random.default_rng(1)
    p = Pair(torch, ctx, 1, 12, 1, 64, 4, 6)
    p.place([70, 20, 300, 10], rng)
    slots, off, counts, picks = [1, 0], [0, 8, 16], [2, 3], [[1, 2, 0], [0, 4, 7]]
    if what == "slot-twice":
        slots = [1, 1]
    elif what == "slot-outside":
        slots = [1, 4]
    elif what == "too-many-rows":
        off = [0, 21, 24]
    elif what == "negative-rows":
        off = [0, 8, 6]
    elif what == "count-negative":
        counts = [2, -1]
    elif what == "count-above-rows":
        counts = [9, 3]
    elif what == "picks-equal":
        picks[1] = [0, 4, 4]
    elif what == "picks-descend":
        picks[0] = [2, 1, 0]
    elif what == "picks-outside":
        picks[1] = [0, 4, 8]
    elif what == "picks-negative":
        picks[1] = [-1, 4, 7]
    elif what == "count-above-width":
        counts = [2, 4]
    elif what == "too-many-drafts":
        slots, off = [1, 2], [0, 8, 265]
    elif what == "bad-page":
        p.cpu.table[0, 1] = 12
    elif what == "free-page":
        p.cpu.refs[p.cpu.table[0, 1]] = 0
    elif what == "bad-length":
        p.cpu.lengths[0] = 6 * 64 + 1
    p.push()
    p.gpu.keep(p.ints(counts), p.ints(off), p.ints(picks).reshape(2, 3), slots=p.ints(slots))
    assert ctx.get_status() == binding.ESSA_ERR_CACHE
    p.assert_same()


def test_keep_refuses_on_the_host(torch, ctx):
    p = Pair(torch, ctx, 1, 4, 1, 64, 2, 2)
    p.place([70, 20], np.random.default_rng(1))
    c, off = p.ints([1, 1]), p.ints([0, 4, 8])
    for call in (lambda: p.gpu.keep(c, p.ints([0, 4])), lambda: p.gpu.keep(c, off, p.ints([0, 0])), lambda: p.gpu.keep(c, off, p.ints([0]).reshape(1, 1)),
                 lambda: p.gpu.keep(c.long(), off), lambda: p.gpu.keep(c, off, slots=p.ints([0])), lambda: p.gpu.keep(p.ints([1, 1, 1]), p.ints([0, 1, 2, 3])),
                 lambda: p.gpu.keep(c, off, torch.zeros((2, 4), dtype=torch.int32, device="cuda")[:, :2])):
        with pytest.raises(binding.EssaError):
            call()
    lib, ws = ctx.lib, torch.empty(256 + 64, dtype=torch.uint8, device="cuda")
    args = lambda **k: (ctx.handle, p.gpu._ref, None, off.data_ptr(), k.get("c", c.data_ptr()), None, k.get("ld", 0), k.get("n", 2), k.get("ws", ws.data_ptr()), k.get("b", 320), None)
    for k in (dict(c=None), dict(n=-1), dict(n=3), dict(ws=None), dict(ws=ws.data_ptr() + 8), dict(b=319)):
        assert lib.essa_cache_keep(*args(**k)) == binding.ESSA_ERR_INVALID_ARG, k
    p.assert_same()
    assert ctx.get_status() == 0


# ------------------------------------------------------------------------------------------------ together
def draft_round(torch, p, model, rng, rot, freq, heads, slots, sizes, steps):
    """Drafting rounds as a program makes them: grow by the drafts, their tree, rotate and append, attend, keep a path; checked against the model each time."""
    layers, _, kv_heads, d = p.cpu.shape
    for _ in range(steps):
        trees = [random_tree(rng, n) for n in sizes]
        off = np.concatenate([[0], np.cumsum(sizes)])
        T = int(off[-1])
        p.gpu.grow(p.ints(slots), p.ints(sizes))
        p.cpu.grow(slots, sizes)
        drafts, positions = p.gpu.tree(p.ints(sum(trees, [])), p.ints(off), max(sizes), slots=p.ints(slots))
        for layer in range(layers):
            q, k, v = (bf16(rng, (T, h, d)) for h in (heads, kv_heads, kv_heads))
            turned = p.gpu.append_rotary(layer, rot, p.bf(q), p.bf(k), p.bf(v), positions, p.ints(off), slots=p.ints(slots))
            out = f32(p.gpu.attend(layer, turned, p.ints(off), slots=p.ints(slots), max_new=max(sizes), tree=drafts))
            pos = positions.cpu().numpy()[None]
            want_q, want_k = (co.rotate(x, pos, freq, [0] * (d // 2)) for x in (q, k))
            assert (np.abs(f32(turned) - want_q) <= rotate_bound(q, want_q, False, 1.0)).all()
            # (a key whose rounding to bf16 the 2^-21 above can turn is stored as the GPU has it)
            stored = f32(p.gpu.ctx.rotary(rot, p.bf(k), positions))
            assert (np.abs(stored - want_k) <= rotate_bound(k, want_k, False, 1.0)).all()
            p.cpu.append(layer, stored, v, off, slots)
            for i, s in enumerate(slots):
                kk, vv, codes, sc = p.cpu.sequence(layer, s)
                mine = f32(turned)[off[i]:off[i + 1]]
                bits, depth = co.ancestors(trees[i])
                assert (pos[0, off[i]:off[i + 1]] == p.cpu.lengths[s] - sizes[i] + depth).all()
                want, w = co.attend_seen(mine, kk, vv, co.seen_mask(int(p.cpu.lengths[s]), sizes[i], drafts=bits), d ** -0.5)
                assert (np.abs(out[off[i]:off[i + 1]] - want) <= attend_bound(mine, vv, codes, sc, want, w, d ** -0.5, kk)).all()
        picks = []
        for tree in trees:  # a path from the history on
            path, at = [], -1
            while True:
                below = [j for j, up in enumerate(tree) if up == at]
                if not below or rng.random() < 0.3:
                    break
                at = int(rng.choice(below))
                path.append(at)
            picks.append(path)
        counts = [len(x) for x in picks]
        table = torch.zeros((len(slots), max(sizes)), dtype=torch.int32, device="cuda")
        for i, x in enumerate(picks):
            table[i, :len(x)] = p.ints(x)
        p.gpu.keep(p.ints(counts), p.ints(off), table, slots=p.ints(slots))
        co.keep(p.cpu, slots, sizes, counts, [x + [0] * (max(sizes) - len(x)) for x in picks])
        p.assert_same()


@pytest.mark.parametrize("heads,kv_heads,d,sizes", [(4, 2, 64, [5, 1, 12]), (6, 1, 128, [33, 20, 7])])
def test_rounds_of_drafts(torch, ctx, heads, kv_heads, d, sizes):
    rng = np.random.default_rng(d)
    p = Pair(torch, ctx, 2, 30, kv_heads, d, 4, 7)
    p.place([100, 3, 64, 200], rng)
    freq = 1e4 ** (-np.arange(d // 2) * 2 / d)
    draft_round(torch, p, None, rng, binding.Rotary(d, base=1e4), freq, heads, [2, 0, 3], sizes, 4)
    assert ctx.get_status() == 0


def test_a_run_between_the_projections_is_captured_and_replayed(torch, ctx):
    """grow, tree, append_rotary, masked attention and keep in one graph, replayed beside an eager run of the same on another cache: the same state and results."""
    rng = np.random.default_rng(21)
    heads, kv_heads, d, n = 8, 2, 128, 3
    a, b = (Pair(torch, ctx, 1, 30, kv_heads, d, n, 6) for _ in range(2))
    for c in (a, b):
        c.place([70, 128, 5], np.random.default_rng(1))
    sizes = [9, 4, 20]
    off, slots, count = a.ints(np.concatenate([[0], np.cumsum(sizes)])), a.ints([0, 1, 2]), a.ints(sizes)
    T = sum(sizes)
    parents = a.ints(sum((random_tree(rng, s) for s in sizes), []))
    picks, kept = a.ints([[0, 3, 0], [1, 2, 3], [5, 0, 0]]).reshape(3, 3), a.ints([2, 3, 1])
    rot = binding.Rotary(d, base=1e6)
    q, k, v = (torch.empty((T, h, d), dtype=torch.bfloat16, device="cuda") for h in (heads, kv_heads, kv_heads))

    def step(g):
        g.grow(slots, count)
        drafts, pos = g.tree(parents, off, max(sizes), slots=slots)
        turned = g.append_rotary(0, rot, q, k, v, pos, off, slots=slots)
        out = g.attend(0, turned, off, slots=slots, max_new=max(sizes), tree=drafts)
        win = g.attend(0, turned, off, slots=slots, max_new=max(sizes), window=40, sinks=2)
        g.keep(kept, off, picks, slots=slots)
        return out, win

    side = torch.cuda.Stream()
    state = [t.clone() for t in (a.gpu.pages, a.gpu.table, a.gpu.lengths, a.gpu.refs)]
    with torch.cuda.stream(side):
        for x in (q, k, v):
            x.normal_()
        step(a.gpu)  # warm-up
        for t, s in zip((a.gpu.pages, a.gpu.table, a.gpu.lengths, a.gpu.refs), state):
            t.copy_(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        outs = step(a.gpu)
    for t, s in zip((a.gpu.pages, a.gpu.table, a.gpu.lengths, a.gpu.refs), state):
        t.copy_(s)
    for _ in range(5):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, device="cuda"))
        graph.replay()
        want = step(b.gpu)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, want))
        for name in ("pages", "table", "lengths", "refs"):
            assert torch.equal(getattr(a.gpu, name), getattr(b.gpu, name)), name
    assert ctx.get_status() == 0


def test_two_graphs_at_once(torch, ctx):
    """Two masked calls captured on one stream, replayed side by side on two: each has a workspace of its own (both are joined from parts)."""
    rng = np.random.default_rng(23)
    p = Pair(torch, ctx, 1, 700, 2, 128, 2, 340)
    p.place([20001, 19000], rng)
    tree = p.gpu.tree(p.ints([-1, 0, 0, 2, 1, 3, 3, -1]), p.ints([0, 8]), 8, slots=p.ints([0]))[0]
    q, off, a, b = p.bf(bf16(rng, (8, 14, 128))), p.ints([0, 8]), p.ints([0]), p.ints([1])
    calls = [lambda: p.gpu.attend(0, q, off, slots=a, max_new=8, tree=tree), lambda: p.gpu.attend(0, q[:1], off[:2] // 8, slots=b, window=15000, sinks=70),
             lambda: p.gpu.attend(0, q, off, slots=b, max_new=8, window=18000, sinks=1)]
    want = [f() for f in calls]
    side, streams, graphs, outs = torch.cuda.Stream(), [torch.cuda.Stream() for _ in calls], [], []
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        [f() for f in calls]
    torch.cuda.synchronize()
    for f in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            outs.append(f())
    for _ in range(20):
        for x in outs:
            x.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, want))
    assert ctx.get_status() == 0


def test_on_a_stream_that_is_not_current(torch, ctx):
    """Every call on a stream of its own, while another one is current and busy: the same results, in that stream's order."""
    rng = np.random.default_rng(22)
    heads, kv_heads, d, sizes = 4, 2, 64, [6, 3]
    a, b = (Pair(torch, ctx, 1, 10, kv_heads, d, 2, 4) for _ in range(2))
    for c in (a, b):
        c.place([70, 20], np.random.default_rng(1))
    off, T = a.ints([0, 6, 9]), 9
    parents, picks, kept = a.ints([-1, 0, 0, 1, 2, -1, -1, 0, 1]), a.ints([[2, 4], [0, 0]]).reshape(2, 2), a.ints([2, 1])
    q, k, v = (a.bf(bf16(rng, (T, h, d))) for h in (heads, kv_heads, kv_heads))
    rot, st = binding.Rotary(d), torch.cuda.Stream()
    torch.cuda.synchronize()
    results = []
    for c, kw in ((a, {}), (b, {"stream": st})):
        if kw:
            torch.cuda._sleep(2_000_000)
        g = c.gpu
        g.grow(None, c_sizes := c.ints(sizes)) if not kw else (torch.cuda.synchronize(), g.grow(None, c_sizes := c.ints(sizes), **kw))
        drafts, pos = g.tree(parents, off, 6, **kw)
        turned = g.append_rotary(0, rot, q, k, v, pos, off, **kw)
        out = g.attend(0, turned, off, max_new=6, tree=drafts, **kw)
        again = ctx.rotary(rot, q, pos, **kw)
        g.keep(kept, off, picks, **kw)
        torch.cuda.synchronize()
        results.append((drafts, pos, turned, out, again, g.pages, g.table, g.lengths, g.refs))
    for x, y in zip(*results):
        assert torch.equal(x, y)
    assert torch.equal(results[0][2], results[0][4]) and ctx.get_status() == 0


def test_pages_beyond_32_bits(torch, ctx):
    """A pool of more than 2^32 bytes: rotated tokens are stored, attended to and moved at their own addresses."""
    kv_heads, d = 8, 128
    page_bytes = 72 * kv_heads * d
    pages = (1 << 32) // page_bytes + 40
    g = ctx.kv_cache(1, pages, kv_heads, d, 2, 4)
    rng = np.random.default_rng(3)
    ints = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    g.refs[:pages - 6] = 1
    g.grow(ints([0]), ints([150]))
    q, k, v = (to_dev(torch, bf16(rng, (150, h, d)), torch.bfloat16) for h in (16, kv_heads, kv_heads))
    off, rot = ints([0, 150]), binding.Rotary(d)
    turned = g.append_rotary(0, rot, q, k, v, None, off, slots=ints([0]))
    rk, rv = g.read(0, off, 150, slots=ints([0]))
    pos = torch.arange(150, dtype=torch.int32, device="cuda")
    want = wl.round_to_bf16(co.dequantize(*co.quantize(f32(ctx.rotary(rot, k, pos)))).astype(np.float32))
    np.testing.assert_array_equal(f32(rk), want)
    out = g.attend(0, turned[149:], ints([0, 1]), slots=ints([0]), window=80, sinks=3)
    vals = [np.moveaxis(f32(x).astype(np.float64), 0, 1) for x in (rk, rv)]
    ref, _ = co.attend_seen(f32(turned[149:]), *vals, co.seen_mask(150, 1, 80, 3), d ** -0.5)
    assert norm_error(f32(out), ref).max() <= 2 * NORM_LIMIT  # (the values that were read back are rounded to bf16 too)
    g.keep(ints([3]), ints([0, 60]), ints([[5, 40, 59]]).reshape(1, 3), slots=ints([0]))
    k3, v3 = g.read(0, ints([0, 3]), 3, slots=ints([0]))
    assert torch.equal(k3, rk[[95, 130, 149]]) and torch.equal(v3, rv[[95, 130, 149]]) and g.lengths.tolist() == [93, 0]
    assert g.table[0].tolist() == [pages - 6, pages - 5, -1, -1] and ctx.get_status() == 0


def test_more_elements_than_32_bits(torch, ctx):
    """q of more than 2^31 elements: the last rows are turned, attended to and written at their own addresses."""
    heads, kv_heads, d, T = 64, 1, 128, (1 << 18) + 300
    rng = np.random.default_rng(31)
    g = ctx.kv_cache(1, T // 64 + 1, kv_heads, d, 1, T // 64 + 1)
    ints = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    q = torch.empty((T, heads, d), dtype=torch.bfloat16, device="cuda")
    assert q.numel() > 1 << 31
    some = to_dev(torch, bf16(rng, (300, heads, d)), torch.bfloat16)
    q.copy_(some[:1].expand_as(q))
    q[-300:] = some
    rot, pos = binding.Rotary(d, base=1e4), torch.arange(T, dtype=torch.int32, device="cuda")
    k, v = (torch.randn((T, kv_heads, d), device="cuda").bfloat16() for _ in range(2))
    g.grow(None, ints([T]))
    out = g.append_rotary(0, rot, q, k, v, None, ints([0, T]), q_out=q)
    assert torch.equal(q[-300:], ctx.rotary(rot, some, pos[-300:])) and torch.equal(ctx.rotary(rot, out, -pos)[-300:], ctx.rotary(rot, out[-300:], -pos[-300:]))
    want = g.attend(0, q[-300:], ints([0, 300]), max_new=300, window=90, sinks=5)
    got = g.attend(0, out, ints([0, T]), max_new=T, window=90, sinks=5)
    assert ctx.get_status() == 0
    # (row blocks begin at other rows: other tiles, the same numbers but for their roundings)
    assert norm_error(f32(got[-300:]), f32(want).astype(np.float64)).max() <= 2 * NORM_LIMIT
    kk, vv = g.read(0, ints([0, T]), T)
    vals = [np.moveaxis(f32(torch.cat([x[:5], x[-90:]])).astype(np.float64), 0, 1) for x in (kk, vv)]
    ref, _ = co.attend_seen(f32(q[-1:]), *vals, np.ones((1, 95), bool), d ** -0.5)
    assert norm_error(f32(got[-1:]), ref).max() <= 2 * NORM_LIMIT  # (the values that were read back are rounded to bf16 too)
