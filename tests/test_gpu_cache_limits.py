"""GPU tests of the paged 4-bit key / value cache where its limits lie: stored values beyond fp16, tables that are damaged, long sequences."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from paper_2507_04453_b200 import binding
from tests.cache_utils import NORM_LIMIT, Pair, attend_bound, bf16, norm_error

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


# ------------------------------------------------------------------------------------------------ values beyond fp16
# (minimum, scale) on both sides of +-65440: inside, the largest inside, above it, far above it, below it, on both sides
RANGES = [(-2.5, 0.3), (20000, 3028), (-60000, 12000), (0, 65504), (-65504, 4000), (-65504, 12000), (65504, 0), (65440, 0)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hint", [1, 100])
@pytest.mark.parametrize("where", ["k", "v", "both"])
def test_stored_values_beyond_fp16(torch, ctx, where, hint, d):
    """A value beyond +-65440 counts as it is (few rows) or as +-65440 (many rows); its neighbours in the group are what they are."""
    rng = np.random.default_rng(30)
    p = Pair(torch, ctx, 1, 8, 2, d, 2, 4)
    p.place([200, 70], rng)
    for half, name in enumerate("kv"):
        if where not in (name, "both"):
            continue
        kind = rng.integers(0, len(RANGES), p.cpu.scale[:, :, :, half].shape)
        stale = np.isnan(p.cpu.low[:, :, :, half])
        for a, i in ((p.cpu.low, 0), (p.cpu.scale, 1)):
            a[:, :, :, half] = np.where(stale, a[:, :, :, half], np.array(RANGES, np.float16)[kind, i])
        p.cpu.codes[:, :, :, half] = rng.integers(0, 16, p.cpu.codes[:, :, :, half].shape)
    p.push()
    off, q = [0, 30, 60], bf16(rng, (60, 4, d))
    scale = d ** -0.5 / (1 if where == "v" else 2e5)  # (scores of a few units)
    got = p.gpu.attend(0, p.bf(q), p.ints(off), max_new=hint, scale=scale).float().cpu().numpy()
    assert ctx.get_status() == 0 and np.isfinite(got).all()
    for s in range(2):
        k, v, codes, sc = p.cpu.sequence(0, s)
        if hint > 1:
            k, v = np.clip(k, -65440, 65440), np.clip(v, -65440, 65440)
        mine, out = q[off[s]:off[s + 1]], got[off[s]:off[s + 1]]
        want, w = co.attend(mine, k, v, int(p.cpu.lengths[s]), scale)
        err = np.abs(out - want)
        tol = attend_bound(mine, v, codes, sc, want, w, scale, k)
        assert (err <= tol).all(), float(np.max(err / tol))
        assert norm_error(out, want).max() <= NORM_LIMIT, float(norm_error(out, want).max())


# ------------------------------------------------------------------------------------------------ damaged tables
@pytest.mark.parametrize("hint", [1, 100])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,bad", [(1, [0]), (30, [0]), (30, [0, 1]), (20, [0, 2]), (70, [0])])
def test_pages_that_are_not_there_before_scores_far_below_zero(torch, ctx, rows, bad, d, hint):
    """A sequence whose first pages are missing and whose scores all lie where e^score is no fp32 number: the softmax of what is left.  Keys are
    whole numbers and queries multiples of 1/4, so that the scores (-128 and a few units) are sums of numbers that the products hold exactly."""
    rng = np.random.default_rng(31)
    p = Pair(torch, ctx, 1, 20, 1, d, 2, 8)
    p.place([340, 90], rng)
    here = ~np.isnan(p.cpu.low[0, :, :, 0, :, 0])                    # tokens of the two sequences
    codes = rng.integers(0, 16, p.cpu.codes[0, :, :, 0].shape)
    codes[..., np.arange(d) % 64 < 32] = 0                            # half of every group is -8
    p.cpu.codes[0, :, :, 0][here] = codes[here]
    p.cpu.scale[0, :, :, 0][here], p.cpu.low[0, :, :, 0][here] = 1, -8
    p.push()
    p.gpu.table[0, p.ints(bad).long()] = 20
    q = np.where(np.arange(d) % 64 < 32, 4.0, rng.integers(-2, 3, (2 * rows, 4, d)) / 4).astype(np.float32)
    scale = 8 / d
    got = p.gpu.attend(0, p.bf(q), p.ints([0, rows, 2 * rows]), max_new=hint, scale=scale).float().cpu().numpy()
    assert ctx.get_status() == binding.ESSA_ERR_CACHE
    for s, mine, out in ((0, q[:rows], got[:rows]), (1, q[rows:], got[rows:])):
        k, v, codes, sc = p.cpu.sequence(0, s)
        n = k.shape[1]
        keep = np.array([i for i in range(n) if s or i // co.PAGE not in bad])
        for j in range(rows):  # (row by row: the tokens that it sees are not a row's number away from a common end)
            see = keep[keep < n - rows + j + 1]
            want, w = co.attend(mine[j:j + 1], k[:, see], v[:, see], len(see), scale)
            tol = attend_bound(mine[j:j + 1], v[:, see], codes[:, :, see], sc[:, :, see], want, w, scale, k[:, see])
            assert (np.abs(out[j:j + 1] - want) <= tol).all() and norm_error(out[j:j + 1], want).max() <= NORM_LIMIT, (s, j)


def damaged(torch, ctx, entry):
    """Five sequences, two of them on a shared page, and a table entry that names no page in use."""
    p = Pair(torch, ctx, 2, 12, 1, 64, 6, 5)
    p.place([70, 64 + 10, 64, 10, 1, 0], np.random.default_rng(32))
    p.gpu.fork(p.ints([1]), p.ints([5]))
    p.cpu.fork([1], [5])
    free = int(np.flatnonzero(p.cpu.refs == 0)[-1])
    value = {"behind": 12, "far-behind": 1 << 30, "negative": -2, "free": free, "far-negative": -(1 << 31)}[entry]
    return p, value


ENTRIES = ["behind", "far-behind", "negative", "far-negative", "free"]


@pytest.mark.parametrize("entry", ENTRIES)
@pytest.mark.parametrize("at", [(0, 1), (3, 0), (3, 4)])
def test_free_of_a_damaged_row_changes_nothing(torch, ctx, entry, at):
    p, value = damaged(torch, ctx, entry)
    p.cpu.table[at] = value
    p.push()
    p.gpu.free(p.ints([5, 0, 1, 3]))
    assert ctx.get_status() == binding.ESSA_ERR_CACHE
    p.assert_same()
    slots = [s for s in (5, 1, 4) if s != at[0]]  # the other sequences can still be freed
    p.gpu.free(p.ints(slots))
    p.cpu.free(slots)
    assert ctx.get_status() == 0
    p.assert_same()


@pytest.mark.parametrize("n,max_pages", [(1, 1), (1, 5000), (40, 700), (1400, 9), (3000, 40)])
def test_free_sees_damage_in_any_row(torch, ctx, n, max_pages):
    """From one entry to more than the thread blocks look at in one round: refused for a bad entry at the start, in between, at the end; done without."""
    p = Pair(torch, ctx, 1, 9000, 1, 64, n, max_pages)
    rng = np.random.default_rng(n + max_pages)
    counts = rng.integers(0, min(64 * max_pages, 64 * 8000 // n) + 1, n)
    p.gpu.grow(None, p.ints(counts))
    p.cpu.grow(range(n), counts)
    assert ctx.get_status() == 0
    slots = rng.permutation(n)
    for i, j in ((0, 0), (n // 2, max_pages // 2), (n - 1, max_pages - 1), (int(rng.integers(n)), int(rng.integers(max_pages)))):
        at = (slots[i], j)
        keep, p.cpu.table[at] = p.cpu.table[at], 9000
        p.gpu.table.copy_(torch.from_numpy(p.cpu.table))
        p.gpu.free(p.ints(slots))
        assert ctx.get_status() == binding.ESSA_ERR_CACHE
        p.assert_same(pages=False)
        p.cpu.table[at] = keep
    p.gpu.table.copy_(torch.from_numpy(p.cpu.table))
    p.gpu.free(p.ints(slots))
    p.cpu.free(slots)
    assert ctx.get_status() == 0
    p.assert_same(pages=False)


@pytest.mark.parametrize("entry", ENTRIES)
@pytest.mark.parametrize("at", [(0, 1), (3, 0), (3, 4), (4, 0)])
def test_fork_between_damaged_rows_changes_nothing(torch, ctx, entry, at):
    """A source's page (0, 1), a destination's page (3, 0) and what stands behind its pages (3, 4): refused; a row that the fork does not touch: done."""
    p, value = damaged(torch, ctx, entry)
    p.cpu.table[at] = value
    p.push()
    p.gpu.fork(p.ints([0, 1]), p.ints([3, 2]))
    if at[0] == 4:
        p.cpu.fork([0, 1], [3, 2])
        assert ctx.get_status() == 0
    else:
        assert ctx.get_status() == binding.ESSA_ERR_CACHE
    p.assert_same()


def test_fork_looks_only_at_the_pages_that_it_takes(torch, ctx):
    """Damage behind the tokens that are forked does not matter; in the last of them it does."""
    for value in (12, -2):
        p = Pair(torch, ctx, 1, 12, 1, 64, 3, 5)
        p.place([200, 70, 0], np.random.default_rng(33))
        p.cpu.table[0, 3] = value
        p.push()
        p.gpu.fork(p.ints([0]), p.ints([1]), p.ints([192]))
        p.cpu.fork([0], [1], [192])
        assert ctx.get_status() == 0
        p.assert_same()
        p.gpu.fork(p.ints([0]), p.ints([1]), p.ints([193]))
        assert ctx.get_status() == binding.ESSA_ERR_CACHE
        p.assert_same()


@pytest.mark.parametrize("entry", ENTRIES)
@pytest.mark.parametrize("at", [(0, 1), (3, 0), (3, 4), (5, 4)])
def test_compact_of_a_damaged_table_changes_nothing(torch, ctx, entry, at):
    p, value = damaged(torch, ctx, entry)
    p.cpu.table[at] = value
    p.push()
    used = torch.full((1,), -7, dtype=torch.int32, device="cuda")
    for u in (used, None):
        p.gpu.compact(u)
        assert ctx.get_status() == binding.ESSA_ERR_CACHE
        p.assert_same()
    assert int(used) == -7


@pytest.mark.parametrize("n,max_pages", [(1, 1), (1, 5000), (1400, 9), (3000, 120)])
def test_compact_sees_damage_anywhere_in_the_table(torch, ctx, n, max_pages):
    p = Pair(torch, ctx, 1, 9000, 1, 64, n, max_pages)
    rng = np.random.default_rng(n + max_pages)
    counts = rng.integers(0, min(64 * max_pages, 64 * 8000 // n) + 1, n)
    gone = rng.permutation(n)[:n // 2]
    p.gpu.grow(None, p.ints(counts))
    p.cpu.grow(range(n), counts)
    p.gpu.free(p.ints(gone))
    p.cpu.free(gone)
    assert ctx.get_status() == 0
    for at in ((0, 0), (n // 2, max_pages // 2), (n - 1, max_pages - 1), (int(rng.integers(n)), int(rng.integers(max_pages)))):
        keep, p.cpu.table[at] = p.cpu.table[at], 9000
        p.gpu.table.copy_(torch.from_numpy(p.cpu.table))
        p.gpu.compact()
        assert ctx.get_status() == binding.ESSA_ERR_CACHE
        p.assert_same(pages=False)
        p.cpu.table[at] = keep
    p.gpu.table.copy_(torch.from_numpy(p.cpu.table))
    used = torch.zeros(1, dtype=torch.int32, device="cuda")
    p.gpu.compact(used)
    assert int(used) == p.cpu.compact() and ctx.get_status() == 0
    p.assert_same(pages=False)


# ------------------------------------------------------------------------------------------------ long sequences
@pytest.mark.parametrize("heads,kv_heads,d,lengths,rows,hint", [
    (14, 2, 128, [24901, 77], [1, 1], 1), (14, 2, 128, [24901, 77], [2, 1], 2), (14, 2, 128, [24901, 77], [37, 1], 64), (16, 1, 64, [60001], [1], 1),
    (8, 8, 64, [9000, 5000, 3], [1, 1, 1], 1), (10, 2, 128, [5000, 4999, 130], [90, 65, 130], 130), (5, 1, 64, [3000, 2000], [700, 1], 700)])
def test_long_sequences_by_the_norm_of_the_error(torch, ctx, heads, kv_heads, d, lengths, rows, hint):
    """Each row and head by itself: no part of a row block that several thread blocks share is lost, counted twice or taken from another's."""
    rng = np.random.default_rng(len(lengths) * 1000 + heads)
    p = Pair(torch, ctx, 1, sum(co.pages_of(n) for n in lengths) + 3, kv_heads, d, len(lengths), co.pages_of(max(lengths)) + 40)
    p.place(lengths, rng)
    off = np.concatenate([[0], np.cumsum(rows)])
    q = bf16(rng, (int(off[-1]), heads, d))
    got = p.gpu.attend(0, p.bf(q), p.ints(off), max_new=hint).float().cpu().numpy()
    assert ctx.get_status() == 0
    for s in range(len(lengths)):
        k, v, _, _ = p.cpu.sequence(0, s)
        want, _ = co.attend(q[off[s]:off[s + 1]], k, v, lengths[s], d ** -0.5)
        err = norm_error(got[off[s]:off[s + 1]], want)
        assert err.max() <= NORM_LIMIT, (s, float(err.max()))


# ------------------------------------------------------------------------------------------------ scores beyond fp32
@pytest.mark.parametrize("hint", [1, 100])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("up,scale", [(0, 2.0 ** 127), (0, 2.0 ** 60), (60, 2.0 ** 80), (100, 2.0 ** 20), (-100, 2.0 ** 127)])
@pytest.mark.parametrize("width", [30, 40])  # pages of the table: row blocks in one piece, and divided between thread blocks
def test_scores_beyond_fp32_leave_the_largest(torch, ctx, up, scale, d, hint, width):
    """Products of q and k that fp32 holds, and a scale that takes them out of its range (or far enough for one key to have all the weight): the
    values of the keys with the largest product.  Keys are whole numbers and queries multiples of 1/4 times a power of two: products are exact, and
    equal ones are equal."""
    rng = np.random.default_rng(34)
    p = Pair(torch, ctx, 1, 40, 1, d, 2, width)
    p.place([340, 1500], rng)
    here = ~np.isnan(p.cpu.low[0, :, :, 0, :, 0])
    p.cpu.codes[0, :, :, 0][here] = rng.integers(0, 16, p.cpu.codes[0, :, :, 0].shape)[here]
    p.cpu.scale[0, :, :, 0][here], p.cpu.low[0, :, :, 0][here] = 1, -8
    p.push()
    q = (rng.integers(-2, 3, (40, 4, d)) / 4 * 2.0 ** up).astype(np.float32)
    got = p.gpu.attend(0, p.bf(q), p.ints([0, 20, 40]), max_new=hint, scale=scale).float().cpu().numpy()
    assert ctx.get_status() == 0 and np.isfinite(got).all()
    for s in range(2):
        k, v, _, _ = p.cpu.sequence(0, s)
        want, _ = co.attend(q[20 * s:20 * s + 20], k, v, k.shape[1], scale)
        err = norm_error(got[20 * s:20 * s + 20], want)
        assert err.max() <= NORM_LIMIT, (s, float(err.max()))


# ------------------------------------------------------------------------------------------------ graphs
def test_page_operations_captured_into_a_graph(torch, ctx):
    """free, fork, grow and compact in one graph, replayed: each replay is the model's next round, and one that is refused changes nothing."""
    rng = np.random.default_rng(35)
    p = Pair(torch, ctx, 2, 60, 1, 64, 8, 6)
    p.place([200, 70, 64, 10, 130, 0, 300, 1], rng)
    src, dst, gone, more = p.ints([0, 1, 0]), p.ints([3, 4, 5]), p.ints([6]), p.ints([20] * 8)
    used = p.ints([0])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        p.gpu.free(gone)
        p.gpu.fork(src, dst)
        p.gpu.grow(None, more)
        p.gpu.compact(used)
    p.push()
    for step in range(4):
        graph.replay()
        p.cpu.free([6])
        p.cpu.fork([0, 1, 0], [3, 4, 5])
        p.cpu.grow(range(8), [20] * 8)
        assert p.cpu.compact() == int(used) and ctx.get_status() == 0
        p.assert_same()
    p.cpu.table[7, 5] = 60
    p.push()
    gone.fill_(7)
    graph.replay()  # the free and the compact of row 7 are refused, the fork and the growth between them are not
    p.cpu.fork([0, 1, 0], [3, 4, 5])
    p.cpu.grow(range(8), [20] * 8)
    assert ctx.get_status() == binding.ESSA_ERR_CACHE
    p.assert_same()
