"""GPU tests of calls around the key / value cache that meet one another: sequences shortened into pages that others share and grown again, pages that
have left every window, padded batches, far positions, masks that hide nothing."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from paper_2507_04453_b200 import binding
from tests.cache_utils import Pair, attend_bound, bf16
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


# ------------------------------------------------------------------------------------------------ shortened into a shared page
def fork(p, src, dst, lens=None):
    p.gpu.fork(p.ints(src), p.ints(dst), p.ints(lens))
    p.cpu.fork(src, dst, lens)


def shorten(p, slots, lengths):
    """The sequences slots[i] to lengths[i] tokens."""
    rows = [int(p.cpu.lengths[s]) for s in slots]
    p.gpu.keep(p.ints(lengths), p.ints(np.concatenate([[0], np.cumsum(rows)])), slots=p.ints(slots))
    co.keep(p.cpu, slots, rows, lengths)


def grow_and_append(p, rng, slots, counts):
    p.gpu.grow(p.ints(slots), p.ints(counts))
    p.cpu.grow(slots, counts)
    off = np.concatenate([[0], np.cumsum(counts)])
    layers, _, kv_heads, d = p.cpu.shape
    for layer in range(layers):
        k, v = bf16(rng, (off[-1], kv_heads, d)), bf16(rng, (off[-1], kv_heads, d))
        p.gpu.append(layer, p.bf(k), p.bf(v), p.ints(off), slots=p.ints(slots))
        p.cpu.append(layer, k, v, off, slots)


@pytest.mark.parametrize("kv_heads,d", [(1, 64), (3, 128)])
@pytest.mark.parametrize("end,add", [(12, 1), (63, 1), (63, 2), (65, 5), (100, 130), (64, 3), (128, 1), (0, 7), (190, 10)])
def test_a_sequence_shortened_into_a_shared_page_grows_on_a_copy_of_it(torch, ctx, kv_heads, d, end, add):
    """What both sequences hold and what is attended to afterwards is the model's; tokens go to the page of the one that grows."""
    rng = np.random.default_rng(end + d)
    p = Pair(torch, ctx, 2, 14, kv_heads, d, 3, 6)
    p.place([200, 0, 10], rng)
    fork(p, [0], [1])
    shorten(p, [1], [end])
    p.assert_same()
    grow_and_append(p, rng, [1, 2], [add, 3])
    p.assert_same()
    assert ctx.get_status() == 0
    q = bf16(rng, (2, 2 * kv_heads, d))
    for layer in range(2):
        out = f32(p.gpu.attend(layer, p.bf(q), slots=p.ints([1, 0])))
        for i, s in enumerate((1, 0)):
            k, v, codes, sc = p.cpu.sequence(layer, s)
            want, w = co.attend(q[i:i + 1], k, v, int(p.cpu.lengths[s]), d ** -0.5)
            assert (np.abs(out[i:i + 1] - want) <= attend_bound(q[i:i + 1], v, codes, sc, want, w, d ** -0.5, k)).all()
    assert ctx.get_status() == 0


def test_sequences_that_end_in_the_same_page_grow_together(torch, ctx):
    """Three of four sequences shortened into one page and grown by one call each get a copy; one that does not grow keeps its share; the last
    holder of a page needs none; a page that nobody holds any more is free."""
    rng = np.random.default_rng(1)
    p = Pair(torch, ctx, 2, 20, 2, 64, 5, 4)
    p.place([130, 0, 0, 0, 64], rng)
    fork(p, [0, 0, 0], [1, 2, 3])
    shorten(p, [0, 1, 2, 3], [70, 90, 127, 100])
    p.assert_same()
    grow_and_append(p, rng, [2, 4, 0, 1, 3], [1, 70, 60, 0, 2])  # (sequence 1 stays as it is)
    p.assert_same()
    assert p.cpu.refs[p.cpu.table[1, 1]] == 1
    before = int(p.cpu.table[1, 1])
    grow_and_append(p, rng, [1], [3])
    p.assert_same()
    assert int(p.cpu.table[1, 1]) == before
    shorten(p, [0, 3], [10, 20])  # page 0 of all four
    grow_and_append(p, rng, [3, 0], [1, 1])
    p.assert_same()
    shorten(p, [1, 2], [33, 34])
    grow_and_append(p, rng, [1, 2], [1, 1])  # both, though the second could have had the page itself
    p.assert_same()
    assert ctx.get_status() == 0


def test_growing_on_a_copy_needs_a_page_for_it(torch, ctx):
    """Too few pages with the copy among them: refused, nothing changes; enough for the rest after another sequence has gone."""
    rng = np.random.default_rng(2)
    p = Pair(torch, ctx, 1, 4, 1, 64, 3, 4)
    p.place([130, 0, 0], rng)
    fork(p, [0], [1])  # pages: two shared, two of their own
    shorten(p, [1], [100])
    fork(p, [0], [2], [64])
    grow_and_append(p, rng, [2], [1])  # the page that the shortened one gave back
    p.gpu.grow(p.ints([1]), p.ints([1]))
    assert ctx.get_status() == binding.ESSA_ERR_CACHE
    with pytest.raises(co.Refused):
        p.cpu.grow([1], [1])
    p.assert_same()
    p.gpu.free(p.ints([0]))
    p.cpu.free([0])
    grow_and_append(p, rng, [1], [1])
    p.assert_same()
    assert ctx.get_status() == 0


def test_more_sequences_than_threads_grow_on_copies(torch, ctx):
    rng = np.random.default_rng(3)
    n = 1500
    p = Pair(torch, ctx, 1, 2 * n + 10, 1, 64, n + 1, 3)
    p.place([64] + [0] * n, rng)
    others = list(range(1, n + 1))
    fork(p, [0] * n, others)
    shorten(p, others, [int(x) for x in rng.integers(1, 65, n)])
    counts = [int(x) for x in rng.integers(0, 90, n)]
    order = [int(s) for s in 1 + rng.permutation(n)]
    grow_and_append(p, rng, order, counts)
    p.assert_same()
    assert ctx.get_status() == 0


def test_a_captured_growth_copies_when_it_is_replayed(torch, ctx):
    """The graph is captured while no end is shared, and replayed when one is."""
    rng = np.random.default_rng(4)
    p = Pair(torch, ctx, 2, 14, 2, 64, 2, 4)
    p.place([150, 0], rng)
    slots, counts = p.ints([1]), p.ints([1])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        p.gpu.grow(slots, counts)
    torch.cuda.current_stream().wait_stream(stream)
    fork(p, [0], [1])
    shorten(p, [1], [70])
    for _ in range(3):
        graph.replay()
        p.cpu.grow([1], [1])
        p.assert_same()
    assert ctx.get_status() == 0


# ------------------------------------------------------------------------------------------------ pages that no draft sees
@pytest.mark.parametrize("hint", [1, 100])
@pytest.mark.parametrize("past,window,sinks,gone", [(127, 64, 0, [0]), (127, 64, 1, []), (319, 128, 70, [2]), (255, 64, 0, [0, 1, 2]), (256, 64, 0, [0, 1, 2])])
def test_pages_that_no_draft_sees_may_be_missing(torch, ctx, hint, past, window, sinks, gone):
    """A tree's first draft sees the tokens from past - window + 1 on: a page that ends right before that one may be missing, and no other."""
    rng = np.random.default_rng(past)
    sizes = [5, 20]
    p = Pair(torch, ctx, 1, 24, 2, 64, 2, 7)
    p.place([past + 5, past + 20], rng)
    trees = [[-1, 0, 0, 1, -1], [-1] + list(range(19))]
    off = p.ints([0, 5, 25])
    q = p.bf(bf16(rng, (25, 6, 64)))
    drafts, _ = p.gpu.tree(p.ints(sum(trees, [])), off, 20)
    want = p.gpu.attend(0, q, off, max_new=hint, window=window, sinks=sinks, tree=drafts)
    assert ctx.get_status() == 0
    for s in range(2):
        for j in gone:
            p.gpu.table[s, j] = -1
    assert torch.equal(p.gpu.attend(0, q, off, max_new=hint, window=window, sinks=sinks, tree=drafts), want)
    assert ctx.get_status() == 0
    for s in range(2):
        keep, first = p.gpu.table[s].clone(), (past - window + 1) // 64
        for j in [first] + ([0] if sinks else []):  # (seen by the first draft)
            p.gpu.table[s, j] = 99
            p.gpu.attend(0, q, off, max_new=hint, window=window, sinks=sinks, tree=drafts)
            assert ctx.get_status() == binding.ESSA_ERR_CACHE
            p.gpu.table[s] = keep
    none = drafts.clone()
    none[3] = 0  # a row that sees no draft is at past - 1, and sees a token more
    p.gpu.attend(0, q, off, max_new=hint, window=window, sinks=sinks, tree=none)
    assert ctx.get_status() == (binding.ESSA_ERR_CACHE if (past - window) // 64 in gone else 0)




# ------------------------------------------------------------------------------------------------ padded batches
def test_empty_entries_of_a_tree_need_no_sequence(torch, ctx):
    """A batch padded with entries without rows and slots of -1, as append, attend and read take them."""
    p = Pair(torch, ctx, 1, 4, 1, 64, 2, 2)
    p.place([10, 40], np.random.default_rng(0))
    slots, off, parents = p.ints([1, -1, 0, -1]), p.ints([0, 3, 3, 5, 5]), p.ints([-1, 0, 0, -1, 0])
    drafts, pos = p.gpu.tree(parents, off, 3, slots=slots)
    assert ctx.get_status() == 0
    assert pos.tolist() == [37, 38, 38, 8, 9] and drafts[:, 0].tolist() == [1, 3, 5, 1, 3]
    x = torch.zeros((5, 1, 64), dtype=torch.bfloat16, device="cuda")
    p.gpu.append_rotary(0, binding.Rotary(64), x, x, x, pos, off, slots=slots)
    p.gpu.attend(0, x, off, slots=slots, max_new=3, tree=drafts)
    p.gpu.read(0, off, 5, slots=slots)
    assert ctx.get_status() == 0


# ------------------------------------------------------------------------------------------------ rotation
# Of a pair (a, b): the angle is wrong by the position times 0.51 2^-64 of a turn (2^-30 radians for 2^31); cosine and sine, nearest fp32 numbers of at most 1, by
# 2^-25, and by as much again when they are multiplied with the magnitude; the products and their sum are rounded to fp32 (2^-24 each, of no more than
# magnitude (|a| + |b|)), the result to bf16 (2^-8 of it, or 2^-134 absolutely).  So before bf16 (2^-24 + 2^-30 + 2 2^-24) magnitude (|a| + |b|).
def rotate_bound(x, want, adjacent, magnitude):
    y = np.abs(x.astype(np.float64))
    d = x.shape[-1]
    both = (y[..., 0::2] + y[..., 1::2]) if adjacent else (y[..., :d // 2] + y[..., d // 2:])
    both = np.repeat(both, 2, -1) if adjacent else np.concatenate([both, both], -1)
    return 2.0 ** -8 * np.abs(want) + 3.03 * 2.0 ** -24 * (1 + 2.0 ** -8) * abs(magnitude) * both + 2.0 ** -133


@pytest.mark.parametrize("d,adjacent", [(64, False), (128, True), (48, False)])
@pytest.mark.parametrize("top", [1.0, 1e5, 4e9])
def test_far_positions_of_any_frequency(torch, ctx, d, adjacent, top):
    rng = np.random.default_rng(int(top) + d)
    freq = top * rng.uniform(-1, 1, d // 2)
    pos = np.concatenate([2 ** 31 - 1 - np.arange(20), -2 ** 31 + np.arange(20), rng.integers(-2 ** 31, 2 ** 31, 60)]).astype(np.int32)
    x = bf16(rng, (100, 3, d))
    want = co.rotate(x, pos[None], freq, [0] * (d // 2), adjacent, 0.75)
    got = f32(ctx.rotary(binding.Rotary(d, frequencies=freq, adjacent=adjacent, magnitude=0.75), to_dev(torch, x, torch.bfloat16), torch.from_numpy(pos).cuda()))
    assert (np.abs(got - want) <= rotate_bound(x, want, adjacent, 0.75)).all()


# ------------------------------------------------------------------------------------------------ masks that hide nothing
@pytest.mark.parametrize("heads,kv_heads,d", [(1, 1, 64), (14, 2, 128), (8, 8, 64)])
@pytest.mark.parametrize("hint", [1, 100])
@pytest.mark.parametrize("window,sinks", [(10 ** 6, 7), (513, 0), (1, 10 ** 6), (200, 400)])
def test_a_mask_that_hides_nothing_gives_what_no_mask_gives(torch, ctx, heads, kv_heads, d, hint, window, sinks):
    """The kernels with a mask (a window of 2^31 - 1 would choose those without): the model's values; and the bits of no mask where the work is divided alike,
    which it is but for several row blocks of few rows (without a mask each walks all of the entry's pages)."""
    rng = np.random.default_rng(heads + hint)
    lengths, rows = [1, 5, 64, 130, 200, 257, 300, 90, 513], [1, 5, 64, 3, 77, 257, 0, 90, 2]
    p = Pair(torch, ctx, 1, 45, kv_heads, d, len(lengths), 9)
    p.place(lengths, rng)
    ends = np.concatenate([[0], np.cumsum(rows)])
    q, off = bf16(rng, (sum(rows), heads, d)), p.ints(ends)
    got, want = p.gpu.attend(0, p.bf(q), off, max_new=hint, window=window, sinks=sinks), p.gpu.attend(0, p.bf(q), off, max_new=hint)
    assert hint == 1 or torch.equal(got, want)
    for i, n in enumerate(lengths):
        if rows[i] == 0:
            continue
        k, v, codes, sc = p.cpu.sequence(0, i)
        mine, here = q[ends[i]:ends[i + 1]], f32(got)[ends[i]:ends[i + 1]]
        model, w = co.attend(mine, k, v, n, d ** -0.5)
        assert (np.abs(here - model) <= attend_bound(mine, v, codes, sc, model, w, d ** -0.5, k)).all()
    one = p.bf(bf16(rng, (len(lengths), heads, d)))
    assert torch.equal(p.gpu.attend(0, one, max_new=hint, window=window, sinks=sinks), p.gpu.attend(0, one, max_new=hint))
    assert ctx.get_status() == 0
