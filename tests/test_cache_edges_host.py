"""Host side of calls around the key / value cache that meet one another (no GPU)."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import cache_oracle as co
from paper_2507_04453_b200 import binding

# pi in 60 digits: the angle of 2^32 radians is some 2^96 units of 2^-64 turns, of which it leaves 2^-100
TWO_PI = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494")


def test_the_model_grows_on_a_copy_of_a_shared_page():
    """fork, shorten into a page that both share, grow: a page of its own with the same tokens, and the other sequence's as they were."""
    c, rng = co.Cache(2, 8, 1, 64, 2, 4), np.random.default_rng(0)
    c.grow([0], [150])
    for layer in range(2):
        c.append(layer, *(rng.standard_normal((150, 1, 64)).astype(np.float32) for _ in range(2)), [0, 150], [0])
    c.fork([0], [1])
    co.keep(c, [1], [150], [70])
    shared, before = int(c.table[0, 1]), [c.sequence(layer, 0) for layer in range(2)]
    assert int(c.table[1, 1]) == shared and c.refs[shared] == 2
    c.grow([1], [2])
    assert int(c.table[1, 1]) != shared and c.refs[shared] == c.refs[c.table[1, 1]] == 1 and c.refs[c.table[0, 0]] == 2
    x = rng.standard_normal((2, 1, 64)).astype(np.float32)
    for layer in range(2):
        c.append(layer, x, x, [0, 2], [1])
        for a, b in zip(before[layer], c.sequence(layer, 0)):
            np.testing.assert_array_equal(a, b)
        for a, b in zip(before[layer][:2], c.sequence(layer, 1)[:2]):
            np.testing.assert_array_equal(a[:, :70], b[:, :70])
    c.grow([1], [1])
    assert c.refs.sum() == (c.table >= 0).sum()


@pytest.fixture
def cache():
    """A KvCache on CPU tensors whose library only notes the masks that it is called with."""
    import torch

    class Library:
        masks = []

        def essa_cache_attend_workspace(self, cache, heads, max_new, sms, out):
            out._obj.value = 16
            return binding.ESSA_OK

        def essa_cache_attend(self, *args):
            self.masks.append(None)
            return binding.ESSA_OK

        def essa_cache_attend_masked(self, handle, cache, mask, *args):
            self.masks.append(mask._obj)
            return binding.ESSA_OK

    class Ctx:
        handle = None

    kv, Ctx.torch = binding.KvCache.__new__(binding.KvCache), torch
    kv.ctx, kv._lib, kv._ref, kv.device, kv._index = Ctx, Library(), None, torch.device("cpu"), -1
    kv.head_dim, kv.kv_heads, kv._sms, kv._scale, kv._attend_ws = 64, 1, 148, 0.125, {}
    kv._int32, kv._bf16, kv._empty_like = torch.int32, torch.bfloat16, torch.empty_like
    kv._raw, kv._workspace = lambda stream: None, lambda n, raw, stream: torch.empty(n, dtype=torch.uint8)
    return kv


def test_a_tree_without_words_is_refused(cache):
    """(Not taken for a call without a tree, in which the drafts see one another.)"""
    torch = cache.ctx.torch
    q, off = torch.zeros((3, 2, 64), dtype=torch.bfloat16), torch.tensor([0, 3], dtype=torch.int32)
    for T in (3, 0):
        with pytest.raises(binding.EssaError):
            cache.attend(0, q[:T], off, max_new=3, tree=torch.zeros((T, 0), dtype=torch.int32))
        cache.attend(0, q[:T], off, max_new=3, tree=torch.zeros((T, 1), dtype=torch.int32))
    assert len(cache._lib.masks) == 2 and cache._lib.masks[0].draft_words == 1


def test_a_call_has_a_mask_of_its_own(cache):
    """What one call hands over is not what another makes of it (ctypes lets other threads run before the library reads it)."""
    torch = cache.ctx.torch
    q, off = torch.zeros((3, 2, 64), dtype=torch.bfloat16), torch.tensor([0, 3], dtype=torch.int32)
    tree = torch.zeros((3, 2), dtype=torch.int32)
    cache.attend(0, q, off, max_new=3, window=100, sinks=7, tree=tree)
    cache.attend(0, q, off, max_new=3, window=5, sinks=1)
    first, second = cache._lib.masks
    assert (first.window, first.sinks, first.draft_words, first.drafts) == (100, 7, 2, tree.data_ptr())
    assert (second.window, second.sinks, second.draft_words, second.drafts) == (5, 1, 0, None)


@pytest.mark.parametrize("scale", [0, 10, 20, 31])
def test_turns_are_exact_however_high_the_frequency(scale):
    """The nearest 64-bit fraction of a turn (half a unit, and the hundredth of one that the constant's end may cost)."""
    rng = np.random.default_rng(scale)
    freq = np.ldexp(rng.uniform(1, 2, 128), scale) * rng.choice([-1, 1], 128)
    freq[:5] = 2.0 ** 32, -2.0 ** 32, 2.0 ** 32 - 2.0 ** -20, 5e-324, np.pi * 2.0 ** (scale - 1)
    r = binding.Rotary(256, frequencies=freq)
    for t, f in zip(r.desc.turns, freq):
        want = Fraction(float(f)) / TWO_PI * 2 ** 64
        off = abs(int(t) - want) % 2 ** 64
        assert min(off, 2 ** 64 - off) <= Fraction(51, 100), f


@pytest.mark.parametrize("f", [np.nextafter(2.0 ** 32, np.inf), -1e10, 1e19, 1e300])
def test_frequencies_that_no_position_needs_are_refused(f):
    with pytest.raises(binding.EssaError):
        binding.Rotary(16, frequencies=[0.5] * 7 + [f])
