"""Host side of the operators around the cache (no GPU): the table of turns, its refusals, workspace sizes, and pins of the model's masks, trees and rotation."""
import ctypes as C
from fractions import Fraction

import numpy as np
import pytest

from oracle import cache_oracle as co
from paper_2507_04453_b200 import binding

TWO_PI = Fraction("6.28318530717958647692528676655900576839433879875021")


def test_turns_are_the_frequencies_in_64_bit_fractions_of_a_turn():
    freq = np.array([1.0, 0.5, 1e-7, 0.0, -0.25, 123456.789, 2 * np.pi, 1e-30])
    r = binding.Rotary(16, frequencies=freq)
    for i, f in enumerate(freq):
        part = Fraction(float(f)) / TWO_PI
        part -= part.numerator // part.denominator
        # long double: the quotient is rounded to 2^-64 of itself, in turns of the whole angle; the fraction is cut to 2^-64
        lim = 1 + abs(Fraction(float(f)) / TWO_PI) * 2
        off = abs(int(r.desc.turns[i]) - part * 2 ** 64)
        assert min(off, 2 ** 64 - off) <= lim, i
    assert list(r.desc.axis)[:8] == [0] * 8 and r.desc.magnitude == 1.0


def test_base_gives_the_usual_frequencies():
    r, f = binding.Rotary(128, base=1e6), [1e6 ** (-2 * i / 128) for i in range(64)]
    got = np.array([float(Fraction(int(t), 2 ** 64) * TWO_PI) for t in list(r.desc.turns)[:64]])
    # (a turn is cut to 2^-64, which is 2 pi 2^-64 radians whatever the frequency)
    np.testing.assert_allclose(got, f, rtol=1e-14, atol=2 * np.pi * 2.0 ** -64)


@pytest.mark.parametrize("sections,interleaved,axis", [
    ([5, 2, 1], False, [0, 0, 0, 0, 0, 1, 1, 2]), ([4, 2, 2], True, [0, 1, 2, 0, 1, 2, 0, 0]), ([8], True, [0] * 8),
    ([0, 8], False, [1] * 8), ([2, 2, 2, 2], True, [0, 1, 2, 3, 0, 1, 2, 3])])
def test_sections_and_turns_of_the_axes(sections, interleaved, axis):
    r = binding.Rotary(16, sections=sections, interleaved=interleaved)
    assert list(r.desc.axis)[:8] == axis and r.axes == len(sections) and r.desc.axes == len(sections)
    assert list(binding.Rotary(16, axis=axis).desc.axis)[:8] == axis


@pytest.mark.parametrize("kw", [dict(head_dim=0), dict(head_dim=24), dict(head_dim=272), dict(head_dim=-16), dict(head_dim=16, base=0.0), dict(head_dim=16, base=float("nan")),
                                dict(head_dim=16, sections=[4, 3]), dict(head_dim=16, sections=[9, -1]), dict(head_dim=16, sections=[2, 2, 2, 1, 1]),
                                dict(head_dim=16, frequencies=[1.0] * 7), dict(head_dim=16, frequencies=[float("inf")] * 8), dict(head_dim=16, frequencies=[float("nan")] * 8),
                                dict(head_dim=16, axis=[0] * 7), dict(head_dim=16, axis=[0] * 7 + [-1]), dict(head_dim=16, axis=[0] * 7 + [4]),
                                dict(head_dim=16, sections=[8], axis=[0] * 8), dict(head_dim=16, magnitude=float("inf")), dict(head_dim=16, magnitude=float("nan"))])
def test_rotary_refusals(kw):
    with pytest.raises(binding.EssaError):
        binding.Rotary(**kw)


def test_make_refuses_null():
    lib = binding.load_library()
    f = (C.c_double * 8)()
    out = binding.RotaryDesc()
    assert lib.essa_rotary_make(16, 1, 0, 1.0, None, None, C.byref(out)) == binding.ESSA_ERR_INVALID_ARG
    assert lib.essa_rotary_make(16, 1, 0, 1.0, f, None, None) == binding.ESSA_ERR_INVALID_ARG
    assert lib.essa_rotary_make(16, 0, 0, 1.0, f, None, C.byref(out)) == binding.ESSA_ERR_UNSUPPORTED_SHAPE
    assert lib.essa_rotary_make(16, 5, 0, 1.0, f, None, C.byref(out)) == binding.ESSA_ERR_UNSUPPORTED_SHAPE
    assert lib.essa_rotary_make(16, 1, 0, 1.0, f, None, C.byref(out)) == binding.ESSA_OK


def test_calls_without_a_context_are_refused():
    lib = binding.load_library()
    desc = binding.CacheDesc(1, 1, 1, 64, 1, 1, 16, 16, 16, 16)
    r = binding.Rotary(64)
    assert lib.essa_cache_attend_masked(None, C.byref(desc), None, 0, None, 0, 1, 1, None, None, 1, 1, 1.0, None, 0, None, 0, None) == binding.ESSA_ERR_INVALID_ARG
    assert lib.essa_cache_tree(None, C.byref(desc), None, 1, None, None, 1, None, 1, None, None) == binding.ESSA_ERR_INVALID_ARG
    assert lib.essa_cache_keep(None, C.byref(desc), None, None, None, None, 0, 1, None, 0, None) == binding.ESSA_ERR_INVALID_ARG
    assert lib.essa_rotary_apply(None, r._ref, None, 0, 1, 1, None, 0, None, 0, None) == binding.ESSA_ERR_INVALID_ARG
    assert lib.essa_cache_append_rotary(None, C.byref(desc), 0, r._ref, None, 0, 1, None, 0, None, 0, 1, None, 0, None, None, 1, None, 0, None) == binding.ESSA_ERR_INVALID_ARG


def test_keep_workspace():
    lib = binding.load_library()
    b = C.c_int64(-1)
    assert lib.essa_cache_keep_workspace(3, C.byref(b)) == 0 and b.value == 256 + 3 * 32
    assert lib.essa_cache_keep_workspace(0, C.byref(b)) == 0 and lib.essa_cache_keep_workspace(1, None) == binding.ESSA_ERR_INVALID_ARG
    assert lib.essa_cache_keep_workspace(-1, C.byref(b)) == binding.ESSA_ERR_INVALID_ARG


# -- the model itself
def test_rotation_is_a_complex_product_and_turns_back():
    rng = np.random.default_rng(0)
    x, pos = rng.standard_normal((3, 2, 16)), np.array([[0, 5, -7], [1, 2, 3]])
    freq, axis = 10.0 ** -rng.uniform(0, 3, 8), np.array([0, 1] * 4)
    for adjacent in (False, True):
        y = co.rotate(x, pos, freq, axis, adjacent)
        a, b = (slice(0, None, 2), slice(1, None, 2)) if adjacent else (slice(0, 8), slice(8, 16))
        z = (x[..., a] + 1j * x[..., b]) * np.exp(1j * pos[axis].T * freq)[:, None]
        np.testing.assert_allclose(y[..., a] + 1j * y[..., b], z, atol=1e-12)
        np.testing.assert_allclose(co.rotate(y, -pos, freq, axis, adjacent), x, atol=1e-12)


def test_window_of_everything_is_causal_and_sinks_stay():
    assert (co.seen_mask(9, 4) == co.seen_mask(9, 4, window=9)).all()
    s = co.seen_mask(10, 2, window=3, sinks=2)
    assert s.astype(int).tolist() == [[1, 1, 0, 0, 0, 0, 1, 1, 1, 0], [1, 1, 0, 0, 0, 0, 0, 1, 1, 1]]
    assert not co.seen_mask(2, 4)[:2].any()


def test_a_chain_of_drafts_is_causal_and_a_tree_is_not():
    bits, depth = co.ancestors([-1, 0, 1, 2])
    assert (co.seen_mask(9, 4, drafts=bits) == co.seen_mask(9, 4)).all() and depth.tolist() == [0, 1, 2, 3]
    bits, depth = co.ancestors([-1, 0, 0, 2, -1])
    assert bits.astype(int).tolist() == [[1, 0, 0, 0, 0], [1, 1, 0, 0, 0], [1, 0, 1, 0, 0], [1, 0, 1, 1, 0], [0, 0, 0, 0, 1]] and depth.tolist() == [0, 1, 1, 2, 0]
    assert co.pack_bits(bits, 1)[:, 0].tolist() == [1, 3, 5, 13, 16]


def test_attend_seen_agrees_with_attend():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 4, 64)), rng.standard_normal((2, 8, 64)), rng.standard_normal((2, 8, 64))
    np.testing.assert_allclose(co.attend_seen(q, k, v, co.seen_mask(8, 3), 0.1)[0], co.attend(q, k, v, 8, 0.1)[0])
