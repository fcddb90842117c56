"""The cache's model against what its definition fixes, the page layout's byte order, and the library's host-only calls.  No kernel runs."""
import ctypes as C

import numpy as np
import pytest

from oracle import cache_oracle as co
from paper_2507_04453_b200 import binding
from tests.cache_utils import bf16


@pytest.fixture(scope="module")
def lib():
    from paper_2507_04453_b200 import build
    build.build()
    return binding.load_library()


def test_sixteen_evenly_spaced_values_are_stored_exactly():
    x = np.tile(np.arange(16, dtype=np.float32), 4) * 0.5 - 2
    codes, scale, low = co.quantize(x[None])
    assert scale[0, 0] == 0.5 and low[0, 0] == -2 and np.array_equal(codes[0], np.tile(np.arange(16), 4))
    np.testing.assert_array_equal(co.dequantize(codes, scale, low)[0], x)


def test_stored_values_are_within_half_a_step():
    rng = np.random.default_rng(0)
    x = bf16(rng, (50, 3, 128), 3.0)
    y = co.dequantize(*co.quantize(x))
    g = x.reshape(50, 3, 2, 64).astype(np.float64)
    step = (g.max(-1) - g.min(-1)) / 15
    # the minimum and the scale are rounded to fp16 (2^-11 relative): the code range shifts by that much
    assert np.all(np.abs(y.reshape(g.shape) - g) <= (0.5 * step + 2.0 ** -11 * (np.abs(g.min(-1)) + 15 * step) * 1.01)[..., None])


def test_constant_groups_and_tokens_that_do_not_fit():
    x = np.full((1, 1, 64), 1.25, np.float32)
    codes, scale, low = co.quantize(x)
    assert scale[0, 0, 0] == 0 and np.all(codes == 0) and np.all(co.dequantize(codes, scale, low) == 1.25)
    k, v = np.zeros((4, 1, 64), np.float32), np.zeros((4, 1, 64), np.float32)
    k[1, 0, 3], v[2, 0, 9], k[3, 0, 0] = np.inf, np.nan, -1e5
    (kc, ks, kl), (vc, vs, vl) = co.quantize_tokens(k, v)
    assert np.isnan(kl[1:]).all() and (vl[1:] == 0).all() and (ks[1:] == 0).all() and (vs[1:] == 0).all() and np.isfinite(kl[0]).all()


def test_bytes_of_a_page():
    """Token 5, channel 35 of V of kv head 1: a nibble and an fp16 pair at the places the layout names."""
    c = co.Cache(1, 2, 2, 128, 1, 1)
    c.codes[0, 1, 1, 1, 5, 35] = 9
    c.scale[0, 1, 1, 1, 5, 1], c.low[0, 1, 1, 1, 5, 1] = 0.5, -3
    raw = c.to_bytes()
    run = raw[0, 1, 72 * 128:]
    at = 64 * 64 + 1 * 1024 + 5 * 16 + 1                    # codes of K, chunk 1, token 5, byte (35 - 32) / 2
    assert run[at] == 9 << 4 and np.count_nonzero(run[:64 * 128]) == 1
    meta = run[64 * 128:].view(np.float16).reshape(2, 2, 64, 2)
    assert meta[1, 1, 5, 0] == 0.5 and meta[1, 1, 5, 1] == -3 and np.count_nonzero(meta) == 2
    d = co.Cache(1, 2, 2, 128, 1, 1)
    d.load_bytes(raw)
    assert np.array_equal(d.codes, c.codes) and np.array_equal(d.scale, c.scale) and np.array_equal(d.low, c.low)


def test_attention_of_the_model_against_closed_forms():
    rng = np.random.default_rng(1)
    v = rng.standard_normal((1, 5, 64))
    out, p = co.attend(np.zeros((2, 2, 64)), rng.standard_normal((1, 5, 64)), v, 5, 1.0)
    np.testing.assert_allclose(out[0, 0], v[0, :4].mean(0))   # equal scores: the mean of what the row sees
    np.testing.assert_allclose(out[1, 1], v[0].mean(0))
    out, p = co.attend(np.ones((7, 1, 64)), np.ones((1, 3, 64)), v[:, :3], 3, 1.0)
    assert np.all(out[:4] == 0)                               # rows before the sequence's first token
    np.testing.assert_allclose(out[4, 0], v[0, 0])


def test_model_refuses_and_shares_pages():
    c = co.Cache(1, 6, 1, 64, 4, 3)
    c.grow([0, 1], [100, 64])
    assert c.table[0].tolist() == [0, 1, -1] and c.table[1].tolist() == [2, -1, -1]
    c.fork([0], [2])
    assert c.table[2].tolist() == [0, 3, -1] and c.refs.tolist() == [2, 1, 1, 1, 0, 0]
    with pytest.raises(co.Refused):
        c.grow([0, 2], [100, 100])
    c.free([0, 1])
    assert c.refs.tolist() == [1, 0, 0, 1, 0, 0]
    assert c.compact() == 2 and c.table[2].tolist() == [0, 1, -1] and c.refs.tolist() == [1, 1, 0, 0, 0, 0]


# ------------------------------------------------------------------------------------------------ the library's host-only calls
def desc(**kw):
    d = dict(layers=1, num_pages=4, kv_heads=2, head_dim=64, max_seqs=3, max_pages=5, pages=4096, table=4096, lengths=4096, refs=4096)
    d.update(kw)
    return binding.CacheDesc(**d)


def test_page_bytes(lib):
    assert lib.essa_cache_page_bytes(8, 128) == 72 * 8 * 128 and lib.essa_cache_page_bytes(1, 64) == 72 * 64
    assert lib.essa_cache_page_bytes(1, 96) == 0 and lib.essa_cache_page_bytes(0, 64) == 0


@pytest.mark.parametrize("change,status", [({}, 0), ({"layers": 0}, -1), ({"num_pages": 0}, -1), ({"kv_heads": 0}, -1), ({"max_seqs": 0}, -1), ({"max_pages": -1}, -1),
                                           ({"pages": None}, -1), ({"table": None}, -1), ({"lengths": None}, -1), ({"refs": None}, -1), ({"pages": 4104}, -1),
                                           ({"table": 4097}, -1), ({"head_dim": 96}, -2), ({"head_dim": 256}, -2), ({"max_seqs": 65537}, -2), ({"max_pages": 1 << 25}, -2),
                                           ({"max_pages": (1 << 25) - 1}, 0), ({"max_seqs": 65536}, 0)])
def test_descriptor_validation(lib, change, status):
    assert lib.essa_cache_validate(C.byref(desc(**change))) == status
    n = C.c_int64(0)
    assert lib.essa_cache_pages_workspace(C.byref(desc(**change)), C.byref(n)) == status
    assert (n.value > 0) == (status == 0)


def test_null_descriptor_and_context_are_refused(lib):
    assert lib.essa_cache_validate(None) == binding.ESSA_ERR_INVALID_ARG
    d = desc()
    assert lib.essa_cache_reset(None, C.byref(d), None) == binding.ESSA_ERR_INVALID_ARG
    assert lib.essa_cache_grow(None, C.byref(d), None, None, 1, None, 0, None) == binding.ESSA_ERR_INVALID_ARG
    assert lib.essa_cache_free(None, C.byref(d), None, 1, None) == binding.ESSA_ERR_INVALID_ARG
    assert lib.essa_cache_attend(None, C.byref(d), 0, None, 0, 4, 1, None, None, 1, 1, 1.0, None, 0, None, 0, None) == binding.ESSA_ERR_INVALID_ARG


def test_attend_workspace(lib):
    n = C.c_int64(0)
    ok = lambda heads, new, sms=148: lib.essa_cache_attend_workspace(C.byref(desc()), heads, new, sms, C.byref(n))
    assert ok(4, 1) == 0 and n.value > 0 and n.value % 16 == 0
    assert ok(3, 1) == binding.ESSA_ERR_INVALID_ARG   # not a multiple of kv_heads
    assert ok(4, 0) == binding.ESSA_ERR_INVALID_ARG and ok(0, 1) == binding.ESSA_ERR_INVALID_ARG and ok(4, 1, 0) == binding.ESSA_ERR_INVALID_ARG
    assert ok(2 * 1000, 1 << 20) == 0 and n.value < 1 << 30  # bounded by the grid, whatever the call's size
