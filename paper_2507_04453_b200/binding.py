"""ctypes binding of libessa.so: argument marshalling only.

Every function here forwards to the C entry point of the same name (``essa_`` prefix dropped on the
methods of :class:`Context`); all arithmetic runs in the library's CUDA kernels.  torch supplies device
memory (``tensor.data_ptr()``) and streams, nothing else.  There is no fallback: if the library has not
been built, or no sm_100 GPU is present, the calls raise.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
from typing import Optional

import numpy as np

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG_DIR, "libessa.so")

ESSA_OK = 0
ESSA_ERR_INVALID_ARG = -1
ESSA_ERR_UNSUPPORTED_SHAPE = -2
ESSA_ERR_ALLOC = -3
ESSA_ERR_CUDA = -4
ESSA_ERR_DEVICE_TIMEOUT = -5
ESSA_ERR_NO_DEVICE = -6
ESSA_ERR_CACHE = -7
ESSA_W0_BF16 = 0
ESSA_W0_INT8_PERCHANNEL = 1
ESSA_W0_INT4_GROUP128 = 2
ESSA_OPT_PAIR_TILES = 1
ESSA_OPT_FUSE_DOWN = 2
ESSA_OPT_WAIT_LIMIT_MCYCLES = 3
ESSA_OPT_DEBUG_STALL_RANK_ROWS = 4
ESSA_OPT_DECODE_PAIRS = 5
ESSA_OPT_DECODE_DOWN_CTAS = 6
ESSA_OPT_WIDE_TILES = 7
ESSA_OPT_DOWN_SPLITS = 8
ESSA_OPT_L2_HINTS = 9
ESSA_OPT_DOWN_PAIRS = 10
ESSA_OPT_DOWN_TILE_UNITS = 11

EXPORTED_SYMBOLS = (
    "essa_version", "essa_status_string", "essa_create", "essa_destroy", "essa_last_error", "essa_get_status",
    "essa_reserve", "essa_load_adapter", "essa_free_adapter", "essa_sample_population",
    "essa_sample_population_range", "essa_apply_projection", "essa_apply_projection_host",
    "essa_apply_projection_simt", "essa_plan_projection", "essa_validate_segments", "essa_debug_stream_words",
    "essa_debug_philox", "essa_debug_segment_map", "essa_debug_core_matrix", "essa_profile_begin", "essa_profile_end",
    "essa_apply_projection_static", "essa_get_launch_count", "essa_reserve_dequant", "essa_apply_block", "essa_apply_block_host", "essa_set_option",
    "essa_top_alpha_index", "essa_sample_population_masked", "essa_export_candidates", "essa_sample_apply_block",
    "essa_apply_layers", "essa_cma_create", "essa_cma_destroy", "essa_cma_ask", "essa_tell", "essa_cma_set", "essa_cma_get", "essa_cma_params",
    "essa_cache_page_bytes", "essa_cache_validate", "essa_cache_pages_workspace", "essa_cache_attend_workspace",
    "essa_cache_reset", "essa_cache_grow", "essa_cache_append", "essa_cache_read", "essa_cache_attend", "essa_cache_fork",
    "essa_cache_free", "essa_cache_compact", "essa_cache_attend_masked", "essa_cache_tree", "essa_cache_keep_workspace", "essa_cache_keep",
    "essa_rotary_make", "essa_rotary_apply", "essa_cache_append_rotary",
)


def top_alpha_index(n_factors: int, rank: int, alpha) -> list:
    """essa_top_alpha_index: columns of the floor(alpha * rank) leading entries of each of n_factors slices of `rank`
    columns.  alpha may be a float, a string or a Fraction; it is turned into an exact ratio of integers first."""
    from fractions import Fraction
    fr = alpha if isinstance(alpha, Fraction) else Fraction(str(alpha))
    lib = load_library()
    cnt = C.c_int32(0)
    st = lib.essa_top_alpha_index(n_factors, rank, fr.numerator, fr.denominator, None, C.byref(cnt))
    if st != ESSA_OK:
        raise EssaError(st, "top_alpha_index: bad arguments")
    out = (C.c_int32 * max(cnt.value, 1))()
    st = lib.essa_top_alpha_index(n_factors, rank, fr.numerator, fr.denominator, out, C.byref(cnt))
    if st != ESSA_OK:
        raise EssaError(st, "top_alpha_index: bad arguments")
    return [int(out[i]) for i in range(cnt.value)]


class EssaError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"essa status {status}: {message}")
        self.status = status


class AdapterDesc(C.Structure):
    _fields_ = [("d_in", C.c_int32), ("d_out", C.c_int32), ("rank", C.c_int32), ("w0_dtype", C.c_int32),
                ("W0", C.c_void_p), ("w0_scale", C.c_void_p), ("U_A", C.c_void_p), ("V_A", C.c_void_p),
                ("U_B", C.c_void_p), ("V_B", C.c_void_p), ("on_device", C.c_int32)]


class BlockItem(C.Structure):
    _fields_ = [("adapter", C.c_void_p), ("x", C.c_void_p), ("sA_col", C.c_int32), ("sB_col", C.c_int32), ("y", C.c_void_p)]


class CacheDesc(C.Structure):
    _fields_ = [("layers", C.c_int32), ("num_pages", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("max_seqs", C.c_int32), ("max_pages", C.c_int32), ("pages", C.c_void_p), ("table", C.c_void_p),
                ("lengths", C.c_void_p), ("refs", C.c_void_p)]


CACHE_MAX_DRAFTS = 256
ROTARY_MAX_DIM = 256


class AttendMask(C.Structure):
    _fields_ = [("window", C.c_int32), ("sinks", C.c_int32), ("drafts", C.c_void_p), ("draft_words", C.c_int32)]


class RotaryDesc(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("axes", C.c_int32), ("adjacent", C.c_int32), ("magnitude", C.c_float),
                ("turns", C.c_uint64 * (ROTARY_MAX_DIM // 2)), ("axis", C.c_uint8 * (ROTARY_MAX_DIM // 2))]


class Plan(C.Structure):
    _fields_ = [("block_m", C.c_int32), ("block_n", C.c_int32), ("block_k", C.c_int32), ("stages", C.c_int32),
                ("k_blocks", C.c_int32), ("splits", C.c_int32), ("tiles", C.c_int32), ("grid", C.c_int32),
                ("down_splits", C.c_int32), ("down_grid", C.c_int32), ("scratch_bytes", C.c_int64),
                ("decode", C.c_int32), ("x_stages", C.c_int32)]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class Profile(C.Structure):
    _fields_ = [("rank_down_ms", C.c_double), ("base_up_ms", C.c_double), ("calls", C.c_int32), ("dropped", C.c_int32)]


_lib = None


def load_library() -> C.CDLL:
    """dlopen libessa.so (built by ``python -m paper_2507_04453_b200.build``) and declare signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(f"{LIB_PATH} not built: run `python -m paper_2507_04453_b200.build` (or __graft_entry__.build())")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, u64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64, C.c_float
    sig = {
        "essa_version": (i32, []),
        "essa_status_string": (C.c_char_p, [i32]),
        "essa_create": (i32, [C.POINTER(vp), i32]),
        "essa_destroy": (i32, [vp]),
        "essa_last_error": (C.c_char_p, [vp]),
        "essa_get_status": (i32, [vp, C.POINTER(i32)]),
        "essa_reserve": (i32, [vp, i64, i32, i32]),
        "essa_get_launch_count": (i32, [vp, C.POINTER(i64)]),
        "essa_reserve_dequant": (i32, [vp, i32, i32]),
        "essa_set_option": (i32, [vp, i32, i32]),
        "essa_apply_block": (i32, [vp, C.POINTER(BlockItem), i32, i64, vp, i32, vp, i32, vp]),
        "essa_apply_block_host": (i32, [vp, C.POINTER(BlockItem), i32, i64, vp, i32, vp, i32, vp]),
        "essa_apply_layers": (i32, [vp, C.POINTER(BlockItem), i32, i32, i64, vp, i32, vp, i32, vp]),
        "essa_sample_apply_block": (i32, [vp, vp, f32, vp, vp, i32, u64, i32, i32, vp, C.POINTER(BlockItem), i32, i64, vp, vp]),
        "essa_cma_create": (i32, [vp, i32, i32, vp, f32, C.POINTER(vp)]),
        "essa_cma_destroy": (i32, [vp, vp]),
        "essa_cma_ask": (i32, [vp, vp, u64, i32, i32, vp, vp]),
        "essa_tell": (i32, [vp, vp, vp, i32, vp, vp]),
        "essa_cma_set": (i32, [vp, vp, vp, vp, vp, vp, vp, i32, vp]),
        "essa_cma_get": (i32, [vp, vp, vp, vp, vp, vp, vp, vp, vp, C.POINTER(i32), C.POINTER(i32)]),
        "essa_cma_params": (i32, [vp, vp]),
        "essa_load_adapter": (i32, [vp, C.POINTER(AdapterDesc), C.POINTER(vp), vp]),
        "essa_free_adapter": (i32, [vp, vp]),
        "essa_sample_population": (i32, [vp, vp, f32, vp, vp, i32, u64, i32, vp, vp]),
        "essa_sample_population_range": (i32, [vp, vp, f32, vp, vp, i32, u64, i32, i32, vp, vp]),
        "essa_top_alpha_index": (i32, [i32, i32, i32, i32, vp, vp]),
        "essa_export_candidates": (i32, [vp, vp, vp, i32, i32, i32, i32, i32, vp, vp, vp]),
        "essa_sample_population_masked": (i32, [vp, vp, vp, vp, f32, vp, vp, i32, i32, u64, i32, i32, vp, vp]),
        "essa_apply_projection": (i32, [vp, vp, vp, i64, vp, i32, vp, i32, i32, i32, vp, vp]),
        "essa_apply_projection_host": (i32, [vp, vp, vp, i64, vp, i32, vp, i32, i32, i32, vp, vp]),
        "essa_apply_projection_simt": (i32, [vp, vp, vp, i64, vp, i32, vp, i32, i32, i32, vp, vp]),
        "essa_apply_projection_static": (i32, [vp, vp, vp, i64, vp, i32, vp, i32, i32, i32, vp, vp]),
        "essa_plan_projection": (i32, [i32, i32, i32, i32, i64, i32, C.POINTER(Plan)]),
        "essa_validate_segments": (i32, [vp, i32, i64]),
        "essa_debug_stream_words": (i32, [vp, u64, i32, i32, i32, vp, vp]),
        "essa_debug_philox": (i32, [vp, C.POINTER(C.c_uint32), C.POINTER(C.c_uint32), C.POINTER(C.c_uint32)]),
        "essa_debug_segment_map": (i32, [vp, vp, i32, i64, vp, vp]),
        "essa_debug_core_matrix": (i32, [vp, vp, vp]),
        "essa_profile_begin": (i32, [vp, i32]),
        "essa_profile_end": (i32, [vp, C.POINTER(Profile)]),
        "essa_cache_page_bytes": (i64, [i32, i32]),
        "essa_cache_validate": (i32, [C.POINTER(CacheDesc)]),
        "essa_cache_pages_workspace": (i32, [C.POINTER(CacheDesc), C.POINTER(i64)]),
        "essa_cache_attend_workspace": (i32, [C.POINTER(CacheDesc), i32, i32, i32, C.POINTER(i64)]),
        "essa_cache_reset": (i32, [vp, C.POINTER(CacheDesc), vp]),
        "essa_cache_grow": (i32, [vp, C.POINTER(CacheDesc), vp, vp, i32, vp, i64, vp]),
        "essa_cache_append": (i32, [vp, C.POINTER(CacheDesc), i32, vp, i64, vp, i64, i32, vp, vp, i32, vp]),
        "essa_cache_read": (i32, [vp, C.POINTER(CacheDesc), i32, vp, vp, i32, vp, vp, i32, vp]),
        "essa_cache_attend": (i32, [vp, C.POINTER(CacheDesc), i32, vp, i64, i32, i32, vp, vp, i32, i32, f32, vp, i64, vp, i64, vp]),
        "essa_cache_fork": (i32, [vp, C.POINTER(CacheDesc), vp, vp, vp, i32, vp, i64, vp]),
        "essa_cache_free": (i32, [vp, C.POINTER(CacheDesc), vp, i32, vp]),
        "essa_cache_compact": (i32, [vp, C.POINTER(CacheDesc), vp, vp, i64, vp]),
        "essa_cache_attend_masked": (i32, [vp, C.POINTER(CacheDesc), C.POINTER(AttendMask), i32, vp, i64, i32, i32, vp, vp, i32, i32, f32, vp, i64, vp, i64, vp]),
        "essa_cache_tree": (i32, [vp, C.POINTER(CacheDesc), vp, i32, vp, vp, i32, vp, i32, vp, vp]),
        "essa_cache_keep_workspace": (i32, [i32, C.POINTER(i64)]),
        "essa_cache_keep": (i32, [vp, C.POINTER(CacheDesc), vp, vp, vp, vp, i64, i32, vp, i64, vp]),
        "essa_rotary_make": (i32, [i32, i32, i32, f32, vp, vp, C.POINTER(RotaryDesc)]),
        "essa_rotary_apply": (i32, [vp, C.POINTER(RotaryDesc), vp, i64, i32, i32, vp, i64, vp, i64, vp]),
        "essa_cache_append_rotary": (i32, [vp, C.POINTER(CacheDesc), i32, C.POINTER(RotaryDesc), vp, i64, i32, vp, i64, vp, i64, i32, vp, i64, vp, vp, i32, vp, i64, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def plan_projection(d_in: int, d_out: int, rank: int, w0_dtype: int, T: int, sm_count: int = 148) -> dict:
    """essa_plan_projection: the schedule a call would use (host arithmetic, no device needed)."""
    lib = load_library()
    p = Plan()
    st = lib.essa_plan_projection(d_in, d_out, rank, w0_dtype, T, sm_count, C.byref(p))
    if st != ESSA_OK:
        raise EssaError(st, lib.essa_status_string(st).decode())
    return p.as_dict()


def validate_segments(seg_offsets, T: int) -> int:
    """essa_validate_segments on a host int32 array; returns the status code."""
    lib = load_library()
    seg = np.ascontiguousarray(seg_offsets, dtype=np.int32)
    return lib.essa_validate_segments(seg.ctypes.data_as(C.c_void_p), len(seg) - 1, T)


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream or None


class AdapterHandle:
    def __init__(self, ctx: "Context", handle: int, d_in: int, d_out: int, rank: int, w0_dtype: int):
        self.ctx, self.handle = ctx, handle
        self.d_in, self.d_out, self.rank, self.w0_dtype = d_in, d_out, rank, w0_dtype

    def free(self):
        if self.handle:
            self.ctx._check(self.ctx.lib.essa_free_adapter(self.ctx.handle, self.handle))
            self.handle = None


class PreparedBlock:
    """essa_apply_block with its arguments marshalled ahead of time (see Context.prepare_block)."""

    def __init__(self, ctx, adapters, xs, seg_offsets, sigma, cols, outs):
        n = len(adapters)
        T = xs[0].shape[0]
        self.keep = (list(adapters), list(xs), seg_offsets, sigma, list(outs))
        self.arr = (BlockItem * n)()
        for i in range(n):
            self.arr[i] = BlockItem(adapters[i].handle, xs[i].data_ptr() if T else None, cols[i][0], cols[i][1],
                                    outs[i].data_ptr() if T else None)
        self.ctx = ctx
        self.fn = ctx.lib.essa_apply_block
        self.args = (ctx.handle, self.arr, n, T, seg_offsets.data_ptr(), seg_offsets.numel() - 1, sigma.data_ptr(),
                     sigma.stride(0) if sigma.dim() == 2 else sigma.numel())

    def run(self, stream_handle):
        """stream_handle: the integer cudaStream_t (torch's ``stream.cuda_stream``; 0 / None = default stream)."""
        st = self.fn(*self.args, stream_handle or None)
        if st != ESSA_OK:
            self.ctx._check(st)


class PreparedLayers:
    """essa_apply_layers with its arguments marshalled ahead of time (see Context.prepare_layers)."""

    def __init__(self, ctx, layers, seg_offsets, sigma):
        n_layers, n_items = len(layers), len(layers[0])
        T = layers[0][0][1].shape[0]
        self.keep = (layers, seg_offsets, sigma)
        self.arr = (BlockItem * (n_layers * n_items))()
        for l, layer in enumerate(layers):
            assert len(layer) == n_items
            for i, (ad, x, cols, y) in enumerate(layer):
                self.arr[l * n_items + i] = BlockItem(ad.handle, x.data_ptr() if T else None, cols[0], cols[1],
                                                      y.data_ptr() if T else None)
        self.ctx = ctx
        self.fn = ctx.lib.essa_apply_layers
        self.args = (ctx.handle, self.arr, n_layers, n_items, T, seg_offsets.data_ptr(), seg_offsets.numel() - 1,
                     sigma.data_ptr(), sigma.stride(0) if sigma.dim() == 2 else sigma.numel())

    def run(self, stream_handle):
        st = self.fn(*self.args, stream_handle or None)
        if st != ESSA_OK:
            self.ctx._check(st)


class PreparedSampleBlock:
    """essa_sample_apply_block with its arguments marshalled ahead of time (see Context.prepare_sample_block)."""

    def __init__(self, ctx, mean, step, Bfactor, Dvec, seed, P, sigma_out, adapters, xs, seg_offsets, cols, outs, k_begin):
        n = len(adapters)
        T = xs[0].shape[0]
        self.keep = (mean, Bfactor, Dvec, sigma_out, list(adapters), list(xs), seg_offsets, list(outs))
        self.arr = (BlockItem * n)()
        for i in range(n):
            self.arr[i] = BlockItem(adapters[i].handle, xs[i].data_ptr() if T else None, cols[i][0], cols[i][1],
                                    outs[i].data_ptr() if T else None)
        self.ctx = ctx
        self.fn = ctx.lib.essa_sample_apply_block
        self.args = (ctx.handle, mean.data_ptr(), step, _ptr(Bfactor), _ptr(Dvec), mean.numel(), seed, k_begin, P,
                     sigma_out.data_ptr(), self.arr, n, T, seg_offsets.data_ptr())

    def run(self, stream_handle):
        st = self.fn(*self.args, stream_handle or None)
        if st != ESSA_OK:
            self.ctx._check(st)


class PreparedSample:
    """essa_sample_population(_range) with its arguments marshalled ahead of time (see Context.prepare_sample)."""

    def __init__(self, ctx, mean, step, Bfactor, Dvec, seed, P, out, k_begin):
        self.keep = (mean, Bfactor, Dvec, out)
        self.ctx = ctx
        d = mean.numel()
        if k_begin == 0:
            self.fn = ctx.lib.essa_sample_population
            self.args = (ctx.handle, mean.data_ptr(), step, _ptr(Bfactor), _ptr(Dvec), d, seed, P, out.data_ptr())
        else:
            self.fn = ctx.lib.essa_sample_population_range
            self.args = (ctx.handle, mean.data_ptr(), step, _ptr(Bfactor), _ptr(Dvec), d, seed, k_begin, P, out.data_ptr())

    def run(self, stream_handle):
        st = self.fn(*self.args, stream_handle or None)
        if st != ESSA_OK:
            self.ctx._check(st)


class CmaState:
    """Device-resident search-distribution state (essa_cma_*): argument marshalling only."""

    def __init__(self, ctx, d: int, lam: int, mean0, step0: float):
        self.ctx, self.d, self.lam = ctx, d, lam
        m = np.ascontiguousarray(mean0, dtype=np.float32)
        h = C.c_void_p()
        ctx._check(ctx.lib.essa_cma_create(ctx.handle, d, lam, m.ctypes.data_as(C.c_void_p), float(step0), C.byref(h)))
        self.handle = h.value

    def close(self):
        if self.handle:
            self.ctx.lib.essa_cma_destroy(self.ctx.handle, self.handle)
            self.handle = None

    def ask(self, seed: int, P=None, out=None, k_begin: int = 0, stream=None):
        """essa_cma_ask: candidates k_begin .. k_begin + P - 1 of the population, [P, d] fp32 on the device."""
        torch = self.ctx.torch
        P = self.lam if P is None else P
        if out is None:
            out = torch.empty((P, self.d), dtype=torch.float32, device=self.ctx.device)
        self.ctx._check(self.ctx.lib.essa_cma_ask(self.ctx.handle, self.handle, seed, k_begin, P, out.data_ptr(), _stream(stream)))
        return out

    def tell(self, population, rewards, stream=None):
        """essa_tell: population [lambda, ld] fp32 and rewards [lambda] fp32, both on the device."""
        self.ctx._check(self.ctx.lib.essa_tell(self.ctx.handle, self.handle, population.data_ptr(), population.stride(0),
                                               rewards.data_ptr(), _stream(stream)))

    def set(self, mean=None, step=None, C_=None, p_sigma=None, p_c=None, generation: int = -1, stream=None):
        """essa_cma_set from host fp64 arrays (None = keep)."""
        keep = []

        def ptr(a, shape):
            if a is None:
                return None
            a = np.ascontiguousarray(np.asarray(a, dtype=np.float64).reshape(shape))
            keep.append(a)
            return a.ctypes.data_as(C.c_void_p)
        d = self.d
        self.ctx._check(self.ctx.lib.essa_cma_set(self.ctx.handle, self.handle, ptr(mean, (d,)), ptr(step, (1,)), ptr(C_, (d, d)),
                                                  ptr(p_sigma, (d,)), ptr(p_c, (d,)), generation, _stream(stream)))

    def get(self) -> dict:
        """essa_cma_get: the whole state as host fp64 arrays."""
        d = self.d
        out = {"mean": np.empty(d), "step": np.empty(1), "C": np.empty((d, d)), "B": np.empty((d, d)), "D": np.empty(d),
               "p_sigma": np.empty(d), "p_c": np.empty(d)}
        gen, sweeps = C.c_int32(0), C.c_int32(0)
        p = lambda k: out[k].ctypes.data_as(C.c_void_p)
        self.ctx._check(self.ctx.lib.essa_cma_get(self.ctx.handle, self.handle, p("mean"), p("step"), p("C"), p("B"), p("D"),
                                                  p("p_sigma"), p("p_c"), C.byref(gen), C.byref(sweeps)))
        out["step"] = float(out["step"][0])
        out["generation"], out["sweeps"] = gen.value, sweeps.value
        return out

    def params(self) -> dict:
        """essa_cma_params: the strategy parameters in use."""
        v = np.empty(9)
        self.ctx._check(self.ctx.lib.essa_cma_params(self.handle, v.ctypes.data_as(C.c_void_p)))
        names = ("mu", "mu_eff", "c_sigma", "d_sigma", "c_c", "c_1", "c_mu", "c_m", "chi_n")
        return dict(zip(names, (float(x) for x in v)))


class Rotary:
    """Which turn every pair of channels makes per position (essa_rotary), made on the host once per model.

    head_dim: a multiple of 16 up to 256.  base: pair i turns by base ** (-2 i / head_dim) radians per position; or frequencies: head_dim / 2 of them,
    up to 2 ** 32 in magnitude.
    sections: how many pairs each axis has (their sum is head_dim / 2; None: one axis), one axis after another or, interleaved, the axes in turns until
    each has its share; or axis: the axis of every pair.  adjacent: pairs are channels 2 i and 2 i + 1 instead of i and i + head_dim / 2.
    magnitude: what cosine and sine are multiplied with."""

    def __init__(self, head_dim: int, base: float = 10000.0, sections=None, interleaved: bool = False, adjacent: bool = False, frequencies=None, axis=None,
                 magnitude: float = 1.0):
        half = head_dim // 2
        if frequencies is None:
            if not base > 0:
                raise EssaError(ESSA_ERR_INVALID_ARG, "rotary: base must be positive")
            frequencies = float(base) ** (-2.0 * np.arange(half) / max(head_dim, 1))
        frequencies = np.ascontiguousarray(frequencies, dtype=np.float64)
        if axis is None:
            left = [half] if sections is None else [int(n) for n in sections]
            if sum(left) != half or min(left, default=-1) < 0:
                raise EssaError(ESSA_ERR_INVALID_ARG, "rotary: the sections must add up to head_dim / 2")
            self.axes, axis = len(left), []
            while len(axis) < half:
                for a, n in enumerate(left):
                    take = min(n, 1) if interleaved else n
                    axis += [a] * take
                    left[a] -= take
        elif sections is not None:
            raise EssaError(ESSA_ERR_INVALID_ARG, "rotary: pass sections or axis, not both")
        else:
            self.axes = int(max(axis, default=0)) + 1
        axis = np.ascontiguousarray(axis, dtype=np.int32)
        if frequencies.shape != (half,) or axis.shape != (half,):
            raise EssaError(ESSA_ERR_INVALID_ARG, "rotary: frequencies and axis must have head_dim / 2 elements")
        self.head_dim, self.desc = head_dim, RotaryDesc()
        lib = load_library()
        st = lib.essa_rotary_make(head_dim, self.axes, int(adjacent), magnitude, frequencies.ctypes.data_as(C.c_void_p), axis.ctypes.data_as(C.c_void_p),
                                  C.byref(self.desc))
        if st != ESSA_OK:
            raise EssaError(st, "rotary: " + lib.essa_status_string(st).decode())
        self._ref = C.byref(self.desc)

    def _positions(self, torch, positions, T, index):
        """Checks positions, [axes, T] (or [T] for one axis) int32 with contiguous rows; (pointer, elements between rows)."""
        shape, axes, ld = positions.shape, self.axes, T
        ok = positions.dtype is torch.int32 and positions.get_device() == index and shape[-1:] == (T,) and shape[:-1] in ((axes,), () if axes == 1 else (axes,))
        if ok and not positions.is_contiguous():
            ok = T < 2 or positions.stride(-1) == 1
            if ok and axes > 1:
                ld = positions.stride(0)
                ok = ld >= T  # (rows that do not overlap)
        if not ok:
            raise EssaError(ESSA_ERR_INVALID_ARG, f"rotary: positions must be int32 [{axes}, {T}] with contiguous rows, on the data's device")
        return positions.data_ptr() or None, ld


class KvCache:
    """A paged 4-bit key / value cache (essa_cache_*): four torch tensors and the calls on them, argument marshalling only.

    pages [layers, num_pages, page_bytes] uint8, table [max_seqs, max_pages], lengths [max_seqs], refs [num_pages] int32.
    Index and count arguments are int32 tensors on the cache's device.  ``stream``: a torch.cuda.Stream; None = the current
    stream of the cache's device.  Workspaces and outputs come from torch's allocator, on that
    stream.  Not thread-safe, as its context."""

    def __init__(self, ctx, layers, num_pages, kv_heads, head_dim, max_seqs, max_pages, pages=None, table=None, lengths=None, refs=None):
        torch = ctx.torch
        page_bytes = ctx.lib.essa_cache_page_bytes(kv_heads, head_dim)
        if page_bytes == 0:
            raise EssaError(ESSA_ERR_UNSUPPORTED_SHAPE, "kv_cache: head_dim must be 64 or 128, kv_heads positive")
        given = [t is not None for t in (pages, table, lengths, refs)]
        if any(given) != all(given):
            raise EssaError(ESSA_ERR_INVALID_ARG, "kv_cache: pass all four buffers or none")
        self.ctx, self.device = ctx, ctx.device
        fresh = not all(given)
        if fresh:
            pages = torch.empty((layers, num_pages, page_bytes), dtype=torch.uint8, device=self.device)
            table = torch.empty((max_seqs, max_pages), dtype=torch.int32, device=self.device)
            lengths = torch.empty(max_seqs, dtype=torch.int32, device=self.device)
            refs = torch.empty(num_pages, dtype=torch.int32, device=self.device)
        for name, t, dtype, shape in (("pages", pages, torch.uint8, (layers, num_pages, page_bytes)), ("table", table, torch.int32, (max_seqs, max_pages)),
                                      ("lengths", lengths, torch.int32, (max_seqs,)), ("refs", refs, torch.int32, (num_pages,))):
            if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous() or t.device != self.device:
                raise EssaError(ESSA_ERR_INVALID_ARG, f"kv_cache: {name} must be a contiguous {dtype} tensor of shape {shape} on {self.device}")
        self.pages, self.table, self.lengths, self.refs = pages, table, lengths, refs
        self.kv_heads, self.head_dim, self.max_seqs = kv_heads, head_dim, max_seqs
        self.desc = CacheDesc(layers, num_pages, kv_heads, head_dim, max_seqs, max_pages, pages.data_ptr(), table.data_ptr(),
                              lengths.data_ptr(), refs.data_ptr())
        st = ctx.lib.essa_cache_validate(C.byref(self.desc))
        if st != ESSA_OK:
            raise EssaError(st, "kv_cache: " + ctx.lib.essa_status_string(st).decode())
        need = C.c_int64(0)
        ctx._check(ctx.lib.essa_cache_pages_workspace(C.byref(self.desc), C.byref(need)))
        self._pages_ws = need.value
        self._sms = torch.cuda.get_device_properties(self.device).multi_processor_count
        self._attend_ws = {}  # (q_heads, max_new) -> bytes
        self._ws = {}         # cudaStream_t -> workspace
        self._lib, self._ref, self._index = ctx.lib, C.byref(self.desc), self.device.index
        self._int32, self._bf16, self._scale = torch.int32, torch.bfloat16, head_dim ** -0.5
        self._none = torch.empty(0, dtype=torch.bfloat16, device=self.device)
        self._empty_like = torch.empty_like
        self._current_stream = torch._C._cuda_getCurrentRawStream
        if fresh:
            self.reset()

    # -- plumbing (a decode step makes these calls once per layer: they take a few microseconds each, so the checks are terse)
    def _raw(self, stream):
        """The cudaStream_t to enqueue on (None: torch's current stream of the cache's device)."""
        return (self._current_stream(self._index) if stream is None else stream.cuda_stream) or None

    def _fail(self, name, what):
        raise EssaError(ESSA_ERR_INVALID_ARG, f"kv_cache: {name} must be {what} on {self.device}")

    def _ints(self, name, t, n=None):
        """Checks an int32 index tensor; its pointer (None for None)."""
        if t is None:
            return None
        if t.dtype is not self._int32 or t.dim() != 1 or t.get_device() != self._index or not t.is_contiguous() or (n is not None and t.shape[0] != n):
            self._fail(name, "a contiguous int32 vector" + ("" if n is None else f" of {n} elements"))
        return t.data_ptr() or None

    def _entries(self, T, slots, tok_offsets):
        n = T if tok_offsets is None else tok_offsets.shape[0] - 1
        if n < 0:
            raise EssaError(ESSA_ERR_INVALID_ARG, "kv_cache: tok_offsets is empty")
        return self._ints("slots", slots, n), self._ints("tok_offsets", tok_offsets), n

    def _rows(self, name, t, heads):
        """Checks a token-major [T, heads, head_dim] or [T, heads * head_dim] bf16 tensor; (pointer, elements between rows)."""
        shape, d = t.shape, self.head_dim
        width = heads * d
        ok = t.dtype is self._bf16 and t.get_device() == self._index
        if ok and len(shape) == 3:
            ok = shape[1] == heads and shape[2] == d
        elif ok:
            ok = len(shape) == 2 and shape[1] == width
        if ok and t.is_contiguous():
            return t.data_ptr() or None, width
        if ok and shape[0]:
            stride = t.stride()
            if stride[-1] == 1 and (len(shape) == 2 or heads == 1 or stride[1] == d):
                return t.data_ptr(), (stride[0] if shape[0] > 1 else width)
        self._fail(name, f"a bf16 tensor [T, {heads}, {d}] whose rows are contiguous")

    def _workspace(self, bytes_, raw, stream):
        """A workspace for a call on stream `raw`: one buffer per stream serves its calls in turn.  A call that is being captured
        gets its own, from the graph's pool: the graph may be replayed beside later calls on the stream it was captured on."""
        torch = self.ctx.torch
        if stream is not None:
            with torch.cuda.stream(stream):
                return self._workspace(bytes_, raw, None)
        if torch.cuda.current_device() != self._index:  # (whose current stream is not the call's)
            with torch.cuda.device(self._index):
                return self._workspace(bytes_, raw, None)
        if torch.cuda.is_current_stream_capturing():
            return torch.empty(bytes_, dtype=torch.uint8, device=self.device)
        ws = self._ws.get(raw)
        if ws is None or ws.shape[0] < bytes_:
            ws = self._ws[raw] = torch.empty(bytes_, dtype=torch.uint8, device=self.device)
        return ws

    def _empty(self, shape, stream):
        if stream is None:
            return self._none.new_empty(shape)  # (half the time of torch.empty with its keywords)
        with self.ctx.torch.cuda.stream(stream):
            return self._none.new_empty(shape)

    def _check(self, st):
        if st != ESSA_OK:
            self.ctx._check(st)

    # -- pages
    def reset(self, stream=None):
        """essa_cache_reset: all sequences empty, all pages free."""
        self._check(self._lib.essa_cache_reset(self.ctx.handle, self._ref, self._raw(stream)))

    def grow(self, slots, counts, stream=None):
        """essa_cache_grow: sequence slots[i] (None: i) becomes counts[i] tokens longer (on a copy of its last page, if another shares that)."""
        n = counts.shape[0]
        a, b, raw = self._ints("slots", slots, n), self._ints("counts", counts), self._raw(stream)
        ws = self._workspace(self._pages_ws, raw, stream)
        self._check(self._lib.essa_cache_grow(self.ctx.handle, self._ref, a, b, n, ws.data_ptr(), ws.shape[0], raw))

    def fork(self, src, dst, lens=None, stream=None):
        """essa_cache_fork: sequence dst[i] becomes a copy of the first lens[i] (None: all) tokens of src[i]."""
        n = src.shape[0]
        a, b, c, raw = self._ints("src", src), self._ints("dst", dst, n), self._ints("lens", lens, n), self._raw(stream)
        ws = self._workspace(self._pages_ws, raw, stream)
        self._check(self._lib.essa_cache_fork(self.ctx.handle, self._ref, a, b, c, n, ws.data_ptr(), ws.shape[0], raw))

    def free(self, slots, stream=None):
        """essa_cache_free: the sequences become empty."""
        self._check(self._lib.essa_cache_free(self.ctx.handle, self._ref, self._ints("slots", slots), slots.shape[0], self._raw(stream)))

    def compact(self, used=None, stream=None):
        """essa_cache_compact: the pages in use become 0 .. U - 1; used (int32, one element) receives U."""
        u, raw = self._ints("used", used, 1), self._raw(stream)
        ws = self._workspace(self._pages_ws, raw, stream)
        self._check(self._lib.essa_cache_compact(self.ctx.handle, self._ref, u, ws.data_ptr(), ws.shape[0], raw))

    def keep(self, counts, tok_offsets=None, picks=None, slots=None, stream=None):
        """essa_cache_keep: of the last tok_offsets[i + 1] - tok_offsets[i] (None: 1) tokens of the sequence slots[i] (None: i), the counts[i] that
        picks[i, :counts[i]] names (ascending; None: the first) stay and move together; the sequence's end behind them is given back."""
        n = counts.shape[0]
        a, b, c, raw = self._ints("slots", slots, n), self._ints("tok_offsets", tok_offsets, n + 1), self._ints("counts", counts), self._raw(stream)
        pp, ldp = None, 0
        if picks is not None:
            if picks.dtype is not self._int32 or picks.dim() != 2 or picks.shape[0] != n or picks.get_device() != self._index or not picks.is_contiguous():
                self._fail("picks", f"a contiguous int32 tensor of {n} rows")
            # (without a column nothing can be picked: counts other than 0 are refused as with any that are too large)
            pp, ldp = picks.data_ptr() or self.refs.data_ptr(), picks.shape[1]
        ws = self._workspace(256 + 32 * n, raw, stream)
        self._check(self._lib.essa_cache_keep(self.ctx.handle, self._ref, a, b, c, pp, ldp, n, ws.data_ptr(), ws.shape[0], raw))

    # -- tokens
    def append_rotary(self, layer: int, rotary, q, k, v, positions=None, tok_offsets=None, slots=None, q_out=None, stream=None):
        """essa_cache_append_rotary: q [T, heads, head_dim] and k turned by positions [axes, T] int32 (None: every axis is the token's position in its
        sequence); k and v become the last tokens of the entries' sequences, as append does it.  Returns the turned q (q_out may be q)."""
        shape = q.shape
        T = shape[0]
        if v.shape[0] != T or k.shape[0] != T:
            raise EssaError(ESSA_ERR_INVALID_ARG, "kv_cache: q, k and v must have the same number of rows")
        heads = shape[1] if len(shape) == 3 else shape[-1] // self.head_dim
        pq, ldq = self._rows("q", q, heads)
        pk, ldk = self._rows("k", k, self.kv_heads)
        pv, ldv = self._rows("v", v, self.kv_heads)
        a, b, n = self._entries(T, slots, tok_offsets)
        pp, ldp = (None, 0) if positions is None else rotary._positions(self.ctx.torch, positions, T, self._index)
        if q_out is None:
            q_out = self._empty_like(q) if stream is None and q.is_contiguous() else self._empty(shape, stream)
            po, ldo = q_out.data_ptr() or None, heads * self.head_dim
        else:
            if q_out.shape != shape:
                raise EssaError(ESSA_ERR_INVALID_ARG, "kv_cache: q_out must have q's shape")
            po, ldo = self._rows("q_out", q_out, heads)
        self._check(self._lib.essa_cache_append_rotary(self.ctx.handle, self._ref, layer, rotary._ref, pq, ldq, heads, pk, ldk, pv, ldv, T, pp, ldp, a, b, n,
                                                       po, ldo, self._raw(stream)))
        return q_out

    def tree(self, parents, tok_offsets, max_new: int, slots=None, positions: bool = True, stream=None):
        """essa_cache_tree: (drafts, positions) of the drafted tokens that are the entries' rows: parents [T] int32, the place of a row's parent among its entry's
        rows (-1: the token before them).  drafts [T, words] int32 is attend's `tree`; positions [T] int32 (None unless asked for) is for append_rotary.
        max_new: the most rows of an entry, up to CACHE_MAX_DRAFTS.  (Rows outside all entries are not written.)"""
        if not 1 <= max_new <= CACHE_MAX_DRAFTS:
            raise EssaError(ESSA_ERR_UNSUPPORTED_SHAPE, f"kv_cache: a tree has 1 .. {CACHE_MAX_DRAFTS} tokens")
        T, words = parents.shape[0], (max_new + 31) // 32
        p = self._ints("parents", parents)
        a, b, n = self._entries(T, slots, tok_offsets)
        if stream is None:
            drafts, pos = parents.new_empty((T, words)), self._empty_like(parents) if positions else None
        else:
            with self.ctx.torch.cuda.stream(stream):
                drafts, pos = parents.new_empty((T, words)), self._empty_like(parents) if positions else None
        self._check(self._lib.essa_cache_tree(self.ctx.handle, self._ref, p, T, a, b, n, drafts.data_ptr() or None, words, pos.data_ptr() or None if positions else None,
                                              self._raw(stream)))
        return drafts, pos

    def append(self, layer: int, k, v, tok_offsets=None, slots=None, stream=None):
        """essa_cache_append: k, v [T, kv_heads, head_dim] bf16 become the last tokens of the entries' sequences."""
        T = k.shape[0]
        if v.shape[0] != T:
            raise EssaError(ESSA_ERR_INVALID_ARG, "kv_cache: k and v must have the same number of rows")
        pk, ldk = self._rows("k", k, self.kv_heads)
        pv, ldv = self._rows("v", v, self.kv_heads)
        a, b, n = self._entries(T, slots, tok_offsets)
        self._check(self._lib.essa_cache_append(self.ctx.handle, self._ref, layer, pk, ldk, pv, ldv, T, a, b, n, self._raw(stream)))

    def read(self, layer: int, tok_offsets, T: int, slots=None, k_out=None, v_out=None, stream=None):
        """essa_cache_read: (k, v) [T, kv_heads, head_dim] bf16, the last tokens of the entries' sequences as they are stored."""
        a, b, n = self._entries(T, slots, tok_offsets)
        shape = (T, self.kv_heads, self.head_dim)
        if k_out is None and v_out is None:
            k_out, v_out = self._empty(shape, stream), self._empty(shape, stream)
            pk, pv = k_out.data_ptr() or None, v_out.data_ptr() or None
        else:
            k_out = self._empty(shape, stream) if k_out is None else k_out
            v_out = self._empty(shape, stream) if v_out is None else v_out
            pk, pv = self._rows("k_out", k_out, self.kv_heads)[0], self._rows("v_out", v_out, self.kv_heads)[0]
            if k_out.shape[0] != T or v_out.shape[0] != T or not (k_out.is_contiguous() and v_out.is_contiguous()):
                self._fail("k_out and v_out", f"contiguous tensors of {T} rows")
        self._check(self._lib.essa_cache_read(self.ctx.handle, self._ref, layer, pk, pv, T, a, b, n, self._raw(stream)))
        return k_out, v_out

    def _mask(self, window, sinks, tree, T):
        """The mask of a call (None: rows see all up to themselves)."""
        words, ptr = 0, None
        if tree is not None:
            if tree.dtype is not self._int32 or tree.dim() != 2 or tree.shape[0] != T or tree.get_device() != self._index or not tree.is_contiguous():
                self._fail("tree", f"a contiguous int32 tensor [{T}, words]")
            words, ptr = tree.shape[1], tree.data_ptr() or None
            if words < 1:  # (its pointer is NULL, which would stand for no tree)
                raise EssaError(ESSA_ERR_UNSUPPORTED_SHAPE, "kv_cache: a tree has at least one word of bits per row")
        if window is not None and window < 1:
            raise EssaError(ESSA_ERR_INVALID_ARG, "kv_cache: a window has at least one token")
        # (beyond 32 bits: all tokens; the structure would take the low bits)
        return C.byref(AttendMask(min(window or 0, 0x7fffffff), max(min(sinks, 0x7fffffff), -1), ptr, words))

    def attend(self, layer: int, q, tok_offsets=None, slots=None, max_new: int = 1, scale=None, out=None, stream=None, window=None, sinks: int = 0, tree=None):
        """essa_cache_attend: q [T, heads, head_dim] (or [T, heads * head_dim]) bf16 over the cached tokens; the result has q's
        shape.  max_new: the most rows an entry is expected to have (chooses the schedule only); scale: None = head_dim ** -0.5.
        essa_cache_attend_masked: window: a row sees the last `window` tokens up to itself (None: all), and the first `sinks` of its sequence; tree: an
        entry's rows are drafted tokens that see what comes before the rows and the drafts whose bits [T, words] int32 (of tree()) are set."""
        shape = q.shape
        heads = shape[1] if len(shape) == 3 else shape[-1] // self.head_dim
        pq, ldq = self._rows("q", q, heads)
        a, b, n = self._entries(shape[0], slots, tok_offsets)
        need = self._attend_ws.get((heads, max_new))
        if need is None:
            got = C.c_int64(0)
            st = self._lib.essa_cache_attend_workspace(self._ref, heads, max_new, self._sms, C.byref(got))
            if st != ESSA_OK:
                raise EssaError(st, "kv_cache: the number of query heads must be a multiple of kv_heads and max_new at least 1")
            need = self._attend_ws[(heads, max_new)] = got.value
        mask = None if window is None and tree is None and sinks == 0 else self._mask(window, sinks, tree, shape[0])
        if out is None:
            out = self._empty_like(q) if stream is None and q.is_contiguous() else self._empty(shape, stream)
            po, ldo = out.data_ptr() or None, heads * self.head_dim
        else:
            if out.shape != shape:
                raise EssaError(ESSA_ERR_INVALID_ARG, "kv_cache: out must have q's shape")
            po, ldo = self._rows("out", out, heads)
        raw = self._raw(stream)
        ws = self._workspace(need, raw, stream)
        scale = self._scale if scale is None else scale
        if mask is None:
            st = self._lib.essa_cache_attend(self.ctx.handle, self._ref, layer, pq, ldq, heads, shape[0], a, b, n, max_new, scale, po, ldo, ws.data_ptr(), ws.shape[0], raw)
        else:
            st = self._lib.essa_cache_attend_masked(self.ctx.handle, self._ref, mask, layer, pq, ldq, heads, shape[0], a, b, n, max_new, scale, po, ldo, ws.data_ptr(),
                                                    ws.shape[0], raw)
        self._check(st)
        return out


class Context:
    """Owns one essa_ctx on a CUDA device."""

    def __init__(self, device: int = 0):
        import torch
        self.lib = load_library()
        self.torch = torch
        self.device = torch.device("cuda", device)
        h = C.c_void_p()
        st = self.lib.essa_create(C.byref(h), device)
        if st != ESSA_OK:
            raise EssaError(st, self.lib.essa_status_string(st).decode())
        self.handle = h.value

    # -- plumbing
    def _check(self, st: int):
        if st != ESSA_OK:
            raise EssaError(st, self.lib.essa_last_error(self.handle).decode() or self.lib.essa_status_string(st).decode())

    def close(self):
        if self.handle:
            self.lib.essa_destroy(self.handle)
            self.handle = None

    @property
    def gpu_launches(self) -> int:
        """essa_get_launch_count: kernels of this library enqueued through this context so far."""
        v = C.c_int64(0)
        self._check(self.lib.essa_get_launch_count(self.handle, C.byref(v)))
        return v.value

    def get_status(self) -> int:
        v = C.c_int32(0)
        self._check(self.lib.essa_get_status(self.handle, C.byref(v)))
        return v.value

    def reserve(self, max_tokens: int, max_d_in: int, max_d_out: int):
        self._check(self.lib.essa_reserve(self.handle, max_tokens, max_d_in, max_d_out))

    def set_option(self, option: int, value: int):
        """essa_set_option (ESSA_OPT_PAIR_TILES = 1, ESSA_OPT_FUSE_DOWN = 2)."""
        self._check(self.lib.essa_set_option(self.handle, option, value))

    def reserve_dequant(self, max_d_in: int, max_d_out: int):
        """essa_reserve_dequant: pre-size the scratch that prefill calls on INT8-stored adapters dequantise into."""
        self._check(self.lib.essa_reserve_dequant(self.handle, max_d_in, max_d_out))

    # -- adapters
    def load_adapter(self, ad) -> AdapterHandle:
        """essa_load_adapter from a workloads.Adapter (host arrays; values already bf16/fp16/int8 exact)."""
        torch = self.torch
        bf = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16).contiguous()
        keep = {k: bf(getattr(ad, k)) for k in ("U_A", "V_A", "U_B", "V_B")}
        if ad.w0_dtype == "bf16":
            keep["W0"] = bf(ad.W0)
            dtype, scale_ptr = ESSA_W0_BF16, None
        elif ad.w0_dtype == "int4":  # two 4-bit codes per byte, fp16 scale per (channel, group of 128 features)
            keep["W0"] = torch.from_numpy(np.ascontiguousarray(ad.W0_q, dtype=np.uint8))
            keep["scale"] = torch.from_numpy(np.ascontiguousarray(ad.W0_scale, dtype=np.float16))
            dtype, scale_ptr = ESSA_W0_INT4_GROUP128, keep["scale"].data_ptr()
        else:
            keep["W0"] = torch.from_numpy(np.ascontiguousarray(ad.W0_q, dtype=np.int8))
            keep["scale"] = torch.from_numpy(np.ascontiguousarray(ad.W0_scale, dtype=np.float16))
            dtype, scale_ptr = ESSA_W0_INT8_PERCHANNEL, keep["scale"].data_ptr()
        desc = AdapterDesc(ad.d_in, ad.d_out, ad.rank, dtype, keep["W0"].data_ptr(), scale_ptr, keep["U_A"].data_ptr(),
                           keep["V_A"].data_ptr(), keep["U_B"].data_ptr(), keep["V_B"].data_ptr(), 0)
        h = C.c_void_p()
        self._check(self.lib.essa_load_adapter(self.handle, C.byref(desc), C.byref(h), _stream(None)))
        return AdapterHandle(self, h.value, ad.d_in, ad.d_out, ad.rank, dtype)

    def load_adapter_device(self, d_in, d_out, rank, W0, U_A, V_A, U_B, V_B, w0_scale=None) -> AdapterHandle:
        """essa_load_adapter from device tensors (bf16 bases; W0 bf16, or int8 with fp16 w0_scale)."""
        dtype = ESSA_W0_BF16 if w0_scale is None else ESSA_W0_INT8_PERCHANNEL
        desc = AdapterDesc(d_in, d_out, rank, dtype, W0.data_ptr(), _ptr(w0_scale), U_A.data_ptr(), V_A.data_ptr(),
                           U_B.data_ptr(), V_B.data_ptr(), 1)
        h = C.c_void_p()
        self._check(self.lib.essa_load_adapter(self.handle, C.byref(desc), C.byref(h), _stream(None)))
        return AdapterHandle(self, h.value, d_in, d_out, rank, dtype)

    def cma_state(self, d: int, lam: int, mean0, step0: float) -> "CmaState":
        """essa_cma_create: search-distribution state (m_0 = mean0 host array, sigma_0 = step0, C_0 = I) on the device."""
        return CmaState(self, d, lam, mean0, step0)

    def kv_cache(self, layers: int, num_pages: int, kv_heads: int, head_dim: int, max_seqs: int, max_pages: int, **buffers) -> "KvCache":
        """A paged 4-bit key / value cache on this context's device; buffers: the four tensors of an existing one."""
        return KvCache(self, layers, num_pages, kv_heads, head_dim, max_seqs, max_pages, **buffers)

    def rotary(self, rotary: "Rotary", x, positions, out=None, stream=None):
        """essa_rotary_apply: x [T, heads, head_dim] bf16 (rows may be strided) turned by positions [axes, T] int32 (or [T] for one axis); out may be x."""
        torch, index, shape = self.torch, self.device.index, x.shape
        if len(shape) != 3 or shape[2] != rotary.head_dim or shape[1] < 1:
            raise EssaError(ESSA_ERR_INVALID_ARG, f"rotary: x must be a tensor [T, heads, {rotary.head_dim}]")
        T, heads, d = shape

        def pitch(name, t):  # elements between rows
            ok = t.dtype is torch.bfloat16 and t.get_device() == index and t.shape == shape
            if ok and t.is_contiguous():
                return heads * d
            if ok and T:
                stride = t.stride()
                if stride[2] == 1 and (heads == 1 or stride[1] == d):
                    return stride[0] if T > 1 else heads * d
            raise EssaError(ESSA_ERR_INVALID_ARG, f"rotary: {name} must be a bf16 tensor [T, heads, {d}] on {self.device} whose rows are contiguous")
        ldx = pitch("x", x)
        pp, ldp = rotary._positions(torch, positions, T, index)
        if out is not None:
            ldo = pitch("out", out)
        else:
            ldo = heads * d
            if stream is None:
                out = torch.empty_like(x) if x.is_contiguous() else x.new_empty(shape)
            else:
                with torch.cuda.stream(stream):
                    out = x.new_empty(shape)
        raw = (torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream) or None
        self._check(self.lib.essa_rotary_apply(self.handle, rotary._ref, x.data_ptr() or None, ldx, heads, T, pp, ldp, out.data_ptr() or None, ldo, raw))
        return out

    # -- sampling
    def sample_population(self, mean, step: float, Bfactor, Dvec, seed: int, P: int, out=None, k_begin: int = 0,
                          stream=None):
        """essa_sample_population(_range): sigma[P, d] fp32 on the device."""
        torch = self.torch
        d = mean.numel()
        if out is None:
            out = torch.empty((P, d), dtype=torch.float32, device=self.device)
        if k_begin == 0:
            st = self.lib.essa_sample_population(self.handle, mean.data_ptr(), step, _ptr(Bfactor), _ptr(Dvec), d,
                                                 seed, P, out.data_ptr(), _stream(stream))
        else:
            st = self.lib.essa_sample_population_range(self.handle, mean.data_ptr(), step, _ptr(Bfactor), _ptr(Dvec),
                                                       d, seed, k_begin, P, out.data_ptr(), _stream(stream))
        self._check(st)
        return out

    def sample_population_masked(self, frozen, index, mean_t, step: float, Bfactor_t, Dvec_t, seed: int, P: int,
                                 out=None, k_begin: int = 0, stream=None):
        """essa_sample_population_masked: sigma[P, d] with the columns `index` (int32, device) drawn around mean_t
        and every other column equal to frozen."""
        torch = self.torch
        d = frozen.numel()
        d_t = 0 if index is None else index.numel()
        if out is None:
            out = torch.empty((P, d), dtype=torch.float32, device=self.device)
        st = self.lib.essa_sample_population_masked(self.handle, frozen.data_ptr(), _ptr(index) if d_t else None,
                                                    _ptr(mean_t) if d_t else None, step, _ptr(Bfactor_t), _ptr(Dvec_t),
                                                    d, d_t, seed, k_begin, P, out.data_ptr(), _stream(stream))
        self._check(st)
        return out

    def export_candidates(self, adapter, sigma, sA_col: int, sB_col: int, k_begin: int, k_count: int, want_a=True,
                          want_b=True, stream=None):
        """essa_export_candidates: (A'[k_count, rank, d_in], B'[k_count, d_out, rank]) bf16 on the device."""
        torch = self.torch
        A = torch.empty((k_count, adapter.rank, adapter.d_in), dtype=torch.bfloat16, device=self.device) if want_a else None
        B = torch.empty((k_count, adapter.d_out, adapter.rank), dtype=torch.bfloat16, device=self.device) if want_b else None
        st = self.lib.essa_export_candidates(self.handle, adapter.handle, sigma.data_ptr(), sigma.stride(0), sA_col, sB_col,
                                             k_begin, k_count, _ptr(A) if k_count else None, _ptr(B) if k_count else None,
                                             _stream(stream))
        self._check(st)
        return A, B

    # -- projection
    def _proj(self, fn, adapter, x, seg_offsets, sigma, sA_col, sB_col, out, stream):
        torch = self.torch
        T = x.shape[0]
        P = seg_offsets.numel() - 1
        if out is None:
            out = torch.empty((T, adapter.d_out), dtype=torch.bfloat16, device=self.device)
        st = fn(self.handle, adapter.handle, x.data_ptr() if T else None, T, seg_offsets.data_ptr(), P, sigma.data_ptr(),
                sigma.stride(0) if sigma.dim() == 2 else sigma.numel(), sA_col, sB_col, out.data_ptr() if T else None,
                _stream(stream))
        self._check(st)
        return out

    def apply_projection(self, adapter, x, seg_offsets, sigma, sA_col: int, sB_col: int, out=None, stream=None):
        """essa_apply_projection: y[T, d_out] bf16 (one launch at decode sizes, else rank-down then base + up)."""
        y = self._proj(self.lib.essa_apply_projection, adapter, x, seg_offsets, sigma, sA_col, sB_col, out, stream)
        return y

    def apply_block(self, adapters, xs, seg_offsets, sigma, cols, outs=None, stream=None):
        """essa_apply_block: several projections over the same tokens / segments / sigma table in one call.

        adapters, xs, cols (pairs (sA_col, sB_col)) and outs are parallel sequences; returns the list of outputs."""
        torch = self.torch
        T = xs[0].shape[0]
        P = seg_offsets.numel() - 1
        n = len(adapters)
        if outs is None:
            outs = [torch.empty((T, a.d_out), dtype=torch.bfloat16, device=self.device) for a in adapters]
        arr = (BlockItem * n)()
        for i in range(n):
            arr[i] = BlockItem(adapters[i].handle, xs[i].data_ptr() if T else None, cols[i][0], cols[i][1],
                               outs[i].data_ptr() if T else None)
        st = self.lib.essa_apply_block(self.handle, arr, n, T, seg_offsets.data_ptr(), P, sigma.data_ptr(),
                                       sigma.stride(0) if sigma.dim() == 2 else sigma.numel(), _stream(stream))
        self._check(st)
        return outs

    def prepare_block(self, adapters, xs, seg_offsets, sigma, cols, outs):
        """The arguments of one essa_apply_block call marshalled once; ``run(stream)`` then issues the call with a
        single foreign-function call (at decode sizes the Python-side marshalling of a step is otherwise comparable
        to the step's device time).  The tensors must stay alive and in place while the object is used."""
        return PreparedBlock(self, adapters, xs, seg_offsets, sigma, cols, outs)

    def prepare_layers(self, layers, seg_offsets, sigma):
        """The arguments of one essa_apply_layers call marshalled once.  layers: a list (one entry per layer) of lists
        of (adapter, x, (sA_col, sB_col), y) tuples; ``run(stream)`` issues the call."""
        return PreparedLayers(self, layers, seg_offsets, sigma)

    def apply_layers(self, layers, seg_offsets, sigma, stream=None):
        """essa_apply_layers: the blocks of several layers in one call (see prepare_layers for the argument layout)."""
        PreparedLayers(self, layers, seg_offsets, sigma).run(_stream(stream))

    def prepare_sample_block(self, mean, step: float, Bfactor, Dvec, seed: int, P: int, sigma_out, adapters, xs, seg_offsets,
                             cols, outs, k_begin: int = 0):
        """The arguments of one essa_sample_apply_block call (population draw + the block's projections) marshalled
        once; ``run(stream)`` issues it."""
        return PreparedSampleBlock(self, mean, step, Bfactor, Dvec, seed, P, sigma_out, adapters, xs, seg_offsets, cols, outs,
                                   k_begin)

    def sample_apply_block(self, mean, step: float, Bfactor, Dvec, seed: int, P: int, adapters, xs, seg_offsets, cols,
                           sigma_out=None, outs=None, k_begin: int = 0, stream=None):
        """essa_sample_apply_block: draw the population into sigma_out[P, d] and run the block's projections on it.
        Returns (sigma_out, outs)."""
        torch = self.torch
        d = mean.numel()
        T = xs[0].shape[0]
        if sigma_out is None:
            sigma_out = torch.empty((P, d), dtype=torch.float32, device=self.device)
        if outs is None:
            outs = [torch.empty((T, a.d_out), dtype=torch.bfloat16, device=self.device) for a in adapters]
        prep = PreparedSampleBlock(self, mean, step, Bfactor, Dvec, seed, P, sigma_out, adapters, xs, seg_offsets, cols, outs,
                                   k_begin)
        prep.run(_stream(stream))
        return sigma_out, outs

    def prepare_sample(self, mean, step: float, Bfactor, Dvec, seed: int, P: int, out, k_begin: int = 0):
        """The arguments of one essa_sample_population(_range) call marshalled once; ``run(stream)`` issues it."""
        return PreparedSample(self, mean, step, Bfactor, Dvec, seed, P, out, k_begin)

    def apply_projection_static(self, adapter, x, seg_offsets, sigma, sA_col: int, sB_col: int, out, stream=None):
        """essa_apply_projection_static: same result as apply_projection without any device allocation.

        For callers that cannot allocate when they call (another allocator owns the GPU memory, or no implicit
        synchronisation is tolerable): the library's fixed 512 KB array is the only scratch, so T is limited to
        ESSA_STATIC_MAX_TOKENS (4096) and `out` must be supplied by the caller (this wrapper allocates nothing).
        Calls share that array: keep them ordered on the GPU.
        """
        if out is None:
            raise ValueError("apply_projection_static needs a caller-provided output tensor")
        y = self._proj(self.lib.essa_apply_projection_static, adapter, x, seg_offsets, sigma, sA_col, sB_col, out, stream)
        return y

    def apply_projection_simt(self, adapter, x, seg_offsets, sigma, sA_col: int, sB_col: int, out=None, stream=None):
        """essa_apply_projection_simt: CUDA-core cross-check of the same formula."""
        y = self._proj(self.lib.essa_apply_projection_simt, adapter, x, seg_offsets, sigma, sA_col, sB_col, out, stream)
        return y

    def apply_projection_host(self, adapter, x_host, seg_offsets_host, sigma_host, sA_col: int, sB_col: int, y_host,
                              stream=None):
        """essa_apply_projection_host: host tensors in (bf16 x, int32 offsets, fp32 sigma), host bf16 y out."""
        T = x_host.shape[0]
        P = seg_offsets_host.numel() - 1
        st = self.lib.essa_apply_projection_host(self.handle, adapter.handle, x_host.data_ptr(), T,
                                                 seg_offsets_host.data_ptr(), P, sigma_host.data_ptr(),
                                                 sigma_host.stride(0), sA_col, sB_col, y_host.data_ptr(), _stream(stream))
        self._check(st)
        return y_host

    def apply_block_host(self, adapters, xs_host, seg_offsets_host, sigma_host, cols, ys_host, stream=None):
        """essa_apply_block_host: apply_block with host tensors (bf16 x per projection, int32 offsets, fp32 sigma) and
        host bf16 outputs."""
        T = xs_host[0].shape[0]
        P = seg_offsets_host.numel() - 1
        n = len(adapters)
        arr = (BlockItem * n)()
        for i in range(n):
            arr[i] = BlockItem(adapters[i].handle, xs_host[i].data_ptr() if T else None, cols[i][0], cols[i][1],
                               ys_host[i].data_ptr() if T else None)
        st = self.lib.essa_apply_block_host(self.handle, arr, n, T, seg_offsets_host.data_ptr(), P, sigma_host.data_ptr(),
                                            sigma_host.stride(0), _stream(stream))
        self._check(st)
        return ys_host

    def profile_begin(self, max_calls: int):
        """essa_profile_begin: record per-kernel CUDA events inside the following apply_projection calls."""
        self._check(self.lib.essa_profile_begin(self.handle, max_calls))

    def profile_end(self) -> dict:
        """essa_profile_end: {rank_down_ms, base_up_ms, calls, dropped} summed over the recorded calls."""
        p = Profile()
        self._check(self.lib.essa_profile_end(self.handle, C.byref(p)))
        return {"rank_down_ms": p.rank_down_ms, "base_up_ms": p.base_up_ms, "calls": p.calls, "dropped": p.dropped}

    # -- diagnostics
    def debug_philox(self, ctr, key):
        c = (C.c_uint32 * 4)(*[int(v) for v in ctr])
        k = (C.c_uint32 * 2)(*[int(v) for v in key])
        o = (C.c_uint32 * 4)()
        self._check(self.lib.essa_debug_philox(self.handle, c, k, o))
        return [int(v) for v in o]

    def debug_stream_words(self, seed: int, k_begin: int, k_count: int, n_blocks: int):
        torch = self.torch
        out = torch.empty((k_count, n_blocks, 4), dtype=torch.int32, device=self.device)
        self._check(self.lib.essa_debug_stream_words(self.handle, seed, k_begin, k_count, n_blocks, out.data_ptr(), _stream(None)))
        return out

    def debug_segment_map(self, seg_offsets, T: int):
        torch = self.torch
        out = torch.empty((T,), dtype=torch.int32, device=self.device)
        self._check(self.lib.essa_debug_segment_map(self.handle, seg_offsets.data_ptr(), seg_offsets.numel() - 1, T,
                                                    out.data_ptr() if T else None, _stream(None)))
        return out

    def debug_core_matrix(self, adapter) -> np.ndarray:
        M = np.empty((adapter.rank, adapter.rank), dtype=np.float32)
        self._check(self.lib.essa_debug_core_matrix(self.handle, adapter.handle, M.ctypes.data_as(C.c_void_p)))
        return M
