// Rotary positions with several axes: rows of q (or any rows) turned pair by pair, and, in the same launch, keys turned and stored with their
// values in the paged 4-bit cache.
//
// Pair (a, b) with t = position * frequency: (a cos t - b sin t, b cos t + a sin t).  In fp32 the angle of a far position loses its fraction (2^-24 of
// 10^5 radians is a hundredth); here a frequency is a 64-bit fraction of a turn, and the product with a position modulo 2^64 is the angle's fraction, exact but for
// the frequency's own 2^-64: one wide multiplication, then sincospif of its upper 32 bits.
//
// What bounds it: bytes.  Sine and cosine depend on the token and the pair only, so a thread block computes them once for its tokens and
// all their heads use them: a lane keeps those of its eight pairs in registers while its warp walks the heads.
#include <cmath>

#include "cache_api.cuh"
#include "cache_store.cuh"

namespace essa {
namespace {

constexpr int kRotaryWarps = 8;

struct RotaryArgs {
  essa_rotary r;
  const int32_t* positions;  // NULL: the tokens' positions in their sequences
  int64_t ld_pos;
  const __nv_bfloat16* q;
  __nv_bfloat16* q_out;
  int64_t ld_q, ld_q_out;
  int32_t q_heads, T;
};

// Two channels times (cos, sin): the low halves of a and b, then the high ones.
__device__ __forceinline__ void turn_pair(uint32_t& a, uint32_t& b, float2 c0, float2 c1) {
  const float a0 = __uint_as_float(a << 16), a1 = __uint_as_float(a & 0xffff0000u), b0 = __uint_as_float(b << 16), b1 = __uint_as_float(b & 0xffff0000u);
  a = pack_bf16x2(fmaf(a0, c0.x, -b0 * c0.y), fmaf(a1, c1.x, -b1 * c1.y));
  b = pack_bf16x2(fmaf(b0, c0.x, a0 * c0.y), fmaf(b1, c1.x, a1 * c1.y));
}
// Two neighbouring channels as one pair.
__device__ __forceinline__ uint32_t turn_word(uint32_t w, float2 c) {
  const float a = __uint_as_float(w << 16), b = __uint_as_float(w & 0xffff0000u);
  return pack_bf16x2(fmaf(a, c.x, -b * c.y), fmaf(b, c.x, a * c.y));
}
// A lane's sixteen channels of a row: eight pairs.
struct Chunk {
  uint4 lo, hi;  // half a row apart (channels 8 c .. and D / 2 + 8 c ..), or neighbours (16 c .., 16 c + 8 ..)
};
__device__ __forceinline__ void turn(Chunk& x, const float2 (&cs)[8], bool adjacent) {
  uint32_t* lo = &x.lo.x;
  uint32_t* hi = &x.hi.x;
  if (adjacent) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo[i] = turn_word(lo[i], cs[i]);
      hi[i] = turn_word(hi[i], cs[4 + i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) turn_pair(lo[i], hi[i], cs[2 * i], cs[2 * i + 1]);
  }
}

// What a thread block knows of one of its tokens.
struct TokenPlace {
  int page, offset;  // page -1: of no entry, -2: not in the cache
  int pos;           // -1: unknown
};

// A warp has 32 / (D / 16) tokens, D / 16 lanes each (D = 0: of a.r.head_dim channels, some lanes may have none); the thread block's warps take the
// heads in turn, those of blockIdx.y too.  STORE: K and V are stored (D = 64 or 128).
template <int D, bool STORE>
__global__ void __launch_bounds__(kRotaryWarps * 32) rotary_kernel(const __grid_constant__ RotaryArgs a, CacheView v, CacheEntries e, const __nv_bfloat16* k, int64_t ld_k,
                                                                   const __nv_bfloat16* val, int64_t ld_v, int32_t* status) {
  const int dim = D ? D : a.r.head_dim, lanes = dim / 16, tokens = 32 / lanes, half = dim / 2;
  __shared__ float2 cs_of[256];  // [token][pair]
  __shared__ TokenPlace place[16];
  __shared__ int32_t offsets[STORE ? kOffsetsMax : 1];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t t0 = (int64_t)blockIdx.x * tokens;
  const bool adjacent = a.r.adjacent != 0;
  if (STORE) {
    stage_offsets(e, offsets);
    if (tid < tokens) {
      TokenPlace p{-1, 0, -1};
      const int64_t t = t0 + tid;
      const int i = t < a.T ? entry_of(e, offsets, (int)t) : -1;
      if (i >= 0) {
        const EntryInfo info = load_entry(v, e, i);
        const int pos = info.len - info.rows + ((int)t - info.row0);
        p.page = -2;
        if (t < info.row0 + info.rows && info.slot >= 0 && pos >= 0) {
          p.pos = pos;
          p.offset = pos % kPageTokens;
          const int page = __ldg(v.table + (int64_t)info.slot * v.max_pages + pos / kPageTokens);
          if (page >= 0 && page < v.num_pages && __ldg(v.refs + page) == 1) p.page = page;  // (shared or free: not this sequence's to write)
        }
        if (p.page == -2 && blockIdx.y == 0) cache_fault(status);
      }
      place[tid] = p;
    }
    __syncthreads();
  }
  for (int i = tid; i < tokens * half; i += kRotaryWarps * 32) {
    const int j = i / half, pair = i - j * half;
    const int64_t t = t0 + j;
    int pos = 0;
    if (a.positions) {
      if (t < a.T) pos = a.positions[a.r.axis[pair] * a.ld_pos + t];
    } else if (STORE) {
      pos = place[j].pos;
    }
    const uint64_t turns = (uint64_t)(int64_t)pos * a.r.turns[pair] + (1ull << 31);
    float s, c;
    sincospif((float)(int32_t)(turns >> 32) * 0x1p-31f, &s, &c);
    cs_of[i] = make_float2(c * a.r.magnitude, s * a.r.magnitude);
  }
  __syncthreads();
  const int token = lane / lanes, l = lane % lanes;
  const int64_t t = t0 + token;
  // which eight pairs: with halves of a row apart, lanes l and l + lanes / 2 have neighbouring ones (see below)
  const int chunk = adjacent || !STORE ? l : 2 * (l % (lanes / 2)) + l / (lanes / 2);
  const int lo_at = adjacent ? 16 * chunk : 8 * chunk, hi_at = adjacent ? lo_at + 8 : half + lo_at;
  float2 cs[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) cs[i] = token < tokens ? cs_of[token * half + 8 * chunk + i] : make_float2(0.f, 0.f);
  const bool in = token < tokens && t < a.T;
  TokenPlace p{-1, 0, -1};
  if (STORE && in) p = place[token];
  const bool writes_q = in && (!STORE || (p.page != -1 && (a.positions || p.pos >= 0)));
  const int first = blockIdx.y * kRotaryWarps + warp, step = gridDim.y * kRotaryWarps;
  int h = first;
  if (writes_q) {
    const __nv_bfloat16* from = a.q + t * a.ld_q;
    __nv_bfloat16* to = a.q_out + t * a.ld_q_out;
    for (; h < a.q_heads; h += step) {
      Chunk x;
      x.lo = *reinterpret_cast<const uint4*>(from + (int64_t)h * dim + lo_at);
      x.hi = *reinterpret_cast<const uint4*>(from + (int64_t)h * dim + hi_at);
      turn(x, cs, adjacent);
      *reinterpret_cast<uint4*>(to + (int64_t)h * dim + lo_at) = x.lo;
      *reinterpret_cast<uint4*>(to + (int64_t)h * dim + hi_at) = x.hi;
    }
  }
  if constexpr (STORE) {
    constexpr int L = D / 16;
    h = first - a.q_heads % step;  // (the warps go on in turn)
    if (h < 0) h += step;
    for (; h < v.kv_heads; h += step) {
      Chunk xk;
      Piece pk, pv;
      xk.lo = xk.hi = pv.raw[0] = pv.raw[1] = make_uint4(0, 0, 0, 0);
      if (in && p.page >= 0) {
        const __nv_bfloat16* from = k + t * ld_k + h * D;
        xk.lo = *reinterpret_cast<const uint4*>(from + lo_at);
        xk.hi = *reinterpret_cast<const uint4*>(from + hi_at);
        const uint4* from_v = reinterpret_cast<const uint4*>(val + t * ld_v + h * D + l * 16);
        pv.raw[0] = from_v[0];
        pv.raw[1] = from_v[1];
      }
      turn(xk, cs, adjacent);
      if (adjacent) {
        pk.raw[0] = xk.lo;
        pk.raw[1] = xk.hi;
      } else {
        // Lane l is to have channels 16 l .. 16 l + 15 (a group of 64 is four lanes): of the first half of the lanes, both chunks' first halves
        const bool upper = l >= L / 2;
        uint4 mine = upper ? xk.hi : xk.lo, other = upper ? xk.lo : xk.hi;
        other.x = __shfl_xor_sync(0xffffffffu, other.x, L / 2);
        other.y = __shfl_xor_sync(0xffffffffu, other.y, L / 2);
        other.z = __shfl_xor_sync(0xffffffffu, other.z, L / 2);
        other.w = __shfl_xor_sync(0xffffffffu, other.w, L / 2);
        pk.raw[0] = upper ? other : mine;
        pk.raw[1] = upper ? mine : other;
      }
      store_token<D>(v, h, l, in ? p.page : -1, p.offset, pk, pv);
    }
  }
}

const char* rotary_problem(const essa_rotary* r, int32_t* code) {
  *code = ESSA_ERR_INVALID_ARG;
  if (!r) return "rotary is NULL";
  *code = ESSA_ERR_UNSUPPORTED_SHAPE;
  if (r->head_dim < 16 || r->head_dim > ESSA_ROTARY_MAX_DIM || r->head_dim % 16) return "head_dim must be a multiple of 16 up to ESSA_ROTARY_MAX_DIM";
  if (r->axes < 1 || r->axes > ESSA_ROTARY_MAX_AXES) return "axes outside 1 .. ESSA_ROTARY_MAX_AXES";
  *code = ESSA_ERR_INVALID_ARG;
  for (int i = 0; i < r->head_dim / 2; ++i)
    if (r->axis[i] >= r->axes) return "a pair's axis is not below axes";
  *code = ESSA_OK;
  return nullptr;
}
int32_t check_positions(essa_ctx* ctx, const char* what, const int32_t* positions, int64_t ld, int32_t T) {
  if (reinterpret_cast<uintptr_t>(positions) & 3) return fail(ctx, ESSA_ERR_INVALID_ARG, std::string(what) + ": positions must be 4-byte aligned");
  if (ld < T) return fail(ctx, ESSA_ERR_INVALID_ARG, std::string(what) + ": the rows of positions must hold T of them");
  return ESSA_OK;
}
// Heads are dealt to blockIdx.y until there are two thread blocks for every SM (a decode step's few tokens), a head or more for each warp.
int head_splits(const essa_ctx* ctx, int64_t blocks, int heads) {
  int splits = 1;
  while (blocks * splits < 2 * ctx->sm_count && splits * kRotaryWarps < heads) splits *= 2;
  return splits;
}

}  // namespace
}  // namespace essa

using namespace essa;

extern "C" {

int32_t essa_rotary_make(int32_t head_dim, int32_t axes, int32_t adjacent, float magnitude, const double* frequencies, const int32_t* axis, essa_rotary* out) {
  if (!out || !frequencies || !(fabsf(magnitude) <= 3.4028234e38f)) return ESSA_ERR_INVALID_ARG;
  essa_rotary r = {};
  r.head_dim = head_dim;
  r.axes = axes;
  r.adjacent = adjacent != 0;
  r.magnitude = magnitude;
  int32_t code;
  if (rotary_problem(&r, &code)) return code;
  for (int i = 0; i < head_dim / 2; ++i) {
    if (!(std::fabs(frequencies[i]) <= 1e300)) return ESSA_ERR_INVALID_ARG;
    if (axis && (axis[i] < 0 || axis[i] >= axes)) return ESSA_ERR_INVALID_ARG;
    const long double turn = (long double)frequencies[i] / 6.283185307179586476925286766559005768L, part = turn - std::floor(turn);
    r.turns[i] = part >= 1.0L ? 0 : (uint64_t)(part * 18446744073709551616.0L);
    r.axis[i] = (uint8_t)(axis ? axis[i] : 0);
  }
  *out = r;
  return ESSA_OK;
}

int32_t essa_rotary_apply(essa_ctx* ctx, const essa_rotary* rotary, const void* x, int64_t ld_x, int32_t heads, int32_t T, const int32_t* positions,
                          int64_t ld_positions, void* out, int64_t ld_out, void* stream_v) {
  if (!ctx) return ESSA_ERR_INVALID_ARG;
  int32_t code;
  if (const char* why = rotary_problem(rotary, &code)) return fail(ctx, code, std::string("rotary_apply: ") + why);
  if (heads < 1 || T < 0) return fail(ctx, ESSA_ERR_INVALID_ARG, "rotary_apply: heads must be positive, T not negative");
  if (T == 0) return ESSA_OK;
  const int64_t width = (int64_t)heads * rotary->head_dim;
  ESSA_TRY(check_rows(ctx, "rotary_apply", "x", x, ld_x, width));
  ESSA_TRY(check_rows(ctx, "rotary_apply", "out", out, ld_out, width));
  if (out == x && ld_out != ld_x) return fail(ctx, ESSA_ERR_INVALID_ARG, "rotary_apply: in place, the pitches must be the same");
  if (!positions) return fail(ctx, ESSA_ERR_INVALID_ARG, "rotary_apply: positions is NULL");
  ESSA_TRY(check_positions(ctx, "rotary_apply", positions, ld_positions, T));
  DeviceGuard guard(ctx->device);
  const RotaryArgs a{*rotary, positions, ld_positions, static_cast<const __nv_bfloat16*>(x), static_cast<__nv_bfloat16*>(out), ld_x, ld_out, heads, T};
  const int64_t tokens = 32 / (rotary->head_dim / 16), blocks = (T + tokens - 1) / tokens;
  const dim3 grid((unsigned)blocks, head_splits(ctx, blocks, heads));
  const auto run = [&](auto kernel) {
    kernel<<<grid, kRotaryWarps * 32, 0, static_cast<cudaStream_t>(stream_v)>>>(a, CacheView{}, CacheEntries{}, nullptr, 0, nullptr, 0, ctx->d_status);
  };
  if (rotary->head_dim == 64) run(rotary_kernel<64, false>);
  else if (rotary->head_dim == 128) run(rotary_kernel<128, false>);
  else run(rotary_kernel<0, false>);
  return launched(ctx, "rotary_apply", 1);
}

int32_t essa_cache_append_rotary(essa_ctx* ctx, const essa_cache_desc* cache, int32_t layer, const essa_rotary* rotary, const void* q, int64_t ld_q, int32_t q_heads,
                                 const void* k, int64_t ld_k, const void* val, int64_t ld_v, int32_t T, const int32_t* positions, int64_t ld_positions,
                                 const int32_t* slots, const int32_t* tok_offsets, int32_t n, void* q_out, int64_t ld_q_out, void* stream_v) {
  CacheView v;
  ESSA_TRY(view_of(ctx, "cache_append_rotary", cache, layer, &v));
  int32_t code;
  if (const char* why = rotary_problem(rotary, &code)) return fail(ctx, code, std::string("cache_append_rotary: ") + why);
  if (rotary->head_dim != v.head_dim) return fail(ctx, ESSA_ERR_INVALID_ARG, "cache_append_rotary: the rotary's head_dim is not the cache's");
  const CacheEntries e{slots, tok_offsets, n, T};
  ESSA_TRY(check_entries(ctx, "cache_append_rotary", e));
  if (q_heads < 1) return fail(ctx, ESSA_ERR_INVALID_ARG, "cache_append_rotary: q_heads must be positive");
  if (T == 0 || n == 0) return ESSA_OK;
  const int64_t width = (int64_t)v.kv_heads * v.head_dim, q_width = (int64_t)q_heads * v.head_dim;
  ESSA_TRY(check_rows(ctx, "cache_append_rotary", "q", q, ld_q, q_width));
  ESSA_TRY(check_rows(ctx, "cache_append_rotary", "q_out", q_out, ld_q_out, q_width));
  ESSA_TRY(check_rows(ctx, "cache_append_rotary", "k", k, ld_k, width));
  ESSA_TRY(check_rows(ctx, "cache_append_rotary", "v", val, ld_v, width));
  if (q_out == q && ld_q_out != ld_q) return fail(ctx, ESSA_ERR_INVALID_ARG, "cache_append_rotary: in place, the pitches must be the same");
  if (positions) ESSA_TRY(check_positions(ctx, "cache_append_rotary", positions, ld_positions, T));
  DeviceGuard guard(ctx->device);
  const RotaryArgs a{*rotary, positions, ld_positions, static_cast<const __nv_bfloat16*>(q), static_cast<__nv_bfloat16*>(q_out), ld_q, ld_q_out, q_heads, T};
  const int64_t tokens = 32 / (v.head_dim / 16), blocks = (T + tokens - 1) / tokens;
  const dim3 grid((unsigned)blocks, head_splits(ctx, blocks, q_heads + v.kv_heads));
  const auto run = [&](auto kernel) {
    kernel<<<grid, kRotaryWarps * 32, 0, static_cast<cudaStream_t>(stream_v)>>>(a, v, e, static_cast<const __nv_bfloat16*>(k), ld_k, static_cast<const __nv_bfloat16*>(val),
                                                                               ld_v, ctx->d_status);
  };
  v.head_dim == 64 ? run(rotary_kernel<64, true>) : run(rotary_kernel<128, true>);
  return launched(ctx, "cache_append_rotary", 1);
}

}  // extern "C"
