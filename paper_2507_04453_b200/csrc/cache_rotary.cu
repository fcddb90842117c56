// Rotary positions with several axes: rows of q (or any rows) turned pair by pair, and, in the same launch, keys turned and stored with their
// values in the paged 4-bit cache.
//
// Pair (a, b) with t = position * frequency: (a cos t - b sin t, b cos t + a sin t).  In fp32 the angle of a far position loses its fraction (2^-24 of
// 10^5 radians is a hundredth); here a frequency is a 64-bit fraction of a turn, and the product with a position modulo 2^64 is the angle's fraction, exact but for
// the frequency's own 2^-65: one wide multiplication, then sincospi.
//
// What bounds it: bytes.  Sine and cosine depend on the token and the pair only, so a thread block computes them once for its tokens and
// all their heads use them: a lane keeps those of its eight pairs in registers while its warp walks the heads.
// 33 thousand tokens of 40 + 8 heads of 128, stored too (844 MB): 160 us, 5.3 TB/s.  217 us with one head's loads at a time, three thread blocks per SM and four
// tokens per thread block; two heads at a time 199, eight tokens 175, four thread blocks per SM 160.  Four heads at a time, sixteen tokens: the same.
#include <cmath>

#include "cache_api.cuh"
#include "cache_store.cuh"

namespace essa {
namespace {

constexpr int kRotaryWarps = 8;
constexpr int kUnroll = 2;     // heads of a warp whose loads are on their way together
constexpr int kMaxGroups = 2;  // see rotary_kernel
static_assert(ESSA_ROTARY_MAX_HEADS <= 1 << 30, "");  // (a warp's walk passes the last head by a step or two, in 32 bits)

struct RotaryArgs {
  essa_rotary r;
  const int32_t* positions;  // NULL: the tokens' positions in their sequences
  int64_t ld_pos;
  const __nv_bfloat16* q;
  __nv_bfloat16* q_out;
  int64_t ld_q, ld_q_out;
  int32_t q_heads, T;
};

// Both products rounded, so that the pair's two members are treated alike (a multiply-add would round one product and not the other).
__device__ __forceinline__ float turned(float x, float y, float c, float s) { return __fadd_rn(__fmul_rn(x, c), __fmul_rn(y, s)); }
// Two channels times (cos, sin): the low halves of a and b, then the high ones.
__device__ __forceinline__ void turn_pair(uint32_t& a, uint32_t& b, float2 c0, float2 c1) {
  const float a0 = __uint_as_float(a << 16), a1 = __uint_as_float(a & 0xffff0000u), b0 = __uint_as_float(b << 16), b1 = __uint_as_float(b & 0xffff0000u);
  a = pack_bf16x2(turned(a0, b0, c0.x, -c0.y), turned(a1, b1, c1.x, -c1.y));
  b = pack_bf16x2(turned(b0, a0, c0.x, c0.y), turned(b1, a1, c1.x, c1.y));
}
// Two neighbouring channels as one pair.
__device__ __forceinline__ uint32_t turn_word(uint32_t w, float2 c) {
  const float a = __uint_as_float(w << 16), b = __uint_as_float(w & 0xffff0000u);
  return pack_bf16x2(turned(a, b, c.x, -c.y), turned(b, a, c.x, c.y));
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

// A warp has 32 / (D / 16) tokens, D / 16 lanes each (D = 0: of a.r.head_dim channels, some lanes may have none).  A thread block has `groups` times as many
// (1 or 2): that many sets of warps, each of which deals the heads to its warps and to blockIdx.y in turn.  STORE: K and V are stored (D = 64 or 128).
template <int D, bool STORE>
__global__ void __launch_bounds__(kRotaryWarps * 32, 4)
    rotary_kernel(const __grid_constant__ RotaryArgs a, CacheView v, CacheEntries e, const __nv_bfloat16* k, int64_t ld_k, const __nv_bfloat16* val, int64_t ld_v,
                  int groups, int32_t* status) {
  const int dim = D ? D : a.r.head_dim, lanes = dim / 16, tokens = 32 / lanes, half = dim / 2;
  __shared__ float2 cs_of[256 * kMaxGroups];  // [token][pair]
  __shared__ TokenPlace place[8 * kMaxGroups];
  __shared__ int32_t offsets[STORE ? kOffsetsMax : 1];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t t0 = (int64_t)blockIdx.x * tokens * groups;
  const bool adjacent = a.r.adjacent != 0;
  const int set = kRotaryWarps / groups;  // warps that share tokens
  const int token = lane / lanes + warp / set * tokens, l = lane % lanes;
  const int64_t t = t0 + token;
  const bool in = lane / lanes < tokens && t < a.T;
  // which eight pairs: with halves of a row apart, lanes l and l + lanes / 2 have neighbouring ones (see below)
  const int chunk = adjacent || !STORE ? l : 2 * (l % (lanes / 2)) + l / (lanes / 2);
  const int lo_at = adjacent ? 16 * chunk : 8 * chunk, hi_at = adjacent ? lo_at + 8 : half + lo_at;
  const int first = blockIdx.y * set + warp % set, step = gridDim.y * set;
  const __nv_bfloat16* from = a.q + t * a.ld_q;
  Chunk x[kUnroll];
  const auto load = [&](int h) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (h + u * step >= a.q_heads) break;
      x[u].lo = *reinterpret_cast<const uint4*>(from + (int64_t)(h + u * step) * dim + lo_at);
      x[u].hi = *reinterpret_cast<const uint4*>(from + (int64_t)(h + u * step) * dim + hi_at);
    }
  };
  if (in) load(first);  // (on its way while the tokens are looked up)
  if (STORE) {
    stage_offsets(e, offsets);
    if (tid < tokens * groups) {
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
  for (int i = tid; i < groups * tokens * half; i += kRotaryWarps * 32) {
    const int j = i / half, pair = i - j * half;
    const int64_t t = t0 + j;
    int pos = 0;
    if (a.positions) {
      if (t < a.T) pos = a.positions[a.r.axis[pair] * a.ld_pos + t];
    } else if (STORE) {
      pos = place[j].pos;
    }
    const uint64_t turns = (uint64_t)(int64_t)pos * a.r.turns[pair];
    // (in fp64: no slower here, and sine and cosine are the nearest fp32 numbers)
    double s, c;
    sincospi((double)(int64_t)turns * 0x1p-63, &s, &c);
    cs_of[i] = make_float2((float)c * a.r.magnitude, (float)s * a.r.magnitude);
  }
  __syncthreads();
  float2 cs[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) cs[i] = in ? cs_of[token * half + 8 * chunk + i] : make_float2(0.f, 0.f);
  TokenPlace p{-1, 0, -1};
  if (STORE && in) p = place[token];
  const bool writes_q = in && (!STORE || (p.page != -1 && (a.positions || p.pos >= 0)));
  if (writes_q) {
    __nv_bfloat16* to = a.q_out + t * a.ld_q_out;
    for (int h = first; h < a.q_heads;) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (h + u * step >= a.q_heads) break;
        turn(x[u], cs, adjacent);
        *reinterpret_cast<uint4*>(to + (int64_t)(h + u * step) * dim + lo_at) = x[u].lo;
        *reinterpret_cast<uint4*>(to + (int64_t)(h + u * step) * dim + hi_at) = x[u].hi;
      }
      h += kUnroll * step;
      load(h);
    }
  }
  if constexpr (STORE) {
    constexpr int L = D / 16;
    int h = first - a.q_heads % step;  // (the warps go on in turn)
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
// frac(f / 2 pi) in units of 2^-64, to the nearest, for |f| <= kMaxFrequency: |f| is an integer m below 2^53 times 2^e, e <= -20, and 2^128 / 2 pi (the
// constant, in two halves) times m has to be shifted by 64 - e.  The constant's missing end is m 2^(e - 64) < 2^-31 units, what
// the product leaves out 2^-20.
constexpr double kMaxFrequency = 4294967296.0;
uint64_t turns_of(double f) {
  constexpr uint64_t kHigh = 0x28be60db9391054aull, kLow = 0x7f09d5f47d4d3770ull;
  int e;
  const uint64_t m = (uint64_t)std::ldexp(std::frexp(std::fabs(f), &e), 53);
  const int shift = 53 - e;  // (by 64 already)
  if (shift > 120) return 0;  // (less than half a unit)
  const unsigned __int128 product = (unsigned __int128)m * kHigh + (uint64_t)((unsigned __int128)m * kLow >> 64);  // < 2^115
  const uint64_t turns = (uint64_t)((product + ((unsigned __int128)1 << (shift - 1))) >> shift);
  return f < 0 ? 0 - turns : turns;
}
// How a call of T tokens is divided: token groups of a thread block, and what share of the heads.
struct RotaryGrid {
  dim3 grid;
  int groups;
};
// Two groups share a thread block's look-ups where that leaves every SM two thread blocks (9 thousand tokens of 14 heads of 64: 10 us, with one group 11.5); a
// decode step's few tokens have their heads dealt to several thread blocks, until there are two for every SM or a head for each warp.
RotaryGrid rotary_grid(const essa_ctx* ctx, int64_t T, int head_dim, int heads) {
  const int64_t tokens = 32 / (head_dim / 16);
  int groups = kMaxGroups;
  while (groups > 1 && (T + tokens * groups - 1) / (tokens * groups) < 2 * ctx->sm_count) groups /= 2;
  const int64_t blocks = (T + tokens * groups - 1) / (tokens * groups);
  int splits = 1;
  while (blocks * splits < 2 * ctx->sm_count && splits * (kRotaryWarps / groups) < heads) splits *= 2;
  return {dim3((unsigned)blocks, splits), groups};
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
    if (!(std::fabs(frequencies[i]) <= kMaxFrequency)) return ESSA_ERR_INVALID_ARG;
    if (axis && (axis[i] < 0 || axis[i] >= axes)) return ESSA_ERR_INVALID_ARG;
    r.turns[i] = turns_of(frequencies[i]);
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
  if (heads > ESSA_ROTARY_MAX_HEADS) return fail(ctx, ESSA_ERR_UNSUPPORTED_SHAPE, "rotary_apply: heads > ESSA_ROTARY_MAX_HEADS");
  if (T == 0) return ESSA_OK;
  const int64_t width = (int64_t)heads * rotary->head_dim;
  ESSA_TRY(check_rows(ctx, "rotary_apply", "x", x, ld_x, width));
  ESSA_TRY(check_rows(ctx, "rotary_apply", "out", out, ld_out, width));
  if (out == x && ld_out != ld_x) return fail(ctx, ESSA_ERR_INVALID_ARG, "rotary_apply: in place, the pitches must be the same");
  if (!positions) return fail(ctx, ESSA_ERR_INVALID_ARG, "rotary_apply: positions is NULL");
  ESSA_TRY(check_positions(ctx, "rotary_apply", positions, ld_positions, T));
  DeviceGuard guard(ctx->device);
  const RotaryArgs a{*rotary, positions, ld_positions, static_cast<const __nv_bfloat16*>(x), static_cast<__nv_bfloat16*>(out), ld_x, ld_out, heads, T};
  const RotaryGrid g = rotary_grid(ctx, T, rotary->head_dim, heads);
  const auto run = [&](auto kernel) {
    kernel<<<g.grid, kRotaryWarps * 32, 0, static_cast<cudaStream_t>(stream_v)>>>(a, CacheView{}, CacheEntries{}, nullptr, 0, nullptr, 0, g.groups, ctx->d_status);
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
  if (q_heads > ESSA_ROTARY_MAX_HEADS) return fail(ctx, ESSA_ERR_UNSUPPORTED_SHAPE, "cache_append_rotary: q_heads > ESSA_ROTARY_MAX_HEADS");
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
  const RotaryGrid g = rotary_grid(ctx, T, v.head_dim, q_heads + v.kv_heads);
  const auto run = [&](auto kernel) {
    kernel<<<g.grid, kRotaryWarps * 32, 0, static_cast<cudaStream_t>(stream_v)>>>(a, v, e, static_cast<const __nv_bfloat16*>(k), ld_k,
                                                                                 static_cast<const __nv_bfloat16*>(val), ld_v, g.groups, ctx->d_status);
  };
  v.head_dim == 64 ? run(rotary_kernel<64, true>) : run(rotary_kernel<128, true>);
  return launched(ctx, "cache_append_rotary", 1);
}

}  // extern "C"
