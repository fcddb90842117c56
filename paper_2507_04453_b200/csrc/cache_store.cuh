// What the kernels that store and move tokens share: which entry a row belongs to, where its token is cached, 4-bit storage of a group, and
// checks of the page table.
#pragma once

#include "cache_list.cuh"

namespace essa {

#ifdef __CUDACC__
constexpr int kOffsetsMax = 2048;  // offsets that a thread block searches in shared memory

// The offsets of a call in shared memory, if they fit (all threads of the block; a search of dependent loads from L2 would take
// longer than the rest of a decode step's append).
__device__ __forceinline__ void stage_offsets(const CacheEntries& e, int32_t* sm) {
  if (!e.off || e.n >= kOffsetsMax) return;
  for (int i = threadIdx.x; i <= e.n; i += blockDim.x) sm[i] = __ldg(e.off + i);
  __syncthreads();
}
// The entry that row t belongs to (off[i] <= t < off[i + 1]); -1 if none.
__device__ __forceinline__ int entry_of(const CacheEntries& e, const int32_t* sm, int t) {
  if (!e.off) return t;
  if (e.n == 0) return -1;
  if (e.n >= kOffsetsMax) return t < __ldg(e.off) || t >= __ldg(e.off + e.n) ? -1 : find_candidate(e.off, e.n, t);
  if (t < sm[0] || t >= sm[e.n]) return -1;
  int lo = 0, hi = e.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sm[mid] <= t) lo = mid; else hi = mid;
  }
  return lo;
}

// Where row t of the call is cached: page (>= 0) and offset in it; -1 if the row belongs to no entry, -2 if it should be in
// the cache and is not.
__device__ __forceinline__ int locate_token(const CacheView& v, const CacheEntries& e, const int32_t* sm, int t, int* offset, int* end) {
  *end = t + 1;  // (rows up to here follow in the same entry and page)
  const int i = entry_of(e, sm, t);
  if (i < 0) return -1;
  const EntryInfo info = load_entry(v, e, i);
  const int pos = info.len - info.rows + (t - info.row0);
  if (info.slot < 0 || t >= info.row0 + info.rows || pos < 0) return -2;
  const int page = __ldg(v.table + (int64_t)info.slot * v.max_pages + pos / kPageTokens);
  if (page < 0 || page >= v.num_pages) return -2;
  *offset = pos % kPageTokens;
  *end = min(t + kPageTokens - *offset, info.row0 + info.rows);
  return page;
}

// Sixteen channels of a group of 64; the other three neighbours (lanes of an aligned group of four) hold the rest.  (With eight channels a
// lane, what every lane does for a token made it 20 instructions a value instead of 16: 54 us for 32 thousand tokens of 8 heads of 128, now 51.)
struct Piece {
  uint4 raw[2];  // bf16
  __device__ __forceinline__ float value(int i) const {
    const uint4& r = raw[i >> 3];
    const uint32_t w = (i & 7) < 2 ? r.x : (i & 7) < 4 ? r.y : (i & 7) < 6 ? r.z : r.w;
    return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
  }
};
struct Packed {
  uint2 codes;
  __half scale, low;
  bool fits;
};
__device__ __forceinline__ __nv_bfloat162 as_bf162(uint32_t v) { return *reinterpret_cast<__nv_bfloat162*>(&v); }

// 4-bit storage of the group.  The minimum and maximum are found on bf16 pairs (exact, NaN stays NaN); one shuffle a step carries
// (max, -min).
__device__ __forceinline__ Packed pack_group(const Piece& x) {
  __nv_bfloat162 top = as_bf162(x.raw[0].x), low = top;
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    const uint4& r = x.raw[i >> 2];
    const __nv_bfloat162 v = as_bf162((i & 3) == 0 ? r.x : (i & 3) == 1 ? r.y : (i & 3) == 2 ? r.z : r.w);
    top = __hmax2_nan(top, v);
    low = __hmin2_nan(low, v);
  }
  low = __hneg2(low);
  __nv_bfloat162 both = __hmax2_nan(__lows2bfloat162(top, low), __highs2bfloat162(top, low));
#pragma unroll
  for (int step = 1; step < 4; step <<= 1) both = __hmax2_nan(both, __shfl_xor_sync(0xffffffffu, both, step));
  const float high = __low2float(both);
  Packed p;
  p.low = __float2half_rn(-__high2float(both));
  const float base = __half2float(p.low);
  // (high - base) / 15, correctly rounded (Markstein: a quotient from the rounded reciprocal, corrected by its exact remainder)
  const float range = high - base, q0 = range * (1.f / 15.f);
  p.scale = __float2half_rn(fmaf(fmaf(-15.f, q0, range), 1.f / 15.f, q0));
  const float s = __half2float(p.scale);
  p.fits = s < INFINITY && fabsf(base) < INFINITY;  // (false for NaN)
  p.codes = make_uint2(0, 0);
  if (s > 0.f) {
    // rint((x - base) / s), clipped to 0 .. 15, as x * k - base * k with k = 1 / (15 s): the saturating multiply-add clips it to 0 .. 1 and
    // the next one takes it to 0 .. 15 and rounds.  With |base| <= 100 s the products are wrong by (115 + 100) 2^-22 < 10^-4 steps at most,
    // which matters next to a half only; then, and with a larger base, the division is made.  (The division, the rounding and the conversion of
    // every value kept the kernel at a quarter of the memory's rate: 128 us for 32 thousand tokens of 8 heads of 128, 209 MB; a subtraction, a
    // multiplication and two comparisons to clip every value: 64 us, so 54.)
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
    const float magic = 12582912.f;  // 1.5 * 2^23: what is added to it is rounded to an integer, ties to even
    const float k = inv * (1.f / 15.f), offset = -base * k;
    const uint64_t magic2 = pack_f32x2(magic, magic), back2 = pack_f32x2(-magic, -magic), up2 = pack_f32x2(15.f, 15.f), down2 = pack_f32x2(-15.f, -15.f);
    float far = fabsf(base) <= 100.f * s ? 0.f : 1.f;
    uint32_t half[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float n[4], first = 0.f;
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        const uint64_t t = pack_f32x2(__saturatef(fmaf(x.value(4 * j + i), k, offset)), __saturatef(fmaf(x.value(4 * j + i + 1), k, offset)));
        const uint64_t c = fma_f32x2(t, up2, magic2), r = add_f32x2(c, back2);
        float c0, c1, d0, d1;
        unpack_f32x2(c, c0, c1);
        unpack_f32x2(r, n[i], n[i + 1]);
        unpack_f32x2(fma_f32x2(t, down2, r), d0, d1);
        far = fmaxf(far, fmaxf(fabsf(d0), fabsf(d1)));
        if (i == 0) first = c0;
      }
      half[j] = __float_as_uint(fmaf(n[3], 4096.f, fmaf(n[2], 256.f, fmaf(n[1], 16.f, first))));  // (four codes in the lowest 16 bits)
    }
    p.codes = make_uint2(__byte_perm(half[0], half[1], 0x5410), __byte_perm(half[2], half[3], 0x5410));
    if (far > 0.4999f) {
      p.codes = make_uint2(0, 0);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        (i < 8 ? p.codes.x : p.codes.y) |= (__float_as_uint(fminf(fmaxf(__fdiv_rn(x.value(i) - base, s), 0.f), 15.f) + magic) & 15u) << (4 * (i & 7));
    }
  }
  return p;
}

// Stores a token of kv head h: lane `lane` of its D / 16 neighbouring ones has channels 16 lane .. of K and V.  page < 0: nothing is stored (all
// lanes of the warp take part all the same).
template <int D>
__device__ __forceinline__ void store_token(const CacheView& v, int h, int lane, int page, int offset, const Piece& k, const Piece& val) {
  constexpr int L = D / 16;
  Packed pk = pack_group(k), pv = pack_group(val);
  // one lane that does not fit makes the token (its L lanes) NaN
  const uint32_t misfits = __ballot_sync(0xffffffffu, !(pk.fits && pv.fits)) >> ((threadIdx.x & 31) / L * L) & ((1u << L) - 1);
  if (misfits) {
    pk.codes = pv.codes = make_uint2(0, 0);
    pk.scale = pv.scale = pv.low = __ushort_as_half(0);  // (V 0: it meets weights 0 in the rows that do not see the token)
    pk.low = __ushort_as_half(0x7e00);
  }
  if (page < 0) return;
  uint8_t* run = v.pages + page * v.page_bytes + (int64_t)h * 72 * D;
  uint8_t* code = run + (lane >> 1) * 1024 + offset * 16 + (lane & 1) * 8;
  *reinterpret_cast<uint2*>(code) = pk.codes;
  *reinterpret_cast<uint2*>(code + 32 * D) = pv.codes;
  if ((lane & 3) == 0) {
    __half2* meta = reinterpret_cast<__half2*>(run + 64 * D + ((lane >> 2) * kPageTokens + offset) * 4);
    meta[0] = __halves2half2(pk.scale, pk.low);
    meta[D] = __halves2half2(pv.scale, pv.low);
  }
}

// ---- pages
__device__ __forceinline__ int pages_of(int tokens) { return tokens / kPageTokens + (tokens % kPageTokens != 0); }

// How many sequences hold the page that a table entry names: 0 for one that is free, or not in the pool.
__device__ __forceinline__ int holders(const CacheView& v, int page) { return page >= 0 && page < v.num_pages ? v.refs[page] : 0; }

// Whether the n slots lie in [0, max_seqs) and are distinct.  `seen`: shared bitmap of max_seqs bits, left with the slots' bits
// set.  Every thread of the block gets the answer.
__device__ inline bool slots_distinct(const int32_t* slots, int n, int max_seqs, uint32_t* seen) {
  for (int i = threadIdx.x; i < (max_seqs + 31) / 32; i += blockDim.x) seen[i] = 0;
  __syncthreads();
  bool ok = true;
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int s = slots ? slots[i] : i;
    if (s < 0 || s >= max_seqs) { ok = false; continue; }
    if (atomicOr(&seen[s >> 5], 1u << (s & 31)) >> (s & 31) & 1) ok = false;
  }
  return __syncthreads_and(ok);
}
#endif

}  // namespace essa
