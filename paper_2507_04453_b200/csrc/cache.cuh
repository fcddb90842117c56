// Paged 4-bit key / value cache: the device view of a cache and what its kernels share.
//
// A page holds kPageTokens tokens of one layer: for each kv head one run of 72 * head_dim bytes,
//   codes of K, codes of V   [head_dim / 32][64 tokens][16 bytes], two 4-bit codes per byte, low nibble = even channel;
//   (scale, minimum) of K, of V   [head_dim / 64][64 tokens] half2, one pair per group of 64 channels.
// Why this order: a (page, kv head) run is one contiguous bulk copy; eight tokens of a 32-channel chunk are 128 contiguous
// bytes, so that ldmatrix reads them without bank conflicts, as they are for K and transposed for V.
#pragma once

#include "common.cuh"

namespace essa {

constexpr int kPageTokens = ESSA_CACHE_PAGE_TOKENS;
constexpr int kCacheGroup = ESSA_CACHE_GROUP;

struct CacheView {
  uint8_t* pages;  // of the layer in question
  int32_t* table;
  int32_t* lengths;
  int32_t* refs;
  int64_t page_bytes, layer_bytes;
  int32_t num_pages, kv_heads, head_dim, max_seqs, max_pages, layers;
};

// One call's entries: entry i adds / asks for rows [off[i], off[i+1]) on sequence slots[i].
struct CacheEntries {
  const int32_t* slots;  // NULL: entry i is sequence i
  const int32_t* off;    // NULL: entry i has the one row i
  int32_t n;
  int32_t T;
};

// What entry i stands for, with everything that comes from device memory brought into range: a slot outside the cache
// gives slot -1 (and length 0), offsets are clamped to [0, T], a length to what the page table can hold.
struct EntryInfo {
  int slot, row0, rows, len;
};

struct AttendArgs;  // cache_list.cuh
// cache_attend.cu (few query rows per sequence) and cache_tiles.cu (many): rows_hint = most query rows (tokens x heads of a group)
// that an entry is expected to have; both are right for any number.
int64_t attend_decode_workspace(int head_dim, int64_t rows_hint, int sm_count);
int32_t launch_attend_decode(essa_ctx* ctx, AttendArgs& a, int64_t rows_hint, cudaStream_t stream);
int64_t attend_tiles_workspace(int head_dim, int sm_count);
int32_t launch_attend_tiles(essa_ctx* ctx, AttendArgs& a, cudaStream_t stream);

#ifdef __CUDACC__
__device__ __forceinline__ EntryInfo load_entry(const CacheView& v, const CacheEntries& e, int i) {
  EntryInfo r;
  int lo = i, hi = i + 1;
  if (e.off) { lo = __ldg(e.off + i); hi = __ldg(e.off + i + 1); }
  lo = min(max(lo, 0), e.T);
  hi = min(max(hi, 0), e.T);
  r.row0 = lo;
  r.rows = max(hi - lo, 0);
  r.slot = e.slots ? __ldg(e.slots + i) : i;
  if (r.slot < 0 || r.slot >= v.max_seqs) r.slot = -1;
  r.len = r.slot < 0 ? 0 : min(max(v.lengths[r.slot], 0), v.max_pages * kPageTokens);
  return r;
}

// A device-side condition that the call could not check on the host: recorded once, read by essa_get_status.
__device__ __forceinline__ void cache_fault(int32_t* status) { atomicCAS(status, 0, ESSA_ERR_CACHE); }

// Exclusive prefix of `x` over the block's threads (all of them call it) and the block's total.  blockDim.x is a multiple of 32.
__device__ __forceinline__ long long block_scan(long long x, long long* total, long long* smem /* [33] */) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  long long s = x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, s, d);
    if (lane >= d) s += y;
  }
  __syncthreads();  // (smem may still be read from the call before)
  if (lane == 31) smem[warp] = s;
  __syncthreads();
  if (warp == 0) {
    long long w = lane < warps ? smem[lane] : 0;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, w, d);
      if (lane >= d) w += y;
    }
    smem[lane] = w;
  }
  __syncthreads();
  *total = smem[warps - 1];
  return (warp ? smem[warp - 1] : 0) + s - x;
}
#endif

}  // namespace essa
