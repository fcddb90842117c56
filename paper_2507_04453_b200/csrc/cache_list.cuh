// How an attention call over the cache is divided: the list of (entry, kv head, row block, key tile) is cut into equal runs, one per
// thread block, wherever the cuts fall.  A row block inside one run is finished there; one that is cut leaves partial
// results (O, maximum, sum per row, fp32) in the workspace, two slots per run at most, and attend_join_kernel adds them in
// run order.  Ragged lengths, causal prompts and single long sequences balance alike, results do not depend on timing, and
// the workspace is bounded by the grid.
// A row block also costs its queries' way in and its results' way out, so it stands in the list as kSetup elements without work,
// followed by its key tiles; a cut between those leaves it whole to the run behind the cut.
//
// A list policy L gives R (query rows of a row block), tiles(info, args, rb) >= 1 (key tiles of a row block, so that rows that
// see nothing are still written), per_head(info, args) (the elements of all row blocks of an entry), kSetup and kMinRun.
#pragma once

#include "cache.cuh"
#include "tc_ptx.cuh"

namespace essa {

// Division by the number of heads of a group (rows are token * group + head) as a multiplication: for n < 2^31,
// n / d = (umulhi(mul, n) + n) >> shift with shift = ceil(log2 d), mul = floor(2^32 (2^shift - d) / d) + 1.
struct Divisor {
  uint32_t d, mul, shift;
  static Divisor of(uint32_t d) {
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;
    return {d, (uint32_t)(((1ull << 32) * ((1ull << s) - d)) / d + 1), s};
  }
#ifdef __CUDACC__
  __device__ __forceinline__ int operator()(int n) const { return (int)((__umulhi(mul, (uint32_t)n) + (uint32_t)n) >> shift); }
#endif
};

struct AttendArgs {
  CacheView v;
  CacheEntries e;
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  int64_t ld_q, ld_out;
  int32_t group;
  Divisor by_group;
  float scale;  // softmax scale * log2(e)
  float* ws;
  int32_t* status;
};

#ifdef __CUDACC__
// 2^x by the special function unit (results below the normal range are 0, which no weight notices).
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ uint32_t half2_bits(__half2 v) { return *reinterpret_cast<uint32_t*>(&v); }
__device__ __forceinline__ __half2 as_half2(uint32_t v) { return *reinterpret_cast<__half2*>(&v); }
// Two codes as fp16 numbers: (w & MASK) | magic, magic = 0x64006400, is 1024 + code for the nibbles 0 and 4 of w (MASK 0x000f000f) and
// 1024 + 16 code for the nibbles 1 and 5 (MASK 0x00f000f0).  One instruction; left to the compiler it becomes two.
template <uint32_t MASK>
__device__ __forceinline__ __half2 nibble_half2(uint32_t w, uint32_t magic) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "n"(MASK), "r"(magic));
  return as_half2(r);
}
// code - 8 of the nibbles 0 and 4, and of the nibbles 1 and 5: exact.
__device__ __forceinline__ __half2 centred_low(uint32_t w, uint32_t magic) { return __hsub2(nibble_half2<0x000f000fu>(w, magic), as_half2(0x64086408u) /* 1032 */); }
__device__ __forceinline__ __half2 centred_high(uint32_t w, uint32_t magic) {
  return __hfma2(nibble_half2<0x00f000f0u>(w, magic), as_half2(0x2c002c00u) /* 1 / 16 */, as_half2(0xd480d480u) /* -72 */);
}

struct Cursor {  // a place in the list
  int entry, kvh, rb, at, blocks, tiles;  // at: element of the row block
  EntryInfo info;
};

// (rows * group < 2^31 is checked on the host)
__device__ __forceinline__ int row_blocks(const EntryInfo& e, int group, int R) { return (int)(((uint32_t)e.rows * (uint32_t)group + R - 1) / R); }

// Elements of the list; all threads of the block.  sm: shared [33].
template <class L>
__device__ long long list_total(const AttendArgs& a, long long* sm) {
  long long total = 0;
  for (int base = 0; base < a.e.n; base += blockDim.x) {
    const int i = base + threadIdx.x;
    long long w = 0, t;
    if (i < a.e.n) w = L::per_head(load_entry(a.v, a.e, i), a) * a.v.kv_heads;
    block_scan(w, &t, sm);
    total += t;
  }
  return total;
}

// The place of element `at` < total; all threads of the block.  found: shared [2].
template <class L>
__device__ void list_seek(const AttendArgs& a, long long at, Cursor& c, long long* sm, long long* found) {
  long long before = 0;
  for (int base = 0; base < a.e.n; base += blockDim.x) {
    const int i = base + threadIdx.x;
    long long w = 0, t;
    if (i < a.e.n) w = L::per_head(load_entry(a.v, a.e, i), a) * a.v.kv_heads;
    const long long pre = before + block_scan(w, &t, sm);
    if (w > 0 && at >= pre && at < pre + w) {
      found[0] = i;
      found[1] = at - pre;
    }
    before += t;
    __syncthreads();
    if (at < before) break;
  }
  c.entry = (int)found[0];
  c.info = load_entry(a.v, a.e, c.entry);
  c.blocks = row_blocks(c.info, a.group, L::R);
  const long long per = L::per_head(c.info, a);
  c.kvh = (int)(found[1] / per);
  long long rest = found[1] % per;
  for (c.rb = 0; (c.tiles = L::tiles(c.info, a, c.rb)) + L::kSetup <= rest; ++c.rb) rest -= c.tiles + L::kSetup;
  c.at = (int)rest;
}

// Takes what is left of c's row block from a run that has `left` elements to go: key tiles first .. stop - 1 (none, if the run ends
// before the first) are the run's.
template <class L>
__device__ __forceinline__ void take_block(const Cursor& c, long long& left, int& first, int& stop) {
  const int n = (int)min((long long)(c.tiles + L::kSetup - c.at), left);
  first = max(c.at - L::kSetup, 0);
  stop = max(c.at + n - L::kSetup, 0);
  left -= n;
}
// The row block after c's; must not be called at the end of the list.
template <class L>
__device__ __forceinline__ void next_block(const AttendArgs& a, Cursor& c) {
  c.at = 0;
  if (++c.rb >= c.blocks) {
    c.rb = 0;
    if (++c.kvh >= a.v.kv_heads) {
      c.kvh = 0;
      do {
        if (++c.entry >= a.e.n) return;
        c.info = load_entry(a.v, a.e, c.entry);
        c.blocks = row_blocks(c.info, a.group, L::R);
      } while (c.blocks == 0);
    }
  }
  c.tiles = L::tiles(c.info, a, c.rb);
}

__device__ __forceinline__ long long run_start(long long total, int runs, int c) { return total * c / runs; }
// Runs that share the list: L::kMinRun elements each at least (a shorter one would pay its fixed cost and a join for little).
template <class L>
__device__ __forceinline__ int run_count(long long total, int grid) {
  return (int)max(1LL, min((long long)grid, (total + L::kMinRun - 1) / L::kMinRun));
}

template <class L, int D>
struct Partial {
  static constexpr int kFloats = L::R * (D + 2);  // O [R][D], maximum [R], sum [R]
};
// Slot of the partial result that run `run` leaves for a row block: 1 if the row block begins in this run, else 0.
template <class L, int D>
__device__ __forceinline__ float* partial_of(const AttendArgs& a, int run, bool begins) {
  return a.ws + ((int64_t)run * 2 + (begins ? 1 : 0)) * Partial<L, D>::kFloats;
}

// Joins the row blocks that run boundaries cut.  Thread blocks (c, *) look at the boundary between runs c and c + 1 and work if it
// is the first one between key tiles of its row block; gridDim.y of them share its rows.  Launched to start beside the attention kernel: it finds
// its row block meanwhile and waits for the partial results.
template <class L, int D>
__global__ void __launch_bounds__(128) attend_join_kernel(AttendArgs a, int grid) {
  constexpr int R = L::R;
  __shared__ long long scan_sm[33];
  __shared__ long long found[2];
  const long long total = list_total<L>(a, scan_sm);
  const int runs = total ? run_count<L>(total, grid) : 0;
  Cursor c;
  long long first = 0;
  const int run = blockIdx.x;
  bool work = run + 1 < runs;
  if (work) {
    const long long edge = run_start(total, runs, run + 1);
    list_seek<L>(a, edge, c, scan_sm, found);
    first = edge - c.at;  // the row block's first element
    work = c.at > L::kSetup && first + L::kSetup >= run_start(total, runs, run);
  }
  grid_dep_wait();
  if (!work) return;
  const long long stop = first + L::kSetup + c.tiles;
  const int rows = c.info.rows * a.group, r0 = c.rb * R;
  int last = run;  // the runs run .. last have a part of the row block
  while (last + 1 < runs && run_start(total, runs, last + 1) < stop) ++last;
  for (int x = blockIdx.y * 128 + threadIdx.x; x < R * (D / 4); x += gridDim.y * 128) {
    const int row = x / (D / 4), d4 = (x % (D / 4)) * 4, r = r0 + row;
    if (r >= rows) break;
    float m = -INFINITY, sum = 0.f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k = run; k <= last; ++k) {
      const float* p = partial_of<L, D>(a, k, k == run);
      const float pm = p[R * D + row], mn = fmaxf(m, pm);
      const float f0 = m == -INFINITY ? 0.f : ex2((m - mn) * a.scale), f1 = pm == -INFINITY ? 0.f : ex2((pm - mn) * a.scale);
      const float4 y = *reinterpret_cast<const float4*>(p + row * D + d4);
      sum = fmaf(f0, sum, f1 * p[R * D + R + row]);
      v.x = fmaf(f0, v.x, f1 * y.x);
      v.y = fmaf(f0, v.y, f1 * y.y);
      v.z = fmaf(f0, v.z, f1 * y.z);
      v.w = fmaf(f0, v.w, f1 * y.w);
      m = mn;
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const int j = a.by_group(r), hd = r - j * a.group;
    uint2 y;
    y.x = pack_bf16x2(v.x * inv, v.y * inv);
    y.y = pack_bf16x2(v.z * inv, v.w * inv);
    *reinterpret_cast<uint2*>(a.out + (int64_t)(c.info.row0 + j) * a.ld_out + (int64_t)(c.kvh * a.group + hd) * D + d4) = y;
  }
}

template <class L, int D>
int32_t launch_join(essa_ctx* ctx, const AttendArgs& a, int grid, int row_split, cudaStream_t stream) {
  if (grid < 2) return ESSA_OK;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid - 1, row_split);
  cfg.blockDim = dim3(128);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, attend_join_kernel<L, D>, a, grid);
  if (e != cudaSuccess) return check_cuda(ctx, e, "attend join launch");
  ++ctx->launches;
  return ESSA_OK;
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ float2 lds_half2(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return __half22float2(*reinterpret_cast<__half2*>(&v));
}
// The copies into `slots` ring slots that were filled `filled` times in all land (a bounded wait each); for leaving early.
__device__ __forceinline__ void drain_ring(uint32_t full, int slots, int filled) {
  for (int s = 0; s < slots && s < filled; ++s) {
    const uint32_t last = ((filled - 1 - s) / slots) & 1;
    const long long t0 = clock64();
    while (!mbar_try_wait(full + 8 * s, last) && clock64() - t0 < kWaitLimitCycles / 16) {}
  }
}
#endif

}  // namespace essa
