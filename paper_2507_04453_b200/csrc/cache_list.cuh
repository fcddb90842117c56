// How an attention call over the cache is divided: the list of (entry, kv head, row block, key tile) is cut into equal runs, one per
// thread block, wherever the cuts fall.  A row block inside one run is finished there; one that is cut leaves partial
// results (O, maximum, sum per row, fp32) in the workspace, two slots per run at most, and attend_join_kernel adds them in
// run order.  Ragged lengths, causal prompts and single long sequences balance alike, results do not depend on timing, and
// the workspace is bounded by the grid.
// Where that is cheaper (whole_blocks), cuts move to the row blocks' ends instead: nothing is left to join.
// A row block also costs its queries' way in and its results' way out, so it stands in the list as kSetup elements without work,
// followed by its key tiles; a cut between those leaves it whole to the run behind the cut.
//
// A list policy L gives R (query rows of a row block), tiles(info, args, rb) >= 1 (key tiles of a row block, so that rows that
// see nothing are still written), per_head(info, args) (the elements of all row blocks of an entry), kSetup and kMinRun.
#pragma once

#include <atomic>

#include "cache.cuh"
#include "tc_ptx.cuh"

namespace essa {

// Division by the number of heads of a group (rows are token * group + head) as a multiplication (T. Granlund and P. Montgomery, Division by
// invariant integers using multiplication, 1994): for n < 2^31,
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
  int64_t partials_at;  // floats before the partial results
  int32_t whole;        // a run has the row blocks that begin in it, to their ends
  int32_t* status;
};

// Bytes of the workspace for `grid` thread blocks, two partial results of `floats` each; the partial results begin after the run places.
constexpr int64_t kRunPlaceBytes = 40;
inline int64_t partials_at(int grid) { return (kRunPlaceBytes * grid + 255) / 256 * 64; }
inline int64_t attend_workspace(int grid, int64_t floats) { return (partials_at(grid) + (int64_t)grid * 2 * floats) * 4; }

// Whether a call is divided between row blocks only.  Cut anywhere, all thread blocks end together, but partial results are written, read and
// joined, which costs about as much as kJoin key tiles; cut between row blocks, the last round leaves some idle for a row block's length (for
// many rounds, of lengths that vary, half of them).  Lengths are known on the host as an upper bound only, hence kWholePages.
// Cut anywhere / between row blocks, us in a graph, heads of 128 channels: one token of 16 sequences, 4 kv heads: 2 pages 10 / 7, 8 pages 11 / 9,
// 16 pages 12.5 / 15; of 50, 8 heads: 13.9 / 8.4, 19.1 / 13.4, 25.2 / 19.9; of 256, 4 heads: 19.8 / 16.6, 32.2 / 29.9, 49.2 / 49.5, 32 pages 79 / 83;
// 64 tokens of 15 sequences, 8 kv heads of 5: 33 / 21, 55 / 34, 70 / 51, 96 / 83; prompts of 1 .. 1024 tokens of 64: 498 / 479.
// (A launch less on the host, too: 13 -> 10 us a call.)
constexpr int kWholePages = 32, kJoin = 16;
template <class L>
bool whole_blocks(const AttendArgs& a, int grid) {
  const int64_t by_rows = (int64_t)a.e.T * ((a.group + L::R - 1) / L::R), by_entries = (int64_t)a.e.T * a.group / L::R + a.e.n;
  const int64_t blocks = (by_rows < by_entries ? by_rows : by_entries) * a.v.kv_heads;  // at most
  const int64_t idle = blocks > 4 * (int64_t)grid ? grid / 2 : (blocks + grid - 1) / grid * grid - blocks;
  return a.v.max_pages <= kWholePages && idle * (a.v.max_pages + L::kSetup) <= (int64_t)kJoin * grid;
}

#ifdef __CUDACC__
// 2^x by the special function unit (results below the normal range are 0, which no weight notices).
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// What a difference of scores is multiplied with to be an exponent of 2, kept away from 0 and infinity: hidden scores are -infinity and equal ones
// 0 apart, either of which would make NaN of it.  Scores in units of 2^13 .. 2^14 of a row of q and fp16's smallest numbers of K differ by 2^-48
// or not at all: from 2^80 on, and well before, every difference is a weight of 0.
__device__ __forceinline__ float softmax_scale(float x) { return fminf(fmaxf(x, 0x1p-126f), 0x1p80f); }

// Two fp32 operations in one instruction.
__device__ __forceinline__ uint64_t pack_f32x2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpack_f32x2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add_f32x2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

__device__ __forceinline__ uint32_t half2_bits(__half2 v) { return *reinterpret_cast<uint32_t*>(&v); }
__device__ __forceinline__ __half2 as_half2(uint32_t v) { return *reinterpret_cast<__half2*>(&v); }
// Two codes as fp16 numbers (a published technique for 4-bit weights; the last place of an fp16 number from 1024 on is 1, so that a code
// dropped into its mantissa is added to it): (w & MASK) | magic, magic = 0x64006400, is 1024 + code for the nibbles 0 and 4 of w (MASK 0x000f000f) and
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

// Where a run begins, as its thread block has found it (the workspace's first part, one for each thread block).
struct RunPlace {
  long long total;
  int runs, entry, kvh, rb, at, tiles, row0, rows;
};
static_assert(sizeof(RunPlace) == kRunPlaceBytes, "");
__device__ __forceinline__ RunPlace* run_places(const AttendArgs& a) { return reinterpret_cast<RunPlace*>(a.ws); }

struct Cursor {  // a place in the list
  int entry, kvh, rb, at, blocks, tiles;  // at: element of the row block
  EntryInfo info;
};

// (rows * group < 2^31 is checked on the host)
__device__ __forceinline__ int row_blocks(const EntryInfo& e, int group, int R) { return (int)(((uint32_t)e.rows * (uint32_t)group + R - 1) / R); }

__device__ __forceinline__ long long run_start(long long total, int runs, int c) { return total * c / runs; }
// Runs that share the list: L::kMinRun elements each at least (a shorter one would pay its fixed cost and a join for little).
template <class L>
__device__ __forceinline__ int run_count(long long total, int grid) {
  return (int)max(1LL, min((long long)grid, (total + L::kMinRun - 1) / L::kMinRun));
}

struct RunShared {
  long long scan[33];
  long long rest;
  int entry;
};
// This thread block's run: its first element's place and its length (0: none); all threads of the block.  Every thread sums a stretch
// of the entries; the one whose stretch holds the place walks it again.
template <class L>
__device__ __forceinline__ void next_block(const AttendArgs& a, Cursor& c);
template <class L>
__device__ long long find_run(const AttendArgs& a, Cursor& c, RunShared& sm) {
  const int per = (a.e.n + blockDim.x - 1) / blockDim.x, lo = min((int)threadIdx.x * per, a.e.n), hi = min(lo + per, a.e.n);
  long long sum = 0, total;
  for (int i = lo; i < hi; ++i) sum += L::per_head(load_entry(a.v, a.e, i), a) * a.v.kv_heads;
  const long long pre = block_scan(sum, &total, sm.scan);
  if (total == 0) {
    if (blockIdx.x == 0 && threadIdx.x == 0) run_places(a)[0].runs = 0;
    return 0;
  }
  const int runs = run_count<L>(total, gridDim.x);
  if ((int)blockIdx.x >= runs) return 0;
  const long long begin = run_start(total, runs, blockIdx.x), end = run_start(total, runs, blockIdx.x + 1);
  if (begin >= pre && begin < pre + sum) {
    long long rest = begin - pre;
    for (int i = lo; i < hi; ++i) {
      const long long w = L::per_head(load_entry(a.v, a.e, i), a) * a.v.kv_heads;
      if (rest < w) {
        sm.entry = i;
        sm.rest = rest;
        break;
      }
      rest -= w;
    }
  }
  __syncthreads();
  c.entry = sm.entry;
  c.info = load_entry(a.v, a.e, c.entry);
  c.blocks = row_blocks(c.info, a.group, L::R);
  const long long per_head = L::per_head(c.info, a);
  c.kvh = (int)(sm.rest / per_head);
  long long rest = sm.rest % per_head;
  for (c.rb = 0; (c.tiles = L::tiles(c.info, a, c.rb)) + L::kSetup <= rest; ++c.rb) rest -= c.tiles + L::kSetup;
  c.at = (int)rest;
  if (a.whole) {  // (attend_join_kernel does not run)
    if (c.at == 0) return end - begin;
    const long long left = end - begin - (c.tiles + L::kSetup - c.at);
    if (left > 0) next_block<L>(a, c);
    return max(left, 0LL);
  }
  if (threadIdx.x == 0) {  // for attend_join_kernel
    RunPlace p;
    p.total = total;
    p.runs = runs;
    p.entry = c.entry;
    p.kvh = c.kvh;
    p.rb = c.rb;
    p.at = c.at;
    p.tiles = c.tiles;
    p.row0 = c.info.row0;
    p.rows = c.info.rows;
    run_places(a)[blockIdx.x] = p;
  }
  return end - begin;
}

// Takes what is left of c's row block from a run that has `left` elements to go: key tiles first .. stop - 1 (none, if the run ends
// before the first) are the run's.
template <class L>
__device__ __forceinline__ void take_block(const AttendArgs& a, const Cursor& c, long long& left, int& first, int& stop) {
  const int all = c.tiles + L::kSetup - c.at, n = a.whole ? all : (int)min((long long)all, left);
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

template <class L, int D>
struct Partial {
  static constexpr int kFloats = L::R * (D + 2);  // O [R][D], maximum [R], sum [R]
};
// Slot of the partial result that run `run` leaves for a row block: 1 if the row block begins in this run, else 0.
template <class L, int D>
__device__ __forceinline__ float* partial_of(const AttendArgs& a, int run, bool begins) {
  return a.ws + a.partials_at + ((int64_t)run * 2 + (begins ? 1 : 0)) * Partial<L, D>::kFloats;
}

// Joins the row blocks that run boundaries cut.  Thread blocks (c, *) look at the boundary between runs c and c + 1 and work if it
// is the first one between key tiles of its row block; gridDim.y of them share its rows.  A warp takes a row and adds its parts
// in run order.
template <class L, int D>
__global__ void __launch_bounds__(128) attend_join_kernel(AttendArgs a) {
  constexpr int R = L::R, V = D / 32;  // V floats of a row per lane
  grid_dep_wait();
  const int run = blockIdx.x;
  const int runs = run_places(a)[0].runs;  // (0: no entry has a row)
  if (run + 1 >= runs) return;
  const RunPlace p = run_places(a)[run + 1];
  const long long edge = run_start(p.total, runs, run + 1), first = edge - p.at, begin = run_start(p.total, runs, run);
  if (p.at <= L::kSetup || first + L::kSetup < begin) return;
  const long long stop = first + L::kSetup + p.tiles;
  // the runs run .. last have a part of the row block: floor(total k / runs) < stop for k < stop * runs / total
  const int last = (int)min((long long)runs - 1, (stop * runs + p.total - 1) / p.total - 1);
  const int rows = p.rows * a.group, r0 = p.rb * R, lane = threadIdx.x & 31;
  for (int row = blockIdx.y * 4 + (threadIdx.x >> 5); row < R; row += gridDim.y * 4) {
    const int r = r0 + row;
    if (r >= rows) break;
    float m = -INFINITY, sum = 0.f, v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = 0.f;
    for (int k0 = run; k0 <= last; k0 += 32) {  // a lane has the maximum and the sum of a run's part
      const int n = min(last + 1 - k0, 32);
      float pm = -INFINITY, ps = 0.f;
      if (lane < n) {
        const float* q = partial_of<L, D>(a, k0 + lane, k0 + lane == run) + R * D + row;
        pm = q[0];
        ps = q[R];
      }
      float top = fmaxf(m, pm);
#pragma unroll
      for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      const float f0 = m == -INFINITY ? 0.f : ex2((m - top) * a.scale), f = pm == -INFINITY ? 0.f : ex2((pm - top) * a.scale);
      float add = f * ps;  // (NaN where a part has seen nothing but NaN)
#pragma unroll
      for (int d = 16; d; d >>= 1) add += __shfl_xor_sync(0xffffffffu, add, d);
      sum = fmaf(f0, sum, add);
      m = top;
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] *= f0;
      for (int k = 0; k < n; k += 8) {  // eight parts' loads are on their way together: L2's latency, not its rate, is what a row would wait for
        float x[8][V];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int at = k0 + min(k + u, n - 1);
          const float* q = partial_of<L, D>(a, at, at == run) + row * D + lane * V;
#pragma unroll
          for (int i = 0; i < V; i += 2) {
            const float2 y = *reinterpret_cast<const float2*>(q + i);
            x[u][i] = y.x;
            x[u][i + 1] = y.y;
          }
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const float w = __shfl_sync(0xffffffffu, f, min(k + u, n - 1));
#pragma unroll
          for (int i = 0; i < V; ++i) v[i] = fmaf(k + u < n ? w : 0.f, x[u][i], v[i]);
        }
      }
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const int j = a.by_group(r), hd = r - j * a.group;
    uint32_t* out = reinterpret_cast<uint32_t*>(a.out + (int64_t)(p.row0 + j) * a.ld_out + (int64_t)(p.kvh * a.group + hd) * D + lane * V);
#pragma unroll
    for (int i = 0; i < V; i += 2) out[i / 2] = pack_bf16x2(v[i] * inv, v[i + 1] * inv);
  }
}

// A kernel's dynamic shared memory allowance, raised on its first launch on a device (the call costs about a microsecond).
template <auto kKernel>
cudaError_t allow_shared(int bytes, int device) {
  static std::atomic<uint64_t> done{0};  // a bit per device
  const uint64_t bit = device < 64 ? 1ull << device : 0;
  if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

template <class L, int D>
int32_t launch_join(essa_ctx* ctx, const AttendArgs& a, int grid, int row_split, cudaStream_t stream) {
  if (grid < 2 || a.whole) return ESSA_OK;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid - 1, row_split);
  cfg.blockDim = dim3(128);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, attend_join_kernel<L, D>, a);
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
