// Attention over the paged 4-bit cache for few rows per sequence (decode steps): softmax(scale q K^T) V with
// K = code * scale + minimum per token and group of 64 channels.
//
// What bounds it: the cache is read once and each byte carries two values, so a B200 streams ~46 codes per clock and SM
// from HBM; what the kernel has to keep up with is widening them.  The mathematics is arranged so that a code needs little more than an
// and-or.  A nibble dropped into the mantissa of the fp16 number 1024 is 1024 + c, or 1024 + 16 c one nibble further up, so
// that a word of eight codes needs one shift.
//   S = sum_g s_g (q_g . c_g) + min_g sum(q_g).  The tensor core multiplies q, or q / 16, by those numbers as they are and starts from
//   minus what the 1024 will add (a sum over q), so that the offset has gone when it has finished.  (On the way the sum is up to 1024 sum |q|,
//   whose last place in fp32 takes up to ten bits of the score's: some 10^-4 of a score's unit for 128 channels of N(0, 1).)
//   O = sum_k p_k (s_k (c_k - 8) + (min_k + 8 s_k)): one operation more takes a number to c - 8; the weight times the scale is rounded to
//   fp16 (2^-11 of a centred value; with the codes not centred it would be 2^-11 of a number 2.6 times as large), the second term stays
//   on the CUDA cores in fp32.  (Leaving the 1024 in and subtracting it from the sum at the end loses the result in fp32.)
// fp16 holds what it has to: a query row is brought to a largest element of 2^13 .. 2^14 by a power of two, and scales are taken
// relative to a power of two near the largest that the warp has met (products 2^-14 below it lose bits).
// 910 MB of cache (128 sequences of 4 to 8 thousand tokens, 8 kv heads, 8 query heads each): 200 to 219 us (by clocks), 4.2 to 4.6 TB/s; ALU 47 % and
// issue slots 60 % busy, HBM 55 %, tensor 24 %: none is full; 3.4 warps per scheduler leave fixed latencies uncovered, and their 128 registers spill 64 bytes.  The first
// version, with bf16 operands (three shifts and twice the roundings per word of codes): 289 us.  Tried and no faster:
// four consuming warps that copy for themselves in four thread blocks per SM, one slice of 16 tokens per warp.
// K and V are the M = 16 operand of mma.m16n8k16, the query rows (heads of the group x tokens) are the N = 8 columns: a
// group of up to eight heads fills the tensor core's tile, where q as the M operand would leave half of it empty.
//
// Work split: cache_list.cuh, with row blocks of 8 or 16 query rows and key tiles of one page.
// With a mask the list has the pages that a row block can see, and a page at an edge (of a window, of the first tokens, among drafts) is masked by 32 bits per row.
// A window of 1024 and 4 first tokens of those long sequences (156 MB): 59 us, 2.6 TB/s: seventeen pages of a row block beside five pages' worth of fixed cost, and
// a join of 5 us.  Queries and row blocks found ahead by the copying warp: 58 (and 36 -> 34 for 256 short ones), left out for its second path of synchronisation.
// Tokens per column instead of limits, and a mask per different token: 35.9 -> 35.3 for the short ones.  The masked instance spills 208 bytes a thread (64 without a
// mask; heads of 64 with two column tiles 192, and none).
#include "cache_list.cuh"

namespace essa {
namespace {

constexpr int kWarps = 4;                     // consuming warps: two share a page (32 tokens each), pages go to the pairs in turn
constexpr int KS = 2;                         // slices of 16 tokens per warp: independent chains of products that hide one another's latency
constexpr int kThreads = kWarps * 32 + 32;    // + one copying warp

// Row blocks of R rows; every row block of an entry walks all its pages (the few rows of an entry see nearly the same ones).
// kSetup: 256 sequences of up to 1024 tokens take 43.3 us with 2, 40.2 with 3, 38.8 with 5, 38.6 with 7, 39.6 with 10 (cut anywhere).
template <int ROWS, bool MASKED>
struct DecodeList {
  static constexpr int R = ROWS, kMinRun = 2, kSetup = 5;
  static int64_t most_tiles(const AttendArgs& a) { return MASKED ? most_masked_tiles(a, (R - 1) / a.group + 2) : a.v.max_pages; }
  __device__ static Span span(const EntryInfo& e, const AttendArgs& a, int rb) {
    if (!MASKED) return {0, 0, max((e.len + kPageTokens - 1) / kPageTokens, 1)};
    return span_of(e, a.m, first_token(a, rb, R), last_token(e, a, rb, R));
  }
  __device__ static int tiles(const EntryInfo& e, const AttendArgs& a, int rb) { return span(e, a, rb).tiles; }
  __device__ static long long per_head(const EntryInfo& e, const AttendArgs& a) {
    const int blocks = row_blocks(e, a.group, R);
    if (!MASKED) return (long long)blocks * (tiles(e, a, 0) + kSetup);
    long long sum = 0;
    for (int rb = 0; rb < blocks; ++rb) sum += tiles(e, a, rb) + kSetup;
    return sum;
  }
};

__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ void mma_f16(float (&d)[4], __half2 a0, __half2 a1, __half2 a2, __half2 a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(half2_bits(a0)), "r"(half2_bits(a1)), "r"(half2_bits(a2)), "r"(half2_bits(a3)), "r"(b0), "r"(b1));
}

// mbar_wait for the warp that fills a deep ring: it sleeps between probes and leaves the issue slots to the warps that compute.
__device__ __forceinline__ bool wait_napping(uint32_t bar, uint32_t parity, volatile int* abort_flag, int32_t* status) {
  const long long t0 = clock64();
  while (!mbar_test_wait(bar, parity)) {
    __nanosleep(64);
    if (*abort_flag) return false;
    if (clock64() - t0 > kWaitLimitCycles) {
      *abort_flag = 1;
      atomicCAS(status, 0, ESSA_ERR_DEVICE_TIMEOUT);
      return false;
    }
  }
  return true;
}
// mma_f16 with the accumulator's start in registers of its own (they stay).
__device__ __forceinline__ void mma_f16_from(float (&d)[4], const float (&c)[4], __half2 a0, __half2 a1, __half2 a2, __half2 a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(half2_bits(a0)), "r"(half2_bits(a1)), "r"(half2_bits(a2)), "r"(half2_bits(a3)), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}

template <int D, int NT>
struct Shape {
  static constexpr int R = 8 * NT;             // query rows of a row block
  static constexpr int kBytes = 72 * D;        // a (page, kv head) run
  static constexpr int kStages = (D == 128 ? 6 : 10);
  static constexpr int kCol = D + 4;           // floats of a column's O in the join (padded: the lanes of a store have columns of their own)
  static constexpr int kWarpJoin = R * (kCol + 2);
  static constexpr int kJoin = kWarps * kWarpJoin * 4;
  static_assert(kStages % 2 == 0, "");
  static constexpr int kSmem = kStages * kBytes + kJoin + 256;
};

// Thread blocks per SM: what shared memory and registers allow.
constexpr int attend_blocks_per_sm(int head_dim, int nt) { return nt == 1 ? 3 : 2; }

template <int D, int NT, bool MASKED>
__global__ void __launch_bounds__(kThreads, attend_blocks_per_sm(D, NT)) attend_decode_kernel(AttendArgs a) {
  using S = Shape<D, NT>;
  constexpr int R = S::R, G = D / kCacheGroup, CH = D / 32;
  using L = DecodeList<R, MASKED>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ RunShared run_sm;
  __shared__ volatile int abort_flag;
  __shared__ int bad_page[S::kStages];
  __shared__ __align__(8) uint64_t bars[2 * S::kStages];
  float* join = reinterpret_cast<float*>(smem + S::kStages * S::kBytes);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t ring = smem_u32(smem), full = smem_u32(bars), empty = full + 8 * S::kStages;
  if (!a.whole) grid_dep_launch();  // (else the launch that follows is not the join)
  if (tid == 0) {
    abort_flag = 0;
    for (int s = 0; s < S::kStages; ++s) { mbar_init(full + 8 * s, 1); mbar_init(empty + 8 * s, 2); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  Cursor c;
  long long left = find_run<L>(a, c, run_sm);
  if (left == 0) return;

  if (warp == kWarps) {  // ---------------------------------------------------------------- copying warp
    if (lane != 0) return;
    int st = 0, filled = 0;
    uint32_t phase = 0;
    bool ok = true;
    while (ok && left > 0) {
      int tile, stop;
      take_block<L>(a, c, left, tile, stop);
      const int32_t* row = a.v.table + (int64_t)max(c.info.slot, 0) * a.v.max_pages;
      const bool none = c.info.len == 0;
      const Span span = L::span(c.info, a, c.rb);
      for (; tile < stop; ++tile) {
        if (filled >= S::kStages && !wait_napping(empty + 8 * st, phase ^ 1, &abort_flag, a.status)) { ok = false; break; }
        const int at = MASKED ? span.page(tile) : tile, page = none ? -1 : __ldg(row + at);
        const bool there = page >= 0 && page < a.v.num_pages;
        if (!there && (!none || c.info.slot < 0) && (!MASKED || page_seen(a.m, c.info, first_token(a, c.rb, R), last_token(c.info, a, c.rb, R), at))) cache_fault(a.status);
        bad_page[st] = !there;
        if (there) {
          mbar_expect_tx(full + 8 * st, S::kBytes);
          bulk_load(ring + st * S::kBytes, a.v.pages + page * a.v.page_bytes + (int64_t)c.kvh * S::kBytes, S::kBytes, full + 8 * st);
        } else {
          mbar_arrive(full + 8 * st);
        }
        ++filled;
        if (++st == S::kStages) { st = 0; phase ^= 1; }
      }
      if (left > 0) next_block<L>(a, c);
    }
    if (!ok) drain_ring(full, S::kStages, filled);  // before the block's shared memory goes away
    return;
  }

  // ----------------------------------------------------------------------------------------- consuming warps
  const int g = lane >> 2, t = lane & 3;
  const int key0 = (warp & 1) * 32;                                           // this warp's tokens of a page
  const uint32_t k_lane = (uint32_t)(key0 + (lane & 15)) * 16 + (uint32_t)(lane >> 4) * 1024;  // ldmatrix row addresses: (tokens 0-7, 8-15) x two chunks
  int st = warp >> 1;  // (an even number of stages: a pair's pages stay in its stages)
  uint32_t phase = 0;
  int mine_at = warp >> 1;  // the pair's first tile of a row block, counted from the run's first tile of it
  uint32_t magic = 0x64006400u;
  asm volatile("" : "+r"(magic));  // (in a register, where the and-or can take it)
  bool dead = false;  // a wait ran out: the warp goes through the barriers with the others and does nothing else
  for (; left > 0; next_block<L>(a, c)) {
    int first, stop;
    take_block<L>(a, c, left, first, stop);
    if (first == stop) break;  // (the run ends before the row block's first tile)
    const int rows = c.info.rows * a.group;  // (fits: T * group is checked on the host)
    const int r0 = c.rb * R;
    // --- query operand: lane (g, t) holds channels 32 h + 8 t .. + 7 of column g, in the order that the nibbles come in:
    // (0, 4), (1, 5) / 16, (2, 6), (3, 7) / 16
    uint32_t qf[NT][CH][4];
    float qsum[NT][G][2], start[NT][G][4];  // per group: the sum of q; minus what the 1024 in the codes' numbers adds
    float sc[NT][2], back[NT][2];           // softmax scale in the units of the row; what the row was divided by
    int limit[NT][2], lowest = 0x7fffffff;  // (with a mask: the token of the entry that the column is; without a row, the last one)
    Span span;
    int reach = 0;
    if (MASKED) {
      span = L::span(c.info, a, c.rb);
      lowest = seen_by_all(a.m, c.info, first_token(a, c.rb, R));
      reach = hidden_to_some(a.m, c.info, last_token(c.info, a, c.rb, R));
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = r0 + nt * 8 + g;
      const int j = a.by_group(r), hd = r - j * a.group;
      const bool there = r < rows;
      const uint4* src = reinterpret_cast<const uint4*>(a.q + (int64_t)(c.info.row0 + (there ? j : 0)) * a.ld_q + (int64_t)(c.kvh * a.group + hd) * D) + t;
      uint4 u[CH];
      float big = 0.f;
#pragma unroll
      for (int h = 0; h < CH; ++h) u[h] = there ? __ldg(src + h * 4) : make_uint4(0, 0, 0, 0);
      const auto at = [&](int h, int x) {
        const uint32_t w = x < 2 ? u[h].x : x < 4 ? u[h].y : x < 6 ? u[h].z : u[h].w;
        return __uint_as_float(x & 1 ? w & 0xffff0000u : w << 16);
      };
#pragma unroll
      for (int h = 0; h < CH; ++h)
#pragma unroll
        for (int x = 0; x < 8; ++x) big = fmaxf(big, fabsf(at(h, x)));
      big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
      big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
      // a power of two (1 for a row of zeros, or one with an infinity)
      const int e = big > 0.f && big < INFINITY ? max((int)(__float_as_uint(big) >> 23), 27) - 127 - 13 : 0;
      const float up = __uint_as_float((uint32_t)(127 - e) << 23), down = __uint_as_float((uint32_t)(127 + e) << 23);
      float even[G], odd[G];
#pragma unroll
      for (int i = 0; i < G; ++i) even[i] = odd[i] = 0.f;
#pragma unroll
      for (int h = 0; h < CH; ++h)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float f = x & 1 ? up * 0.0625f : up;
          const __half2 v = __floats2half2_rn(at(h, x) * f, at(h, x + 4) * f);
          qf[nt][h][x] = half2_bits(v);
          (x & 1 ? odd : even)[h / 2] += __low2float(v) + __high2float(v);
        }
#pragma unroll
      for (int i = 0; i < G; ++i) {
        even[i] += __shfl_xor_sync(0xffffffffu, even[i], 1);
        even[i] += __shfl_xor_sync(0xffffffffu, even[i], 2);
        odd[i] += __shfl_xor_sync(0xffffffffu, odd[i], 1);
        odd[i] += __shfl_xor_sync(0xffffffffu, odd[i], 2);
        const float all = fmaf(16.f, odd[i], even[i]), off = -1024.f * (even[i] + odd[i]);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          qsum[nt][i][x] = __shfl_sync(0xffffffffu, all, 8 * t + 4 * x);
          start[nt][i][x] = start[nt][i][2 + x] = __shfl_sync(0xffffffffu, off, 8 * t + 4 * x);
        }
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        back[nt][x] = __shfl_sync(0xffffffffu, down, 8 * t + 4 * x);
        sc[nt][x] = softmax_scale(a.scale * back[nt][x]);
        const int rc = r0 + nt * 8 + 2 * t + x;  // tokens that column 2 t + x sees; a column without a row sees all and is not written
        if (MASKED) {
          limit[nt][x] = a.by_group(min(rc, rows - 1));
        } else {
          limit[nt][x] = rc < rows ? c.info.len - c.info.rows + a.by_group(rc) + 1 : 0x7fffffff;
          lowest = min(lowest, limit[nt][x]);
        }
      }
    }
    if (!MASKED) {
      lowest = min(lowest, __shfl_xor_sync(0xffffffffu, lowest, 1));
      lowest = min(lowest, __shfl_xor_sync(0xffffffffu, lowest, 2));
    }
    float o[NT][CH][2][4];
    // running maximum, the score that moves it, what weights are relative to (the maximum, or 0 before there is one); sum of weights; second
    // term of O
    float mx[NT][2], high[NT][2], ref[NT][2], l[NT][2], om[NT][G][2];
    float per_unit[G];  // scales are relative to a power of two, the unit of o: this is its inverse; before the first scale any makes a new one
#pragma unroll
    for (int i = 0; i < G; ++i) per_unit[i] = 0x1p40f;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int h = 0; h < CH; ++h)
#pragma unroll
        for (int x = 0; x < 8; ++x) o[nt][h][x >> 2][x & 3] = 0.f;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        mx[nt][x] = high[nt][x] = -INFINITY;
        ref[nt][x] = l[nt][x] = 0.f;
#pragma unroll
        for (int i = 0; i < G; ++i) om[nt][i][x] = 0.f;
      }
    }
    for (int tile = first + mine_at; tile < stop; tile += 2) {
      if (!dead) dead = !__all_sync(0xffffffffu, mbar_wait(full + 8 * st, phase, &abort_flag, a.status));
      if (dead) continue;
      const uint32_t blk = ring + st * S::kBytes;
      const __half2* meta = reinterpret_cast<const __half2*>(smem + st * S::kBytes + 64 * D) + key0 + g;  // (scale, minimum) of K, then of V
      const int pos0 = (MASKED ? span.page(tile) : tile) * kPageTokens + key0, pos = pos0 + g;  // tokens of this lane's scores: pos + 8 n, n < 2 KS
      if (!bad_page[st] && pos0 < c.info.len) {
        // --- scores; of slice k: token pos + 16 k in [0..1], + 8 in [2..3]
        float s[KS][NT][4];
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int x = 0; x < 4; ++x) s[k][nt][x] = 0.f;
#pragma unroll
        for (int i = 0; i < G; ++i) {
          float acc[KS][NT][4];
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            uint32_t w[4];  // chunk 2i: tokens g, g + 8; chunk 2i + 1: tokens g, g + 8
            ldmatrix_x4(blk + k_lane + i * 2048 + k * 256, w);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t u0 = w[2 * h], u1 = w[2 * h + 1], v0 = u0 >> 8, v1 = u1 >> 8;
              const __half2 a00 = nibble_half2<0x000f000fu>(u0, magic), a01 = nibble_half2<0x000f000fu>(u1, magic), a02 = nibble_half2<0x00f000f0u>(u0, magic),
                            a03 = nibble_half2<0x00f000f0u>(u1, magic);
              const __half2 a10 = nibble_half2<0x000f000fu>(v0, magic), a11 = nibble_half2<0x000f000fu>(v1, magic), a12 = nibble_half2<0x00f000f0u>(v0, magic),
                            a13 = nibble_half2<0x00f000f0u>(v1, magic);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                if (h == 0) mma_f16_from(acc[k][nt], start[nt][i], a00, a01, a02, a03, qf[nt][2 * i][0], qf[nt][2 * i][1]);
                else mma_f16(acc[k][nt], a00, a01, a02, a03, qf[nt][2 * i + 1][0], qf[nt][2 * i + 1][1]);
                mma_f16(acc[k][nt], a10, a11, a12, a13, qf[nt][2 * i + h][2], qf[nt][2 * i + h][3]);
              }
            }
          }
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            const float2 m0 = __half22float2(meta[i * kPageTokens + 16 * k]), m1 = __half22float2(meta[i * kPageTokens + 16 * k + 8]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                s[k][nt][x] = fmaf(m0.x, acc[k][nt][x], fmaf(m0.y, qsum[nt][i][x], s[k][nt][x]));
                s[k][nt][2 + x] = fmaf(m1.x, acc[k][nt][2 + x], fmaf(m1.y, qsum[nt][i][x], s[k][nt][2 + x]));
              }
          }
        }
        // --- the values' scales and minima: (scale, minimum + 8 scale)
        float2 mv[KS][2][G];
        bool grow = false;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int i = 0; i < G; ++i) mv[k][y][i] = __half22float2(meta[(G + i) * kPageTokens + 16 * k + 8 * y]);
        if (MASKED && (pos0 + 16 * KS > lowest || pos0 + 16 * KS > c.info.len || (pos0 < reach && pos0 + 16 * KS > a.m.sinks))) {
          uint32_t see = 0;
          int of = 0;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              if (nt + x == 0 || limit[nt][x] != of) see = visible(a.m, c.info, limit[nt][x], pos0);  // (a decode step's columns are one token)
              of = limit[nt][x];
#pragma unroll
              for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int y = 0; y < 2; ++y)
                  if (!(see >> (g + 16 * k + 8 * y) & 1)) s[k][nt][2 * y + x] = -INFINITY;
            }
#pragma unroll
          for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
              for (int i = 0; i < G; ++i)
                if (pos + 16 * k + 8 * y >= c.info.len) mv[k][y][i] = make_float2(0.f, 0.f);
        }
        if (!MASKED && (pos0 + 16 * KS > lowest || pos0 + 16 * KS > c.info.len)) {
          // hidden tokens (whatever their scores are, NaN too); behind the sequence's end the page holds anything
#pragma unroll
          for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const int at = pos + 16 * k + 8 * y;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int x = 0; x < 2; ++x)
                  if (at >= min(limit[nt][x], c.info.len)) s[k][nt][2 * y + x] = -INFINITY;
#pragma unroll
              for (int i = 0; i < G; ++i)
                if (at >= c.info.len) mv[k][y][i] = make_float2(0.f, 0.f);
            }
        }
#pragma unroll
        for (int i = 0; i < G; ++i) {
          float top = 0.f;
#pragma unroll
          for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              float2& m = mv[k][y][i];
              m.y = fmaf(8.f, m.x, m.y);
              m.x *= per_unit[i];
              top = fmaxf(top, m.x);
            }
          grow |= top > 16.f;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float top = -INFINITY;
#pragma unroll
            for (int k = 0; k < KS; ++k) top = fmaxf(top, fmaxf(s[k][nt][x], s[k][nt][2 + x]));
            grow |= top > high[nt][x];
          }
        if (__any_sync(0xffffffffu, grow)) {
          // The maximum moves only when a score is 2^6 above it in the softmax, the unit of the scales when one is 2^4 above it
          // (weights stay below 2^6, their products with scales below 2^10): seldom.
          float f[NT][2];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              float m = mx[nt][x];
#pragma unroll
              for (int k = 0; k < KS; ++k) m = fmaxf(m, fmaxf(s[k][nt][x], s[k][nt][2 + x]));
              m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
              m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
              m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
              f[nt][x] = m == mx[nt][x] ? 1.f : ex2((mx[nt][x] - m) * sc[nt][x]);
              mx[nt][x] = m;
              ref[nt][x] = m == -INFINITY ? 0.f : m;  // (a column that sees nothing yet: all weights 0)
              high[nt][x] = m == -INFINITY ? m : m + 6.f / sc[nt][x];
              l[nt][x] *= f[nt][x];
#pragma unroll
              for (int i = 0; i < G; ++i) om[nt][i][x] *= f[nt][x];
            }
#pragma unroll
          for (int i = 0; i < G; ++i) {
            float top = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k) top = fmaxf(top, fmaxf(mv[k][0][i].x, mv[k][1][i].x));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
            float by = 1.f;
            if (top > 1.f) by = __uint_as_float((254u << 23) - (__float_as_uint(top) & 0x7f800000u));  // the power of two that brings it to 1 .. 2
#pragma unroll
            for (int k = 0; k < KS; ++k) {
              mv[k][0][i].x *= by;
              mv[k][1][i].x *= by;
            }
            per_unit[i] *= by;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int h = 2 * i; h < 2 * i + 2; ++h)
#pragma unroll
                  for (int jj = 0; jj < 2; ++jj) {
                    o[nt][h][jj][x] *= f[nt][x] * by;
                    o[nt][h][jj][2 + x] *= f[nt][x] * by;
                  }
          }
        }
        // --- weights.  (The difference comes first.  A multiply-add with a rounded product of maximum and scale leaves 2^-24 of that in every
        // exponent, a factor next to other runs' parts, and far out all weights are 0 or infinite: 200 us for the long sequences, this 202.)
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              s[k][nt][x] = ex2((s[k][nt][x] - ref[nt][x]) * sc[nt][x]);
              s[k][nt][2 + x] = ex2((s[k][nt][2 + x] - ref[nt][x]) * sc[nt][x]);
              l[nt][x] += s[k][nt][x] + s[k][nt][2 + x];
            }
        // --- values
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            const float2 m0 = mv[k][0][i], m1 = mv[k][1][i];
            uint32_t p0[NT], p1[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
              for (int x = 0; x < 2; ++x) om[nt][i][x] = fmaf(s[k][nt][x], m0.y, fmaf(s[k][nt][2 + x], m1.y, om[nt][i][x]));
              p0[nt] = movmatrix_trans(half2_bits(__floats2half2_rn(s[k][nt][0] * m0.x, s[k][nt][1] * m0.x)));
              p1[nt] = movmatrix_trans(half2_bits(__floats2half2_rn(s[k][nt][2] * m1.x, s[k][nt][3] * m1.x)));
            }
            uint32_t w[4];
            ldmatrix_x4_trans(blk + 32 * D + k_lane + i * 2048 + k * 256, w);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t u0 = w[2 * h], u1 = w[2 * h + 1], v0 = u0 >> 8, v1 = u1 >> 8;
              const __half2 a00 = centred_low(u0, magic), a01 = centred_high(u0, magic), a02 = centred_low(u1, magic), a03 = centred_high(u1, magic);
              const __half2 a10 = centred_low(v0, magic), a11 = centred_high(v0, magic), a12 = centred_low(v1, magic), a13 = centred_high(v1, magic);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                mma_f16(o[nt][2 * i + h][0], a00, a01, a02, a03, p0[nt], p1[nt]);
                mma_f16(o[nt][2 * i + h][1], a10, a11, a12, a13, p0[nt], p1[nt]);
              }
            }
          }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty + 8 * st);
      st += 2;
      if (st >= S::kStages) { st -= S::kStages; phase ^= 1; }
    }
    mine_at = (mine_at + stop - first) & 1;  // (the pairs take turns over the whole run)

    // --- join the four warps: each leaves O, maximum and sum of its tokens in shared memory
    float* mine = join + warp * S::kWarpJoin;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float sum = l[nt][x];
        float add[G];
#pragma unroll
        for (int i = 0; i < G; ++i) add[i] = om[nt][i][x];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
          sum += __shfl_xor_sync(0xffffffffu, sum, d);
#pragma unroll
          for (int i = 0; i < G; ++i) add[i] += __shfl_xor_sync(0xffffffffu, add[i], d);
        }
        const int col = nt * 8 + 2 * t + x;
#pragma unroll
        for (int h = 0; h < CH; ++h) {
          const auto value = [&](float v) { return fmaf(v, 1.f / per_unit[h / 2], add[h / 2]); };
          *reinterpret_cast<float4*>(mine + col * S::kCol + 32 * h + 4 * g) =
              make_float4(value(o[nt][h][0][x]), value(o[nt][h][0][2 + x]), value(o[nt][h][1][x]), value(o[nt][h][1][2 + x]));
        }
        if (g == 0) { mine[R * S::kCol + col] = mx[nt][x] * back[nt][x]; mine[R * S::kCol + R + col] = sum; }
      }
    epi_bar_sync();
    const bool whole = first == 0 && stop == c.tiles;
    float* part = partial_of<L, D>(a, blockIdx.x, first == 0);
    for (int x = tid; x < R * (D / 4); x += kWarps * 32) {
      const int col = x / (D / 4), d4 = (x % (D / 4)) * 4, r = r0 + col;
      float m = -INFINITY, sum = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) m = fmaxf(m, join[w * S::kWarpJoin + R * S::kCol + col]);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float* p = join + w * S::kWarpJoin;
        const float pm = p[R * S::kCol + col], f = pm == -INFINITY ? 0.f : ex2((pm - m) * a.scale);
        const float4 y = *reinterpret_cast<const float4*>(p + col * S::kCol + d4);
        sum = fmaf(f, p[R * S::kCol + R + col], sum);
        v.x = fmaf(f, y.x, v.x); v.y = fmaf(f, y.y, v.y); v.z = fmaf(f, y.z, v.z); v.w = fmaf(f, y.w, v.w);
      }
      if (!whole) {
        *reinterpret_cast<float4*>(part + col * D + d4) = v;
        if (d4 == 0) { part[R * D + col] = m; part[R * D + R + col] = sum; }
      } else if (r < rows) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;  // a row that sees nothing is 0
        const int j = a.by_group(r), hd = r - j * a.group;
        uint2 y;
        y.x = pack_bf16x2(v.x * inv, v.y * inv);
        y.y = pack_bf16x2(v.z * inv, v.w * inv);
        *reinterpret_cast<uint2*>(a.out + (int64_t)(c.info.row0 + j) * a.ld_out + (int64_t)(c.kvh * a.group + hd) * D + d4) = y;
      }
    }
    epi_bar_sync();
    if (left <= 0) break;
  }
}

template <int D, int NT, bool MASKED>
int32_t launch(essa_ctx* ctx, AttendArgs& a, cudaStream_t stream) {
  using S = Shape<D, NT>;
  using L = DecodeList<S::R, MASKED>;
  const int grid = ctx->sm_count * attend_blocks_per_sm(D, NT);
  a.partials_at = partials_at(grid);
  a.whole = whole_blocks<L>(a, grid);
  cudaError_t e = allow_shared<attend_decode_kernel<D, NT, MASKED>>(S::kSmem, ctx->device);
  if (e != cudaSuccess) return check_cuda(ctx, e, "cudaFuncSetAttribute (attend)");
  attend_decode_kernel<D, NT, MASKED><<<grid, kThreads, S::kSmem, stream>>>(a);
  e = cudaGetLastError();
  if (e != cudaSuccess) return check_cuda(ctx, e, "attend launch");
  ++ctx->launches;
  return launch_join<L, D>(ctx, a, grid, S::R / 4, stream);
}
template <bool MASKED>
int32_t launch_shape(essa_ctx* ctx, AttendArgs& a, int nt, cudaStream_t stream) {
  if (a.v.head_dim == 64) return nt == 1 ? launch<64, 1, MASKED>(ctx, a, stream) : launch<64, 2, MASKED>(ctx, a, stream);
  return nt == 1 ? launch<128, 1, MASKED>(ctx, a, stream) : launch<128, 2, MASKED>(ctx, a, stream);
}

}  // namespace

// Column tiles of eight query rows that a row block takes.
static int attend_nt(int64_t rows_hint) { return rows_hint > 8 ? 2 : 1; }

int64_t attend_decode_workspace(int head_dim, int64_t rows_hint, int sm_count) {
  const int nt = attend_nt(rows_hint);
  return attend_workspace(sm_count * attend_blocks_per_sm(head_dim, nt), (int64_t)(8 * nt) * (head_dim + 2));
}

int32_t launch_attend_decode(essa_ctx* ctx, AttendArgs& a, int64_t rows_hint, cudaStream_t stream) {
  const int nt = attend_nt(rows_hint);
  return a.masked ? launch_shape<true>(ctx, a, nt, stream) : launch_shape<false>(ctx, a, nt, stream);
}

}  // namespace essa
