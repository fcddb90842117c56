// Attention over the paged 4-bit cache for many rows per sequence (prompts, chunks): tcgen05 tiles.
//
// A row block is 256 query rows (token-major: row r of an entry is token r / group, head r % group of a kv head, so the heads that
// share K and V share a tile), two halves of 128; a key tile is one page.  Per key tile and half: S = Q K^T (fp16, M = 128, N = 64)
// into one of two buffers in tensor memory, softmax by eight warps (two threads per row, 32 keys each), P back into the same columns as
// fp16, O += P V (fp16, A from tensor memory, V as stored: MN-major).  Products with K run two tiles ahead.  Four warps widen the pages, one
// copies them in (bulk copies), one issues the MMAs.  Tensor memory: 4 x 64 columns of scores, 2 x head_dim of O.
//
// What bounds it (heads of 128 channels): a key tile takes ~2290 cycles of an SM.  The tensor pipe counts 1024 of them as active, but the MMAs take
// ~1800 (N = 64 makes a product with K read 6 KB of shared memory in its 32 cycles of arithmetic); the exponentials need 1024 of the special
// function units, the warps half of the issue slots.  Two prompts of 450 tokens after 16 thousand, 64 heads (468 GFLOP): 500 to 550 us (by
// clocks), 0.85 to 0.94 PFLOP/s.  A row block costs some six tiles beside its own (queries in, results out): ragged prompts of 1 .. 1024 tokens, 40 heads (231
// GFLOP): 495 to 509 us.
// What was tried, when the ragged prompts stood at 496: a thread per row (eight softmax warps): 558 us, and 495 for the others; key tiles of two pages, products
// with K of N = 128 and one buffer of scores per half: 558 and 455 (the halves' softmax and products then alternate, but a tile of 128
// keys is a coarse grain for short prompts); the same with 80 registers for the softmax instead of 96: 705 and 608;
// an eighth, a quarter or a half of the exponentials by a polynomial on the FMA pipe: 486, 498 and 535 (issue slots are as short as the
// special function units); O through shared memory, so that stores are whole rows: 502 and 481 (an SM stores 32 bytes a cycle either way).
//
// Roundings: K and V become fp16 as their scale and minimum are applied, (code - 8) * scale + (minimum + 8 scale), with the offset and the
// result rounded (2^-11 each).  Q is bf16; a row times a power of two, its largest element at 2^13 .. 2^14, is fp16 without loss (elements
// 2^-27 below the largest lose bits).  P is fp16 (2^-11; weights below 6e-8 of the largest lose bits).  With bf16 operands instead, K's
// three roundings (scale, offset, result: 2^-8 each) made up most of the error: 3.2e-3 of the result's norm against 1.7e-3 from rounding
// the result alone.  S, the maximum, the sums and O are fp32.
// Channel order inside a group of eight channels is (0, 4, 1, 5, 2, 6, 3, 7), what masking nibbles out of a word gives: Q is stored in
// the same order, and O's columns are put back on the way out.
#include "cache_list.cuh"

namespace essa {
namespace {

// kSetup: the ragged prompts take 483 us with 3, 479 with 4, 483 with 5, 493 with 6.
struct TileList {
  static constexpr int R = 256, kKeys = kPageTokens, kMinRun = 2, kSetup = 4;
  // keys that the last row of the row block sees, in tiles
  __device__ static int tiles(const EntryInfo& e, const AttendArgs& a, int rb) {
    const int last = min(e.rows - 1, a.by_group(min(rb * R, 0x7fffffff - R) + R - 1));
    return max((e.len - e.rows + last + 1 + kKeys - 1) / kKeys, 1);
  }
  __device__ static long long per_head(const EntryInfo& e, const AttendArgs& a) {
    long long sum = 0;
    const int blocks = row_blocks(e, a.group, R);
    for (int rb = 0; rb < blocks; ++rb) sum += tiles(e, a, rb) + kSetup;
    return sum;
  }
};

constexpr int kSoftWarps = 16, kWidenWarps = 4;
constexpr int kMmaWarp = kSoftWarps + kWidenWarps, kCopyWarp = kMmaWarp + 1;
constexpr int kThreads = 768;  // six warpgroups; the last two warps only give registers away
// Registers per thread: launched with 80, of which the softmax takes more.  4 * 88 + 2 * 64 = 6 * 80.  (Nothing spills; 96 and 48: 508 us for
// the ragged prompts, 80 and 80: 505, this: 502.)
constexpr int kSoftRegs = 88, kOtherRegs = 64;
constexpr int kRaw = 3;  // pages in flight

constexpr int kRing = 4;  // widened key tiles, K and V

template <int D>
struct Mem {  // offsets from a 1024-byte boundary
  static constexpr int kHalf = D / 64 * 128 * 128;    // one half of Q: [64-channel block][128 rows][128 bytes]
  static constexpr int kSub = 64 * 128;               // 64 keys x 64 channels
  static constexpr int kTile = D / 64 * kSub;         // a key tile of K or V
  static constexpr int kQ = 0, kK = 2 * kHalf, kV = kK + kRing * kTile, kRawAt = kV + kRing * kTile;
  static constexpr int kRun = 72 * D;
  static constexpr int kBars = kRawAt + kRaw * kRun;
  static constexpr int kBytes = kBars + 512;
};
enum Bar { kRawFull = 0, kRawEmpty = kRaw, kTileFull = 2 * kRaw, kTileEmpty = kTileFull + kRing, kQFull = kTileEmpty + kRing, kOFull = kQFull + 2, kSFull = kOFull + 2 /* [half][buffer] */, kPFull = kSFull + 4, kDone = kPFull + 4, kBarCount };
static_assert(kBarCount * 8 <= 512, "");

// Instruction descriptor of kind::f16 with both operands fp16 and M = 128; n_contiguous: B is stored with N contiguous.
__host__ __device__ constexpr uint32_t f16_idesc(int N, bool n_contiguous) {
  return (1u << 4) | ((n_contiguous ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | (8u << 24);
}

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ __nv_bfloat162 as_bf162(uint32_t v) { return *reinterpret_cast<__nv_bfloat162*>(&v); }

// Operands in shared memory are 128-byte rows under the 128-byte swizzle.  Q and K: a row is 64 channels of a row / key (K contiguous).
// V as B operand of O += P V: [64-channel block][key][64 channels], i.e. N contiguous: 64 channels x 8 keys per 1024-byte swizzle atom,
// the next eight keys 1024 bytes on (stride offset), the next 64 channels one sub-tile on (leading offset).
// Registers of a tmem_ld32_issue are valid from here on (they pass through, so that no use of them can move up).
__device__ __forceinline__ void tmem_ld_done(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
                 "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]),
                 "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :
               : "memory");
}
__device__ __forceinline__ void st_global_32(void* p, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]),
               "r"(v[7])
               : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// 16 consecutive columns of the warp's lanes (with the wait).
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr), "r"(v[0]), "r"(v[1]),
               "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
               : "memory");
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
// Barrier of two warps, and whether a predicate holds for any of their threads.
__device__ __forceinline__ void pair_sync(int id) { asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory"); }
__device__ __forceinline__ bool pair_any(int id, bool x) {
  uint32_t r;
  asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 p, %2, 0;\nbar.red.or.pred q, %1, 64, p;\nselp.u32 %0, 1, 0, q;\n}\n" : "=r"(r) : "r"(id), "r"((uint32_t)x) : "memory");
  return r != 0;
}
// One lane of the (converged) warp, the same one every time.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ void prefetch_l2(const void* p, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
}
// A shared-memory matrix descriptor whose address part is `lo` (and the leading offset, bits 16-29): only this half changes between MMAs.
__device__ __forceinline__ uint64_t desc_of(uint32_t lo) {
  constexpr uint32_t hi = (1024u >> 4) | (1u << 14) | (2u << 29);  // stride 1024 bytes, version 1, 128-byte swizzle
  return (uint64_t)hi << 32 | lo;
}

constexpr float kFp16End = 65440.f;  // (65504 less what rounding the centre and the result can add)

// Eight codes -> fp16 (code - 8) * s + c in the order (0, 4, 1, 5, 2, 6, 3, 7).
__device__ __forceinline__ uint4 widen(uint32_t w, __half2 s, __half2 c, uint32_t magic /* 0x64006400 */) {
  const uint32_t x = w >> 8;
  return make_uint4(half2_bits(__hfma2(centred_low(w, magic), s, c)), half2_bits(__hfma2(centred_high(w, magic), s, c)),
                    half2_bits(__hfma2(centred_low(x, magic), s, c)), half2_bits(__hfma2(centred_high(x, magic), s, c)));
}
// Whether some code of a token's group, (scale, minimum) = m, stands for a value beyond +-65440 (false for a minimum of NaN).
__device__ __forceinline__ bool beyond_fp16(float2 m) { return m.y < -kFp16End || fmaf(15.f, m.x, m.y) > kFp16End; }
// The same order for such a group (seldom): every value for itself, in fp32, brought to +-65440, what fp16 rounds it to being finite there.
// (The centre of such a group can lie outside fp16 as well.  Changing the scale or the minimum instead would move its other values.)
__device__ __forceinline__ uint4 widen_clipped(uint32_t w, float2 m) {
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float lo = fmaf((float)(w >> (4 * i) & 15u), m.x, m.y), hi = fmaf((float)(w >> (4 * i + 16) & 15u), m.x, m.y);
    r[i] = pack_f16x2(fminf(fmaxf(lo, -kFp16End), kFp16End), fminf(fmaxf(hi, -kFp16End), kFp16End));
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}
template <int D>
__global__ void __launch_bounds__(kThreads, 1) attend_tiles_kernel(AttendArgs a) {
  using M = Mem<D>;
  using L = TileList;
  extern __shared__ uint8_t smem_raw[];
  __shared__ RunShared run_sm;
  __shared__ volatile int abort_flag;
  __shared__ int raw_bad[kRaw];
  __shared__ int tile_bad[8];  // the key tile's page is not there
  __shared__ uint32_t tmem_slot;
  __shared__ float row_scale[L::R];           // what a row of Q was divided by
  __shared__ float of_part[2][L::R];   // maximum, then sum, of the keys that a row's two threads look at
  // Where the softmax and the widening warps are in the list, between row blocks (in registers it would cost their loops spills).
  struct Place {
    Cursor c;
    long long left;
  };
  __shared__ Place places[kSoftWarps + kWidenWarps];
  __shared__ int out_of[kSoftWarps][2][3];  // a softmax warp's present and next row block: first row of q, kv head, row of the group
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t bars = base + M::kBars;
  const auto bar = [&](int i) { return bars + 8 * i; };
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (!a.whole) grid_dep_launch();  // (else the launch that follows is not the join)
  if (tid == 0) {
    abort_flag = 0;
    for (int i = 0; i < kRaw; ++i) { mbar_init(bar(kRawFull + i), 1); mbar_init(bar(kRawEmpty + i), kWidenWarps); }
    for (int i = 0; i < kRing; ++i) { mbar_init(bar(kTileFull + i), kWidenWarps); mbar_init(bar(kTileEmpty + i), 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(bar(kQFull + i), kSoftWarps / 2); mbar_init(bar(kOFull + i), 1); }
    for (int i = 0; i < 4; ++i) { mbar_init(bar(kSFull + i), 1); mbar_init(bar(kPFull + i), kSoftWarps / 2); }
    mbar_init(bar(kDone), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  Cursor c;
  long long left = find_run<L>(a, c, run_sm);
  if (left == 0) return;
  if (warp == kMmaWarp) {
    tmem_alloc(smem_u32(&tmem_slot), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const auto keep_place = [&](const Cursor& at, long long rest) {
    __syncwarp();
    if (lane == 0) places[warp] = Place{at, rest};
    __syncwarp();
  };
  if (warp < kSoftWarps + kWidenWarps) keep_place(c, left);
  const auto wait = [&](int b, uint32_t parity) { return mbar_wait(bar(b), parity, &abort_flag, a.status); };
  const auto wait_warp = [&](int b, uint32_t parity) { return __all_sync(0xffffffffu, wait(b, parity)) != 0; };

  if (warp < kSoftWarps) {  // ------------------------------------------------------------------ softmax, two threads per row
    // (32 of a tile's 64 keys each, and half of O's channels; the two warps that share 32 rows keep in step by a barrier of their own)
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
    const int h = warp >> 3, part = warp >> 2 & 1, quad = warp & 3, row = quad * 32 + lane, pair = 1 + 4 * h + quad;
    const uint32_t lanes = (uint32_t)quad * 32u << 16;
    const uint32_t o_at = tmem + 256 + D * h + D / 2 * part + lanes;
    int tile = 0;  // key tiles of the run so far
    uint32_t s_ph = 0, o_ph = 0;  // s_ph: a bit per buffer
    bool dead = false;  // a wait ran out: the warp goes on through the barriers with the other one, and waits for nothing else
    const auto await = [&](int b, uint32_t parity) {
      if (!dead) dead = !wait_warp(b, parity);
      tc_fence_after();
    };
    // What a thread needs of the row block that it is at.
    struct Block {
      int first, n;
      int limit, lowest;  // keys that the row sees (0x7fffffff: no such row); the fewest of the warp's rows
      float back;         // what the row of Q was divided by
      bool whole;
    };
    // Moves on to the next row block in which this half has rows (false: none left) and puts its rows of Q into shared memory: D / 8
    // lanes per row, channels in the order of the widened codes.
    int parity = 0;
    const auto enter = [&](Block& b) {
      int rows, r0, row0, kvh, past;
      {
        Cursor c = places[warp].c;
        long long left = places[warp].left;
        for (;; next_block<L>(a, c)) {
          if (left <= 0) return false;
          int stop;
          take_block<L>(a, c, left, b.first, stop);
          b.n = stop - b.first;
          if (b.n == 0) return false;  // (the run ends before the row block's first tile)
          b.whole = b.first == 0 && stop == c.tiles;
          if (c.rb * L::R + h * 128 < c.info.rows * a.group) break;
          tile += b.n;
          if (left <= 0) return false;
        }
        rows = c.info.rows * a.group;
        r0 = c.rb * L::R + h * 128;
        row0 = c.info.row0;
        kvh = c.kvh;
        past = c.info.len - c.info.rows;
        if (left > 0) next_block<L>(a, c);
        keep_place(c, left);
      }
      parity ^= 1;
      if (lane < 3) out_of[warp][parity][lane] = lane == 0 ? row0 : lane == 1 ? kvh : r0;
      constexpr int kLanes = D / 8, kRowsAt = 32 / kLanes, kSteps = 16 / kRowsAt;
      const int ch = lane % kLanes;
      const __nv_bfloat16* q = a.q + (int64_t)row0 * a.ld_q + (int64_t)kvh * a.group * D + ch * 8;
      uint4 x[kSteps];
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int r = r0 + quad * 32 + part * 16 + i * kRowsAt + lane / kLanes, tok = a.by_group(r);
        x[i] = make_uint4(0, 0, 0, 0);
        if (r < rows) x[i] = __ldg(reinterpret_cast<const uint4*>(q + tok * a.ld_q + (r - tok * a.group) * D));
      }
      // fp16 holds the rows as they are if every piece of eight channels has an element between 2^-6 and 2^15; otherwise each row is
      // brought there by a power of two
      __nv_bfloat162 least = as_bf162(0x7f807f80u), most = as_bf162(0u);
      int rr = quad * 32 + part * 16 + lane / kLanes;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const __nv_bfloat162 big = __hmax2_nan(__hmax2_nan(__habs2(as_bf162(x[i].x)), __habs2(as_bf162(x[i].y))), __hmax2_nan(__habs2(as_bf162(x[i].z)), __habs2(as_bf162(x[i].w))));
        most = __hmax2_nan(most, big);
        if (r0 + rr + i * kRowsAt < rows) least = __hmin2_nan(least, big);
      }
      const float low = fminf(__low2float(least), __high2float(least));
      const bool plain = __all_sync(0xffffffffu, __low2float(most) < 32768.f && __high2float(most) < 32768.f && low >= 0.015625f);  // (false for NaN)
#pragma unroll
      for (int i = 0; i < kSteps; ++i, rr += kRowsAt) {
        float f[8] = {__uint_as_float(x[i].x << 16), __uint_as_float(x[i].x & 0xffff0000u), __uint_as_float(x[i].y << 16), __uint_as_float(x[i].y & 0xffff0000u),
                      __uint_as_float(x[i].z << 16), __uint_as_float(x[i].z & 0xffff0000u), __uint_as_float(x[i].w << 16), __uint_as_float(x[i].w & 0xffff0000u)};
        int e = 0;
        if (!plain) {
          float big = 0.f;
#pragma unroll
          for (int k = 0; k < 8; ++k) big = fmaxf(big, fabsf(f[k]));
#pragma unroll
          for (int d = 1; d < kLanes; d <<= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, d));
          // largest element at 2^13 .. 2^14 (not of a row of zeros, or one with an infinity)
          e = big > 0.f && big < INFINITY ? max((int)(__float_as_uint(big) >> 23), 27) - 127 - 13 : 0;
          const float up = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
          for (int k = 0; k < 8; ++k) f[k] *= up;
        }
        if (ch == 0) row_scale[h * 128 + rr] = __uint_as_float((uint32_t)(127 + e) << 23);
        sts_v4(base + M::kQ + h * M::kHalf + (ch >> 3) * (128 * 128) + rr * 128 + (((ch & 7) ^ (rr & 7)) << 4),
               make_uint4(pack_f16x2(f[0], f[4]), pack_f16x2(f[1], f[5]), pack_f16x2(f[2], f[6]), pack_f16x2(f[3], f[7])));
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(kQFull + h));
      pair_sync(pair);  // (row_scale)
      const int r = r0 + row;
      b.back = row_scale[h * 128 + row];
      // rows behind the last one have q = 0 and are not written, whatever they see
      b.limit = r < rows ? past + a.by_group(r) + 1 : 0x7fffffff;
      b.lowest = __shfl_sync(0xffffffffu, b.limit, 0);
      return true;
    };
    const bool wide_out = !(reinterpret_cast<uintptr_t>(a.out) & 31) && a.ld_out % 16 == 0;  // whole 32-byte sectors
    Block b, next;
    b.n = 0;
    // Maximum, sum of weights and softmax scale (in the units of the row).  Weights are 2^(s scale + shift) with shift = -m scale, rounded: 2^-25
    // of the exponent away from being relative to m itself.  That changes nothing in a row's own result, but a partial result is taken back to m
    // (a factor), and an exponent is kept below 2^27, where it is at most 2^4.
    float m = 0.f, sum = 0.f, scale = 0.f;
    const auto shift_of = [&](float top) { return top == -INFINITY ? 0.f : -top * scale; };  // (a row that sees nothing yet: all weights 0)
    for (;;) {
      // --- the next row block's Q (all products with this one's are done), while the last product with V runs
      const bool more = enter(next);
      if (b.n > 0) {
        if (!more) pair_sync(pair);  // (the other warp has read of_part's maxima; enter has a barrier too)
        of_part[part][h * 128 + row] = sum;
        pair_sync(pair);
        sum = of_part[0][h * 128 + row] + of_part[1][h * 128 + row];
        pair_sync(pair);
        await(kOFull + h, o_ph);
        o_ph ^= 1;
        // --- out, or a partial result; columns (0, 4, 1, 5, 2, 6, 3, 7) of eight are the channels in order
        const float inv = sum == 0.f ? 0.f : 1.f / sum;  // a row that sees nothing is 0
        const float fix = ex2(m == -INFINITY ? 0.f : -fmaf(m, scale, shift_of(m)));
        const int rr = h * 128 + row;
        const int* o = out_of[warp][parity ^ (more ? 1 : 0)];
        const int r = o[2] + row, tok = a.by_group(r);
        __nv_bfloat16* out = a.out + (int64_t)(o[0] + tok) * a.ld_out + (int64_t)(o[1] * a.group + r - tok * a.group) * D;
        const bool there = b.limit != 0x7fffffff;
        float* partial = partial_of<L, D>(a, blockIdx.x, b.first == 0);
#pragma unroll 1
        for (int d = 0; d < D / 2; d += 32) {
          uint32_t v[32];
          tmem_ld32_issue(o_at + d, v);
          tmem_ld_done(v);
          const auto at = [&](int i) { return __uint_as_float(v[i]); };
          const int ch = D / 2 * part + d;
          if (there && b.whole) {
#pragma unroll
            for (int i = 0; i < 32; i += 16) {
              uint32_t y[8];
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const int o = i + 8 * k;
                y[4 * k] = pack_bf16x2(at(o) * inv, at(o + 2) * inv);
                y[4 * k + 1] = pack_bf16x2(at(o + 4) * inv, at(o + 6) * inv);
                y[4 * k + 2] = pack_bf16x2(at(o + 1) * inv, at(o + 3) * inv);
                y[4 * k + 3] = pack_bf16x2(at(o + 5) * inv, at(o + 7) * inv);
              }
              if (wide_out) {
                st_global_32(out + ch + i, y);
              } else {
                *reinterpret_cast<uint4*>(out + ch + i) = make_uint4(y[0], y[1], y[2], y[3]);
                *reinterpret_cast<uint4*>(out + ch + i + 8) = make_uint4(y[4], y[5], y[6], y[7]);
              }
            }
          } else if (there) {
#pragma unroll
            for (int i = 0; i < 32; i += 8) {
              *reinterpret_cast<float4*>(partial + rr * D + ch + i) = make_float4(at(i) * fix, at(i + 2) * fix, at(i + 4) * fix, at(i + 6) * fix);
              *reinterpret_cast<float4*>(partial + rr * D + ch + i + 4) = make_float4(at(i + 1) * fix, at(i + 3) * fix, at(i + 5) * fix, at(i + 7) * fix);
            }
          }
        }
        if (!b.whole && part == 0) {
          partial[L::R * D + rr] = m * b.back;
          partial[L::R * D + L::R + rr] = sum * fix;
        }
        tc_fence_before();
      }
      if (!more) break;
      b = next;
      scale = softmax_scale(a.scale * b.back);
      m = -INFINITY;
      sum = 0.f;
      const auto scores_at = [&](int t) { return tmem + 128 * h + 64 * (t & 1) + lanes; };  // (P follows in the first 32 columns)
      // Scores of the block's tile j, the run's tile t: waits for them; hidden ones become -infinity in place (the tiles that hide none
      // pay nothing for it).
      const auto arrived = [&](int j, int t) {
        await(kSFull + 2 * h + (t & 1), s_ph >> (t & 1) & 1);
        s_ph ^= 1u << (t & 1);
        const int key0 = (b.first + j) * L::kKeys, bad = tile_bad[t & 7];
        if (key0 + L::kKeys > b.lowest || bad) {
          const int see = bad ? 0 : b.limit - key0 - 32 * part;  // this thread's keys before this one are seen
          uint32_t v[32];
          tmem_ld32_issue(scores_at(t) + 32 * part, v);
          tmem_ld_done(v);
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (i >= see) v[i] = 0xff800000u;
          tmem_st32(scores_at(t) + 32 * part, v);
        }
      };
      for (int j = 0; j < b.n; ++j, ++tile) {
        arrived(j, tile);
        const uint32_t s_at = scores_at(tile);
        uint32_t p[16];
        float s0, s1;
        // Whether to look for the maximum before the weights: in the first tile, and where the weights by the one so far turn out too large or
        // there is none yet though the row sees the tile (the pages before are not there): weights by 0 could then all vanish.  (A row's two
        // threads have the same m and limit, so the two warps decide alike.)
        bool look = j == 0 || __any_sync(0xffffffffu, m == -INFINITY && b.limit > (b.first + j) * L::kKeys);
        for (;;) {
          uint32_t v[32];
          tmem_ld32_issue(s_at + 32 * part, v);
          tmem_ld_done(v);
          if (look) {
            float t[4] = {m, m, m, m};
#pragma unroll
            for (int i = 0; i < 32; i += 2) t[i >> 1 & 3] = max3(t[i >> 1 & 3], __uint_as_float(v[i]), __uint_as_float(v[i + 1]));
            float top = max3(max3(t[0], t[1], t[2]), t[3], t[3]);
            if (j > 0) pair_sync(pair);  // (the other warp has read what the tile before left in of_part)
            of_part[part][h * 128 + row] = top;
            tc_fence_before();
            pair_sync(pair);
            tc_fence_after();
            top = fmaxf(top, of_part[part ^ 1][h * 128 + row]);
            // Exponents beyond 2^27 (no model has such scores; the products know them to 2^-18 at best) shrink to that: keys whose scores differ
            // by more than 2^-19 of the maximum keep weights of 0.
            if (top != -INFINITY && fabsf(top * scale) > 0x1p27f) scale = 0x1p27f / fabsf(top);
            if (j > 0) {
              // O holds the tiles before this one: their products end before those with the K of the next tile, or (there is none) signal
              if (j + 1 < b.n) await(kSFull + 2 * h + (~tile & 1), s_ph >> (~tile & 1) & 1);
              else await(kOFull + h, o_ph);
              const float f = top == m ? 1.f : m == -INFINITY ? 0.f : ex2(shift_of(top) - shift_of(m));
              sum *= f;
#pragma unroll 1
              for (int d = 0; d < D / 2; d += 16) {
                float y[16];
                tmem_ld16(o_at + d, y);
#pragma unroll
                for (int i = 0; i < 16; ++i) p[i] = __float_as_uint(y[i] * f);
                tmem_st16(o_at + d, p);
              }
            }
            m = top;
          }
          const float shift = shift_of(m);
          const uint64_t scale2 = pack_f32x2(scale, scale), shift2 = pack_f32x2(shift, shift);
          uint64_t sums[2] = {0, 0};
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float x0, x1;
            unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), scale2, shift2), x0, x1);
            x0 = ex2(x0);
            x1 = ex2(x1);
            sums[i & 1] = add_f32x2(sums[i & 1], pack_f32x2(x0, x1));
            p[i] = pack_f16x2(x0, x1);
          }
          unpack_f32x2(add_f32x2(sums[0], sums[1]), s0, s1);
          s0 += s1;
          // No running maximum: the tile's sum says whether a weight can be too large for fp16 (a score 2^14 above the maximum so far in
          // the softmax; seldom).  Then the maximum is looked for, O and the sum are scaled, and the tile is done again.
          // (The barrier, here or above, also stands between the other warp's reading of its scores and P, which goes where they are.)
          if (look) break;
          tc_fence_before();
          const bool again = pair_any(pair, s0 > 16384.f);
          tc_fence_after();
          if (!again) break;
          look = true;
        }
        sum += s0;
        tmem_st16(s_at + 16 * part, p);
        if (j > 0 && j + 1 == b.n) {  // the last two products with V signal: the first of them is seen before the second can start
          await(kOFull + h, o_ph);
          o_ph ^= 1;
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(kPFull + 2 * h + (tile & 1)));
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp == kCopyWarp) {  // ------------------------------------------------------------------ pages -> shared memory
      if (lane == 0) {
        int slot = 0, filled = 0;
        uint32_t phase = 0;
        bool ok = true;
        while (ok && left > 0) {
          int first, stop;
          take_block<L>(a, c, left, first, stop);
          if (first == stop) break;  // (the run ends before the row block's first tile)
          const int pages = (c.info.len + kPageTokens - 1) / kPageTokens;
          const int32_t* row = a.v.table + (int64_t)max(c.info.slot, 0) * a.v.max_pages;
          if (c.info.slot < 0) cache_fault(a.status);
          {  // the row block's part of q into L2, a key tile or more before the softmax warps ask for it
            const int t0 = a.by_group(c.rb * L::R), t1 = min(c.info.rows, a.by_group(min(c.rb * L::R, 0x7fffffff - L::R) + L::R - 1) + 1);
            for (int t = t0; t < t1; ++t) prefetch_l2(a.q + (int64_t)(c.info.row0 + t) * a.ld_q + (int64_t)c.kvh * a.group * D, a.group * D * 2);
          }
          for (int p = first; p < stop; ++p) {
            if (filled >= kRaw && !wait(kRawEmpty + slot, phase ^ 1)) { ok = false; break; }
            const int page = p < pages ? __ldg(row + p) : -1;
            const bool there = page >= 0 && page < a.v.num_pages;
            if (!there && p < pages) cache_fault(a.status);
            raw_bad[slot] = !there;
            if (there) {
              mbar_expect_tx(bar(kRawFull + slot), M::kRun);
              bulk_load(base + M::kRawAt + slot * M::kRun, a.v.pages + page * a.v.page_bytes + (int64_t)c.kvh * M::kRun, M::kRun, bar(kRawFull + slot));
            } else {
              mbar_arrive(bar(kRawFull + slot));
            }
            ++filled;
            if (++slot == kRaw) { slot = 0; phase ^= 1; }
          }
          if (left > 0) next_block<L>(a, c);
        }
        if (!ok) drain_ring(bar(kRawFull), kRaw, filled);
      }
    } else if (warp == kMmaWarp) {  // ------------------------------------------------------------ MMAs
      // (few instructions between two MMAs: what the issuing thread does there delays them)
      if (elect_one()) {
        constexpr uint32_t kQk = f16_idesc(64, false), kPv = f16_idesc(D, true);
        const uint32_t q_lo = (base + M::kQ) >> 4, k_lo = (base + M::kK) >> 4, v_lo = ((base + M::kV) >> 4) | (uint32_t)(M::kSub >> 4) << 16;
        uint32_t q_ph = 0, p_ph = 0;    // a bit per half; per half and buffer
        uint32_t k_at = 0, v_at = 0;    // key tiles of the run whose products with K / V have been issued
        bool ok = true;
        const auto qk = [&](int h) {
          const uint32_t d = tmem + 128 * h + 64 * (k_at & 1), q0 = q_lo + h * (M::kHalf >> 4), k0 = k_lo + k_at % kRing * (M::kTile >> 4);
#pragma unroll
          for (int i = 0; i < D / 16; ++i)
            umma_bf16(d, desc_of(q0 + (((i / 4) * 128 * 128 + (i % 4) * 32) >> 4)), desc_of(k0 + (((i / 4) * M::kSub + (i % 4) * 32) >> 4)), kQk, i > 0);
          umma_commit(bar(kSFull + 2 * h + (k_at & 1)));
        };
        while (ok && left > 0) {
          int first, stop;
          take_block<L>(a, c, left, first, stop);
          const int n = stop - first, halves = c.info.rows * a.group - c.rb * L::R > 128 ? 2 : 1;
          if (n == 0) break;
          // Products with K run two tiles ahead: the scores of a half's next tile are there when its softmax has finished one.
          for (int j = 0; ok && j < min(n, 2); ++j, ++k_at) {
            if (!(ok = wait(kTileFull + k_at % kRing, k_at / kRing & 1))) break;
            for (int h = 0; h < halves; ++h) {
              if (j == 0) {
                if (!(ok = wait(kQFull + h, q_ph >> h & 1))) break;
                q_ph ^= 1u << h;
              }
              tc_fence_after();
              qk(h);
            }
          }
          for (int j = 0; ok && j < n; ++j, ++v_at) {
            const bool more = j + 2 < n;
            for (int h = 0; h < halves; ++h) {
              const uint32_t at = 2 * h + (v_at & 1);
              if (!(ok = wait(kPFull + at, p_ph >> at & 1))) break;
              p_ph ^= 1u << at;
              tc_fence_after();
              const uint32_t d = tmem + 256 + D * h, p0 = tmem + 128 * h + 64 * (v_at & 1), v0 = v_lo + v_at % kRing * (M::kTile >> 4);
#pragma unroll
              for (int i = 0; i < 4; ++i) umma_bf16_ts(d, p0 + 8 * i, desc_of(v0 + i * (2048 >> 4)), kPv, i > 0 || j > 0);
              if (!more) {
                umma_commit(bar(kOFull + h));
                continue;
              }
              if (h == 0 && !(ok = wait(kTileFull + k_at % kRing, k_at / kRing & 1))) break;
              qk(h);
            }
            if (!ok) break;
            // V of this tile, and K of every tile up to it, have been used
            umma_commit(bar(kTileEmpty + v_at % kRing));
            if (more) ++k_at;
          }
          if (left > 0) next_block<L>(a, c);
        }
        if (!ok) {  // MMAs in flight finish (a bounded wait) before tensor memory is given back
          umma_commit(bar(kDone));
          const long long t0 = clock64();
          while (!mbar_try_wait(bar(kDone), 0) && clock64() - t0 < kWaitLimitCycles / 16) {}
        }
      }
      __syncwarp();
    } else if (warp < kMmaWarp) {  // ---------------------------------------------------------- pages -> operands
      const int wt = tid - kSoftWarps * 32;
      const int token = wt & 63, part = wt >> 6;       // D = 128: a 64-channel group each; D = 64: half a group each
      uint32_t magic = 0x64006400u;
      asm volatile("" : "+r"(magic));  // in a register
      constexpr int kWords = D / 16;                   // 32-bit words of codes per thread: 8 or 4
      const int group = D == 128 ? part : 0, word0 = D == 128 ? 0 : part * 4;
      int slot = 0, tile = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (;;) {
        int j, stop, len;
        {
          Cursor c = places[warp].c;
          long long left = places[warp].left;
          if (left <= 0) break;
          take_block<L>(a, c, left, j, stop);
          len = c.info.len;
          if (left > 0) next_block<L>(a, c);
          keep_place(c, left);
        }
        for (; j < stop; ++j, ++tile) {
          const int st = tile % kRing;
          const uint32_t reuse = (tile / kRing & 1) ^ 1;
          const uint32_t k_dst = base + M::kK + st * M::kTile + group * M::kSub + token * 128, v_dst = k_dst + M::kV - M::kK;
          if (!(ok = wait_warp(kRawFull + slot, phase))) break;
          const uint32_t raw = base + M::kRawAt + slot * M::kRun;
          const bool bad = raw_bad[slot] != 0;
          const bool in = !bad && j * kPageTokens + token < len;
          const uint32_t sw = (uint32_t)(token & 7);
          float2 mk = lds_half2(raw + 64 * D + (group * kPageTokens + token) * 4), mv = lds_half2(raw + 68 * D + (group * kPageTokens + token) * 4);
          uint4 ck[kWords / 4], cv[kWords / 4];
#pragma unroll
          for (int i = 0; i < kWords / 4; ++i) {
            const uint32_t at = raw + (D == 128 ? group * 2 + i : part) * 1024 + token * 16;
            ck[i] = lds_v4(at);
            cv[i] = lds_v4(at + 32 * D);
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(kRawEmpty + slot));
          if (++slot == kRaw) { slot = 0; phase ^= 1; }
          if (tile >= kRing && !(ok = wait_warp(kTileEmpty + st, reuse))) break;
          if (wt == 0) tile_bad[tile & 7] = bad;
          if (!in) mk = mv = make_float2(0.f, 0.f);
          const auto put = [&](uint32_t dst, const uint4 (&codes)[kWords / 4], float2 m) {
            const __half2 s = __float2half2_rn(m.x), c = __float2half2_rn(fmaf(8.f, m.x, m.y));
#pragma unroll
            for (int i = 0; i < kWords; ++i) sts_v4(dst + (((word0 + i) ^ sw) << 4), widen(in ? (&codes[i / 4].x)[i % 4] : 0x88888888u, s, c, magic));
          };
          const auto put_clipped = [&](uint32_t dst, const uint4 (&codes)[kWords / 4], float2 m) {
#pragma unroll
            for (int i = 0; i < kWords; ++i) sts_v4(dst + (((word0 + i) ^ sw) << 4), widen_clipped((&codes[i / 4].x)[i % 4], m));
          };
          const bool clip = __any_sync(0xffffffffu, beyond_fp16(mk) | beyond_fp16(mv));
          put(k_dst, ck, mk);
          put(v_dst, cv, mv);
          // (written again, not instead, and by a vote: ragged prompts 488 us without this, 492 so, 497 with a branch per thread, 512 with one around `put`)
          if (clip) {
            if (beyond_fp16(mk)) put_clipped(k_dst, ck, mk);
            if (beyond_fp16(mv)) put_clipped(v_dst, cv, mv);
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(kTileFull + st));
        }
        if (!ok) break;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
}

template <int D>
int32_t launch(essa_ctx* ctx, AttendArgs& a, cudaStream_t stream) {
  constexpr int smem = Mem<D>::kBytes + 1024;
  a.partials_at = partials_at(ctx->sm_count);
  a.whole = whole_blocks<TileList>(a, ctx->sm_count);
  cudaError_t e = allow_shared<attend_tiles_kernel<D>>(smem, ctx->device);
  if (e != cudaSuccess) return check_cuda(ctx, e, "cudaFuncSetAttribute (attend tiles)");
  attend_tiles_kernel<D><<<ctx->sm_count, kThreads, smem, stream>>>(a);
  e = cudaGetLastError();
  if (e != cudaSuccess) return check_cuda(ctx, e, "attend tiles launch");
  ++ctx->launches;
  return launch_join<TileList, D>(ctx, a, ctx->sm_count, 16, stream);
}

}  // namespace

int64_t attend_tiles_workspace(int head_dim, int sm_count) { return attend_workspace(sm_count, (int64_t)TileList::R * (head_dim + 2)); }

int32_t launch_attend_tiles(essa_ctx* ctx, AttendArgs& a, cudaStream_t stream) {
  return a.v.head_dim == 64 ? launch<64>(ctx, a, stream) : launch<128>(ctx, a, stream);
}

}  // namespace essa
