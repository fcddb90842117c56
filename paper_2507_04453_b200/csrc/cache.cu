// Paged 4-bit key / value cache: storing and reading tokens, page management, and the C entry points of include/essa.h.
#include "cache_api.cuh"
#include "cache_list.cuh"
#include "cache_store.cuh"

namespace essa {
namespace {

constexpr int kPlanThreads = 1024;

// ------------------------------------------------------------------------------------------------ tokens
// D / 16 neighbouring lanes take a token of a kv head, sixteen channels of K and of V each, kTokens tokens in turn; a thread block has
// consecutive tokens of a head, so that the pieces of neighbouring tokens (adjacent in a page) meet in one sector.  Bytes: 4 * D in
// and 1.125 * D out per (token, kv head).  32 thousand tokens of 8 heads of 128: 51 us, 3.4 TB/s; two thirds of the issue slots are taken (16
// instructions a value between conversion, comparison and packing).  Five thread blocks per SM: 51.2 us, with the registers of four 53.3; two,
// three and eight tokens per thread instead of four: 53.2 to 57.3.
template <int D, int kTokens>
__global__ void __launch_bounds__(256, 5) append_kernel(CacheView v, CacheEntries e, const __nv_bfloat16* k, int64_t ld_k, const __nv_bfloat16* val, int64_t ld_v,
                                                     int32_t* status) {
  constexpr int L = D / 16;  // lanes per token
  __shared__ int32_t offsets[kOffsetsMax];
  stage_offsets(e, offsets);
  // (heads innermost: thread blocks that run together read the whole rows of their tokens)
  const int h = (int)(blockIdx.x % (uint32_t)v.kv_heads), lane = threadIdx.x % L;
  const int64_t unit = (int64_t)(blockIdx.x / (uint32_t)v.kv_heads) * (256 / L) + threadIdx.x / L;
  int end = -1, page = -1, offset = 0;  // the tokens before `end` follow the last one located in its entry and page
#pragma unroll 1
  for (int j = 0; j < kTokens; ++j) {
    const int64_t at = unit * kTokens + j;
    const bool in = at < e.T;
    const int t = in ? (int)at : 0;
    Piece xk, xv;
    xk.raw[0] = xk.raw[1] = xv.raw[0] = xv.raw[1] = make_uint4(0, 0, 0, 0);
    if (in) {  // (before the look-up: its loads and these need not wait for one another)
      const uint4* from_k = reinterpret_cast<const uint4*>(k + t * ld_k + h * D + lane * 16);
      const uint4* from_v = reinterpret_cast<const uint4*>(val + t * ld_v + h * D + lane * 16);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        xk.raw[i] = from_k[i];
        xv.raw[i] = from_v[i];
      }
    }
    if (in && t < end) {
      ++offset;
    } else if (in) {
      page = locate_token(v, e, offsets, t, &offset, &end);
      if (page >= 0 && __ldg(v.refs + page) != 1) page = -2;  // shared (or free): not this sequence's to write
      if (page == -2) cache_fault(status);
    }
    store_token<D>(v, h, lane, in ? page : -1, offset, xk, xv);
  }
}

// 2^23 + the low four bits of w (a conversion would go through a slower unit).
__device__ __forceinline__ float raised_code(uint32_t w) { return __uint_as_float(0x4B000000u | (w & 15u)); }

// The inverse, eight channels a lane: 1.125 * D bytes in and 4 * D out.  32 thousand tokens of 8 heads of 128: 37 us, 4.7 TB/s
// (a multiplication and an addition for every value: 43).
template <int D, int kTokens>
__global__ void __launch_bounds__(256) read_kernel(CacheView v, CacheEntries e, __nv_bfloat16* k_out, __nv_bfloat16* v_out, int32_t* status) {
  constexpr int L = D / 8;
  __shared__ int32_t offsets[kOffsetsMax];
  stage_offsets(e, offsets);
  const int h = (int)(blockIdx.x % (uint32_t)v.kv_heads), lane = threadIdx.x % L;
  const int64_t unit = (int64_t)(blockIdx.x / (uint32_t)v.kv_heads) * (256 / L) + threadIdx.x / L;
  int end = -1, page = -1, offset = 0;  // the tokens before `end` follow the last one located in its entry and page
#pragma unroll 1
  for (int j = 0; j < kTokens; ++j) {
    const int64_t at = unit * kTokens + j;
    if (at >= e.T) return;
    const int t = (int)at;
    if (t < end) {
      ++offset;
    } else {
      page = locate_token(v, e, offsets, t, &offset, &end);
      if (page == -2) cache_fault(status);
    }
    if (page == -1) continue;
    const uint8_t* run = v.pages + (int64_t)max(page, 0) * v.page_bytes + (int64_t)h * 72 * D;
    const int64_t to = ((int64_t)t * v.kv_heads + h) * D + lane * 8;
    uint32_t w[2] = {0, 0};
    float2 m[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    if (page >= 0) {
      const uint32_t* code = reinterpret_cast<const uint32_t*>(run + (lane >> 2) * 1024 + offset * 16 + (lane & 3) * 4);
      const __half2* meta = reinterpret_cast<const __half2*>(run + 64 * D + ((lane >> 3) * kPageTokens + offset) * 4);
      w[0] = code[0];
      w[1] = code[8 * D];
      m[0] = __half22float2(meta[0]);
      m[1] = __half22float2(meta[D]);
      if (m[0].y != m[0].y) m[1].y = m[0].y;  // (a token that did not fit has NaN keys only)
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __nv_bfloat16* out = which ? v_out : k_out;
      if (!out) continue;
      const uint64_t scale2 = pack_f32x2(m[which].x, m[which].x), low2 = pack_f32x2(m[which].y, m[which].y), back2 = pack_f32x2(-8388608.f, -8388608.f);
      uint32_t y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // code * scale is exact in fp32 (4 bits by 11), the sum is rounded, then once more to bf16
        float a, b;
        const uint64_t codes = add_f32x2(pack_f32x2(raised_code(w[which] >> (8 * i)), raised_code(w[which] >> (8 * i + 4))), back2);
        unpack_f32x2(fma_f32x2(codes, scale2, low2), a, b);
        y[i] = pack_bf16x2(a, b);
      }
      *reinterpret_cast<uint4*>(out + to) = make_uint4(y[0], y[1], y[2], y[3]);
    }
  }
}

// ------------------------------------------------------------------------------------------------ pages
// The plan of a page operation, in the caller's workspace.
constexpr int kCheckBlocks = 60;  // thread blocks that look at the table beside compact's plan, at most
struct PlanHead {
  int32_t ok;      // 0: refused, nothing may change
  int32_t copies;  // pages to copy (from[i] -> to[i], in every layer)
  int32_t used;    // compact: pages in use
  int32_t sound[kCheckBlocks];  // compact: whether each of those thread blocks found its share of the table in order
};
static_assert(sizeof(PlanHead) <= 256, "");
struct PlanSpace {
  PlanHead* head;
  int32_t *from, *to;  // [num_pages] each
  int32_t* extra;      // [max(num_pages, max_seqs)]: fork: new last page of entry i or -1; compact: where page p goes
};
PlanSpace plan_space(void* ws, const CacheView& v) {
  PlanSpace p;
  p.head = static_cast<PlanHead*>(ws);
  p.from = reinterpret_cast<int32_t*>(static_cast<uint8_t*>(ws) + 256);
  p.to = p.from + v.num_pages;
  p.extra = p.to + v.num_pages;
  return p;
}

// The numbers of the first `want` pages with refs 0 into list (in global memory, visible to the block afterwards); false if there are fewer.
__device__ bool first_free(const CacheView& v, int want, int32_t* list, long long* scan_sm) {
  long long have = 0;
  constexpr int kPer = 4;
  for (int base = 0; base < v.num_pages && have < want; base += blockDim.x * kPer) {
    const int p0 = base + threadIdx.x * kPer;
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (p0 + i < v.num_pages && __ldcg(v.refs + p0 + i) == 0) bits |= 1u << i;
    long long total;
    long long at = have + block_scan(__popc(bits), &total, scan_sm);
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (bits >> i & 1) {
        if (at < want) list[at] = p0 + i;
        ++at;
      }
    have += total;
  }
  __syncthreads();
  return have >= want;
}

// Page copies from[i] -> to[i], i < copies, in every layer: units of THREADS (a thread block's) x 4 x 16 bytes over the whole grid.  Bound by HBM: 900
// pages of 288 KB (2 x 265 MB) take 80 us, 6.6 TB/s.
template <int THREADS>
__device__ __forceinline__ void copy_pages(const CacheView& v, const int32_t* from, const int32_t* to, int copies) {
  constexpr int kPer = 4;
  const int per_page = (int)(v.page_bytes / 16);  // 16-byte words (a multiple of 288)
  const int pieces = (per_page + THREADS * kPer - 1) / (THREADS * kPer);
  const int64_t units = (int64_t)copies * v.layers * pieces;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int piece = (int)(u % pieces);
    const int64_t rest = u / pieces;
    const int i = (int)(rest % copies), layer = (int)(rest / copies);
    uint8_t* base = v.pages + layer * v.layer_bytes;
    const uint4* src = reinterpret_cast<const uint4*>(base + from[i] * v.page_bytes);
    uint4* dst = reinterpret_cast<uint4*>(base + to[i] * v.page_bytes);
    uint4 x[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int at = (piece * kPer + j) * THREADS + threadIdx.x;
      if (at < per_page) x[j] = __ldcs(src + at);
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int at = (piece * kPer + j) * THREADS + threadIdx.x;
      if (at < per_page) __stcs(dst + at, x[j]);
    }
  }
}

// A thread per entry.  Tokens may only be written to a page of the sequence's own, so that one that ends in a shared page (it has been shortened)
// gets a copy of it.  This thread block makes the copies too: a kernel behind it would cost every decode step a launch, and copies are rare.  256
// entries by a token: 5.1 us (4.7 without a look at the pages that they end on); one that is copied in 28 layers of 4 heads of 128 (1 MB): 29, sixteen 327.
__global__ void __launch_bounds__(kPlanThreads) grow_kernel(CacheView v, const int32_t* slots, const int32_t* counts, int n, PlanSpace ws, int32_t* status) {
  extern __shared__ uint32_t seen[];
  __shared__ long long scan_sm[33];
  bool ok = slots_distinct(slots, n, v.max_seqs, seen), copies = false;
  long long want = 0, total;
  int page0 = -1, held0 = 0;  // the page that the thread's first entry ends in the middle of, and its holders
  if (ok) {
    bool fine = true;
    for (int base = 0; base < n; base += blockDim.x) {
      const int i = base + threadIdx.x;
      long long need = 0;
      int page = -1;
      if (i < n) {
        const int slot = slots ? slots[i] : i, len = v.lengths[slot], add = counts[i];
        if (len < 0 || add < 0 || (long long)len + add > (long long)v.max_pages * kPageTokens) {
          fine = false;
        } else {
          need = pages_of(len + add) - pages_of(len);
          if (add > 0 && len % kPageTokens) page = v.table[(int64_t)slot * v.max_pages + len / kPageTokens];
        }
      }
      block_scan(need, &total, scan_sm);
      want += total;
      const int held = holders(v, page);
      if (base == 0) {  // (on its way while free pages are looked for)
        page0 = page;
        held0 = held;
      } else if (i < n) {
        ws.extra[i] = held > 1 ? page : -1;
        copies |= held > 1;
      }
    }
    ok = __syncthreads_and(fine) && want <= v.num_pages && first_free(v, (int)want, ws.from, scan_sm);
  }
  copies = __syncthreads_or(ok && (copies || held0 > 1));
  if (copies) {  // pages for them, too
    long long mine = 0;
    if (threadIdx.x < n) ws.extra[threadIdx.x] = held0 > 1 ? page0 : -1;
    for (int i = threadIdx.x; i < n; i += blockDim.x) mine += ws.extra[i] >= 0;
    block_scan(mine, &total, scan_sm);
    want += total;
    ok = want <= v.num_pages && first_free(v, (int)want, ws.from, scan_sm);
  }
  if (!ok) {
    if (threadIdx.x == 0) cache_fault(status);
    return;
  }
  long long before = 0, copied = 0;
  for (int base = 0; base < n; base += blockDim.x) {
    const int i = base + threadIdx.x;
    long long need = 0;
    int slot = 0, len = 0, add = 0, old = -1;  // old: the shared page
    if (i < n) {
      slot = slots ? slots[i] : i;
      len = v.lengths[slot];
      add = counts[i];
      if (copies) old = ws.extra[i];
      need = pages_of(len + add) - pages_of(len) + (old >= 0);
    }
    long long at = before + block_scan(need, &total, scan_sm);
    before += total;
    if (copies) {
      const long long copy = copied + block_scan(old >= 0, &total, scan_sm);
      copied += total;
      if (old >= 0) {  // the first of the entry's pages
        const int page = ws.from[at];
        v.table[(int64_t)slot * v.max_pages + len / kPageTokens] = page;
        v.refs[page] = 1;
        atomicSub(v.refs + old, 1);  // (the page is free when its last holder leaves it)
        ws.extra[copy] = old;        // (copy <= i, and these threads' have been read)
        ws.to[copy] = page;
        ++at;
        --need;
      }
    }
    // A few pages each (decode steps): every thread writes its entry's.  Many (long prompts): the warp writes them, an entry after the
    // other, 32 pages at a time; a thread alone would wait for memory once a page (one sequence of 100 thousand tokens: 64 us, so 14).
    const auto give = [&](int to, int first, int64_t from, int j) {
      const int page = ws.from[from + j];
      v.table[(int64_t)to * v.max_pages + first + j] = page;
      v.refs[page] = 1;
    };
    if (__reduce_max_sync(0xffffffffu, (int)need) <= __reduce_add_sync(0xffffffffu, (int)(need + 31) / 32)) {
      for (int j = 0; j < need; ++j) give(slot, pages_of(len), at, j);
    } else {
      for (int u = 0; u < 32; ++u) {
        const int pages = __shfl_sync(0xffffffffu, (int)need, u), to = __shfl_sync(0xffffffffu, slot, u), first = __shfl_sync(0xffffffffu, pages_of(len), u);
        const long long from = __shfl_sync(0xffffffffu, at, u);
        for (int j = threadIdx.x & 31; j < pages; j += 32) give(to, first, from, j);
      }
    }
    if (i < n) v.lengths[slot] = len + add;
  }
  if (!copies) return;
  __syncthreads();
  copy_pages<kPlanThreads>(v, ws.extra, ws.to, (int)copied);
}

// The entries of n table rows that are one thread's, of `threads` threads: first, and from each to the next.
struct EntryWalk {
  int i, j;  // entry j of row i
  int rows, rest, width;
  __device__ __forceinline__ EntryWalk(const CacheView& v, int thread, int threads)
      : i(thread / v.max_pages), j(thread % v.max_pages), rows(threads / v.max_pages), rest(threads % v.max_pages), width(v.max_pages) {}
  __device__ __forceinline__ void next() {
    i += rows;
    j += rest;
    if (j >= width) {
      j -= width;
      ++i;
    }
  }
};
constexpr int kWalk = 8;  // entries of a thread whose loads are on their way together

// Whether every table entry of the n sequences slots[i] (NULL: i) is -1 or a page in use, of this thread's share of the entries.
__device__ bool rows_sound(const CacheView& v, const int32_t* slots, int n, int thread, int threads) {
  bool sound = true;
  for (EntryWalk at(v, thread, threads); at.i < n;) {
    int page[kWalk], held[kWalk];
#pragma unroll
    for (int u = 0; u < kWalk; ++u, at.next()) page[u] = at.i < n ? v.table[(int64_t)(slots ? slots[at.i] : at.i) * v.max_pages + at.j] : -1;
#pragma unroll
    for (int u = 0; u < kWalk; ++u) held[u] = holders(v, page[u]);
#pragma unroll
    for (int u = 0; u < kWalk; ++u) sound &= page[u] == -1 || held[u] > 0;
  }
  return sound;
}

// Frees the sequences, or does nothing if a slot or an entry of their table rows is bad.  One cluster, whose thread blocks look at a share of the
// entries each and tell one another before any of them changes something: thread blocks of a larger grid would need a workspace to come to one
// verdict.  Between events, with the launch: 16 rows of 32 pages 9 to 10 us, 240 rows 11 to 12, 1000 rows of 64 13, 4096 rows of 256 59 (without
// a look at the rows, in a grid of any size: 7.0, 7.1, 8.2, 13).
constexpr int kFreeCluster = 8, kFreeThreads = 1024;
__global__ void __launch_bounds__(kFreeThreads) free_kernel(CacheView v, const int32_t* slots, int n, int32_t* status) {
  extern __shared__ uint32_t seen[];
  __shared__ uint32_t verdict;
  const int blocks = gridDim.x, threads = blocks * kFreeThreads, thread = blockIdx.x * kFreeThreads + threadIdx.x;
  bool ok = slots_distinct(slots, n, v.max_seqs, seen);
  ok = __syncthreads_and(ok && rows_sound(v, slots, n, thread, threads));
  if (threadIdx.x == 0) verdict = ok;
  cluster_sync_all();
  for (int r = 0; r < blocks; ++r) ok = ok && ld_dsmem_u32(map_to_cta(smem_u32(&verdict), r)) != 0;
  cluster_sync_all();  // (every thread block comes here: one that ended before would take its shared memory with it)
  if (!ok) {
    if (thread == 0) cache_fault(status);
    return;
  }
  for (EntryWalk at(v, thread, threads); at.i < n;) {
    int32_t* entry[kWalk];
    int page[kWalk];
#pragma unroll
    for (int u = 0; u < kWalk; ++u, at.next()) {
      page[u] = -1;
      if (at.i >= n) continue;
      entry[u] = v.table + (int64_t)(slots ? slots[at.i] : at.i) * v.max_pages + at.j;
      page[u] = *entry[u];
    }
#pragma unroll
    for (int u = 0; u < kWalk; ++u)
      if (page[u] >= 0) {
        atomicSub(v.refs + page[u], 1);
        *entry[u] = -1;
      }
  }
  for (int i = thread; i < n; i += threads) v.lengths[slots ? slots[i] : i] = 0;
}

// Adds `by` to the refs of all pages of the sequences dst (warps take sequences in turn).
__device__ void count_rows(const CacheView& v, const int32_t* dst, int n, int by) {
  for (int i = threadIdx.x >> 5; i < n; i += blockDim.x >> 5) {
    const int32_t* row = v.table + (int64_t)dst[i] * v.max_pages;
    for (int j = threadIdx.x & 31; j < v.max_pages; j += 32) {
      const int page = row[j];
      if (page >= 0 && page < v.num_pages) atomicAdd(v.refs + page, by);
    }
  }
  __threadfence();
  __syncthreads();
}

__global__ void __launch_bounds__(kPlanThreads) fork_plan_kernel(CacheView v, const int32_t* src, const int32_t* dst, const int32_t* lens, int n, PlanSpace ws,
                                                                 int32_t* status) {
  grid_dep_launch();
  extern __shared__ uint32_t seen[];
  __shared__ long long scan_sm[33];
  bool ok = slots_distinct(dst, n, v.max_seqs, seen);
  long long want = 0;
  if (ok) {
    bool fine = true;
    for (int base = 0; base < n; base += blockDim.x) {
      const int i = base + threadIdx.x;
      long long need = 0, total;
      if (i < n) {
        const int s = src[i];
        if (s < 0 || s >= v.max_seqs || (seen[s >> 5] >> (s & 31) & 1)) {
          fine = false;
        } else {
          const int have = v.lengths[s], len = lens ? lens[i] : have;
          if (len < 0 || len > have || have > v.max_pages * kPageTokens) fine = false;
          else need = len % kPageTokens != 0;
        }
      }
      block_scan(need, &total, scan_sm);
      want += total;
    }
    ok = __syncthreads_and(fine);
    if (ok) {  // every page that will be shared or copied, and every one that the destinations hold, is a page in use
      for (int i = threadIdx.x >> 5; i < n; i += blockDim.x >> 5) {
        const int32_t* row = v.table + (int64_t)src[i] * v.max_pages;
        const int pages = pages_of(lens ? lens[i] : v.lengths[src[i]]);
        for (int j = threadIdx.x & 31; j < pages; j += 32) fine &= holders(v, row[j]) > 0;
      }
      fine &= rows_sound(v, dst, n, threadIdx.x, blockDim.x);
      ok = __syncthreads_and(fine) && want <= v.num_pages;
    }
  }
  if (ok) {
    count_rows(v, dst, n, -1);  // what the destinations held counts as free
    ok = first_free(v, (int)want, ws.to, scan_sm);
    if (!ok) count_rows(v, dst, n, 1);
  }
  if (threadIdx.x == 0) {
    ws.head->ok = ok;
    ws.head->copies = (int)want;
    if (!ok) cache_fault(status);
  }
  if (!ok) return;
  long long before = 0;
  for (int base = 0; base < n; base += blockDim.x) {
    const int i = base + threadIdx.x;
    long long need = 0, total;
    int len = 0, s = 0;
    if (i < n) {
      s = src[i];
      len = lens ? lens[i] : v.lengths[s];
      need = len % kPageTokens != 0;
    }
    const long long at = before + block_scan(need, &total, scan_sm);
    before += total;
    if (i < n) {
      ws.extra[i] = need ? ws.to[at] : -1;
      if (need) ws.from[at] = v.table[(int64_t)s * v.max_pages + len / kPageTokens];
    }
  }
}

__global__ void __launch_bounds__(256) fork_kernel(CacheView v, const int32_t* src, const int32_t* dst, const int32_t* lens, int n, PlanSpace ws) {
  grid_dep_wait();
  if (!ws.head->ok) return;
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const int s = src[i], d = dst[i], len = lens ? lens[i] : v.lengths[s], full = len / kPageTokens, last = ws.extra[i];
    const int32_t* from = v.table + (int64_t)s * v.max_pages;
    int32_t* to = v.table + (int64_t)d * v.max_pages;
    for (int j = threadIdx.x; j < v.max_pages; j += 256) {
      const int page = j < full ? from[j] : j == full ? last : -1;
      to[j] = page;
      if (page >= 0) atomicAdd(v.refs + page, 1);
    }
    if (threadIdx.x == 0) v.lengths[d] = len;
  }
  copy_pages<256>(v, ws.from, ws.to, ws.head->copies);
}

// Thread block 0 plans, from the counts of the pages; the others look at the table, so that the kernel behind this one can tell before it
// changes anything whether an entry names no page in use (nothing is changed here).
__global__ void __launch_bounds__(kPlanThreads) compact_plan_kernel(CacheView v, PlanSpace ws) {
  grid_dep_launch();
  if (blockIdx.x > 0) {
    const bool sound = __syncthreads_and(rows_sound(v, nullptr, v.max_seqs, (blockIdx.x - 1) * kPlanThreads + threadIdx.x, (gridDim.x - 1) * kPlanThreads));
    if (threadIdx.x == 0) ws.head->sound[blockIdx.x - 1] = sound;
    return;
  }
  __shared__ long long scan_sm[33];
  long long used = 0;
  for (int base = 0; base < v.num_pages; base += blockDim.x) {
    const int p = base + threadIdx.x;
    long long total;
    block_scan(p < v.num_pages && v.refs[p] > 0, &total, scan_sm);
    used += total;
  }
  long long holes = 0, movers = 0;
  for (int base = 0; base < v.num_pages; base += blockDim.x) {
    const int p = base + threadIdx.x;
    const bool in = p < v.num_pages, busy = in && v.refs[p] > 0;
    const bool hole = in && !busy && p < used, mover = busy && p >= used;
    long long total;
    const long long both = block_scan((hole ? 1LL << 32 : 0) + mover, &total, scan_sm);
    if (hole) ws.to[holes + (both >> 32)] = p;
    if (mover) ws.from[movers + (both & 0xffffffff)] = p;
    if (in) ws.extra[p] = p;
    holes += total >> 32;
    movers += total & 0xffffffff;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < movers; i += blockDim.x) ws.extra[ws.from[i]] = ws.to[i];
  if (threadIdx.x == 0) {
    ws.head->copies = (int)movers;
    ws.head->used = (int)used;
  }
}
__global__ void __launch_bounds__(256) compact_kernel(CacheView v, PlanSpace ws, int checks, int32_t* used_out, int32_t* status) {
  grid_dep_wait();
  if (!__syncthreads_and(threadIdx.x >= checks || ws.head->sound[threadIdx.x])) {
    if (blockIdx.x == 0 && threadIdx.x == 0) cache_fault(status);
    return;
  }
  if (used_out && blockIdx.x == 0 && threadIdx.x == 0) *used_out = ws.head->used;
  const int copies = ws.head->copies;
  if (copies == 0) return;
  const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
  for (int64_t i = first; i < copies; i += step) {
    const int from = ws.from[i], to = ws.to[i];
    v.refs[to] = v.refs[from];
    v.refs[from] = 0;
  }
  const int64_t entries = (int64_t)v.max_seqs * v.max_pages;
  for (int64_t i = first; i < entries; i += step) {
    const int page = v.table[i];
    if (page >= 0) {
      const int to = ws.extra[page];
      if (to != page) v.table[i] = to;
    }
  }
  copy_pages<256>(v, ws.from, ws.to, copies);
}

// ------------------------------------------------------------------------------------------------ host side
int64_t pages_workspace(const essa_cache_desc* c) {
  return 256 + 4 * (2 * (int64_t)c->num_pages + (c->num_pages > c->max_seqs ? c->num_pages : c->max_seqs));
}
// Which attention kernel: up to 16 query rows per (entry, kv head) take the one that widens codes straight into mma operands; with more the
// 256-row tiles of tcgen05 re-use a widened page often enough.  Few rows / tiles, us, heads of 128 channels: 32 sequences of 4096 tokens, 8 kv
// heads: 8 rows 47 / 121, 16 rows 79 / 121, 24 rows 138 / 123, 64 rows 258 / 127; one of 30000 tokens: 16 rows 30 / 39, 24 rows 39 / 39.
bool few_rows(int64_t rows) { return rows <= 16; }
size_t seen_bytes(const CacheView& v) { return (size_t)(v.max_seqs + 31) / 32 * 4; }
// Thread blocks of append and read: 256 threads, `channels` of them a thread, take `per` tokens of one head each.
int64_t token_blocks(int32_t T, const CacheView& v, int channels, int per) {
  const int64_t tokens = (int64_t)256 / (v.head_dim / channels) * per;
  return (T + tokens - 1) / tokens * v.kv_heads;
}
// Four tokens per thread share a look-up, as long as that leaves every SM four thread blocks.  32 thousand tokens of 8 heads, stored and read
// back: 124 us, with one token per thread 159 (before other steps); 256 tokens (too few for the rule): 45 us with either.
bool four_tokens(const essa_ctx* ctx, int32_t T, const CacheView& v, int channels) { return token_blocks(T, v, channels, 4) >= 4 * ctx->sm_count; }
constexpr int kAppendChannels = 16, kReadChannels = 8;
}  // namespace
}  // namespace essa

using namespace essa;

extern "C" {

int64_t essa_cache_page_bytes(int32_t kv_heads, int32_t head_dim) {
  return kv_heads < 1 || (head_dim != 64 && head_dim != 128) ? 0 : (int64_t)72 * kv_heads * head_dim;
}

int32_t essa_cache_validate(const essa_cache_desc* cache) {
  int32_t code;
  desc_problem(cache, &code);
  return code;
}

int32_t essa_cache_pages_workspace(const essa_cache_desc* cache, int64_t* bytes) {
  ESSA_TRY(essa_cache_validate(cache));
  if (!bytes) return ESSA_ERR_INVALID_ARG;
  *bytes = pages_workspace(cache);
  return ESSA_OK;
}

int32_t essa_cache_attend_workspace(const essa_cache_desc* cache, int32_t q_heads, int32_t max_new, int32_t sm_count, int64_t* bytes) {
  ESSA_TRY(essa_cache_validate(cache));
  if (!bytes || q_heads < 1 || q_heads % cache->kv_heads || max_new < 1 || sm_count < 1) return ESSA_ERR_INVALID_ARG;
  const int64_t rows = (int64_t)max_new * (q_heads / cache->kv_heads);
  *bytes = few_rows(rows) ? attend_decode_workspace(cache->head_dim, rows, sm_count) : attend_tiles_workspace(cache->head_dim, sm_count);
  return ESSA_OK;
}

int32_t essa_cache_reset(essa_ctx* ctx, const essa_cache_desc* cache, void* stream_v) {
  CacheView v;
  ESSA_TRY(view_of(ctx, "cache_reset", cache, 0, &v));
  DeviceGuard guard(ctx->device);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
  ESSA_TRY(check_cuda(ctx, cudaMemsetAsync(v.table, 0xff, (size_t)v.max_seqs * v.max_pages * 4, stream), "cache_reset"));
  ESSA_TRY(check_cuda(ctx, cudaMemsetAsync(v.lengths, 0, (size_t)v.max_seqs * 4, stream), "cache_reset"));
  return check_cuda(ctx, cudaMemsetAsync(v.refs, 0, (size_t)v.num_pages * 4, stream), "cache_reset");
}

int32_t essa_cache_grow(essa_ctx* ctx, const essa_cache_desc* cache, const int32_t* slots, const int32_t* counts, int32_t n, void* workspace,
                        int64_t workspace_bytes, void* stream) {
  CacheView v;
  ESSA_TRY(view_of(ctx, "cache_grow", cache, 0, &v));
  if (n < 0 || n > v.max_seqs) return fail(ctx, ESSA_ERR_INVALID_ARG, "cache_grow: n outside 0 .. max_seqs");
  if (n == 0) return ESSA_OK;
  if (!counts) return fail(ctx, ESSA_ERR_INVALID_ARG, "cache_grow: counts is NULL");
  ESSA_TRY(check_workspace(ctx, "cache_grow", workspace, workspace_bytes, pages_workspace(cache)));
  DeviceGuard guard(ctx->device);
  grow_kernel<<<1, kPlanThreads, seen_bytes(v), static_cast<cudaStream_t>(stream)>>>(v, slots, counts, n, plan_space(workspace, v), ctx->d_status);
  return launched(ctx, "cache_grow", 1);
}

int32_t essa_cache_append(essa_ctx* ctx, const essa_cache_desc* cache, int32_t layer, const void* k, int64_t ld_k, const void* val, int64_t ld_v, int32_t T,
                          const int32_t* slots, const int32_t* tok_offsets, int32_t n, void* stream_v) {
  CacheView v;
  ESSA_TRY(view_of(ctx, "cache_append", cache, layer, &v));
  const CacheEntries e{slots, tok_offsets, n, T};
  ESSA_TRY(check_entries(ctx, "cache_append", e));
  if (T == 0 || n == 0) return ESSA_OK;
  ESSA_TRY(check_rows(ctx, "cache_append", "k", k, ld_k, (int64_t)v.kv_heads * v.head_dim));
  ESSA_TRY(check_rows(ctx, "cache_append", "v", val, ld_v, (int64_t)v.kv_heads * v.head_dim));
  DeviceGuard guard(ctx->device);
  const bool four = four_tokens(ctx, T, v, kAppendChannels);
  const int64_t grid = token_blocks(T, v, kAppendChannels, four ? 4 : 1);
  if (grid > 0x7fffffff) return fail(ctx, ESSA_ERR_UNSUPPORTED_SHAPE, "cache_append: too many tokens");
  const auto *kk = static_cast<const __nv_bfloat16*>(k), *vv = static_cast<const __nv_bfloat16*>(val);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
  const auto run = [&](auto kernel) { kernel<<<(unsigned)grid, 256, 0, stream>>>(v, e, kk, ld_k, vv, ld_v, ctx->d_status); };
  if (v.head_dim == 64) four ? run(append_kernel<64, 4>) : run(append_kernel<64, 1>);
  else four ? run(append_kernel<128, 4>) : run(append_kernel<128, 1>);
  return launched(ctx, "cache_append", 1);
}

int32_t essa_cache_read(essa_ctx* ctx, const essa_cache_desc* cache, int32_t layer, void* k_out, void* v_out, int32_t T, const int32_t* slots,
                        const int32_t* tok_offsets, int32_t n, void* stream_v) {
  CacheView v;
  ESSA_TRY(view_of(ctx, "cache_read", cache, layer, &v));
  const CacheEntries e{slots, tok_offsets, n, T};
  ESSA_TRY(check_entries(ctx, "cache_read", e));
  if (T == 0 || n == 0 || (!k_out && !v_out)) return ESSA_OK;
  const int64_t width = (int64_t)v.kv_heads * v.head_dim;
  if (k_out) ESSA_TRY(check_rows(ctx, "cache_read", "k_out", k_out, width, width));
  if (v_out) ESSA_TRY(check_rows(ctx, "cache_read", "v_out", v_out, width, width));
  DeviceGuard guard(ctx->device);
  const bool four = four_tokens(ctx, T, v, kReadChannels);
  const int64_t grid = token_blocks(T, v, kReadChannels, four ? 4 : 1);
  if (grid > 0x7fffffff) return fail(ctx, ESSA_ERR_UNSUPPORTED_SHAPE, "cache_read: too many tokens");
  auto *kk = static_cast<__nv_bfloat16*>(k_out), *vv = static_cast<__nv_bfloat16*>(v_out);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
  const auto run = [&](auto kernel) { kernel<<<(unsigned)grid, 256, 0, stream>>>(v, e, kk, vv, ctx->d_status); };
  if (v.head_dim == 64) four ? run(read_kernel<64, 4>) : run(read_kernel<64, 1>);
  else four ? run(read_kernel<128, 4>) : run(read_kernel<128, 1>);
  return launched(ctx, "cache_read", 1);
}

int32_t essa_cache_attend(essa_ctx* ctx, const essa_cache_desc* cache, int32_t layer, const void* q, int64_t ld_q, int32_t q_heads, int32_t T,
                          const int32_t* slots, const int32_t* tok_offsets, int32_t n, int32_t max_new, float scale, void* out, int64_t ld_out,
                          void* workspace, int64_t workspace_bytes, void* stream) {
  return essa_cache_attend_masked(ctx, cache, nullptr, layer, q, ld_q, q_heads, T, slots, tok_offsets, n, max_new, scale, out, ld_out, workspace, workspace_bytes,
                                  stream);
}

int32_t essa_cache_attend_masked(essa_ctx* ctx, const essa_cache_desc* cache, const essa_attend_mask* mask, int32_t layer, const void* q, int64_t ld_q,
                                 int32_t q_heads, int32_t T, const int32_t* slots, const int32_t* tok_offsets, int32_t n, int32_t max_new, float scale, void* out,
                                 int64_t ld_out, void* workspace, int64_t workspace_bytes, void* stream) {
  CacheView v;
  ESSA_TRY(view_of(ctx, "cache_attend", cache, layer, &v));
  const CacheEntries e{slots, tok_offsets, n, T};
  ESSA_TRY(check_entries(ctx, "cache_attend", e));
  if (q_heads < 1 || q_heads % v.kv_heads) return fail(ctx, ESSA_ERR_INVALID_ARG, "cache_attend: q_heads must be a multiple of kv_heads");
  if (max_new < 1) return fail(ctx, ESSA_ERR_INVALID_ARG, "cache_attend: max_new must be at least 1");
  if (!(scale > 0.f && scale <= 0x1p127f)) return fail(ctx, ESSA_ERR_INVALID_ARG, "cache_attend: scale must be positive and at most 2^127");
  const int64_t group = q_heads / v.kv_heads;
  if (group * T > 0x7fffffff) return fail(ctx, ESSA_ERR_UNSUPPORTED_SHAPE, "cache_attend: T * (q_heads / kv_heads) must be below 2^31");
  AttendMask m{0x7fffffff, 0, nullptr, 0};
  if (mask) {
    if (mask->window < 0 || mask->sinks < 0) return fail(ctx, ESSA_ERR_INVALID_ARG, "cache_attend: negative window or sinks");
    if (mask->drafts) {
      if (reinterpret_cast<uintptr_t>(mask->drafts) & 3) return fail(ctx, ESSA_ERR_INVALID_ARG, "cache_attend: drafts must be 4-byte aligned");
      if (mask->draft_words < 1 || mask->draft_words > ESSA_CACHE_MAX_DRAFTS / 32) return fail(ctx, ESSA_ERR_UNSUPPORTED_SHAPE, "cache_attend: draft_words outside 1 .. ESSA_CACHE_MAX_DRAFTS / 32");
      if (mask->window && mask->window < 32 * mask->draft_words) return fail(ctx, ESSA_ERR_UNSUPPORTED_SHAPE, "cache_attend: with drafts, the window must be at least 32 * draft_words");
      m.drafts = mask->drafts;
      m.words = mask->draft_words;
    }
    if (mask->window) {
      m.window = mask->window;
      m.sinks = mask->sinks < v.max_pages * kPageTokens ? mask->sinks : v.max_pages * kPageTokens;  // (first tokens are always seen without a window)
    }
  }
  if (T == 0 || n == 0) return ESSA_OK;
  ESSA_TRY(check_rows(ctx, "cache_attend", "q", q, ld_q, (int64_t)q_heads * v.head_dim));
  ESSA_TRY(check_rows(ctx, "cache_attend", "out", out, ld_out, (int64_t)q_heads * v.head_dim));
  int64_t need;
  ESSA_TRY(essa_cache_attend_workspace(cache, q_heads, max_new, ctx->sm_count, &need));
  ESSA_TRY(check_workspace(ctx, "cache_attend", workspace, workspace_bytes, need));
  DeviceGuard guard(ctx->device);
  AttendArgs a;
  a.v = v;
  a.e = e;
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.out = static_cast<__nv_bfloat16*>(out);
  a.ld_q = ld_q;
  a.ld_out = ld_out;
  a.group = (int32_t)group;
  a.by_group = Divisor::of((uint32_t)group);
  a.scale = scale * 1.4426950408889634f;
  a.ws = static_cast<float*>(workspace);
  a.status = ctx->d_status;
  a.m = m;
  a.masked = m.window != 0x7fffffff || m.drafts;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return few_rows(max_new * group) ? launch_attend_decode(ctx, a, max_new * group, s) : launch_attend_tiles(ctx, a, s);
}

int32_t essa_cache_fork(essa_ctx* ctx, const essa_cache_desc* cache, const int32_t* src, const int32_t* dst, const int32_t* lens, int32_t n, void* workspace,
                        int64_t workspace_bytes, void* stream_v) {
  CacheView v;
  ESSA_TRY(view_of(ctx, "cache_fork", cache, 0, &v));
  if (n < 0 || n > v.max_seqs) return fail(ctx, ESSA_ERR_INVALID_ARG, "cache_fork: n outside 0 .. max_seqs");
  if (n == 0) return ESSA_OK;
  if (!src || !dst) return fail(ctx, ESSA_ERR_INVALID_ARG, "cache_fork: src or dst is NULL");
  ESSA_TRY(check_workspace(ctx, "cache_fork", workspace, workspace_bytes, pages_workspace(cache)));
  DeviceGuard guard(ctx->device);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
  const PlanSpace ws = plan_space(workspace, v);
  fork_plan_kernel<<<1, kPlanThreads, seen_bytes(v), stream>>>(v, src, dst, lens, n, ws, ctx->d_status);
  ESSA_TRY(launched(ctx, "cache_fork", 1));
  ++ctx->launches;
  return check_cuda(ctx, launch_behind_plan(stream, dim3(ctx->sm_count * 8), fork_kernel, v, src, dst, lens, (int)n, ws), "cache_fork");
}

int32_t essa_cache_free(essa_ctx* ctx, const essa_cache_desc* cache, const int32_t* slots, int32_t n, void* stream) {
  CacheView v;
  ESSA_TRY(view_of(ctx, "cache_free", cache, 0, &v));
  if (n < 0 || n > v.max_seqs) return fail(ctx, ESSA_ERR_INVALID_ARG, "cache_free: n outside 0 .. max_seqs");
  if (n == 0) return ESSA_OK;
  DeviceGuard guard(ctx->device);
  // a thread for every four entries, up to a cluster of the portable size
  int blocks = 1;
  while (blocks < kFreeCluster && (int64_t)n * v.max_pages > (int64_t)blocks * kFreeThreads * 4) blocks *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(kFreeThreads);
  cfg.dynamicSmemBytes = seen_bytes(v);
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = blocks;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  ++ctx->launches;
  return check_cuda(ctx, cudaLaunchKernelEx(&cfg, free_kernel, v, slots, (int)n, ctx->d_status), "cache_free");
}

int32_t essa_cache_compact(essa_ctx* ctx, const essa_cache_desc* cache, int32_t* used, void* workspace, int64_t workspace_bytes, void* stream_v) {
  CacheView v;
  ESSA_TRY(view_of(ctx, "cache_compact", cache, 0, &v));
  ESSA_TRY(check_workspace(ctx, "cache_compact", workspace, workspace_bytes, pages_workspace(cache)));
  DeviceGuard guard(ctx->device);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
  const PlanSpace ws = plan_space(workspace, v);
  // four entries of the table for a thread, up to kCheckBlocks thread blocks
  const int64_t want = ((int64_t)v.max_seqs * v.max_pages + 4 * kPlanThreads - 1) / (4 * kPlanThreads);
  const int checks = want < kCheckBlocks ? (int)want : kCheckBlocks;
  compact_plan_kernel<<<1 + checks, kPlanThreads, 0, stream>>>(v, ws);
  ESSA_TRY(launched(ctx, "cache_compact", 1));
  ++ctx->launches;
  return check_cuda(ctx, launch_behind_plan(stream, dim3(ctx->sm_count * 8), compact_kernel, v, ws, checks, used, ctx->d_status), "cache_compact");
}

}  // extern "C"
