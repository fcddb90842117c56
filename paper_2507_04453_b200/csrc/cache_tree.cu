// Trees of drafted tokens: the bits that say which drafts a draft sees and the drafts' positions, made from their parents, and keeping the
// accepted path of a tree in the paged 4-bit cache.
#include "cache_api.cuh"
#include "cache_store.cuh"

namespace essa {
namespace {

// ------------------------------------------------------------------------------------------------ ancestors
// A thread block per entry, a thread per draft, which climbs from parent to parent in shared memory: as many steps as it is deep (a dozen in the
// trees that are drafted, 255 at most).  Bound by latency: 3 us for 64 trees of up to 26 drafts.
constexpr int kMaxDrafts = ESSA_CACHE_MAX_DRAFTS;
__global__ void __launch_bounds__(kMaxDrafts) tree_kernel(CacheView v, CacheEntries e, const int32_t* parents, uint32_t* drafts, int words, int32_t* positions, int32_t* status) {
  __shared__ int16_t parent[kMaxDrafts];
  __shared__ uint32_t bits[kMaxDrafts * (kMaxDrafts / 32 + 1)];  // (a word more per row: the rows' words in different banks)
  const EntryInfo info = load_entry(v, e, blockIdx.x);
  const int rows = min(info.rows, 32 * words), j = threadIdx.x, past = info.len - info.rows;
  bool fault = (info.slot < 0 && info.rows > 0) || info.rows > rows;  // (an entry without rows stands for nothing)
  if (j < rows) {
    const int up = __ldg(parents + info.row0 + j);
    const bool fine = up >= -1 && up < j;
    parent[j] = fine ? (int16_t)up : (int16_t)-1;
    fault |= !fine;
  }
  if (fault) cache_fault(status);
  __syncthreads();
  if (j < rows) {
    uint32_t* mine = bits + j * (kMaxDrafts / 32 + 1);
    for (int w = 0; w < words; ++w) mine[w] = 0;
    int depth = -1;
    for (int at = j; at >= 0; at = parent[at], ++depth) mine[at >> 5] |= 1u << (at & 31);
    if (positions && info.slot >= 0) positions[info.row0 + j] = past + depth;
  }
  __syncthreads();
  uint32_t* out = drafts + (int64_t)info.row0 * words;
  for (int i = threadIdx.x; i < rows * words; i += blockDim.x) out[i] = bits[i / words * (kMaxDrafts / 32 + 1) + i % words];
  for (int64_t i = (int64_t)rows * words + threadIdx.x; i < (int64_t)info.rows * words; i += blockDim.x) out[i] = 0;
  if (positions && info.slot >= 0)
    for (int i = rows + threadIdx.x; i < info.rows; i += blockDim.x) positions[info.row0 + i] = past;
}

// ------------------------------------------------------------------------------------------------ the accepted path
constexpr int kKeepPages = kMaxDrafts / kPageTokens + 1;  // pages that kMaxDrafts tokens can lie on
struct KeepEntry {
  int32_t offset, count;      // of the first of the last tokens in its page; tokens that stay
  int32_t pages[kKeepPages];  // from that page on
  int32_t moves;              // whether any of them moves
};
static_assert(sizeof(KeepEntry) == 32, "");
struct KeepHead {
  int32_t ok;
};
constexpr int kKeepThreads = 1024;

// Checks everything, then writes down where the tokens are that move, and takes the sequences' ends away.  A thread per entry: a few pages each after trees;
// an end of 100 thousand tokens, a load, a check and an atomic per page in turn, takes it 260 us.
__global__ void __launch_bounds__(kKeepThreads) keep_plan_kernel(CacheView v, const int32_t* slots, const int32_t* off, const int32_t* counts, const int32_t* picks,
                                                                 int64_t ld_picks, int n, KeepHead* head, KeepEntry* entries, int32_t* status) {
  grid_dep_launch();
  extern __shared__ uint32_t seen[];
  bool ok = slots_distinct(slots, n, v.max_seqs, seen);
  if (ok) {
    bool fine = true;
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
      const int slot = slots ? slots[i] : i, len = v.lengths[slot], stay = counts[i];
      const long long rows = off ? (long long)off[i + 1] - off[i] : 1;
      if (len < 0 || len > v.max_pages * kPageTokens || rows < 0 || rows > len || stay < 0 || stay > rows || (picks && (rows > kMaxDrafts || stay > ld_picks))) {
        fine = false;
        continue;
      }
      const int base = len - (int)rows, first = base / kPageTokens;
      KeepEntry k = {};
      k.offset = base % kPageTokens;
      k.count = stay;
      int least = stay;  // the first that moves
      if (picks) {
        const int32_t* mine = picks + i * ld_picks;
        int before = -1;
        for (int m = 0; m < stay; ++m) {
          const int p = mine[m];
          fine &= p > before && p < rows;
          before = p;
          if (p != m && least == stay) least = m;
        }
        k.moves = least < stay;
      }
      const int32_t* row = v.table + (int64_t)slot * v.max_pages;
      for (int j = first; j < pages_of(len); ++j) {
        const int page = row[j], held = holders(v, page);
        fine &= held > 0;
        // (the tokens least .. stay - 1 are written)
        if (least < stay && j >= (base + least) / kPageTokens && j <= (base + stay - 1) / kPageTokens) fine &= held == 1;
        if (k.moves) {
#pragma unroll
          for (int u = 0; u < kKeepPages; ++u)
            if (j - first == u) k.pages[u] = page;
        }
      }
      entries[i] = k;
    }
    ok = __syncthreads_and(fine);
  }
  if (threadIdx.x == 0) {
    head->ok = ok;
    if (!ok) cache_fault(status);
  }
  if (!ok) return;
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int slot = slots ? slots[i] : i, len = v.lengths[slot], rows = off ? off[i + 1] - off[i] : 1, now = len - rows + counts[i];
    int32_t* row = v.table + (int64_t)slot * v.max_pages;
    for (int j = pages_of(now); j < pages_of(len); ++j) {
      atomicSub(v.refs + row[j], 1);
      row[j] = -1;
    }
    v.lengths[slot] = now;
  }
}

// A thread block has an entry and a share of the layers (blockIdx.y of gridDim.y); a thread takes one piece (sixteen bytes of codes, or a scale and a minimum) of the
// tokens in one layer and kv head after the other, and walks the tokens that stay.  A token moves forward or not at all, and ascending: eight are read before they are
// written, and what is read later lies behind all that has been written.  Bytes: the tokens that move, in and out; pieces of 16 bytes take half of a sector each.  128 entries of 28 layers and 4 kv heads, three of some 40
// tokens each: 12 us under ncu (28 MB read for 7), 17 with the plan before it.
template <int D>
__global__ void __launch_bounds__(256) keep_move_kernel(CacheView v, const int32_t* picks, int64_t ld_picks, const KeepHead* head, const KeepEntry* entries) {
  constexpr int kCodes = 2 * (D / 32), kPieces = kCodes + 2 * (D / 64);
  __shared__ KeepEntry k;
  __shared__ int32_t mine[kMaxDrafts];
  grid_dep_wait();
  if (!head->ok) return;
  const int i = blockIdx.x, tid = threadIdx.x;
  if (tid < (int)(sizeof(KeepEntry) / 4)) reinterpret_cast<int32_t*>(&k)[tid] = reinterpret_cast<const int32_t*>(entries + i)[tid];
  __syncthreads();
  if (!k.moves) return;
  const int offset = k.offset, count = k.count;
  if (tid < count) mine[tid] = picks[i * ld_picks + tid];
  __syncthreads();
  const int per_layer = v.kv_heads * kPieces, first = (int)((int64_t)v.layers * blockIdx.y / gridDim.y), layers = (int)((int64_t)v.layers * (blockIdx.y + 1) / gridDim.y) - first;
  for (int64_t u = tid; u < (int64_t)layers * per_layer; u += 256) {
    const int layer = first + (int)(u / per_layer), rest = (int)(u % per_layer), h = rest / kPieces, piece = rest % kPieces;
    const bool wide = piece < kCodes;
    uint8_t* base = v.pages + layer * v.layer_bytes + (int64_t)h * 72 * D + (wide ? piece * 1024 : 64 * D + (piece - kCodes) * 256);
    const auto at = [&](int token) {
      const int place = offset + token;
      return base + k.pages[place / kPageTokens] * v.page_bytes + place % kPageTokens * (wide ? 16 : 4);
    };
    for (int m0 = 0; m0 < count; m0 += 8) {
      uint4 x[8];
      int from[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) from[j] = m0 + j < count ? mine[m0 + j] : m0 + j;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (from[j] == m0 + j) continue;
        const uint8_t* p = at(from[j]);
        if (wide) x[j] = *reinterpret_cast<const uint4*>(p);
        else x[j].x = *reinterpret_cast<const uint32_t*>(p);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (from[j] == m0 + j) continue;
        uint8_t* p = at(m0 + j);
        if (wide) *reinterpret_cast<uint4*>(p) = x[j];
        else *reinterpret_cast<uint32_t*>(p) = x[j].x;
      }
    }
  }
}

int64_t keep_workspace(int64_t n) { return 256 + n * (int64_t)sizeof(KeepEntry); }

}  // namespace
}  // namespace essa

using namespace essa;

extern "C" {

int32_t essa_cache_tree(essa_ctx* ctx, const essa_cache_desc* cache, const int32_t* parents, int32_t T, const int32_t* slots, const int32_t* tok_offsets, int32_t n,
                        uint32_t* drafts, int32_t draft_words, int32_t* positions, void* stream) {
  CacheView v;
  ESSA_TRY(view_of(ctx, "cache_tree", cache, 0, &v));
  const CacheEntries e{slots, tok_offsets, n, T};
  ESSA_TRY(check_entries(ctx, "cache_tree", e));
  if (draft_words < 1 || draft_words > kMaxDrafts / 32) return fail(ctx, ESSA_ERR_UNSUPPORTED_SHAPE, "cache_tree: draft_words outside 1 .. ESSA_CACHE_MAX_DRAFTS / 32");
  if (T == 0 || n == 0) return ESSA_OK;
  if (!parents || !drafts) return fail(ctx, ESSA_ERR_INVALID_ARG, "cache_tree: parents or drafts is NULL");
  if ((reinterpret_cast<uintptr_t>(parents) | reinterpret_cast<uintptr_t>(drafts) | reinterpret_cast<uintptr_t>(positions)) & 3)
    return fail(ctx, ESSA_ERR_INVALID_ARG, "cache_tree: parents, drafts and positions must be 4-byte aligned");
  DeviceGuard guard(ctx->device);
  tree_kernel<<<n, 32 * draft_words, 0, static_cast<cudaStream_t>(stream)>>>(v, e, parents, drafts, draft_words, positions, ctx->d_status);
  return launched(ctx, "cache_tree", 1);
}

int32_t essa_cache_keep_workspace(int32_t n, int64_t* bytes) {
  if (!bytes || n < 0) return ESSA_ERR_INVALID_ARG;
  *bytes = keep_workspace(n);
  return ESSA_OK;
}

int32_t essa_cache_keep(essa_ctx* ctx, const essa_cache_desc* cache, const int32_t* slots, const int32_t* tok_offsets, const int32_t* counts, const int32_t* picks,
                        int64_t ld_picks, int32_t n, void* workspace, int64_t workspace_bytes, void* stream_v) {
  CacheView v;
  ESSA_TRY(view_of(ctx, "cache_keep", cache, 0, &v));
  if (n < 0 || n > v.max_seqs) return fail(ctx, ESSA_ERR_INVALID_ARG, "cache_keep: n outside 0 .. max_seqs");
  if (n == 0) return ESSA_OK;
  if (!counts) return fail(ctx, ESSA_ERR_INVALID_ARG, "cache_keep: counts is NULL");
  if (picks && ld_picks < 0) return fail(ctx, ESSA_ERR_INVALID_ARG, "cache_keep: the pitch of picks is negative");
  ESSA_TRY(check_workspace(ctx, "cache_keep", workspace, workspace_bytes, keep_workspace(n)));
  DeviceGuard guard(ctx->device);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
  KeepHead* head = static_cast<KeepHead*>(workspace);
  KeepEntry* entries = reinterpret_cast<KeepEntry*>(static_cast<uint8_t*>(workspace) + 256);
  keep_plan_kernel<<<1, kKeepThreads, (size_t)(v.max_seqs + 31) / 32 * 4, stream>>>(v, slots, tok_offsets, counts, picks, ld_picks, n, head, entries, ctx->d_status);
  ESSA_TRY(launched(ctx, "cache_keep", 1));
  if (!picks) return ESSA_OK;  // (nothing moves)
  ++ctx->launches;
  // eight thread blocks per SM, or one for every layer of every entry
  const int64_t want = (8 * (int64_t)ctx->sm_count + n - 1) / n;
  const dim3 grid(n, (unsigned)(want < v.layers ? want : v.layers));
  const auto move = v.head_dim == 64 ? keep_move_kernel<64> : keep_move_kernel<128>;
  return check_cuda(ctx, launch_behind_plan(stream, grid, move, v, picks, ld_picks, (const KeepHead*)head, (const KeepEntry*)entries), "cache_keep");
}

}  // extern "C"
