// Host side of the cache's C entry points: the checks of their arguments, and how a kernel is launched behind the one that plans for it.
#pragma once

#include "cache.cuh"

namespace essa {

// The context's device is made current for the length of a call (the caller's is put back).
class DeviceGuard {
 public:
  explicit DeviceGuard(int device) {
    if (cudaGetDevice(&before_) != cudaSuccess) before_ = device;
    if (before_ != device) cudaSetDevice(device);
    device_ = device;
  }
  ~DeviceGuard() {
    if (before_ != device_) cudaSetDevice(before_);
  }
  DeviceGuard(const DeviceGuard&) = delete;

 private:
  int before_ = 0, device_ = 0;
};

inline const char* desc_problem(const essa_cache_desc* c, int32_t* code) {
  *code = ESSA_ERR_INVALID_ARG;
  if (!c) return "NULL descriptor";
  if (c->layers < 1 || c->num_pages < 1 || c->kv_heads < 1 || c->max_seqs < 1 || c->max_pages < 1) return "sizes must be positive";
  if (!c->pages || !c->table || !c->lengths || !c->refs) return "NULL buffer in the descriptor";
  if (reinterpret_cast<uintptr_t>(c->pages) & 15) return "pages must be 16-byte aligned";
  if ((reinterpret_cast<uintptr_t>(c->table) | reinterpret_cast<uintptr_t>(c->lengths) | reinterpret_cast<uintptr_t>(c->refs)) & 3) return "table, lengths and refs must be 4-byte aligned";
  *code = ESSA_ERR_UNSUPPORTED_SHAPE;
  if (c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 64 or 128";
  if (c->max_seqs > ESSA_CACHE_MAX_SEQS) return "max_seqs > ESSA_CACHE_MAX_SEQS";
  if (c->max_pages > 0x7fffffff / ESSA_CACHE_PAGE_TOKENS) return "max_pages * 64 must be below 2^31";
  if (c->kv_heads > 4096) return "kv_heads > 4096";
  *code = ESSA_OK;
  return nullptr;
}

inline int32_t view_of(essa_ctx* ctx, const char* what, const essa_cache_desc* c, int32_t layer, CacheView* v) {
  if (!ctx) return ESSA_ERR_INVALID_ARG;
  int32_t code;
  if (const char* why = desc_problem(c, &code)) return fail(ctx, code, std::string(what) + ": " + why);
  if (layer < 0 || layer >= c->layers) return fail(ctx, ESSA_ERR_INVALID_ARG, std::string(what) + ": layer outside the cache");
  v->page_bytes = essa_cache_page_bytes(c->kv_heads, c->head_dim);
  v->layer_bytes = v->page_bytes * c->num_pages;
  v->pages = static_cast<uint8_t*>(c->pages) + layer * v->layer_bytes;
  v->table = c->table;
  v->lengths = c->lengths;
  v->refs = c->refs;
  v->num_pages = c->num_pages;
  v->kv_heads = c->kv_heads;
  v->head_dim = c->head_dim;
  v->max_seqs = c->max_seqs;
  v->max_pages = c->max_pages;
  v->layers = c->layers;
  return ESSA_OK;
}

inline int32_t check_entries(essa_ctx* ctx, const char* what, const CacheEntries& e) {
  if (e.n < 0 || e.T < 0) return fail(ctx, ESSA_ERR_INVALID_ARG, std::string(what) + ": negative n or T");
  if (!e.off && e.n != e.T) return fail(ctx, ESSA_ERR_INVALID_ARG, std::string(what) + ": without tok_offsets every entry has one row (n = T)");
  return ESSA_OK;
}
// A token-major bf16 buffer of `width` elements per row.
inline int32_t check_rows(essa_ctx* ctx, const char* what, const char* name, const void* p, int64_t ld, int64_t width) {
  if (!p) return fail(ctx, ESSA_ERR_INVALID_ARG, std::string(what) + ": " + name + " is NULL");
  if (reinterpret_cast<uintptr_t>(p) & 15) return fail(ctx, ESSA_ERR_INVALID_ARG, std::string(what) + ": " + name + " must be 16-byte aligned");
  if (ld < width || ld % 8) return fail(ctx, ESSA_ERR_INVALID_ARG, std::string(what) + ": the row pitch of " + name + " must be a multiple of 8 elements and hold a row");
  return ESSA_OK;
}
inline int32_t check_workspace(essa_ctx* ctx, const char* what, const void* ws, int64_t bytes, int64_t need) {
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 15)) return fail(ctx, ESSA_ERR_INVALID_ARG, std::string(what) + ": the workspace must be a 16-byte aligned device buffer");
  if (bytes < need) return fail(ctx, ESSA_ERR_INVALID_ARG, std::string(what) + ": the workspace is too small");
  return ESSA_OK;
}
inline int32_t launched(essa_ctx* ctx, const char* what, int kernels) {
  ctx->launches += kernels;
  return check_cuda(ctx, cudaGetLastError(), what);
}

// The kernel behind a plan: its thread blocks are on their SMs when the plan is ready (they wait for the end of the plan's launch).
template <class... Args>
cudaError_t launch_behind_plan(cudaStream_t stream, dim3 grid, void (*kernel)(Args...), Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(256);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace essa

#define ESSA_TRY(call)                     \
  do {                                     \
    const int32_t st_ = (call);            \
    if (st_ != ESSA_OK) return st_;        \
  } while (0)
