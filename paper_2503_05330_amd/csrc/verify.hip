// csd — host side of the verifying pass's cache and attention (csd_verify.h): argument checks, workspace layout, the shape of
// a launch.
#include <cmath>
#include <new>

#include "csd_launch.h"
#include "csd_verify.cuh"

namespace csd {
namespace verify {
namespace {

constexpr int64_t kWorkspaceAlign = 256;
int64_t aligned_up(int64_t x) { return (x + kWorkspaceAlign - 1) / kWorkspaceAlign * kWorkspaceAlign; }

struct CacheLayout {
  int64_t prompt_keys, prompt_values, path_keys, path_values, prompt_scale, path_scale, part_o, part_lse, status, total;
  int64_t prompt_layer, path_layer;      // blocks of a layer
};

int check(const csd_cache_config* c) {
  if (!c || c->n_problems <= 0 || c->n_paths <= 0 || (int64_t)c->n_problems * c->n_paths > (1 << 24)) return CSD_ERR_INVALID_ARG;
  if (c->prompt_cap < 0 || c->prompt_cap > CSD_MAX_CACHE_TOKENS || c->path_cap <= 0 || c->path_cap > CSD_MAX_CACHE_TOKENS) return CSD_ERR_INVALID_ARG;
  if (c->n_layers <= 0 || c->n_layers > CSD_MAX_LAYERS || c->n_kv_heads <= 0 || c->n_heads <= 0 || c->n_heads > CSD_MAX_HEADS || c->n_heads % c->n_kv_heads) return CSD_ERR_INVALID_ARG;
  if (c->max_step < 1 || c->max_step > CSD_MAX_VERIFY_STEP) return CSD_ERR_INVALID_ARG;
  if (c->type != CSD_BF16 && c->type != CSD_F16) return CSD_ERR_INVALID_ARG;
  if (c->fp8 != 0 && c->fp8 != 1) return CSD_ERR_INVALID_ARG;
  const int64_t row_tiles = ((int64_t)c->max_step * (c->n_heads / c->n_kv_heads) + 31) / 32;
  if ((int64_t)c->n_problems * c->n_paths * c->n_kv_heads * row_tiles > CSD_MAX_ROW_TILES) return CSD_ERR_INVALID_ARG;
  if (c->head_dim <= 0) return CSD_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128 && c->head_dim != 256) return CSD_ERR_UNIMPLEMENTED;
  return CSD_OK;
}

// false: too large for an address
bool layout_of(const csd_cache_config* c, CacheLayout* l) {
  const double bytes = (double)c->n_layers * c->n_problems * c->n_kv_heads * 2.0 * block_bytes(c->head_dim, c->fp8) *
                       ((c->prompt_cap + kBlock - 1) / kBlock + (double)c->n_paths * ((c->path_cap + kBlock - 1) / kBlock));
  if (bytes > 1e15) return false;
  const int64_t per_block = block_bytes(c->head_dim, c->fp8);
  l->prompt_layer = (int64_t)c->n_problems * c->n_kv_heads * ((c->prompt_cap + kBlock - 1) / kBlock);
  l->path_layer = (int64_t)c->n_problems * c->n_paths * c->n_kv_heads * ((c->path_cap + kBlock - 1) / kBlock);
  const int64_t rows = (int64_t)c->n_problems * c->n_paths * c->max_step * c->n_heads;
  const int64_t parts = parts_of_rows(rows, c->prompt_cap, c->path_cap);
  int64_t at = 0;
  auto take = [&](int64_t* place, int64_t size) {
    *place = at;
    at += aligned_up(size);
  };
  take(&l->prompt_keys, c->n_layers * l->prompt_layer * per_block);
  take(&l->prompt_values, c->n_layers * l->prompt_layer * per_block);
  take(&l->path_keys, c->n_layers * l->path_layer * per_block);
  take(&l->path_values, c->n_layers * l->path_layer * per_block);
  take(&l->prompt_scale, c->fp8 ? c->n_layers * l->prompt_layer * kScaleBytes : 0);
  take(&l->path_scale, c->fp8 ? c->n_layers * l->path_layer * kScaleBytes : 0);
  take(&l->part_o, parts * c->head_dim * 4);
  take(&l->part_lse, parts * 4);
  take(&l->status, 4);
  l->total = at;
  return true;
}

__global__ void clear_kernel(uint32_t* word) { *word = 0; }

bool misaligned(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 != 0; }
int check_heads(const csd_heads* x) {
  if (!x || !x->data || misaligned(x->data) || x->row_stride < 0 || x->token_stride < 0 || x->head_stride < 0 ||
      x->row_stride % 8 || x->token_stride % 8 || x->head_stride % 8)
    return CSD_ERR_INVALID_ARG;
  return CSD_OK;
}

}  // namespace
}  // namespace verify
}  // namespace csd

struct csd_cache {
  csd_cache_config cfg;
  csd::verify::CacheLayout layout;
  uint8_t* base;

  csd::verify::Held held(bool prompt, int32_t layer) const {
    using namespace csd::verify;
    const int64_t first = layer * (prompt ? layout.prompt_layer : layout.path_layer), at = first * block_bytes(cfg.head_dim, cfg.fp8);
    const int32_t cap = prompt ? cfg.prompt_cap : cfg.path_cap;
    return Held{base + (prompt ? layout.prompt_keys : layout.path_keys) + at, base + (prompt ? layout.prompt_values : layout.path_values) + at,
                cfg.fp8 ? base + (prompt ? layout.prompt_scale : layout.path_scale) + first * kScaleBytes : nullptr, cap,
                (cap + kBlock - 1) / kBlock};
  }
  uint32_t* status() const { return reinterpret_cast<uint32_t*>(base + layout.status); }
};

namespace csd {
namespace verify {
namespace {

int finish(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CSD_OK : hip_fail(e, what);
}

int move(csd_cache* c, bool read, bool prompt, int32_t layer, const csd_heads& k, const csd_heads& v, const int32_t* start,
         const int32_t* counts, int32_t n, void* stream) {
  MoveArgs a;
  a.held = c->held(prompt, layer);
  a.k = k;
  a.v = v;
  a.start = start;
  a.counts = counts;
  a.rows = prompt ? c->cfg.n_problems : (int64_t)c->cfg.n_problems * c->cfg.n_paths;
  a.n = n;
  a.Hk = c->cfg.n_kv_heads;
  a.groups = (n + 7) / 8;
  a.status = c->status();
  if (read) cache_read(a, c->cfg.head_dim, c->cfg.type == CSD_F16, c->cfg.fp8, static_cast<hipStream_t>(stream));
  else cache_write(a, c->cfg.head_dim, c->cfg.type == CSD_F16, c->cfg.fp8, static_cast<hipStream_t>(stream));
  return finish(read ? "csd_cache_read" : "csd_cache_write");
}

int check_move(const csd_cache* c, int32_t layer, int32_t n) {
  if (!c || layer < 0 || layer >= c->cfg.n_layers || n <= 0 || n > CSD_MAX_CACHE_TOKENS) return CSD_ERR_INVALID_ARG;
  return CSD_OK;
}
int write(csd_cache* c, bool prompt, int32_t layer, const csd_heads* k, const csd_heads* v, const int32_t* start, const int32_t* counts,
          int32_t n, void* stream) {
  if (check_move(c, layer, n) != CSD_OK || check_heads(k) != CSD_OK || check_heads(v) != CSD_OK) return CSD_ERR_INVALID_ARG;
  return move(c, false, prompt, layer, *k, *v, start, counts, n, stream);
}
int read(csd_cache* c, bool prompt, int32_t layer, const int32_t* start, const int32_t* counts, int32_t n, void* d_k, void* d_v, void* stream) {
  if (check_move(c, layer, n) != CSD_OK || !d_k || !d_v || misaligned(d_k) || misaligned(d_v)) return CSD_ERR_INVALID_ARG;
  const int64_t D = c->cfg.head_dim, token = D * c->cfg.n_kv_heads;
  return move(c, true, prompt, layer, csd_heads{d_k, n * token, token, D}, csd_heads{d_v, n * token, token, D}, start, counts, n, stream);
}

}  // namespace
}  // namespace verify
}  // namespace csd

extern "C" {

int csd_cache_bytes(const csd_cache_config* cfg, size_t* out_bytes) {
  using namespace csd::verify;
  if (!out_bytes) return CSD_ERR_INVALID_ARG;
  const int rc = check(cfg);
  if (rc != CSD_OK) return rc;
  CacheLayout l;
  if (!layout_of(cfg, &l)) return CSD_ERR_INVALID_ARG;
  *out_bytes = (size_t)l.total;
  return CSD_OK;
}

int csd_cache_create(const csd_cache_config* cfg, void* d_workspace, size_t workspace_bytes, void* stream, csd_cache** out_cache) {
  using namespace csd::verify;
  if (!out_cache) return CSD_ERR_INVALID_ARG;
  *out_cache = nullptr;
  const int rc = check(cfg);
  if (rc != CSD_OK) return rc;
  CacheLayout l;
  if (!d_workspace || !layout_of(cfg, &l)) return CSD_ERR_INVALID_ARG;
  if (workspace_bytes < (size_t)l.total || reinterpret_cast<uintptr_t>(d_workspace) % kWorkspaceAlign) return CSD_ERR_WORKSPACE;
  csd_cache* c = new (std::nothrow) csd_cache{*cfg, l, static_cast<uint8_t*>(d_workspace)};
  if (!c) return CSD_ERR_INVALID_ARG;
  clear_kernel<<<1, 1, 0, static_cast<hipStream_t>(stream)>>>(c->status());
  const int done = finish("csd_cache_create");
  if (done != CSD_OK) {
    delete c;
    return done;
  }
  *out_cache = c;
  return CSD_OK;
}

int csd_cache_destroy(csd_cache* cache) {
  if (!cache) return CSD_ERR_INVALID_ARG;
  delete cache;
  return CSD_OK;
}

int csd_cache_write(csd_cache* cache, int32_t layer, const csd_heads* k, const csd_heads* v, const int32_t* d_start,
                    const int32_t* d_counts, int32_t n, void* stream) {
  return csd::verify::write(cache, false, layer, k, v, d_start, d_counts, n, stream);
}
int csd_cache_write_prompt(csd_cache* cache, int32_t layer, const csd_heads* k, const csd_heads* v, const int32_t* d_start,
                           const int32_t* d_counts, int32_t n, void* stream) {
  return csd::verify::write(cache, true, layer, k, v, d_start, d_counts, n, stream);
}
int csd_cache_read(csd_cache* cache, int32_t layer, const int32_t* d_start, const int32_t* d_counts, int32_t n, void* d_k, void* d_v,
                   void* stream) {
  return csd::verify::read(cache, false, layer, d_start, d_counts, n, d_k, d_v, stream);
}
int csd_cache_read_prompt(csd_cache* cache, int32_t layer, const int32_t* d_start, const int32_t* d_counts, int32_t n, void* d_k,
                          void* d_v, void* stream) {
  return csd::verify::read(cache, true, layer, d_start, d_counts, n, d_k, d_v, stream);
}

int csd_attend(csd_cache* cache, int32_t layer, const csd_heads* q, const int32_t* d_prompt_len, const int32_t* d_path_len,
               const int32_t* d_counts, int32_t n, float scale, int32_t prompt_bound, int32_t path_bound, void* d_out, float* d_lse,
               void* stream) {
  using namespace csd::verify;
  if (check_move(cache, layer, n) != CSD_OK || n > cache->cfg.max_step || check_heads(q) != CSD_OK) return CSD_ERR_INVALID_ARG;
  if (!d_path_len || !d_out || misaligned(d_out) || !std::isfinite(scale) || prompt_bound < 0 || path_bound < 0) return CSD_ERR_INVALID_ARG;
  const csd_cache_config& cfg = cache->cfg;
  AttendArgs a;
  const AttendLaunch how = attend_form(&a, cfg, n, prompt_bound, path_bound);
  a.prompt = cache->held(true, layer);
  a.path = cache->held(false, layer);
  a.q = *q;
  a.prompt_len = d_prompt_len;
  a.path_len = d_path_len;
  a.counts = d_counts;
  a.scale = scale * 1.44269504088896340736f;
  a.out = d_out;
  a.lse = d_lse;
  a.part_o = reinterpret_cast<float*>(cache->base + cache->layout.part_o);
  a.part_lse = reinterpret_cast<float*>(cache->base + cache->layout.part_lse);
  attend_any(a, how, cfg.head_dim, static_cast<hipStream_t>(stream));
  return finish("csd_attend");
}

int csd_attend_form_of(const csd_cache_config* cfg, int32_t n, int32_t prompt_bound, int32_t path_bound, csd_attend_form* out_form) {
  using namespace csd::verify;
  const int rc = check(cfg);
  if (rc != CSD_OK) return rc;
  if (n <= 0 || n > cfg->max_step || prompt_bound < 0 || path_bound < 0 || !out_form) return CSD_ERR_INVALID_ARG;
  AttendArgs a;
  const AttendLaunch how = attend_form(&a, *cfg, n, prompt_bound, path_bound);
  *out_form = csd_attend_form{how.join, a.solo, a.prompt_splits, a.path_splits, (int32_t)how.groups};
  return CSD_OK;
}

int csd_cache_status(csd_cache* cache, uint32_t* host_flags, void* stream) {
  if (!cache || !host_flags) return CSD_ERR_INVALID_ARG;
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e = hipMemcpyAsync(host_flags, cache->status(), sizeof(uint32_t), hipMemcpyDeviceToHost, st);
  if (e == hipSuccess) e = hipStreamSynchronize(st);
  return e == hipSuccess ? CSD_OK : csd::hip_fail(e, "csd_cache_status");
}

}  // extern "C"
