// C ABI of the paged cache: argument checks, workspace carving, launch order.  No kernel lives here.  Every check runs before the
// first launch.
#include <cmath>

#include "paged.h"

using namespace spiffy;

namespace {

constexpr int kMaxPoolPages = 1 << 30, kMaxTable = 1 << 22;
constexpr float kLog2e = 1.4426950408889634f;      // what the kernels' exponentials to base 2 take with the scale
constexpr int64_t kMaxPositions = (int64_t(1) << 31) - (1 << 16);      // rows of a sequence: kernels count some way past them in 31 bits

inline bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
int dev(hipError_t e) { return e == hipSuccess ? SPIFFY_OK : SPIFFY_EDEVICE; }

int check_heads(const spiffy_model_cfg* c) {
  if (!c || (c->dtype != SPIFFY_BF16 && c->dtype != SPIFFY_F32)) return SPIFFY_EINVAL;
  if (c->n_q_heads < 1 || c->n_kv_heads < 1 || c->head_dim < 2) return SPIFFY_EINVAL;
  if (c->n_q_heads % c->n_kv_heads != 0 || c->n_q_heads > 4096) return SPIFFY_ESHAPE;
  if (c->head_dim % 8 != 0 || c->head_dim > 256) return SPIFFY_ESHAPE;
  return SPIFFY_OK;
}
Heads heads(const spiffy_model_cfg* c) { return Heads{c->n_q_heads, c->n_kv_heads, c->head_dim, c->dtype == SPIFFY_F32}; }

int check_sizes(const spiffy_paged_cache* c) {
  if (!c || c->n_pages < 1 || c->page_size < 1 || c->n_seqs < 1 || c->max_pages < 1) return SPIFFY_EINVAL;
  if (c->n_seqs > SPIFFY_MAX_SEQS || c->n_pages > kMaxPoolPages || c->max_pages > kMaxTable) return SPIFFY_ESHAPE;
  if ((int64_t)c->n_seqs * c->max_pages > INT32_MAX) return SPIFFY_ESHAPE;      // pages of all sequences are counted in 31 bits
  if ((int64_t)c->n_pages * c->page_size > INT32_MAX || (int64_t)c->max_pages * c->page_size > kMaxPositions) return SPIFFY_ESHAPE;
  return SPIFFY_OK;
}
int check_cache(const spiffy_paged_cache* c) {
  const int rc = check_sizes(c);
  if (rc) return rc;
  if (!c->refs || !c->table || !c->len) return SPIFFY_EINVAL;
  if (!aligned(c->refs, 4) || !aligned(c->table, 4) || !aligned(c->len, 4)) return SPIFFY_EALIGN;
  return SPIFFY_OK;
}
PagedView view(const spiffy_paged_cache* c) {
  return PagedView{c->n_pages, c->page_size, c->n_seqs, c->max_pages, c->refs, c->table, c->len};
}

int check_layers(int32_t n_layers, const spiffy_page_layer* layers, bool need_kv, bool need_summary) {
  if (n_layers < 1 || !layers) return SPIFFY_EINVAL;
  if (n_layers > SPIFFY_MAX_PAGED_LAYERS) return SPIFFY_ESHAPE;
  for (int l = 0; l < n_layers; ++l) {
    if ((need_kv && (!layers[l].k || !layers[l].v)) || (need_summary && (!layers[l].summary || !layers[l].k))) return SPIFFY_EINVAL;
    if (!aligned(layers[l].k, 16) || !aligned(layers[l].v, 16) || !aligned(layers[l].summary, 16)) return SPIFFY_EALIGN;
  }
  return SPIFFY_OK;
}
// the layers from `from` on that one launch takes
void take_layers(PageLayers& p, const spiffy_page_layer* layers, int from, int n_layers) {
  p.n = n_layers - from < kLayersPerLaunch ? n_layers - from : kLayersPerLaunch;
  for (int l = 0; l < p.n; ++l) {
    p.k[l] = layers[from + l].k;
    p.v[l] = layers[from + l].v;
    p.summary[l] = layers[from + l].summary;
  }
}

int check_workspace(const void* ws, size_t have, size_t need) {
  if (!ws) return SPIFFY_EINVAL;
  if (!aligned(ws, 256)) return SPIFFY_EALIGN;
  return have < need ? SPIFFY_EWORKSPACE : SPIFFY_OK;
}

int check_rows(const int32_t* row_start, int32_t T, const uint64_t* mask, int32_t mask_words) {
  if (!row_start || T < 1 || (mask && mask_words < 1)) return SPIFFY_EINVAL;
  if (T > SPIFFY_MAX_NEW_ROWS || (mask && mask_words > SPIFFY_MAX_TREE / 64)) return SPIFFY_ESHAPE;
  if (!aligned(row_start, 4) || !aligned(mask, 8)) return SPIFFY_EALIGN;
  return SPIFFY_OK;
}
// a row stride in elements: at least the row, whole 16-byte pieces, and T rows within 63 bits of bytes
int check_stride(int64_t stride, int64_t row, int es) {
  if (stride < row) return SPIFFY_EINVAL;
  if (stride > ((int64_t)1 << 38)) return SPIFFY_ESHAPE;
  return stride * es % 16 ? SPIFFY_EALIGN : SPIFFY_OK;
}

}  // namespace

extern "C" {
#pragma GCC visibility push(default)

size_t spiffy_pages_workspace_bytes(const spiffy_paged_cache* cache) {
  return check_sizes(cache) ? 0 : pages_workspace_bytes(view(cache));
}

int spiffy_pages_append(const spiffy_model_cfg* cfg, const spiffy_paged_cache* cache, int32_t n_layers, const spiffy_page_layer* layers,
                        const void* const* rows_k, const void* const* rows_v, int64_t row_stride, const int32_t* row_start, int32_t T,
                        const uint64_t* mask, int32_t mask_words, const int32_t* node, int32_t node_stride, int32_t* status,
                        void* workspace, size_t workspace_bytes, void* stream) {
  int rc;
  if ((rc = check_heads(cfg)) || (rc = check_cache(cache)) || (rc = check_layers(n_layers, layers, true, false))) return rc;
  if (!rows_k || !rows_v || (mask != nullptr) != (node != nullptr) || (node && node_stride < 1)) return SPIFFY_EINVAL;
  if ((rc = check_rows(row_start, T, mask, mask_words))) return rc;
  const Heads h = heads(cfg);
  if ((rc = check_stride(row_stride, (int64_t)h.Hkv * h.hd, h.f32 ? 4 : 2))) return rc;
  for (int l = 0; l < n_layers; ++l) {
    if (!rows_k[l] || !rows_v[l]) return SPIFFY_EINVAL;
    if (!aligned(rows_k[l], 16) || !aligned(rows_v[l], 16)) return SPIFFY_EALIGN;
  }
  if (!aligned(node, 4) || !aligned(status, 4)) return SPIFFY_EALIGN;
  PagesArgs a{};
  a.c = view(cache);
  if ((rc = check_workspace(workspace, workspace_bytes, pages_workspace_bytes(a.c)))) return rc;
  a.h = h;
  a.ws = carve_pages(a.c, workspace);
  a.rows = NewRows{row_start, T, mask, mask_words};
  a.row_stride = row_stride;
  a.node = node;
  a.node_stride = node_stride;
  a.status = status;
  hipStream_t st = (hipStream_t)stream;
  if ((rc = dev(launch_append_plan(a, st)))) return rc;
  for (int l = 0; l < n_layers; l += kLayersPerLaunch) {
    take_layers(a.layers, layers, l, n_layers);
    for (int i = 0; i < a.layers.n; ++i) a.row_layers.k[i] = rows_k[l + i], a.row_layers.v[i] = rows_v[l + i];
    if ((rc = dev(launch_append_rows(a, st)))) return rc;
  }
  return SPIFFY_OK;
}

int spiffy_pages_fork(const spiffy_model_cfg* cfg, const spiffy_paged_cache* cache, int32_t n_layers, const spiffy_page_layer* layers,
                      const int32_t* src, const int32_t* dst, int32_t n, int32_t* status, void* workspace, size_t workspace_bytes,
                      void* stream) {
  int rc;
  if ((rc = check_heads(cfg)) || (rc = check_cache(cache)) || (rc = check_layers(n_layers, layers, true, false))) return rc;
  if (!src || !dst || n < 1) return SPIFFY_EINVAL;
  if (n > SPIFFY_MAX_SEQS) return SPIFFY_ESHAPE;
  if (!aligned(src, 4) || !aligned(dst, 4) || !aligned(status, 4)) return SPIFFY_EALIGN;
  PagesArgs a{};
  a.c = view(cache);
  if ((rc = check_workspace(workspace, workspace_bytes, pages_workspace_bytes(a.c)))) return rc;
  a.h = heads(cfg);
  a.ws = carve_pages(a.c, workspace);
  a.src = src;
  a.dst = dst;
  a.n = n;
  a.status = status;
  hipStream_t st = (hipStream_t)stream;
  if ((rc = dev(launch_fork_plan(a, st)))) return rc;
  for (int l = 0; l < n_layers; l += kLayersPerLaunch) {
    take_layers(a.layers, layers, l, n_layers);
    if ((rc = dev(launch_fork_rows(a, l == 0, st)))) return rc;
  }
  return SPIFFY_OK;
}

int spiffy_pages_free(const spiffy_paged_cache* cache, const int32_t* seqs, int32_t n, void* stream) {
  int rc;
  if ((rc = check_cache(cache))) return rc;
  if (!seqs || n < 1) return SPIFFY_EINVAL;
  if (n > SPIFFY_MAX_SEQS) return SPIFFY_ESHAPE;
  if (!aligned(seqs, 4)) return SPIFFY_EALIGN;
  PagesArgs a{};
  a.c = view(cache);
  a.src = seqs;
  a.n = n;
  return dev(launch_free(a, (hipStream_t)stream));
}

int spiffy_pages_compact(const spiffy_model_cfg* cfg, const spiffy_paged_cache* cache, int32_t n_layers, const spiffy_page_layer* layers,
                         int32_t* n_used, void* workspace, size_t workspace_bytes, void* stream) {
  int rc;
  if ((rc = check_heads(cfg)) || (rc = check_cache(cache)) || (rc = check_layers(n_layers, layers, true, false))) return rc;
  if (!aligned(n_used, 4)) return SPIFFY_EALIGN;
  PagesArgs a{};
  a.c = view(cache);
  if ((rc = check_workspace(workspace, workspace_bytes, pages_workspace_bytes(a.c)))) return rc;
  a.h = heads(cfg);
  a.ws = carve_pages(a.c, workspace);
  a.status = n_used;
  hipStream_t st = (hipStream_t)stream;
  if ((rc = dev(launch_compact_plan(a, st)))) return rc;
  for (int l = 0; l < n_layers; l += kLayersPerLaunch) {
    take_layers(a.layers, layers, l, n_layers);
    if ((rc = dev(launch_compact_rows(a, l == 0, st)))) return rc;
  }
  return SPIFFY_OK;
}

int spiffy_page_summary(const spiffy_model_cfg* cfg, const spiffy_paged_cache* cache, int32_t n_layers, const spiffy_page_layer* layers,
                        const int32_t* start, void* stream) {
  int rc;
  if ((rc = check_heads(cfg)) || (rc = check_cache(cache)) || (rc = check_layers(n_layers, layers, false, true))) return rc;
  if (!aligned(start, 4)) return SPIFFY_EALIGN;
  SummaryArgs a{};
  a.c = view(cache);
  a.h = heads(cfg);
  a.start = start;
  for (int l = 0; l < n_layers; l += kLayersPerLaunch) {
    take_layers(a.layers, layers, l, n_layers);
    if ((rc = dev(launch_page_summary(a, (hipStream_t)stream)))) return rc;
  }
  return SPIFFY_OK;
}

size_t spiffy_page_select_workspace_bytes(const spiffy_model_cfg* cfg, const spiffy_paged_cache* cache) {
  if (check_heads(cfg) || check_sizes(cache)) return 0;
  return page_select_workspace_bytes(view(cache), heads(cfg));
}

int spiffy_page_select(const spiffy_model_cfg* cfg, const spiffy_paged_cache* cache, const spiffy_page_layer* layer, const void* q,
                       int64_t q_stride, const int32_t* row_start, int32_t T, int32_t max_rows, int32_t n_sel, int32_t keep_first,
                       int32_t keep_last, int32_t* selected, void* workspace, size_t workspace_bytes, void* stream) {
  int rc;
  if ((rc = check_heads(cfg)) || (rc = check_cache(cache)) || (rc = check_layers(1, layer, false, true))) return rc;
  if (!q || !selected || max_rows < 1 || n_sel < 1 || keep_first < 0 || keep_last < 0) return SPIFFY_EINVAL;
  if ((rc = check_rows(row_start, T, nullptr, 0))) return rc;
  if (max_rows > SPIFFY_MAX_TREE || n_sel > kMaxTable) return SPIFFY_ESHAPE;
  const Heads h = heads(cfg);
  if ((rc = check_stride(q_stride, (int64_t)h.Hq * h.hd, h.f32 ? 4 : 2))) return rc;
  if (!aligned(q, 16) || !aligned(selected, 4)) return SPIFFY_EALIGN;
  SelectArgs a{};
  a.c = view(cache);
  a.h = h;
  if ((rc = check_workspace(workspace, workspace_bytes, page_select_workspace_bytes(a.c, h)))) return rc;
  a.summary = layer->summary;
  a.q = q;
  a.q_stride = q_stride;
  a.rows = NewRows{row_start, T, nullptr, 0};
  a.max_rows = max_rows;
  a.n_sel = n_sel;
  a.keep_first = keep_first;
  a.keep_last = keep_last;
  a.selected = selected;
  a.scores = reinterpret_cast<double*>(workspace);
  return dev(launch_page_select(a, (hipStream_t)stream));
}

size_t spiffy_tree_attention_workspace_bytes(const spiffy_model_cfg* cfg, const spiffy_paged_cache* cache, int32_t max_rows) {
  if (check_heads(cfg) || check_sizes(cache) || max_rows < 1 || max_rows > SPIFFY_MAX_TREE) return 0;
  return tree_attn_fits(view(cache), heads(cfg), max_rows) ? tree_attn_workspace_bytes(view(cache), heads(cfg), max_rows) : 0;
}

int spiffy_tree_attention(const spiffy_model_cfg* cfg, const spiffy_paged_cache* cache, const spiffy_page_layer* layer, const void* q,
                          int64_t q_stride, const void* k, const void* v, int64_t kv_stride, const int32_t* row_start, int32_t T,
                          int32_t max_rows, const uint64_t* mask, int32_t mask_words, const int32_t* selected, int32_t n_sel, float scale,
                          void* out, int64_t out_stride, void* workspace, size_t workspace_bytes, void* stream) {
  int rc;
  if ((rc = check_heads(cfg)) || (rc = check_cache(cache)) || (rc = check_layers(1, layer, true, false))) return rc;
  if (!q || !k || !v || !out || max_rows < 1 || (selected && n_sel < 1) || !std::isfinite(scale * kLog2e)) return SPIFFY_EINVAL;
  if ((rc = check_rows(row_start, T, mask, mask_words))) return rc;
  if (max_rows > SPIFFY_MAX_TREE || (selected && n_sel > kMaxTable)) return SPIFFY_ESHAPE;
  const Heads h = heads(cfg);
  if (selected && (int64_t)n_sel * cache->page_size > kMaxPositions) return SPIFFY_ESHAPE;
  if (!tree_attn_fits(view(cache), h, max_rows)) return SPIFFY_ESHAPE;
  const int es = h.f32 ? 4 : 2;
  if ((rc = check_stride(q_stride, (int64_t)h.Hq * h.hd, es)) || (rc = check_stride(kv_stride, (int64_t)h.Hkv * h.hd, es)) ||
      (rc = check_stride(out_stride, (int64_t)h.Hq * h.hd, es)))
    return rc;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(selected, 4)) return SPIFFY_EALIGN;
  TreeAttnArgs a{};
  a.c = view(cache);
  if ((rc = check_workspace(workspace, workspace_bytes, tree_attn_workspace_bytes(a.c, h, max_rows)))) return rc;
  a.h = h;
  a.pk = layer->k;
  a.pv = layer->v;
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.kv_stride = kv_stride;
  a.out_stride = out_stride;
  a.rows = NewRows{row_start, T, mask, mask_words};
  a.max_rows = max_rows;
  a.selected = selected;
  a.n_sel = n_sel;
  a.scale = scale;
  a.out = out;
  a.workspace = workspace;
  return dev(launch_tree_attn(a, (hipStream_t)stream));
}

#pragma GCC visibility pop
}  // extern "C"
