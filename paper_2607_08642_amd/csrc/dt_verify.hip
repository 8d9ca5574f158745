// Host side of the verification calls (paged cache, attention, commit): argument checks
// and launches.
#include "dt_cache.h"

namespace dt {
namespace {

// Workgroups along a grid's axis: a launch counts its threads (256 or fewer a group here) in 32 bits.
constexpr int kMaxGroups = 1 << 24;

constexpr float kLog2e = 1.4426950408889634f;

bool positive_pow2(int x) { return x > 0 && (x & (x - 1)) == 0; }

dt_status check_cache(const dt_cache *c, bool data) {
  if (!c) return fail(DT_ERR_NULL, "cache is required");
  if (data && !c->data) return fail(DT_ERR_NULL, "cache.data is required");
  if (c->dtype != DT_F32 && c->dtype != DT_BF16 && c->dtype != DT_F8)
    return fail(DT_ERR_DTYPE, "cache.dtype must be DT_F32, DT_BF16 or DT_F8");
  if (c->layers < 1 || c->pages < 1 || c->kv_heads < 1)
    return fail(DT_ERR_SHAPE, "sizes must be positive (layers=%d pages=%d kv_heads=%d)", c->layers, c->pages,
                c->kv_heads);
  if (!positive_pow2(c->page_size) || c->page_size < 32 || c->page_size > 256)
    return fail(DT_ERR_UNSUPPORTED, "page_size must be 32, 64, 128 or 256 (%d)", c->page_size);
  if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128 && c->head_dim != 256)
    return fail(DT_ERR_UNSUPPORTED, "head_dim must be 64, 96, 128 or 256 (%d)", c->head_dim);
  if (c->kv_heads > 4096 || (double)c->layers * c->pages * c->kv_heads *
                                    (double)head_page_bytes(c->page_size, c->head_dim, c->dtype) > 1e15)
    return fail(DT_ERR_UNSUPPORTED, "cache too large");
  if (data && reinterpret_cast<uintptr_t>(c->data) % 256)
    return fail(DT_ERR_ALIGN, "cache.data must be 256-byte aligned");
  return DT_OK;
}

dt_status check_layer(const dt_cache *c, int layer) {
  if (layer < 0 || layer >= c->layers) return fail(DT_ERR_SHAPE, "layer %d outside [0, %d)", layer, c->layers);
  return DT_OK;
}

dt_status check_chunk(const dt_cache *c, const dt_chunk *k, bool data) {
  if (!k) return fail(DT_ERR_NULL, "chunk is required");
  if (data && (!k->starts || !k->lens || !k->table))
    return fail(DT_ERR_NULL, "chunk.starts, lens and table are required");
  if (k->batch < 1 || k->rows < 1 || k->max_chunk < 1 || k->max_len < 1 || k->table_width < 1)
    return fail(DT_ERR_SHAPE, "sizes must be positive (batch=%d rows=%d max_chunk=%d max_len=%d table_width=%d)",
                k->batch, k->rows, k->max_chunk, k->max_len, k->table_width);
  if (k->batch > 65535) return fail(DT_ERR_UNSUPPORTED, "batch must be <= 65535 (%d)", k->batch);
  if ((int64_t)k->table_width * c->page_size >= (int64_t)1 << 30)
    return fail(DT_ERR_UNSUPPORTED, "table_width * page_size must be < 2^30");
  if (k->max_chunk > k->rows) return fail(DT_ERR_SHAPE, "max_chunk (%d) exceeds rows (%d)", k->max_chunk, k->rows);
  if (k->max_len > k->table_width * c->page_size || k->max_chunk > k->max_len)
    return fail(DT_ERR_SHAPE, "need max_chunk (%d) <= max_len (%d) <= table_width * page_size (%d)", k->max_chunk,
                k->max_len, k->table_width * c->page_size);
  if (data && (reinterpret_cast<uintptr_t>(k->starts) % 4 || reinterpret_cast<uintptr_t>(k->lens) % 4 ||
               reinterpret_cast<uintptr_t>(k->table) % 4))
    return fail(DT_ERR_ALIGN, "starts, lens and table must be naturally aligned");
  return DT_OK;
}

dt_status check_rows(const dt_rows *t, int dtype, const char *name, RowsView *v) {
  if (!t || !t->data) return fail(DT_ERR_NULL, "%s is required", name);
  if (t->row_stride < 0 || t->head_stride < 0) return fail(DT_ERR_SHAPE, "%s: strides must be >= 0", name);
  const int es = elem_bytes(dtype);
  const uintptr_t at = reinterpret_cast<uintptr_t>(t->data);
  if (at % es) return fail(DT_ERR_ALIGN, "%s must be naturally aligned", name);
  v->p = static_cast<char *>(t->data);
  v->row = t->row_stride;
  v->head = t->head_stride;
  v->vec = at % 16 == 0 && t->row_stride * es % 16 == 0 && t->head_stride * es % 16 == 0;
  return DT_OK;
}

// the shape of a store call: cache, layer, chunk, two tensors of rows
dt_status check_store(const dt_cache *cache, int layer, const dt_chunk *chunk, const dt_rows *k, const dt_rows *v,
                      RowsView *kr, RowsView *vr) {
  dt_status st = check_cache(cache, true);
  if (st == DT_OK) st = check_layer(cache, layer);
  if (st == DT_OK) st = check_chunk(cache, chunk, true);
  if (st == DT_OK) st = check_rows(k, data_dtype(cache->dtype), "k", kr);
  if (st == DT_OK) st = check_rows(v, data_dtype(cache->dtype), "v", vr);
  if (st == DT_OK && ((int64_t)chunk->max_chunk / kBlk + 3) * cache->kv_heads >= kMaxGroups)
    st = fail(DT_ERR_UNSUPPORTED, "max_chunk and kv_heads are too large together");
  return st;
}

dt_status check_attend(const dt_cache *c, const dt_chunk *k, int heads, const dt_attend_options *o) {
  if (!o) return fail(DT_ERR_NULL, "opts is required");
  if (heads < 1 || heads % c->kv_heads)
    return fail(DT_ERR_SHAPE, "heads (%d) must be a positive multiple of kv_heads (%d)", heads, c->kv_heads);
  if (heads / c->kv_heads > 1024) return fail(DT_ERR_UNSUPPORTED, "at most 1024 heads per kv head");
  if ((int64_t)k->max_chunk * heads > (int64_t)1 << 28)
    return fail(DT_ERR_UNSUPPORTED, "max_chunk * heads must be <= 2^28");
  const float unit = o->scale * kLog2e;  // (exponents are taken to the base of 2)
  if (!(unit - unit == 0.0f)) return fail(DT_ERR_SHAPE, "scale must be finite, and scale log2 e in fp32");
  if (o->window < 0 || o->sinks < 0 || o->tree_nodes < 0)
    return fail(DT_ERR_SHAPE, "window, sinks and tree_nodes must be >= 0");
  if (o->tree_nodes > kMaxB) return fail(DT_ERR_UNSUPPORTED, "tree_nodes must be <= %d", kMaxB);
  if (o->tree_nodes > k->max_chunk)
    return fail(DT_ERR_SHAPE, "tree_nodes (%d) exceeds max_chunk (%d)", o->tree_nodes, k->max_chunk);
  return DT_OK;
}

// window and sinks as the kernels take them (0: no window)
void effective_window(const dt_chunk *k, const dt_attend_options *o, int *window, int *sinks) {
  *window = o->window < 1 << 30 ? o->window : 1 << 30;  // (wider than any table: sums stay within 32 bits)
  *sinks = o->sinks < k->max_len ? o->sinks : k->max_len;
}

struct AttendWs {
  size_t ml, part, bytes;
};
AttendWs attend_ws(const AttendPlan &p, const dt_chunk *k, int heads, int D) {
  AttendWs w{};
  if (p.splits == 1) return w;
  const size_t rows = (size_t)k->rows * heads;
  w.ml = 0;
  w.part = align_up(rows * (p.splits + 1) * sizeof(float2), 256);
  w.bytes = w.part + align_up(rows * p.splits * D * sizeof(float), 256);
  return w;
}

}  // namespace
}  // namespace dt

using namespace dt;

extern "C" {

dt_status dt_cache_size(const dt_cache *cache, size_t *bytes) {
  if (!bytes) return fail(DT_ERR_NULL, "bytes is required");
  const dt_status st = check_cache(cache, false);
  if (st != DT_OK) return st;
  *bytes = (size_t)cache->layers * cache->pages * cache->kv_heads *
           head_page_bytes(cache->page_size, cache->head_dim, cache->dtype);
  return DT_OK;
}

dt_status dt_cache_append(const dt_cache *cache, int layer, const dt_chunk *chunk, const dt_rows *k,
                          const dt_rows *v, void *stream) {
  RowsView kr, vr;
  const dt_status st = check_store(cache, layer, chunk, k, v, &kr, &vr);
  if (st != DT_OK) return st;
  const hipError_t e = launch_append(cache_view(*cache, layer), cache->dtype, chunk_view(*chunk), kr, vr,
                                     static_cast<hipStream_t>(stream));
  return e == hipSuccess ? DT_OK : hip_fail(e, "append launch");
}

dt_status dt_cache_read(const dt_cache *cache, int layer, const dt_chunk *chunk, const dt_rows *k, const dt_rows *v,
                        void *stream) {
  RowsView kr, vr;
  const dt_status st = check_store(cache, layer, chunk, k, v, &kr, &vr);
  if (st != DT_OK) return st;
  const hipError_t e = launch_read(cache_view(*cache, layer), cache->dtype, chunk_view(*chunk), kr, vr,
                                   static_cast<hipStream_t>(stream));
  return e == hipSuccess ? DT_OK : hip_fail(e, "read launch");
}

dt_status dt_attend_workspace_size(const dt_cache *cache, const dt_chunk *chunk, int heads,
                                   const dt_attend_options *opts, size_t *bytes) {
  if (!bytes) return fail(DT_ERR_NULL, "bytes is required");
  dt_status st = check_cache(cache, false);
  if (st == DT_OK) st = check_chunk(cache, chunk, false);
  if (st == DT_OK) st = check_attend(cache, chunk, heads, opts);
  if (st != DT_OK) return st;
  int window, sinks;
  effective_window(chunk, opts, &window, &sinks);
  const AttendPlan p = attend_plan(cache_view(*cache, 0), chunk_view(*chunk), cache->dtype, heads, window, sinks,
                                   opts->tree_nodes);
  *bytes = attend_ws(p, chunk, heads, cache->head_dim).bytes;
  return DT_OK;
}

dt_status dt_cache_attend(const dt_cache *cache, int layer, const dt_chunk *chunk, int heads, const dt_rows *q,
                          const dt_rows *out, const dt_attend_options *opts, void *workspace, size_t ws_bytes,
                          void *stream) {
  AttendArgs a{};
  dt_status st = check_cache(cache, true);
  if (st == DT_OK) st = check_layer(cache, layer);
  if (st == DT_OK) st = check_chunk(cache, chunk, true);
  if (st == DT_OK) st = check_attend(cache, chunk, heads, opts);
  if (st == DT_OK) st = check_rows(q, data_dtype(cache->dtype), "q", &a.q);
  if (st == DT_OK) st = check_rows(out, data_dtype(cache->dtype), "out", &a.out);
  if (st != DT_OK) return st;
  if (opts->tree_nodes > 0 && (!opts->mask || (opts->window > 0 && !opts->depth)))
    return fail(DT_ERR_NULL, "a tree needs its mask, and with a window its depths");
  if (opts->depth && reinterpret_cast<uintptr_t>(opts->depth) % 4)
    return fail(DT_ERR_ALIGN, "depth must be naturally aligned");
  a.cache = cache_view(*cache, layer);
  a.chunk = chunk_view(*chunk);
  a.dtype = cache->dtype;
  a.heads = heads;
  a.group = heads / cache->kv_heads;
  a.scale_log2e = opts->scale * kLog2e;
  effective_window(chunk, opts, &a.window, &a.sinks);
  a.nodes = opts->tree_nodes;
  a.mask = opts->mask;
  a.depth = opts->depth;
  const AttendPlan p = attend_plan(a.cache, a.chunk, cache->dtype, heads, a.window, a.sinks, a.nodes);
  const AttendWs w = attend_ws(p, chunk, heads, cache->head_dim);
  if (w.bytes) {
    if (!workspace || ws_bytes < w.bytes)
      return fail(DT_ERR_WORKSPACE, "workspace needs %zu bytes, got %zu", w.bytes, workspace ? ws_bytes : 0);
    if (reinterpret_cast<uintptr_t>(workspace) % 256)
      return fail(DT_ERR_ALIGN, "workspace must be 256-byte aligned");
    a.part_ml = reinterpret_cast<float2 *>(static_cast<char *>(workspace) + w.ml);
    a.part = reinterpret_cast<float *>(static_cast<char *>(workspace) + w.part);
  }
  a.splits = p.splits;
  a.split_blocks = p.blocks;
  const hipError_t e = launch_attend(a, p, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? DT_OK : hip_fail(e, "attention launch");
}

dt_status dt_tree_accept(const dt_tree *tree, int batch, int B, const int32_t *target, int32_t *path,
                         int32_t *n_accepted, int32_t *next_token, void *stream) {
  if (!tree || !target || !path || !n_accepted || !next_token || !tree->tokens || !tree->parents || !tree->n_nodes)
    return fail(DT_ERR_NULL, "tree (tokens, parents, n_nodes), target and every output are required");
  if (batch < 1 || B < 1) return fail(DT_ERR_SHAPE, "sizes must be positive (batch=%d B=%d)", batch, B);
  if (B > kMaxB) return fail(DT_ERR_UNSUPPORTED, "B must be <= %d (%d)", kMaxB, B);
  if (batch >= kMaxGroups) return fail(DT_ERR_UNSUPPORTED, "batch must be < %d (%d)", kMaxGroups, batch);
  for (const void *p : {(const void *)tree->tokens, (const void *)tree->parents, (const void *)tree->n_nodes,
                        (const void *)target, (const void *)path, (const void *)n_accepted, (const void *)next_token})
    if (reinterpret_cast<uintptr_t>(p) % 4) return fail(DT_ERR_ALIGN, "tensors must be naturally aligned");
  const hipError_t e = launch_accept(*tree, batch, B, target, path, n_accepted, next_token,
                                     static_cast<hipStream_t>(stream));
  return e == hipSuccess ? DT_OK : hip_fail(e, "accept launch");
}

dt_status dt_cache_commit(const dt_cache *cache, const dt_chunk *chunk, int nodes, const int32_t *path,
                          const int32_t *n_accepted, void *stream) {
  dt_status st = check_cache(cache, true);
  if (st == DT_OK) st = check_chunk(cache, chunk, true);
  if (st != DT_OK) return st;
  if (!path || !n_accepted) return fail(DT_ERR_NULL, "path and n_accepted are required");
  if (reinterpret_cast<uintptr_t>(path) % 4 || reinterpret_cast<uintptr_t>(n_accepted) % 4)
    return fail(DT_ERR_ALIGN, "path and n_accepted must be naturally aligned");
  if (nodes < 1 || nodes > chunk->max_chunk)
    return fail(DT_ERR_SHAPE, "nodes %d outside [1, max_chunk=%d]", nodes, chunk->max_chunk);
  if (nodes > kMaxB) return fail(DT_ERR_UNSUPPORTED, "nodes must be <= %d (%d)", kMaxB, nodes);
  if ((int64_t)cache->layers * cache->kv_heads >= kMaxGroups)
    return fail(DT_ERR_UNSUPPORTED, "layers * kv_heads is too large");
  const hipError_t e = launch_commit(cache_view(*cache, 0), cache->dtype, cache->layers, chunk_view(*chunk), nodes,
                                     path, n_accepted, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? DT_OK : hip_fail(e, "commit launch");
}

}  // extern "C"
