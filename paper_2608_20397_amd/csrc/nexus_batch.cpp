// C-ABI entry points of ragged batches: host-side validation (fail-closed: nothing is enqueued unless every check
// passes) and dispatch.  Stateless; allocates nothing.
#include "api_checks.h"
#include "launch_batch.h"

#include <algorithm>

using namespace nexus;

namespace {

constexpr int32_t kMaxWindowLen = 1 << 29;      // positions, windows and their sums stay within 32 bits

bool aligned16(const void *p) { return (uintptr_t)p % 16 == 0; }

// Whether [a, a + an) and [b, b + bn) bytes share any.
bool overlap(const void *a, uint64_t an, const void *b, uint64_t bn) {
  const uint64_t x = (uint64_t)(uintptr_t)a, y = (uint64_t)(uintptr_t)b;
  return x < y + bn && y < x + an;
}

// Bytes of one layer of K or V.
uint64_t layer_bytes(const nexus_kv_cache *c) {
  return (uint64_t)c->n_phys_pages * c->n_kv_heads * kPageSize * c->head_dim * dtype_bytes(c->dtype);
}

const char *layer_base(const void *p, const nexus_kv_cache *c, int32_t layer) {
  return (const char *)p + layer * layer_bytes(c);
}

// What the workspace of a windowed launch depends on (q_start: any non-null pointer stands for many rows).
nexus_status window_sizes(int32_t n_rows, int32_t n_q_heads, const nexus_kv_cache *cache, const int32_t *q_start,
                          int32_t n_seqs, int32_t max_seq_len, int32_t window, int32_t n_sink, WindowLaunch &L) {
  const nexus_status st = check_cache(cache);
  if (st) return st;
  if (n_rows <= 0 || n_seqs <= 0 || window < 1 || n_sink < 0) return NEXUS_EINVAL;
  if (n_q_heads <= 0 || n_q_heads % cache->n_kv_heads) return NEXUS_ESHAPE;
  if (cache->dtype == NEXUS_BF16
          ? cache->head_dim != 64 && cache->head_dim != 128 && cache->head_dim != 256
          : cache->head_dim < 16 || cache->head_dim > 256)
    return NEXUS_ESHAPE;
  if (max_seq_len < 0 || max_seq_len > kMaxWindowLen) return NEXUS_ERANGE;
  if (n_seqs > 65535 || n_q_heads > 65535) return NEXUS_ESHAPE;
  if ((int64_t)n_rows * n_q_heads * cache->head_dim >= kMaxElems32) return NEXUS_ESHAPE;
  L = WindowLaunch{};
  L.q_start = q_start;
  L.max_len = max_seq_len;
  L.n_seqs = n_seqs;
  L.n_rows = n_rows;
  L.n_phys_pages = cache->n_phys_pages;
  L.n_kv_heads = cache->n_kv_heads;
  L.n_q_heads = n_q_heads;
  L.head_dim = cache->head_dim;
  L.is_bf16 = cache->dtype == NEXUS_BF16;
  L.v_transposed = cache->v_layout == NEXUS_V_TRANSPOSED;
  L.window = std::min(window, std::max(max_seq_len, 1));
  L.sinks = std::min(n_sink, max_seq_len);
  return plan_window(L) ? NEXUS_OK : NEXUS_ESHAPE;
}

nexus_status run_window(const void *q, const nexus_kv_cache *cache, const int32_t *maps, int32_t map_stride,
                        const int32_t *seq_len, int32_t layer, float softcap, int32_t v_layout, float scale,
                        void *out, void *workspace, size_t workspace_bytes, void *stream, WindowLaunch &L) {
  if (!q || !out || !maps || !seq_len || map_stride <= 0) return NEXUS_EINVAL;
  if (!aligned16(q) || !aligned16(out) || !aligned16(cache->k) || !aligned16(cache->v)) return NEXUS_EINVAL;
  if (!valid_layout(v_layout)) return NEXUS_EINVAL;
  if (v_layout != cache->v_layout) return NEXUS_ELAYOUT;
  if (layer < 0 || layer >= cache->n_layers) return NEXUS_ERANGE;
  if ((int64_t)map_stride * kPageSize < L.max_len) return NEXUS_ERANGE;
  if ((int64_t)L.n_seqs * map_stride >= kMaxElems32) return NEXUS_ESHAPE;
  if (!(softcap >= 0.f) || !isfinite(softcap)) return NEXUS_EINVAL;
  if (!(scale >= 0.f) || !isfinite(scale)) return NEXUS_EINVAL;
  const size_t need = window_workspace_bytes(L);
  if (need > 0 && (!workspace || workspace_bytes < need)) return NEXUS_EWORKSPACE;
  if (need > 0 && !aligned16(workspace)) return NEXUS_EINVAL;
  // a workgroup reads its own queries before it writes their rows, so q itself may be written over
  const uint64_t bytes = (uint64_t)L.n_rows * L.n_q_heads * L.head_dim * dtype_bytes(cache->dtype);
  if (out != q && overlap(out, bytes, q, bytes)) return NEXUS_EINVAL;
  if (need > 0 && (overlap(workspace, need, q, bytes) || overlap(workspace, need, out, bytes))) return NEXUS_EINVAL;
  L.q = q;
  L.out = out;
  L.cache_k = layer_base(cache->k, cache, layer);
  L.cache_v = layer_base(cache->v, cache, layer);
  L.maps = maps;
  L.seq_len = seq_len;
  L.map_stride = map_stride;
  L.scale = scale > 0.f ? scale : 1.0f / sqrtf((float)cache->head_dim);
  L.softcap = softcap;
  L.workspace = workspace;
  return from_hip(launch_window(L, as_stream(stream)));
}

const int32_t kSome = 0;     // stands for device starts where only sizes are asked for

}  // namespace

extern "C" {

nexus_status nexus_batch_pages(const int32_t *cached, const int32_t *fresh, int32_t n_seqs,
                               const int32_t *free_pages, const int32_t *n_free, int32_t free_capacity,
                               int32_t *maps, int32_t map_stride, int32_t max_tokens, int32_t *q_start,
                               int32_t *seq_len, int32_t *pos, int32_t *slot, int32_t *n_left, void *stream) {
  if (!cached || !fresh || !free_pages || !n_free || !maps || !q_start || !seq_len || !pos || !slot || !n_left)
    return NEXUS_EINVAL;
  if (n_seqs <= 0 || map_stride <= 0 || max_tokens <= 0 || free_capacity < 0) return NEXUS_EINVAL;
  if (n_seqs > kMaxBatchSeqs || (int64_t)n_seqs * map_stride >= kMaxElems32) return NEXUS_ESHAPE;
  if (map_stride > kMaxWindowLen / kPageSize || max_tokens > (1 << 30)) return NEXUS_ERANGE;
  // workgroups read the lengths and the list while others write: what is written stands apart
  const uint64_t seqs = 4ull * n_seqs, rows = 4ull * max_tokens;
  const struct { const void *p; uint64_t n; } out[] = {
      {maps, seqs * map_stride}, {q_start, seqs + 4}, {seq_len, seqs}, {pos, rows}, {slot, rows}, {n_left, 4}};
  const struct { const void *p; uint64_t n; } in[] = {
      {cached, seqs}, {fresh, seqs}, {free_pages, 4ull * free_capacity}, {n_free, 4}};
  for (int i = 0; i < 6; ++i) {
    for (int j = 0; j < i; ++j)
      if (overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return NEXUS_EINVAL;
    for (const auto &r : in)
      if (overlap(out[i].p, out[i].n, r.p, r.n)) return NEXUS_EINVAL;
  }
  BatchPagesLaunch L{};
  L.cached = cached;
  L.fresh = fresh;
  L.free_pages = free_pages;
  L.n_free = n_free;
  L.maps = maps;
  L.q_start = q_start;
  L.seq_len = seq_len;
  L.pos = pos;
  L.slot = slot;
  L.n_left = n_left;
  L.n_seqs = n_seqs;
  L.free_capacity = free_capacity;
  L.map_stride = map_stride;
  L.max_tokens = max_tokens;
  return from_hip(launch_batch_pages(L, as_stream(stream)));
}

nexus_status nexus_norm_rope_append(const nexus_kv_cache *cache, int32_t layer, const void *q, int64_t q_stride,
                                    const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                                    int32_t n_tokens, int32_t n_q_heads, const float *q_weight,
                                    const float *k_weight, float eps, const int32_t *pos, const int32_t *slot,
                                    void *q_out, void *stream) {
  const nexus_status st = check_cache(cache);
  if (st) return st;
  if (!q || !k || !v || !pos || !slot || !q_out || n_tokens <= 0) return NEXUS_EINVAL;
  if (layer < 0 || layer >= cache->n_layers) return NEXUS_ERANGE;
  if (n_q_heads <= 0 || n_q_heads % cache->n_kv_heads || n_q_heads > 65535 || cache->head_dim > 256)
    return NEXUS_ESHAPE;
  if ((int64_t)n_tokens * n_q_heads * cache->head_dim >= kMaxElems32 || n_tokens > (1 << 22)) return NEXUS_ESHAPE;
  if (!(eps >= 0.f) || !isfinite(eps) || (eps == 0.f && (q_weight || k_weight))) return NEXUS_EINVAL;
  const int es = dtype_bytes(cache->dtype);
  const int64_t q_row = (int64_t)n_q_heads * cache->head_dim, kv_row = (int64_t)cache->n_kv_heads * cache->head_dim;
  for (const void *p : {(const void *)cache->k, (const void *)cache->v, q, k, v, (const void *)q_out})
    if (!aligned16(p)) return NEXUS_EINVAL;
  for (const int64_t s : {q_stride, k_stride, v_stride})
    if (s <= 0 || s >= ((int64_t)1 << 38) || s * es % 16 != 0) return NEXUS_EINVAL;
  if (q_stride < q_row || k_stride < kv_row || v_stride < kv_row) return NEXUS_EINVAL;
  const uint64_t out_bytes = (uint64_t)n_tokens * q_row * es;
  auto bytes = [&](int64_t stride, int64_t row) { return (uint64_t)((n_tokens - 1) * stride + row) * es; };
  // a row is read whole before it is written, so only q itself may be written over
  if (!(q_out == q && q_stride == q_row) && overlap(q_out, out_bytes, q, bytes(q_stride, q_row)))
    return NEXUS_EINVAL;
  if (overlap(q_out, out_bytes, k, bytes(k_stride, kv_row)) || overlap(q_out, out_bytes, v, bytes(v_stride, kv_row)))
    return NEXUS_EINVAL;
  const char *cache_k = layer_base(cache->k, cache, layer), *cache_v = layer_base(cache->v, cache, layer);
  for (const char *to : {cache_k, cache_v})
    if (overlap(to, layer_bytes(cache), q, bytes(q_stride, q_row)) ||
        overlap(to, layer_bytes(cache), k, bytes(k_stride, kv_row)) ||
        overlap(to, layer_bytes(cache), v, bytes(v_stride, kv_row)) ||
        overlap(to, layer_bytes(cache), q_out, out_bytes))
      return NEXUS_EINVAL;
  NormRopeLaunch L{};
  L.q = q;
  L.k = k;
  L.v = v;
  L.q_stride = q_stride;
  L.k_stride = k_stride;
  L.v_stride = v_stride;
  L.q_out = q_out;
  L.cache_k = (void *)cache_k;
  L.cache_v = (void *)cache_v;
  L.q_weight = q_weight;
  L.k_weight = k_weight;
  L.pos = pos;
  L.slot = slot;
  L.n_tokens = n_tokens;
  L.n_q_heads = n_q_heads;
  L.n_kv_heads = cache->n_kv_heads;
  L.head_dim = cache->head_dim;
  L.n_phys_pages = cache->n_phys_pages;
  L.dtype_bytes = es;
  L.v_transposed = cache->v_layout == NEXUS_V_TRANSPOSED;
  L.interleaved = cache->rope_style == NEXUS_ROPE_INTERLEAVED;
  L.eps = eps;
  L.rope_base = cache->rope_base;
  return from_hip(launch_norm_rope(L, as_stream(stream)));
}

nexus_status nexus_window_attn(const void *q, int32_t n_rows, int32_t n_q_heads, const nexus_kv_cache *cache,
                               const int32_t *maps, int32_t map_stride, const int32_t *q_start,
                               const int32_t *seq_len, int32_t n_seqs, int32_t max_seq_len, int32_t window,
                               int32_t n_sink, int32_t layer, float softcap, int32_t v_layout, float scale, void *out,
                               void *workspace, size_t workspace_bytes, void *stream) {
  if (!q_start) return NEXUS_EINVAL;
  WindowLaunch L;
  const nexus_status st = window_sizes(n_rows, n_q_heads, cache, q_start, n_seqs, max_seq_len, window, n_sink, L);
  if (st) return st;
  return run_window(q, cache, maps, map_stride, seq_len, layer, softcap, v_layout, scale, out, workspace,
                    workspace_bytes, stream, L);
}

size_t nexus_window_attn_workspace(int32_t n_rows, int32_t n_q_heads, const nexus_kv_cache *cache, int32_t n_seqs,
                                   int32_t max_seq_len, int32_t window, int32_t n_sink) {
  WindowLaunch L;
  if (window_sizes(n_rows, n_q_heads, cache, &kSome, n_seqs, max_seq_len, window, n_sink, L)) return SIZE_MAX;
  return window_workspace_bytes(L);
}

nexus_status nexus_window_decode_attn(const void *q, int32_t n_seqs, int32_t n_q_heads, const nexus_kv_cache *cache,
                                      const int32_t *maps, int32_t map_stride, const int32_t *seq_len,
                                      int32_t max_seq_len, int32_t window, int32_t n_sink, int32_t layer,
                                      float softcap, int32_t v_layout, float scale, void *out, void *workspace,
                                      size_t workspace_bytes, void *stream) {
  WindowLaunch L;
  const nexus_status st = window_sizes(n_seqs, n_q_heads, cache, nullptr, n_seqs, max_seq_len, window, n_sink, L);
  if (st) return st;
  return run_window(q, cache, maps, map_stride, seq_len, layer, softcap, v_layout, scale, out, workspace,
                    workspace_bytes, stream, L);
}

size_t nexus_window_decode_attn_workspace(int32_t n_seqs, int32_t n_q_heads, const nexus_kv_cache *cache,
                                          int32_t max_seq_len, int32_t window, int32_t n_sink) {
  WindowLaunch L;
  if (window_sizes(n_seqs, n_q_heads, cache, nullptr, n_seqs, max_seq_len, window, n_sink, L)) return SIZE_MAX;
  return window_workspace_bytes(L);
}

}  // extern "C"
