// C-ABI entry points of the 8-bit cache: host-side validation (fail-closed: nothing is enqueued unless every
// check passes) and dispatch.  Stateless; allocates no device memory.
#include "api_checks.h"
#include "attn_common.h"
#include "launch_kv8.h"

#include <new>

using namespace nexus;

namespace {

nexus_status check_kv8(const nexus_kv8_cache *c) {
  if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale) return NEXUS_EINVAL;
  if (c->n_layers <= 0 || c->n_phys_pages <= 0 || c->n_kv_heads <= 0 || c->head_dim <= 0)
    return NEXUS_EINVAL;
  // 16-byte loads of rows and of a page's scales (LDS DMA of keys among them)
  for (const void *p : {c->k, c->v, c->k_scale, c->v_scale})
    if ((uintptr_t)p % 16 != 0) return NEXUS_EINVAL;
  if (c->page_size != kPageSize) return NEXUS_ESHAPE;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return NEXUS_ESHAPE;
  if (!valid_style(c->rope_style)) return NEXUS_EINVAL;
  if (c->n_layers > 65535) return NEXUS_ESHAPE;
  // token positions are 32-bit, and so are offsets within a page; a layer may be of any size
  if ((int64_t)c->n_phys_pages * kPageSize >= kMaxElems32) return NEXUS_ESHAPE;
  if ((int64_t)kPageSize * c->n_kv_heads * c->head_dim >= kMaxElems32) return NEXUS_ESHAPE;
  // ... and offsets among a layer's scales (2^32 rows of K and of V would not fit the memory)
  if ((int64_t)c->n_phys_pages * kPageSize * c->n_kv_heads >= ((int64_t)1 << 32)) return NEXUS_ESHAPE;
  if (!(c->rope_base > 1.0) || !isfinite(c->rope_base)) return NEXUS_EROPE;
  return NEXUS_OK;
}

nexus_status check_map(const nexus_page_table *pt, const nexus_kv8_cache *c) {
  if (!pt || !pt->map || pt->n_logical_pages <= 0) return NEXUS_EINVAL;
  if (pt->n_logical_pages > c->n_phys_pages) return NEXUS_ERANGE;
  return NEXUS_OK;
}

// Rows [n_layers][n_tokens][n_kv_heads][head_dim] that a call reads or writes beside the cache.
nexus_status check_rows(const nexus_kv8_cache *c, const void *k, const void *v, int32_t dtype,
                        int32_t n_tokens) {
  if (!k || !v || n_tokens <= 0) return NEXUS_EINVAL;
  if (!dtype_bytes(dtype)) return NEXUS_EDTYPE;
  if ((uintptr_t)k % 16 != 0 || (uintptr_t)v % 16 != 0) return NEXUS_EINVAL;
  if ((int64_t)n_tokens * c->n_kv_heads * c->head_dim >= kMaxElems32) return NEXUS_ESHAPE;
  return NEXUS_OK;
}

nexus_status check_range(const nexus_page_table *pt, int64_t offset, int32_t n_tokens) {
  // (offset first: the sum must not overflow)
  const int64_t capacity = (int64_t)pt->n_logical_pages * kPageSize;
  if (offset < 0 || offset > capacity || offset + n_tokens > capacity) return NEXUS_ERANGE;
  return NEXUS_OK;
}

Kv8Cache device_cache(const nexus_kv8_cache *c) {
  Kv8Cache d{};
  d.k = (uint8_t *)c->k;
  d.v = (uint8_t *)c->v;
  d.ks = (uint8_t *)c->k_scale;
  d.vs = (uint8_t *)c->v_scale;
  d.n_layers = c->n_layers;
  d.n_phys_pages = c->n_phys_pages;
  d.n_heads = c->n_kv_heads;
  d.head_dim = c->head_dim;
  return d;
}

Kv8WriteLaunch write_launch(const nexus_kv8_cache *c, const void *k, const void *v, int32_t dtype,
                            int32_t n_tokens) {
  Kv8WriteLaunch L{};
  L.c = device_cache(c);
  L.src_k = k;
  L.src_v = v;
  L.dtype_bytes = dtype_bytes(dtype);
  L.n_tokens = n_tokens;
  L.interleaved = c->rope_style == NEXUS_ROPE_INTERLEAVED;
  L.rope_base = c->rope_base;
  return L;
}

// What the attention calls check alike.
nexus_status check_attention(const void *q, const void *out, int32_t n_q_heads, const nexus_kv8_cache *c,
                             int32_t layer, float softcap, float scale) {
  if (!q || !out) return NEXUS_EINVAL;
  if ((uintptr_t)q % 16 != 0 || (uintptr_t)out % 16 != 0) return NEXUS_EINVAL;
  if (layer < 0 || layer >= c->n_layers) return NEXUS_ERANGE;
  if (n_q_heads <= 0 || n_q_heads % c->n_kv_heads) return NEXUS_ESHAPE;
  if (!(softcap >= 0.f) || !isfinite(softcap)) return NEXUS_EINVAL;
  if (!(scale >= 0.f) || !isfinite(scale)) return NEXUS_EINVAL;
  return NEXUS_OK;
}

constexpr int32_t kMaxSuffixes = 32;
// Keys of a sequence: the kernel's positions are 32-bit, and those of a split's end (32768 keys at most), a key tile
// and a query block reach past the last one.
constexpr int64_t kMaxKeys = kMaxElems32 - 65536;

struct Suffixes {
  AttnSeq seq[kMaxSuffixes];
};

// Fills what the plan of a suffix launch depends on; n_seqs in [1, kMaxSuffixes], arrays non-null.
nexus_status plan_launch(int32_t n_seqs, const int32_t *q_start, const int32_t *seq_len,
                         const int64_t *seq_n_past, int32_t n_q_heads, const nexus_kv8_cache *c,
                         Suffixes &s, AttnLaunch &L) {
  int64_t rows = 0;
  for (int32_t b = 0; b < n_seqs; ++b) {
    s.seq[b] = AttnSeq{q_start[b], seq_len[b], seq_n_past[b]};
    if (seq_len[b] <= 0 || q_start[b] < 0) return NEXUS_EINVAL;
    if (seq_n_past[b] < 0 || seq_n_past[b] > kMaxKeys - seq_len[b]) return NEXUS_ERANGE;
    if ((int64_t)q_start[b] + seq_len[b] > kMaxElems32 / 1024) return NEXUS_ERANGE;
    rows += seq_len[b];
    for (int32_t o = 0; o < b; ++o)
      if (q_start[b] < q_start[o] + seq_len[o] && q_start[o] < q_start[b] + seq_len[b])
        return NEXUS_EINVAL;   // two writers of one output row
  }
  if (rows * n_q_heads * c->head_dim >= kMaxElems32) return NEXUS_ESHAPE;
  L = AttnLaunch{};
  L.n_kv_heads = c->n_kv_heads;
  L.n_q_heads = n_q_heads;
  L.head_dim = c->head_dim;
  L.is_bf16 = true;
  L.kv8 = true;
  L.n_seqs = n_seqs;
  L.seqs = s.seq;
  return NEXUS_OK;
}

nexus_status decode_launch(int32_t n_seqs, int32_t n_q_heads, const nexus_kv8_cache *c, int32_t max_seq_len,
                           DecodeLaunch &L) {
  if (n_seqs <= 0) return NEXUS_EINVAL;
  if (max_seq_len < 0 || max_seq_len > INT32_MAX - kPageSize) return NEXUS_ERANGE;   // (pages: rounded up)
  if (n_q_heads <= 0 || n_q_heads % c->n_kv_heads) return NEXUS_ESHAPE;
  // grid limits and 32-bit row offsets of q and out
  if (n_seqs > 65535 || n_q_heads > 65535) return NEXUS_ESHAPE;
  if ((int64_t)n_seqs * n_q_heads * c->head_dim >= kMaxElems32) return NEXUS_ESHAPE;
  L = DecodeLaunch{};
  L.n_seqs = n_seqs;
  L.n_q_heads = n_q_heads;
  L.n_kv_heads = c->n_kv_heads;
  L.head_dim = c->head_dim;
  L.max_len = max_seq_len;
  L.is_bf16 = true;
  return NEXUS_OK;
}

}  // namespace

extern "C" {

nexus_status nexus_kv8_append(const nexus_kv8_cache *cache, const nexus_page_table *pt, const void *k,
                              const void *v, int32_t dtype, int32_t n_tokens, int64_t offset, int64_t pos0,
                              void *stream) {
  nexus_status st = check_kv8(cache);
  if (st) return st;
  if ((st = check_map(pt, cache))) return st;
  if ((st = check_rows(cache, k, v, dtype, n_tokens))) return st;
  if ((st = check_range(pt, offset, n_tokens))) return st;
  if (pos0 < 0 || pos0 > INT64_MAX - n_tokens) return NEXUS_ERANGE;
  Kv8WriteLaunch L = write_launch(cache, k, v, dtype, n_tokens);
  L.mode = Kv8WriteLaunch::kRange;
  L.map = pt->map;
  L.offset = offset;
  L.angle0 = pos0;
  return from_hip(launch_kv8_write(L, as_stream(stream)));
}

nexus_status nexus_kv8_append_step(const nexus_kv8_cache *cache, const int32_t *maps, int32_t map_stride,
                                   const int32_t *seq_len, int32_t n_seqs, int32_t max_seq_len,
                                   const void *k, const void *v, int32_t dtype, void *stream) {
  nexus_status st = check_kv8(cache);
  if (st) return st;
  if (!maps || !seq_len || map_stride <= 0 || n_seqs <= 0) return NEXUS_EINVAL;
  if (max_seq_len < 0 || (int64_t)map_stride * kPageSize < max_seq_len) return NEXUS_ERANGE;
  if ((st = check_rows(cache, k, v, dtype, n_seqs))) return st;
  if (max_seq_len == 0) return NEXUS_OK;
  Kv8WriteLaunch L = write_launch(cache, k, v, dtype, n_seqs);
  L.mode = Kv8WriteLaunch::kStep;
  L.map = maps;
  L.map_stride = map_stride;
  L.lens = seq_len;
  L.max_len = max_seq_len;
  return from_hip(launch_kv8_write(L, as_stream(stream)));
}

nexus_status nexus_kv8_splice(const nexus_kv8_cache *cache, const nexus_page_table *pt,
                              const nexus_block *block, int64_t offset, int64_t dst_pos, void *stream) {
  nexus_status st = check_kv8(cache);
  if (st) return st;
  if ((st = check_block(block))) return st;
  if ((st = check_map(pt, cache))) return st;
  if (block->n_layers != cache->n_layers || block->n_kv_heads != cache->n_kv_heads ||
      block->head_dim != cache->head_dim)
    return NEXUS_ESHAPE;
  if (block->rope_base != cache->rope_base || block->rope_style != cache->rope_style) return NEXUS_EROPE;
  if ((st = check_rows(cache, block->k, block->v, block->dtype, block->n_tokens))) return st;
  if ((st = check_range(pt, offset, block->n_tokens))) return st;
  if (dst_pos < 0) return NEXUS_ERANGE;
  Kv8WriteLaunch L = write_launch(cache, block->k, block->v, block->dtype, block->n_tokens);
  L.mode = Kv8WriteLaunch::kFixed;
  L.map = pt->map;
  L.offset = offset;
  L.angle0 = dst_pos - block->base_pos;
  return from_hip(launch_kv8_write(L, as_stream(stream)));
}

nexus_status nexus_kv8_read(const nexus_kv8_cache *cache, const nexus_page_table *pt, int64_t offset,
                            int32_t n_tokens, int32_t dtype, void *k, void *v, void *stream) {
  nexus_status st = check_kv8(cache);
  if (st) return st;
  if ((st = check_map(pt, cache))) return st;
  if ((st = check_rows(cache, k, v, dtype, n_tokens))) return st;
  if ((st = check_range(pt, offset, n_tokens))) return st;
  Kv8ReadLaunch L{};
  L.c = device_cache(cache);
  L.dst_k = k;
  L.dst_v = v;
  L.dtype_bytes = dtype_bytes(dtype);
  L.n_tokens = n_tokens;
  L.map = pt->map;
  L.offset = offset;
  return from_hip(launch_kv8_read(L, as_stream(stream)));
}

size_t nexus_kv8_suffix_attn_varlen_workspace(int32_t n_seqs, const int32_t *q_start,
                                              const int32_t *seq_len, const int64_t *seq_n_past,
                                              int32_t n_q_heads, const nexus_kv8_cache *cache) try {
  if (check_kv8(cache) || !q_start || !seq_len || !seq_n_past || n_seqs <= 0 || n_seqs > kMaxSuffixes ||
      n_q_heads <= 0 || n_q_heads % cache->n_kv_heads)
    return SIZE_MAX;
  Suffixes s;
  AttnLaunch L;
  if (plan_launch(n_seqs, q_start, seq_len, seq_n_past, n_q_heads, cache, s, L)) return SIZE_MAX;
  AttnPlan plan;
  return plan_attention(L, plan) ? plan.ws_bytes : SIZE_MAX;
} catch (const std::bad_alloc &) {
  return SIZE_MAX;
}

size_t nexus_kv8_suffix_attn_workspace(int32_t n_s, int32_t n_q_heads, const nexus_kv8_cache *cache,
                                       int64_t n_past) {
  const int32_t start = 0;
  return nexus_kv8_suffix_attn_varlen_workspace(1, &start, &n_s, &n_past, n_q_heads, cache);
}

nexus_status nexus_kv8_suffix_attn_varlen(const void *q, int32_t n_seqs, const int32_t *q_start,
                                          const int32_t *seq_len, const int64_t *seq_n_past,
                                          int32_t n_q_heads, const nexus_kv8_cache *cache,
                                          const nexus_page_table *pt, int32_t layer, float softcap,
                                          float scale, void *out, void *workspace, size_t workspace_bytes,
                                          void *stream) try {
  nexus_status st = check_kv8(cache);
  if (st) return st;
  if ((st = check_map(pt, cache))) return st;
  if ((st = check_attention(q, out, n_q_heads, cache, layer, softcap, scale))) return st;
  if (!q_start || !seq_len || !seq_n_past || n_seqs <= 0 || n_seqs > kMaxSuffixes) return NEXUS_EINVAL;
  Suffixes s;
  AttnLaunch L;
  if ((st = plan_launch(n_seqs, q_start, seq_len, seq_n_past, n_q_heads, cache, s, L))) return st;
  for (int32_t b = 0; b < n_seqs; ++b)
    if (seq_n_past[b] + seq_len[b] > (int64_t)pt->n_logical_pages * kPageSize) return NEXUS_ERANGE;
  AttnPlan plan;
  if (!plan_attention(L, plan)) return NEXUS_EINVAL;
  if (plan.ws_bytes > 0 &&
      (!workspace || workspace_bytes < plan.ws_bytes || (uintptr_t)workspace % 16 != 0))
    return NEXUS_EWORKSPACE;
  L.q = q;
  L.out = out;
  L.cache_k = cache->k;
  L.cache_v = cache->v;
  L.k_scale = (const uint8_t *)cache->k_scale;
  L.v_scale = (const uint8_t *)cache->v_scale;
  L.map = pt->map;
  L.layer = layer;
  L.n_layers = cache->n_layers;
  L.n_phys_pages = cache->n_phys_pages;
  L.scale = scale > 0.f ? scale : 1.0f / sqrtf((float)cache->head_dim);
  L.softcap = softcap;
  L.workspace = workspace;
  L.workspace_bytes = workspace ? workspace_bytes : 0;
  return from_hip(launch_attention_kv8(L, plan, as_stream(stream)));
} catch (const std::bad_alloc &) {
  return NEXUS_EHIP;
}

nexus_status nexus_kv8_suffix_attn(const void *q, int32_t n_s, int32_t n_q_heads,
                                   const nexus_kv8_cache *cache, const nexus_page_table *pt, int32_t layer,
                                   int64_t n_past, float softcap, float scale, void *out, void *workspace,
                                   size_t workspace_bytes, void *stream) {
  const int32_t start = 0;
  return nexus_kv8_suffix_attn_varlen(q, 1, &start, &n_s, &n_past, n_q_heads, cache, pt, layer, softcap,
                                      scale, out, workspace, workspace_bytes, stream);
}

size_t nexus_kv8_decode_attn_workspace(int32_t n_seqs, int32_t n_q_heads, const nexus_kv8_cache *cache,
                                       int32_t max_seq_len) {
  DecodeLaunch L;
  if (check_kv8(cache) || decode_launch(n_seqs, n_q_heads, cache, max_seq_len, L)) return SIZE_MAX;
  return decode_kv8_workspace_bytes(L);
}

nexus_status nexus_kv8_decode_attn(const void *q, int32_t n_seqs, int32_t n_q_heads,
                                   const nexus_kv8_cache *cache, const int32_t *maps, int32_t map_stride,
                                   const int32_t *seq_len, int32_t max_seq_len, int32_t layer,
                                   float softcap, float scale, void *out, void *workspace,
                                   size_t workspace_bytes, void *stream) {
  nexus_status st = check_kv8(cache);
  if (st) return st;
  if ((st = check_attention(q, out, n_q_heads, cache, layer, softcap, scale))) return st;
  if (!maps || !seq_len || map_stride <= 0) return NEXUS_EINVAL;
  DecodeLaunch L;
  if ((st = decode_launch(n_seqs, n_q_heads, cache, max_seq_len, L))) return st;
  if ((int64_t)map_stride * kPageSize < max_seq_len) return NEXUS_ERANGE;
  if ((int64_t)n_seqs * map_stride >= kMaxElems32) return NEXUS_ESHAPE;
  const size_t need = decode_kv8_workspace_min(L);
  const bool usable = workspace && (uintptr_t)workspace % 16 == 0;
  if (need > 0 && (!usable || workspace_bytes < need)) return NEXUS_EWORKSPACE;
  L.q = q;
  L.out = out;
  L.cache_k = cache->k;
  L.cache_v = cache->v;
  L.k_scale = (const uint8_t *)cache->k_scale;
  L.v_scale = (const uint8_t *)cache->v_scale;
  L.maps = maps;
  L.lens = seq_len;
  L.map_stride = map_stride;
  L.layer = layer;
  L.n_phys_pages = cache->n_phys_pages;
  L.scale = scale > 0.f ? scale : 1.0f / sqrtf((float)cache->head_dim);
  L.softcap = softcap;
  L.workspace = workspace;
  L.workspace_bytes = usable ? workspace_bytes : 0;
  return from_hip(launch_decode_kv8(L, as_stream(stream)));
}

}  // extern "C"
