// Internal launch descriptors of the ragged-batch calls (pages and slots, head norms with rotation and append,
// windowed attention), between the C-ABI layer (nexus_batch.cpp) and the kernels.  Every descriptor has been
// validated by the caller.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace nexus {

constexpr int kMaxBatchSeqs = 8192;    // sequences of a batch_pages launch (12 bytes of LDS each)

// What a sequence of a layout asks for, and whether it gets it behind the rows and pages that the ones before it asked
// for.  Rows are counted as they are asked for, not cut to the launch's: a sequence that alone is longer than the
// launch is refused too.
struct BatchAsk {
  int64_t rows;           // its fresh tokens, a negative count as none
  int32_t pages;          // new ones, or -1: its lengths are not valid
};
__host__ __device__ inline int32_t batch_pages_of(int64_t tokens) { return (int32_t)((tokens + 15) >> 4); }
__host__ __device__ inline BatchAsk batch_ask(int32_t cached, int32_t fresh, int64_t capacity) {
  BatchAsk a;
  const int64_t n = (int64_t)cached + fresh;
  a.rows = fresh > 0 ? fresh : 0;
  a.pages = cached < 0 || fresh < 0 || n > capacity ? -1 : batch_pages_of(n) - batch_pages_of(cached);
  return a;
}
__host__ __device__ inline bool batch_grants(const BatchAsk &a, int64_t rows_before, int64_t pages_before,
                                             int32_t max_tokens, int32_t n_free) {
  return a.pages >= 0 && (a.rows == 0 || rows_before + a.rows <= max_tokens) &&
         (a.pages == 0 || pages_before + a.pages <= n_free);
}

struct BatchPagesLaunch {
  const int32_t *cached, *fresh;      // [n_seqs]
  const int32_t *free_pages, *n_free; // [free_capacity], [1]
  int32_t *maps;                      // [n_seqs][map_stride]
  int32_t *q_start, *seq_len;         // [n_seqs + 1], [n_seqs]
  int32_t *pos, *slot;                // [max_tokens]
  int32_t *n_left;                    // [1]
  int32_t n_seqs, free_capacity, map_stride, max_tokens;
};
hipError_t launch_batch_pages(const BatchPagesLaunch &p, hipStream_t stream);

struct NormRopeLaunch {
  const void *q, *k, *v;              // rows of n heads x head_dim, strides in elements
  int64_t q_stride, k_stride, v_stride;
  void *q_out;                        // [n_tokens][n_q_heads][head_dim]
  void *cache_k, *cache_v;            // layer bases
  const float *q_weight, *k_weight;   // [head_dim] or null
  const int32_t *pos, *slot;          // [n_tokens]
  int32_t n_tokens, n_q_heads, n_kv_heads, head_dim, n_phys_pages;
  int32_t dtype_bytes;
  bool v_transposed, interleaved;
  float eps;                          // 0: no norm
  double rope_base;
};
hipError_t launch_norm_rope(const NormRopeLaunch &p, hipStream_t stream);

// Windowed attention: rows of several sequences (q_start given) or one row a sequence (q_start null).
struct WindowLaunch {
  const void *q;
  void *out;
  const void *cache_k, *cache_v;      // layer bases
  const int32_t *maps, *q_start, *seq_len;
  int32_t map_stride, max_len, n_seqs, n_rows;
  int32_t n_phys_pages, n_kv_heads, n_q_heads, head_dim;
  int32_t window, sinks;              // window >= 1, sinks >= 0, both at most max(max_len, 1)
  bool v_transposed, is_bf16;
  float scale;                        // resolved (never 0)
  float softcap;                      // 0 = off
  int32_t n_splits;                   // of the keys (plan_window)
  void *workspace;
};
// Chooses n_splits by the sizes (of pointers only q_start's being there counts); false: too many workgroups.
bool plan_window(WindowLaunch &p);
// Workspace bytes of a planned launch.
size_t window_workspace_bytes(const WindowLaunch &p);
hipError_t launch_window(const WindowLaunch &p, hipStream_t stream);

}  // namespace nexus
