// Host checks and conversions shared by the C entry points (internal, not part of the C ABI).
#pragma once

#include "nexus.h"

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

namespace nexus {

constexpr int kPageSize = 16;
constexpr int64_t kMaxElems32 = (int64_t)1 << 31;

inline int dtype_bytes(int32_t dt) { return dt == NEXUS_BF16 ? 2 : dt == NEXUS_F32 ? 4 : 0; }

inline bool valid_style(int32_t s) { return s == NEXUS_ROPE_NEOX || s == NEXUS_ROPE_INTERLEAVED; }
inline bool valid_layout(int32_t v) { return v == NEXUS_V_ROWMAJOR || v == NEXUS_V_TRANSPOSED; }

// rows of 16-byte chunks must tile head_dim, and pairs must tile whole 16-byte chunks
inline bool head_dim_ok(int32_t head_dim, int esize) {
  if (head_dim <= 0 || head_dim % 2) return false;
  const int per16 = 16 / esize;
  if (head_dim % (2 * per16)) return false;           // rephase: pairs per thread
  const int chunks = head_dim * esize / 16;
  if (chunks & (chunks - 1)) return false;            // splice: power-of-two chunks per row
  return head_dim <= 1024;
}

inline nexus_status check_block(const nexus_block *b) {
  if (!b || !b->k || !b->v) return NEXUS_EINVAL;
  if (b->n_layers <= 0 || b->n_tokens <= 0 || b->n_kv_heads <= 0 || b->head_dim <= 0)
    return NEXUS_EINVAL;
  const int es = dtype_bytes(b->dtype);
  if (!es) return NEXUS_EDTYPE;
  if (!valid_style(b->rope_style)) return NEXUS_EINVAL;
  if (!head_dim_ok(b->head_dim, es)) return NEXUS_ESHAPE;
  if (b->n_layers > 65535) return NEXUS_ESHAPE;
  if ((int64_t)b->n_tokens * b->n_kv_heads * b->head_dim >= kMaxElems32) return NEXUS_ESHAPE;
  if ((int64_t)b->n_layers * b->n_tokens * b->n_kv_heads >= kMaxElems32) return NEXUS_ESHAPE;
  if (!(b->rope_base > 1.0) || !isfinite(b->rope_base)) return NEXUS_EROPE;
  if (b->base_pos < 0) return NEXUS_ERANGE;
  return NEXUS_OK;
}

inline nexus_status from_hip(hipError_t e) { return e == hipSuccess ? NEXUS_OK : NEXUS_EHIP; }

inline hipStream_t as_stream(void *s) { return reinterpret_cast<hipStream_t>(s); }

}  // namespace nexus
