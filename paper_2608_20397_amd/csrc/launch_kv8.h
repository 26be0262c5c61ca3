// Internal launch descriptors of the 8-bit cache's kernels, between the C-ABI layer (nexus_kv8.cpp) and
// the kernels.  Every descriptor has been validated by the caller.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "launch.h"
#include "launch_decode.h"

namespace nexus {

// The cache: codes [L][NPP][H][16][D], scale bytes [L][NPP][H][16].
struct Kv8Cache {
  uint8_t *k, *v, *ks, *vs;
  int32_t n_layers, n_phys_pages, n_heads, head_dim;
};

// Rows quantised into pages, keys rotated on the way.
struct Kv8WriteLaunch {
  Kv8Cache c;
  const void *src_k, *src_v;       // [L][T][H][D]
  int32_t dtype_bytes, n_tokens;
  bool interleaved;
  double rope_base;
  enum Mode { kFixed, kRange, kStep } mode;
  // kFixed: every key turned by angle0 positions; kRange: key j to position angle0 + j; both into logical
  // tokens offset + j of `map`
  const int32_t *map;
  int64_t offset, angle0;
  // kStep: key j to position lens[j] - 1 and into that token of map row j; lengths outside [1, max_len]
  // write nothing
  const int32_t *lens;
  int32_t map_stride, max_len;
};
hipError_t launch_kv8_write(const Kv8WriteLaunch &p, hipStream_t stream);

// Logical tokens offset .. + n_tokens as values, [L][T][H][D].
struct Kv8ReadLaunch {
  Kv8Cache c;
  void *dst_k, *dst_v;
  int32_t dtype_bytes, n_tokens;
  const int32_t *map;
  int64_t offset;
};
hipError_t launch_kv8_read(const Kv8ReadLaunch &p, hipStream_t stream);

// Suffix attention over an 8-bit cache (AttnLaunch::kv8 set), with the launch's plan (attn_common.h).
struct AttnPlan;
hipError_t launch_attention_kv8(const AttnLaunch &p, const AttnPlan &plan, hipStream_t stream);

// Decode step over an 8-bit cache (DecodeLaunch::k_scale and v_scale set).
size_t decode_kv8_workspace_bytes(const DecodeLaunch &p);   // all it can use
size_t decode_kv8_workspace_min(const DecodeLaunch &p);     // without shared pages
hipError_t launch_decode_kv8(const DecodeLaunch &p, hipStream_t stream);

}  // namespace nexus
