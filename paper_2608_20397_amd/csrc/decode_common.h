// Shared definitions of the decode-step attention kernels (internal, not part of the C ABI): arguments,
// key splits, wave reductions and partial results.
#pragma once

#include "device_common.h"

namespace nexus {

constexpr int kDecWaves = 4;
// log2 units the reference may lag behind the running maximum.  A moved reference gives the key it
// moves to the probability 1, which bf16 holds exactly, and a few top keys carry much of the
// rounding error: 32 sequences of 17473 keys, relative error against 64 bits 2.20e-3 at a lag of
// 8, 2.08e-3 at 6, 2.04e-3 at 4 (2.15e-3 at 8 with pages taken one by one).
constexpr float kDecSlack = 6.0f;
constexpr int kMaxDecSplits = 1024; // splits per sequence at most (bounds the merge's loop)
constexpr int kMaxSplitPages = 2048;  // pages per split at most (page list in LDS)

struct DecodeArgs {
  const void *q;
  void *out;
  const void *kc;         // layer base of the K cache [NPP][Hkv][16][D]
  const void *vc;         // layer base of V: as K, or [Hkv][D][NPP * 16] when transposed
  const int32_t *maps;    // [n_seqs][map_stride]
  const int32_t *lens;    // [n_seqs]
  float *part;            // [n_seqs][Hq][max_splits][D] unnormalised split outputs
  float *part_ml;         // [n_seqs][Hq][max_splits][2] (reference m, row sum l)
  int32_t map_stride, max_len, n_q_heads, n_kv_heads, group, n_qgroups;
  int32_t split_pages, max_splits;      // max_splits: partial slots per row
  int32_t n_seqs;
  // shared pages (0 groups: none looked for): slots own_splits .. max_splits - 1 of a row belong
  // to the page ranges of its group
  int32_t n_groups, group_seqs, shared_splits, own_splits;
  int32_t share_pages;    // whole pages from which on a sequence is long enough to share them
  int32_t *flags;         // [n_seqs]: ranges of shared pages a sequence has partials of (the merge's use)
  uint32_t n_cols;        // transposed V: NPP * 16
  float scale_log2;       // scale * log2(e)
  float cap_in;           // scale / softcap
  float cap_out;          // softcap * log2(e)
  const uint8_t *ks = nullptr, *vs = nullptr;   // 8-bit cache: layer bases of the scale bytes [NPP][Hkv][16]
};

__device__ __forceinline__ float max_x16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_x32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_x16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float sum_x32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Sequence length as the kernels read it: clamped to [0, max_len].
__device__ __forceinline__ int seq_len_of(const DecodeArgs &a, int b) {
  return min(max(a.lens[b], 0), a.max_len);
}

// 16-byte chunk c of row r of a staged V page lives at chunk c ^ vswz(r): the 16 rows of one
// transposed read (32 bytes each) and the 4 rows of one staging write cover distinct banks.
template <int D>
__device__ __forceinline__ int vswz(int r) {
  return D == 64 ? 2 * ((r >> 1) & 3) : 2 * (r & 7);
}

// Writes the partial (O unnormalised, m, l) of a lane's row; a negative row is skipped.
template <int D>
__device__ __forceinline__ void store_part(const DecodeArgs &a, int row, int slot_of_row,
                                           const f32x4 (&o)[D / 16], float m, float l, int grp) {
  if (row < 0) return;
  const size_t slot = (size_t)row * a.max_splits + slot_of_row;
#pragma unroll
  for (int t = 0; t < D / 16; ++t)
    *reinterpret_cast<f32x4 *>(a.part + slot * D + 16 * t + 4 * grp) = o[t];
  if (grp == 0) {
    a.part_ml[2 * slot] = m;
    a.part_ml[2 * slot + 1] = l;
  }
}

// Merges the partials of every row that has more than one (decode_combine_kernel).
hipError_t launch_decode_combine(const DecodeArgs &a, int head_dim, bool bf16, hipStream_t stream);

}  // namespace nexus
