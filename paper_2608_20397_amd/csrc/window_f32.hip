// Windowed attention over fp32 caches (many rows or one a sequence), the merge of split results and the launch of all
// windowed attention.
//
// fp32: a workgroup is 16 (token, head of the group) pairs of one sequence and KV head; its 4 waves take the pages of
// the list in turn, S^T = K.Q^T and O^T += V^T.P^T on 16x16x4 fp32 MFMA straight from global memory, and merge their
// (m, l, O) through LDS.  Scores, probabilities and sums are fp32 throughout.
#include "decode_common.h"
#include "window_common.h"

#include <algorithm>
#include <type_traits>

namespace nexus {

namespace {

constexpr int kF32Rows = 16;       // (token, head) pairs of an fp32 workgroup
constexpr int kMfmaRows = 128;     // of a bf16 one (window_attn.hip)
constexpr int kWideRows = 256;     // of one of head_dim 256 (window_d256.hip)
constexpr int kMaxSplits = 64;     // of a row's keys: the merge holds one in each lane

}  // namespace

template <int D, bool VT, bool CAP>
__global__ __launch_bounds__(256) void window_f32_kernel(const WindowArgs a) {
  constexpr int DT = D / 16;          // O^T tiles, and 16-feature steps of S^T
  constexpr int MO_LD = D + 4;        // padded row of the merge buffer
  __shared__ float mo[2 * 16 * MO_LD];
  __shared__ float mml[2 * 2 * 16];
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qn = lane & 15, grp = lane >> 4;
  const int kvh = blockIdx.x % a.n_kv_heads;
  const uint32_t rest = blockIdx.x / a.n_kv_heads;
  const int split = rest % a.n_splits;
  const uint32_t u = a.n_units / a.n_kv_heads - 1 - rest / a.n_splits;
  const RowTile rt = find_tile<kF32Rows>(a, u);
  if (rt.b < 0) return;
  const int G = a.group;
  const bool direct = a.n_splits == 1;
  const int pair = min(rt.i0 + qn, rt.n - 1);
  const bool row_ok = rt.i0 + qn < rt.n;
  const int tok = pair / G, qhead = kvh * G + pair - tok * G;
  const size_t row = (size_t)(rt.row0 + tok) * a.n_q_heads + qhead;
  const int pos = rt.past + tok;
  const int p0 = rt.past + rt.i0 / G, p1 = rt.past + min(rt.i0 + kF32Rows - 1, rt.n - 1) / G;
  KeyList kl{};
  int e0 = 0, e1 = 0;
  if (p1 >= 0) {
    kl = key_list(a.window, a.sinks, p0, p1);
    e0 = (int)((int64_t)kl.n * split / a.n_splits);
    e1 = (int)((int64_t)kl.n * (split + 1) / a.n_splits);
  }
  const float *q = reinterpret_cast<const float *>(a.q) + row * D;
  f32x4 qreg[DT];
#pragma unroll
  for (int s = 0; s < DT; ++s) qreg[s] = *reinterpret_cast<const f32x4 *>(q + 16 * s + 4 * grp);

  f32x4 o[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, lsum = 0.f;
  const float *kc = reinterpret_cast<const float *>(a.kc), *vc = reinterpret_cast<const float *>(a.vc);
  const int32_t *map = a.maps + (size_t)rt.b * a.map_stride;
  const float c_scale = CAP ? 1.0f : a.scale_log2;
  for (int e = e0 + wave; e < e1; e += 4) {
    const int page = kl.page(e), key0 = page * kPage;
    const uint32_t phys = (uint32_t)map[page];
    auto from = [&](int s) { return kl.stand_in(key0 + s) & (kPage - 1); };
    const size_t base = ((size_t)phys * a.n_kv_heads + kvh) * kPage * D;
    // lane qn feeds key row qn, features 16 s + 4 grp + i as the k index grp of step (s, i); Q alike
    const float *kr = kc + base + from(qn) * D + 4 * grp;
    f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = 0; st < DT; ++st) {
      const f32x4 k = *reinterpret_cast<const f32x4 *>(kr + 16 * st);
#pragma unroll
      for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i], qreg[st][i], s, 0, 0, 0);
    }
    // the lane's scores: keys 4 grp + i of query column qn
    float x[4], mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int key = key0 + 4 * grp + i;
      const bool vis = key <= pos && (key > pos - a.window || key < a.sinks);
      x[i] = vis ? (CAP ? a.cap_out * tanhf(s[i] * a.cap_in) : s[i]) : -INFINITY;
      mx = fmaxf(mx, x[i]);
    }
    mx = max_x32(max_x16(mx)) * c_scale;
    const float nm = fmaxf(m, mx), ref = nm == -INFINITY ? 0.f : nm;
    const float alpha = nm == -INFINITY ? 1.f : fast_exp2(m - nm);
    m = nm;
    float p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = fast_exp2(fmaf(x[i], c_scale, -ref));
    lsum = fmaf(lsum, alpha, (p[0] + p[1]) + (p[2] + p[3]));
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      f32x4 v;
      if constexpr (VT) {
        v = *reinterpret_cast<const f32x4 *>(vc + ((size_t)kvh * D + 16 * t + qn) * a.n_cols +
                                             (size_t)phys * kPage + 4 * grp);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = kl.seen(key0 + 4 * grp + i) ? v[i] : 0.f;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = vc[base + from(4 * grp + i) * D + 16 * t + qn];
      }
      o[t] *= alpha;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[i], p[i], o[t], 0, 0, 0);
    }
  }

  // ---- merge the 4 waves, pairwise
  lsum = sum_x32(sum_x16(lsum));
  auto store_state = [&](int s) {
#pragma unroll
    for (int t = 0; t < DT; ++t)
      *reinterpret_cast<f32x4 *>(mo + (s * 16 + qn) * MO_LD + 16 * t + 4 * grp) = o[t];
    if (grp == 0) {
      mml[2 * (s * 16 + qn)] = m;
      mml[2 * (s * 16 + qn) + 1] = lsum;
    }
  };
  auto merge_state = [&](int s) {
    const float mb = mml[2 * (s * 16 + qn)], lb = mml[2 * (s * 16 + qn) + 1];
    const float M = fmaxf(m, mb);
    const float wa = m > -INFINITY ? fast_exp2(m - M) : m == M ? 1.f : 0.f;
    const float wb = mb > -INFINITY ? fast_exp2(mb - M) : mb == M ? 1.f : 0.f;
#pragma unroll
    for (int t = 0; t < DT; ++t)
      o[t] = o[t] * wa + *reinterpret_cast<const f32x4 *>(mo + (s * 16 + qn) * MO_LD + 16 * t + 4 * grp) * wb;
    lsum = lsum * wa + lb * wb;
    m = M;
  };
  if (wave >= 2) store_state(wave - 2);
  __syncthreads();
  if (wave < 2) merge_state(wave);
  __syncthreads();
  if (wave == 1) store_state(0);
  __syncthreads();
  if (wave != 0) return;
  merge_state(0);

  const bool empty = pos < 0 || e0 == e1;
  const float inv = direct ? (empty ? 0.f : 1.0f / lsum) : lsum > 0.f ? 1.0f / lsum : 0.f;
  float check = 0.f;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[t][i] = empty ? 0.f : o[t][i] * inv;       // (0 x NaN is NaN)
      check = fmaf(o[t][i], 0.f, check);
    }
  check = sum_x32(sum_x16(check));
  const bool bad = row_ok && !empty && (!(check == 0.f) || lsum != lsum);
  const size_t slot = (size_t)split * a.n_rows * a.n_q_heads + row;
  if (row_ok && !bad) {
    float *to = direct ? reinterpret_cast<float *>(a.out) + row * D : a.part + slot * D;
#pragma unroll
    for (int t = 0; t < DT; ++t) *reinterpret_cast<f32x4 *>(to + 16 * t + 4 * grp) = o[t];
    if (!direct && grp == 0) a.part_ml[slot] = float2{part_max(m, pos >= 0, split), empty ? 0.f : lsum};
  }
  uint32_t left = (uint32_t)__builtin_amdgcn_ballot_w64(bad && grp == 0);
  while (left) {
    const int r = __builtin_ctz(left);
    left &= left - 1;
    const int rp = __builtin_amdgcn_readlane(pair, r), rtok = rp / G, rhead = kvh * G + rp - rtok * G;
    const size_t rrow = (size_t)(rt.row0 + rtok) * a.n_q_heads + rhead;
    float res[(D + 63) / 64], ma, la;
    row_again<float, D, VT, CAP>(a, kl, rt.b, kvh, reinterpret_cast<const float *>(a.q) + rrow * D, rt.past + rtok,
                                 e0, e1, res, ma, la);
    store_again<float, D>(a, rrow, split, direct, res, ma, la);
  }
}

hipError_t launch_window_f32(const WindowArgs &a, int head_dim, bool vt, bool cap, hipStream_t stream) {
  const dim3 grid(a.n_units * a.n_splits);
  auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a);
    return hipGetLastError();
  };
  auto with_d = [&](auto d) {
    if (vt) return cap ? run(window_f32_kernel<d(), true, true>) : run(window_f32_kernel<d(), true, false>);
    return cap ? run(window_f32_kernel<d(), false, true>) : run(window_f32_kernel<d(), false, false>);
  };
  switch (head_dim) {
    case 16: return with_d(std::integral_constant<int, 16>{});
    case 32: return with_d(std::integral_constant<int, 32>{});
    case 64: return with_d(std::integral_constant<int, 64>{});
    case 128: return with_d(std::integral_constant<int, 128>{});
    default: return with_d(std::integral_constant<int, 256>{});
  }
}

namespace {

// Merge of a row's splits: out = sum w_s O_s / sum w_s with w_s = l_s 2^(m_s - M), in split order within each share of
// the wave.  One wave a (row, query head); lane s holds (m, l) of split s.  Rows of no sequence stay as they are.
template <bool BF16>
__global__ __launch_bounds__(256) void window_combine_kernel(const WindowArgs a, int D, int lpr_shift) {
  const int lane = threadIdx.x & 63;
  const uint32_t row = blockIdx.x * 4 + (threadIdx.x >> 6);       // row of q and out, times heads, plus head
  if (row >= (uint32_t)a.n_rows * a.n_q_heads) return;
  if (a.q_start != nullptr) {
    const int r = row / a.n_q_heads;
    if (r < row_start(a, 0) || r >= row_start(a, a.n_seqs)) return;
  }
  const size_t stride = (size_t)a.n_rows * a.n_q_heads;
  const float2 ml = lane < a.n_splits ? a.part_ml[lane * stride + row] : float2{-INFINITY, 0.f};
  const int share = lane >> lpr_shift, n_shares = 64 >> lpr_shift;
  const int d = 4 * (lane & ((1 << lpr_shift) - 1));
  float M = ml.x;
  for (int off = 32; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor(M, off));
  // (l is NaN where scores were; an empty split's partial holds nothing)
  const float w = ml.y == 0.f ? 0.f : ml.y * (M == -INFINITY ? 1.f : fast_exp2(ml.x - M));
  float total = w;
  for (int off = 32; off > 0; off >>= 1) total += __shfl_xor(total, off);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < a.n_splits; s0 += n_shares) {
    const int s = s0 + share;
    const float ls = __shfl(ml.y, s & 63), ws = __shfl(w, s & 63);
    if (s < a.n_splits && ls != 0.f)
      o += *reinterpret_cast<const f32x4 *>(a.part + (s * stride + row) * D + d) * ws;
  }
  for (int off = 32; off >= 1 << lpr_shift; off >>= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], off);
  if (share != 0) return;
  // no key at all: zeros
  if (M == -INFINITY && total == 0.f) total = 1.f;
  const float inv = 1.0f / total;
  if (BF16)
    *reinterpret_cast<u32x2 *>(reinterpret_cast<uint16_t *>(a.out) + (size_t)row * D + d) =
        u32x2{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
  else
    *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(a.out) + (size_t)row * D + d) = o * inv;
}

int64_t tile_rows(const WindowLaunch &p) {
  return !p.is_bf16 ? kF32Rows : p.head_dim == 256 ? kWideRows : kMfmaRows;
}

// (row tile, KV head) pairs of a launch; sequences of a decode step take theirs by query group in bf16.
int64_t window_units(const WindowLaunch &p) {
  const int64_t group = p.n_q_heads / p.n_kv_heads;
  if (p.q_start == nullptr) {
    const int64_t per = (group + 15) / 16;
    return p.n_seqs * p.n_kv_heads * per;
  }
  const int64_t r = tile_rows(p);
  return (p.n_rows * group / r + p.n_seqs) * p.n_kv_heads;
}

// Splits of the keys: as many as fill the chip once, of at least 4 tiles (256 keys) each.
int window_splits(const WindowLaunch &p) {
  const int64_t group = p.n_q_heads / p.n_kv_heads, units = window_units(p);
  // workgroups the chip holds at once
  const int64_t slots = p.q_start != nullptr && p.is_bf16 && p.head_dim == 256 ? 256 : 512;
  const int64_t rows = p.q_start == nullptr ? 1 : tile_rows(p) / group + 1;
  const int64_t keys = std::min<int64_t>((int64_t)p.window + p.sinks + rows + 32, p.max_len);
  int64_t s = std::min<int64_t>((slots + units - 1) / units, (keys + 255) / 256);
  return (int)std::max<int64_t>(1, std::min<int64_t>(s, kMaxSplits));
}

}  // namespace

size_t window_workspace_bytes(const WindowLaunch &p) {
  const size_t s = (size_t)window_splits(p);
  return s == 1 ? 0 : s * p.n_rows * p.n_q_heads * (p.head_dim + 2) * sizeof(float);
}

bool window_grid_ok(const WindowLaunch &p) { return window_units(p) * window_splits(p) < (1 << 24); }

hipError_t launch_window(const WindowLaunch &p, hipStream_t stream) {
  WindowArgs a{};
  a.q = p.q;
  a.out = p.out;
  a.kc = p.cache_k;
  a.vc = p.cache_v;
  a.maps = p.maps;
  a.q_start = p.q_start;
  a.lens = p.seq_len;
  a.map_stride = p.map_stride;
  a.max_len = p.max_len;
  a.n_seqs = p.n_seqs;
  a.n_rows = p.n_rows;
  a.n_q_heads = p.n_q_heads;
  a.n_kv_heads = p.n_kv_heads;
  a.group = p.n_q_heads / p.n_kv_heads;
  a.n_qgroups = (a.group + 15) / 16;
  a.window = p.window;
  a.sinks = p.sinks;
  a.n_splits = window_splits(p);
  a.n_cols = (uint32_t)p.n_phys_pages * 16u;
  a.n_units = (uint32_t)window_units(p);
  a.part = reinterpret_cast<float *>(p.workspace);
  a.part_ml = a.n_splits == 1 ? nullptr
                              : reinterpret_cast<float2 *>(a.part + (size_t)a.n_splits * p.n_rows * p.n_q_heads *
                                                                        p.head_dim);
  const float log2e = 1.4426950408889634f;
  a.scale_log2 = p.scale * log2e;
  a.cap_in = p.softcap > 0.f ? p.scale / p.softcap : 0.f;
  a.cap_out = p.softcap * log2e;
  a.cap_k = p.softcap > 0.f ? 2.0f * p.scale * log2e / p.softcap : 0.f;
  const bool cap = p.softcap > 0.f;
  hipError_t e;
  if (!p.is_bf16) e = launch_window_f32(a, p.head_dim, p.v_transposed, cap, stream);
  else if (p.q_start == nullptr) e = launch_window_decode(a, p.head_dim, p.v_transposed, cap, stream);
  else if (p.head_dim == 256) e = launch_window_d256(a, p.v_transposed, cap, stream);
  else e = launch_window_rows(a, p.head_dim, p.v_transposed, cap, stream);
  if (e != hipSuccess || a.n_splits == 1) return e;
  const dim3 grid(((uint32_t)p.n_rows * p.n_q_heads + 3) / 4);
  int lpr_shift = 0;                  // log2 of the lanes that cover a partial row
  while ((4 << lpr_shift) < p.head_dim) ++lpr_shift;
  if (p.is_bf16) hipLaunchKernelGGL((window_combine_kernel<true>), grid, dim3(256), 0, stream, a, p.head_dim, lpr_shift);
  else hipLaunchKernelGGL((window_combine_kernel<false>), grid, dim3(256), 0, stream, a, p.head_dim, lpr_shift);
  return hipGetLastError();
}

}  // namespace nexus
