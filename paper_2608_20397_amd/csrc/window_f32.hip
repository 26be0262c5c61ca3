// Windowed attention over fp32 caches (many rows or one a sequence), the merge of split results and the launch of all
// windowed attention.
//
// fp32: a workgroup is 16 (token, head of the group) pairs of one sequence and KV head, or 32 (f32_blocks); its waves
// (f32_waves) take the pages of the list in turn, S^T = K.Q^T and O^T += V^T.P^T on 16x16x4 fp32 MFMA straight from
// global memory (a page's values and the next one's keys are loading while a page's scores are formed), and merge their
// (m, l, O) through LDS.  Scores, probabilities and sums are fp32 throughout.  122 rows of 4 heads of 64 in a window of
// 256: 8.3 us, a chain of round trips; 512 rows of 40 heads of 128 in one of 1024: 143 us, 76 TFLOP/s: a page serves 16
// pairs, 8 operations a byte, so keys and values come out of the caches at 9.5 TB/s; and five workgroups a CU of which
// four run together.  A decode step of 32 sequences, window 4096, 8 KV heads of 128: 184 us, 5.8 TB/s (transposed V 265).
#include "decode_common.h"
#include "window_common.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace nexus {

namespace {

constexpr int kPre = 8;            // partials of a row that a lane of the merge loads at once
// Of a row's keys, where rows are few: bounds the workspace (64 fp32 rows and records for each) and the merge, whose lanes
// take 0.7 us for each split beyond their first eight (a sequence of 17473 fp32 keys, 2 KV heads of 128 in 64 splits: 37
// us, 23 of them the merge; bf16, 8 of 256 in 32: 49, 23).
constexpr int kMaxSplits = 64;

}  // namespace

template <int D, bool VT, bool CAP, int NW, int RB>
__global__ __launch_bounds__(64 * NW, D == 256 || RB == 2 ? 2 : D == 128 ? 3 : 4) void window_f32_kernel(
    const WindowArgs a) {
  constexpr int DT = D / 16;          // O^T tiles, and 16-feature steps of S^T
  constexpr int MO_LD = D + 4;        // padded row of the merge buffer
  __shared__ float mo[NW / 2 * 16 * MO_LD];
  __shared__ float mml[NW / 2 * 2 * 16];
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qn = lane & 15, grp = lane >> 4;
  const int kvh = blockIdx.x % a.n_kv_heads;
  const uint32_t rest = blockIdx.x / a.n_kv_heads;
  const int split = rest % a.n_splits;
  const uint32_t u = a.n_units / a.n_kv_heads - 1 - rest / a.n_splits;
  static_assert(kF32Rows == 16, "columns of the MFMA");
  constexpr int R = kF32Rows * RB;    // pairs of the workgroup, in RB blocks
  const RowTile rt = find_tile<R>(a, u);
  if (rt.b < 0) return;
  const int G = a.group;
  const bool direct = a.n_splits == 1;
  // this lane's pair in each block
  int pair[RB], pos[RB];
  size_t row[RB];
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    pair[r] = min(rt.i0 + 16 * r + qn, rt.n - 1);
    const int tok = pair[r] / G;
    row[r] = (size_t)(rt.row0 + tok) * a.n_q_heads + kvh * G + pair[r] - tok * G;
    pos[r] = rt.past + tok;
  }
  const int p0 = rt.past + rt.i0 / G, p1 = rt.past + min(rt.i0 + R - 1, rt.n - 1) / G;
  KeyList kl{};
  int e0 = 0, e1 = 0;
  if (p1 >= 0) {
    kl = key_list(a.window, a.sinks, p0, p1);
    e0 = (int)((int64_t)kl.n * split / a.n_splits);
    e1 = (int)((int64_t)kl.n * (split + 1) / a.n_splits);
  }
  f32x4 qreg[RB][DT], o[RB][DT];
  float m[RB], lsum[RB];
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    const float *q = reinterpret_cast<const float *>(a.q) + row[r] * D;
#pragma unroll
    for (int s = 0; s < DT; ++s) qreg[r][s] = *reinterpret_cast<const f32x4 *>(q + 16 * s + 4 * grp);
#pragma unroll
    for (int t = 0; t < DT; ++t) o[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    m[r] = -INFINITY;
    lsum[r] = 0.f;
  }
  const float *kc = reinterpret_cast<const float *>(a.kc), *vc = reinterpret_cast<const float *>(a.vc);
  const int32_t *map = a.maps + (size_t)rt.b * a.map_stride;
  const float c_scale = CAP ? 1.0f : a.scale_log2;
  auto from = [&](int k) { return kl.stand_in(k) & (kPage - 1); };
  auto page_base = [&](uint32_t phys) { return ((size_t)phys * a.n_kv_heads + kvh) * kPage * D; };
  // A page's keys and values come in NH parts of the features.  In one: a page's values are loading while its scores are
  // formed, the next page's keys from there on.  In two (head_dim 256): both take the same registers in turn, a part's
  // values as soon as its keys have been used, the next page's keys as soon as the values have, so that a SIMD has two
  // waves (four sequences of 700 to 1557 rows from 0, transposed V, capped: 708 -> 594 us; 20 x 100 rows at 100 122 ->
  // 90).
  constexpr int NH = D == 256 ? 2 : 1, HT = DT / NH;
  // lane qn feeds key row qn, features 16 s + 4 grp + i as the k index grp of step (s, i); Q alike
  auto load_k = [&](f32x4 (&to)[HT], int h, int key0, uint32_t phys) {
    const float *kr = kc + page_base(phys) + from(key0 + qn) * D + 4 * grp + 16 * HT * h;
#pragma unroll
    for (int st = 0; st < HT; ++st) to[st] = *reinterpret_cast<const f32x4 *>(kr + 16 * st);
  };
  auto load_v = [&](f32x4 (&to)[HT], int h, int key0, uint32_t phys) {
    if constexpr (VT) {
      const float *vr = vc + ((size_t)kvh * D + 16 * HT * h + qn) * a.n_cols + (size_t)phys * kPage + 4 * grp;
#pragma unroll
      for (int t = 0; t < HT; ++t) to[t] = *reinterpret_cast<const f32x4 *>(vr + (size_t)(16 * t) * a.n_cols);
    } else {
      const float *vr = vc + page_base(phys) + qn + 16 * HT * h;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float *row = vr + from(key0 + 4 * grp + i) * D;       // (once a key, not once a feature block)
#pragma unroll
        for (int t = 0; t < HT; ++t) to[t][i] = row[16 * t];
      }
    }
  };
  f32x4 s2[RB][2];                    // two chains of MFMAs a block, added at the end
  auto scores = [&](const f32x4 (&k)[HT], int h) {
#pragma unroll
    for (int st = 0; st < HT; ++st)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < RB; ++r)
          s2[r][i & 1] =
              __builtin_amdgcn_mfma_f32_16x16x4f32(k[st][i], qreg[r][HT * h + st][i], s2[r][i & 1], 0, 0, 0);
  };
  float p[RB][4];
  auto outputs = [&](f32x4 (&v)[HT], int h, int key0) {
    if constexpr (VT) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool in = kl.seen(key0 + 4 * grp + i);    // other slots may hold anything
#pragma unroll
        for (int t = 0; t < HT; ++t) v[t][i] = in ? v[t][i] : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < HT; ++t)
#pragma unroll
        for (int r = 0; r < RB; ++r)
          o[r][HT * h + t] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[t][i], p[r][i], o[r][HT * h + t], 0, 0, 0);
  };
  f32x4 k[NH][HT], v[HT];
  int e = e0 + wave, page = 0;
  uint32_t phys = 0, phys_next = 0;
  if (e < e1) {
    page = kl.page(e);
    phys = (uint32_t)map[page];
    phys_next = (uint32_t)map[kl.page(min(e + NW, e1 - 1))];
#pragma unroll
    for (int h = 0; h < NH; ++h) load_k(k[h], h, page * kPage, phys);
  }
  for (; e < e1; e += NW) {
    const int key0 = page * kPage;
#pragma unroll
    for (int r = 0; r < RB; ++r) s2[r][0] = s2[r][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    if constexpr (NH == 1) {
      load_v(v, 0, key0, phys);
      scores(k[0], 0);
    } else {
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        scores(k[h], h);
        __builtin_amdgcn_sched_barrier(0);
        load_v(k[h], h, key0, phys);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    // the next page (past the list's end the last one again, unused)
    page = kl.page(min(e + NW, e1 - 1));
    phys = phys_next;
    if constexpr (NH == 1) load_k(k[0], 0, page * kPage, phys);
    phys_next = (uint32_t)map[kl.page(min(e + 2 * NW, e1 - 1))];
    // the lane's scores: keys 4 grp + i of query column qn
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      const f32x4 s = s2[r][0] + s2[r][1];
      float x[4], mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = key0 + 4 * grp + i;
        const bool vis = key <= pos[r] && (key > pos[r] - a.window || key < a.sinks);
        x[i] = vis ? (CAP ? a.cap_out * tanhf(s[i] * a.cap_in) : s[i]) : -INFINITY;
        mx = fmaxf(mx, x[i]);
      }
      mx = max_x32(max_x16(mx)) * c_scale;
      const float nm = fmaxf(m[r], mx), ref = nm == -INFINITY ? 0.f : nm;
      const float alpha = nm == -INFINITY ? 1.f : fast_exp2(m[r] - nm);
      m[r] = nm;
#pragma unroll
      for (int i = 0; i < 4; ++i) p[r][i] = fast_exp2(fmaf(x[i], c_scale, -ref));
      lsum[r] = fmaf(lsum[r], alpha, (p[r][0] + p[r][1]) + (p[r][2] + p[r][3]));
#pragma unroll
      for (int t = 0; t < DT; ++t) o[r][t] *= alpha;
    }
    if constexpr (NH == 1) {
      outputs(v, 0, key0);
    } else {
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        outputs(k[h], h, key0);
        __builtin_amdgcn_sched_barrier(0);
        load_k(k[h], h, page * kPage, phys);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }

  // ---- merge the waves, pairwise, a block at a time; wave 0 writes it
  auto finish = [&](f32x4 (&o)[DT], float m, float lsum, int pair, int pos, size_t row, bool row_ok, bool first) {
    lsum = sum_x32(sum_x16(lsum));
#pragma unroll
    for (int half = NW / 2; half > 0; half /= 2) {
      if (!first || half < NW / 2) __syncthreads();       // the slots of the step before have been read
      if (wave >= half && wave < 2 * half) {
        const int s = wave - half;
#pragma unroll
        for (int t = 0; t < DT; ++t)
          *reinterpret_cast<f32x4 *>(mo + (s * 16 + qn) * MO_LD + 16 * t + 4 * grp) = o[t];
        if (grp == 0) {
          mml[2 * (s * 16 + qn)] = m;
          mml[2 * (s * 16 + qn) + 1] = lsum;
        }
      }
      __syncthreads();
      if (wave < half) {
        const int s = wave;
        const float mb = mml[2 * (s * 16 + qn)], lb = mml[2 * (s * 16 + qn) + 1];
        const float M = fmaxf(m, mb);
        const float wa = m > -INFINITY ? fast_exp2(m - M) : m == M ? 1.f : 0.f;
        const float wb = mb > -INFINITY ? fast_exp2(mb - M) : mb == M ? 1.f : 0.f;
#pragma unroll
        for (int t = 0; t < DT; ++t)
          o[t] = o[t] * wa + *reinterpret_cast<const f32x4 *>(mo + (s * 16 + qn) * MO_LD + 16 * t + 4 * grp) * wb;
        lsum = lsum * wa + lb * wb;
        m = M;
      }
    }
    if (wave != 0) return;

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
      float *to = direct ? reinterpret_cast<float *>(a.out) + row * D : reinterpret_cast<float *>(a.part) + slot * D;
#pragma unroll
      for (int t = 0; t < DT; ++t) *reinterpret_cast<f32x4 *>(to + 16 * t + 4 * grp) = o[t];
      const float lw = empty ? 0.f : lsum;
      if (!direct && grp == 0) a.part_ml[slot] = f32x4{part_max(m, pos >= 0, split), lw, 0.f, 0.f};
    }
    uint32_t left = (uint32_t)__builtin_amdgcn_ballot_w64(bad && grp == 0);
    while (left) {
      const int j = __builtin_ctz(left);
      left &= left - 1;
      const int rp = __builtin_amdgcn_readlane(pair, j), rtok = rp / G, rhead = kvh * G + rp - rtok * G;
      const size_t rrow = (size_t)(rt.row0 + rtok) * a.n_q_heads + rhead;
      float res[(D + 63) / 64], ma, la;
      row_again<float, D, VT, CAP>(a, kl, rt.b, kvh, reinterpret_cast<const float *>(a.q) + rrow * D, rt.past + rtok,
                                   e1 - e0, [&](int i) { return e0 + i; }, res, ma, la);
      store_again<float, D, false>(a, rrow, split, direct, res, ma, la);
    }
  };
  finish(o[0], m[0], lsum[0], pair[0], pos[0], row[0], rt.i0 + qn < rt.n, true);
  if constexpr (RB == 2) finish(o[1], m[1], lsum[1], pair[1], pos[1], row[1], rt.i0 + 16 + qn < rt.n, false);
}

hipError_t launch_window_f32(const WindowArgs &a, int head_dim, bool vt, bool cap, int waves, int blocks,
                             hipStream_t stream) {
  const dim3 grid(a.n_units * a.n_splits);
  auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(64 * waves), 0, stream, a);
    return hipGetLastError();
  };
  auto with_w = [&](auto d, auto v, auto c) {
    if constexpr (d() == 128) {
      if (blocks == 2) return run(window_f32_kernel<d(), v(), c(), 4, 2>);
    }
    if (waves == 2) return run(window_f32_kernel<d(), v(), c(), 2, 1>);
    if constexpr (d() < 256) {
      if (waves == 8) return run(window_f32_kernel<d(), v(), c(), 8, 1>);
    }
    return run(window_f32_kernel<d(), v(), c(), 4, 1>);
  };
  auto with_v = [&](auto d, auto v) {
    return cap ? with_w(d, v, std::true_type{}) : with_w(d, v, std::false_type{});
  };
  auto with_d = [&](auto d) { return vt ? with_v(d, std::true_type{}) : with_v(d, std::false_type{}); };
  switch (head_dim) {
    case 16: return with_d(std::integral_constant<int, 16>{});
    case 32: return with_d(std::integral_constant<int, 32>{});
    case 64: return with_d(std::integral_constant<int, 64>{});
    case 128: return with_d(std::integral_constant<int, 128>{});
    default: return with_d(std::integral_constant<int, 256>{});
  }
}

namespace {

// Merge of a row's splits: out = sum w_s O_s, w_s = l_s 2^(m_s - M) / (their sum), in a fixed order.  The weights are
// divided by their sum before a partial is multiplied, so that finite partials have a finite result.  Rows of no sequence
// stay as they are.  A partial row lies in 2^lpr_shift lanes, 16 bytes each; 2^spr_shift neighbouring groups of them
// share the splits of a row, and what is left of the wave takes other rows.  The first eight partials of a group are
// loaded beside their (m, l), in one round trip; the ones behind them come one after another.
template <bool BF16, bool HALF>
__global__ __launch_bounds__(256) void window_combine_kernel(const WindowArgs a, int D, int lpr_shift, int spr_shift) {
  constexpr int E = HALF ? 8 : 4;
  constexpr int kRest = HALF ? 1 : 8;      // records of further splits at a time (rows in fp16 have 16 splits at most)
  const int lane = threadIdx.x & 63;
  const uint32_t n = (uint32_t)a.n_rows * a.n_q_heads;
  const uint32_t group = blockIdx.x * 4 + (threadIdx.x >> 6);
  const uint32_t row = (group << (6 - lpr_shift - spr_shift)) + (lane >> (lpr_shift + spr_shift));
  bool live = row < n;
  if (a.q_start != nullptr && live) {
    const int r = row / a.n_q_heads;
    live = r >= row_start(a, 0) && r < row_start(a, a.n_seqs);
  }
  const int spr = 1 << spr_shift, share = (lane >> lpr_shift) & (spr - 1);
  const int d = E * (lane & ((1 << lpr_shift) - 1));
  const int S = live ? a.n_splits : 0;
  auto load = [&](int s) {
    const size_t slot = (size_t)s * n + row;
    return *reinterpret_cast<const u32x4 *>(reinterpret_cast<const char *>(a.part) + (slot * D + d) * (16 / E));
  };
  u32x4 pre[kPre];
  f32x4 ml[kPre];
  float M = -INFINITY;
#pragma unroll
  for (int i = 0; i < kPre; ++i) {
    const int s = share + i * spr;
    if (s >= S) continue;
    pre[i] = load(s);
    ml[i] = a.part_ml[(size_t)s * n + row];
  }
#pragma unroll
  for (int i = 0; i < kPre; ++i)
    if (share + i * spr < S) M = fmaxf(M, ml[i][0]);
#pragma unroll kRest
  for (int s = share + kPre * spr; s < S; s += spr) M = fmaxf(M, a.part_ml[(size_t)s * n + row][0]);
  for (int off = 1 << lpr_shift; off < 1 << (lpr_shift + spr_shift); off <<= 1) M = fmaxf(M, __shfl_xor(M, off));
  // l 2^(m - M); 0 where nothing is seen (l is NaN where scores were)
  auto weight = [&](const f32x4 &r) { return r[1] == 0.f ? 0.f : r[1] * (M == -INFINITY ? 1.f : fast_exp2(r[0] - M)); };
  float total = 0.f;
#pragma unroll
  for (int i = 0; i < kPre; ++i) {
    if (share + i * spr >= S) continue;
    ml[i][3] = weight(ml[i]);
    total += ml[i][3];
  }
#pragma unroll kRest
  for (int s = share + kPre * spr; s < S; s += spr) total += weight(a.part_ml[(size_t)s * n + row]);
  for (int off = 1 << lpr_shift; off < 1 << (lpr_shift + spr_shift); off <<= 1) total += __shfl_xor(total, off);
  if (M == -INFINITY && total == 0.f) total = 1.f;      // no key at all: zeros
  const float inv = 1.0f / total;
  float o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f * inv;         // (NaN where every score is -inf: 0 / 0)
  auto add = [&](const f32x4 &r, float w, const u32x4 &x) {
    if (r[1] == 0.f) return;                            // nothing seen: the partial holds nothing
    const int ex = (int)r[2];
    w *= inv;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (HALF) {
        const f32x2 v = unpack_f16x2(x[i]);
        o[2 * i] = fmaf(ldexpf(v[0], ex), w, o[2 * i]);
        o[2 * i + 1] = fmaf(ldexpf(v[1], ex), w, o[2 * i + 1]);
      } else {
        o[i] = fmaf(__uint_as_float(x[i]), w, o[i]);
      }
    }
  };
#pragma unroll
  for (int i = 0; i < kPre; ++i)
    if (share + i * spr < S) add(ml[i], ml[i][3], pre[i]);
  for (int s = share + kPre * spr; s < S; s += spr) {
    const f32x4 r = a.part_ml[(size_t)s * n + row];
    add(r, weight(r), load(s));
  }
  for (int off = 1 << lpr_shift; off < 1 << (lpr_shift + spr_shift); off <<= 1) {
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] += __shfl_xor(o[e], off);
  }
  if (share != 0 || !live) return;
  if constexpr (BF16) {
    uint16_t *out = reinterpret_cast<uint16_t *>(a.out) + (size_t)row * D + d;
#pragma unroll
    for (int e = 0; e < E; e += 4)
      *reinterpret_cast<u32x2 *>(out + e) = u32x2{pack_bf16x2(o[e], o[e + 1]), pack_bf16x2(o[e + 2], o[e + 3])};
  } else {
    *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(a.out) + (size_t)row * D + d) = f32x4{o[0], o[1], o[2], o[3]};
  }
}

// Whether a launch's partials are fp16.
bool half_parts(const WindowLaunch &p) { return p.is_bf16 && p.q_start != nullptr; }

// Blocks of 16 pairs of an fp32 workgroup.  Two (of 4 waves) read keys and values half as often and leave a SIMD two
// waves; for that a launch has to have long lists and workgroups enough, sooner with a transposed V, whose pieces of 64
// bytes cost the caches more (head_dim 128, 40 heads over 8, one block and two: 263 + 130 rows, window 2420, transposed V
// 386, 211 us; 16 x 100 rows at 500 319, 223, row-major 235, 231; 2000 rows from 0 503, 450; but 512 rows, window 1024,
// 140, 152; 256 rows, window 512, transposed V 50, 55; 334 rows from 0 28, 31; head_dim 64, 16 x 100 at 500 95, 99).
int f32_blocks(const WindowLaunch &p) {
  if (p.is_bf16 || p.q_start == nullptr || p.head_dim != 128) return 1;
  const int64_t wgs = ((int64_t)p.n_rows * (p.n_q_heads / p.n_kv_heads) / (2 * kF32Rows) + p.n_seqs) * p.n_kv_heads;
  const int64_t keys = std::min<int64_t>((int64_t)p.window + p.sinks, p.max_len);
  return keys > 512 && wgs > (p.v_transposed ? 384 : 1024) ? 2 : 1;
}

int64_t tile_rows(const WindowLaunch &p) {
  return !p.is_bf16 ? kF32Rows * f32_blocks(p) : p.head_dim == 256 ? kWideRows : kMfmaRows;
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

// Microseconds per key tile of n workgroups that are on the chip together (128 rows x 64 keys, head_dim 256: 256 rows
// x 32 keys), by launches of 96 to 1280 equal workgroups: those of a CU share its units, and a chip that is not full
// clocks higher.
double tile_us(const WindowLaunch &p, double n) {
  const double layers = n / 256.;
  if (p.head_dim == 64) return layers <= 1. ? 0.85 : 0.65 * ceil(layers);
  if (p.head_dim == 128) return layers <= 1. ? 1.2 : 1.2 + 0.8 * (layers - 1.);
  // (with a soft cap 1.6 + 1.1 layers, without 1.6 + 0.45: the workspace knows of none)
  return 1.6 + 0.8 * layers;
}

// Pages of the longest list of a row tile.
int64_t list_pages(const WindowLaunch &p) {
  const int64_t group = p.n_q_heads / p.n_kv_heads, rows = p.q_start == nullptr ? 1 : tile_rows(p) / group + 1;
  return (std::min<int64_t>((int64_t)p.window + p.sinks + rows + 16, p.max_len) + 15) / 16;
}

// Waves of an fp32 workgroup.  Eight where the chip has room for every workgroup at once and a list's length is what a
// launch takes; with more workgroups fewer merge less, and of short lists two (8, 4, 2 waves; 40 heads over 8 of 128 and
// 32 of 64: 60 rows at 1000 30, 50, 61 us; 334 at 0 31, 27, 31; 1024 at 0, head_dim 64, 62, 57, 71; 43 sequences of 62
// rows at 10 101, 72, 60, at 100 232, 165, 115; 2000 rows, window 64, 96, 71, 60; 64 x 16 at 200 101, 79, 82).  head_dim
// 256 has four for eight (200 rows at 1000 70, 62, 108; 20 x 100 at 100 -, 102, 90; 480 at 0 50, 52, 64).
int f32_waves(const WindowLaunch &p) {
  const int64_t wgs = window_units(p) * p.n_splits;
  if (wgs > 4 * 256 && list_pages(p) <= 16) return 2;
  return wgs > 2 * 256 || p.head_dim == 256 || f32_blocks(p) == 2 ? 4 : 8;
}

// Splits of the keys of every row tile.
int window_splits(const WindowLaunch &p) {
  const int64_t group = p.n_q_heads / p.n_kv_heads;
  constexpr int64_t kCUs = 256;
  const int64_t pages = list_pages(p);
  if (p.q_start == nullptr || !p.is_bf16) {
    // One workgroup a CU, of at least 20 pages in bf16 and 8 in fp32 (whose 8 waves take a page each), lists of under
    // twice and four times that whole (a merge costs 4 us of host time); from three quarters of the CUs on one split,
    // which needs no merge, is as fast or faster (8 KV heads of 128, window 4096: one sequence 49 us, in 12 splits 12.9,
    // in 24 13.9; 8 sequences 55, in 3 or 4 28, in 8 29.5; 24: 73, in 2 82; 32: 96, in 2 100), but for long windows and
    // between one workgroup a CU and one and a half (40 sequences 142, in 3 125; window 1024, head_dim 64: 20.6, in 3
    // 20.7).
    const int64_t units = window_units(p);
    int64_t s = 4 * units >= 3 * kCUs ? 1 : kCUs / units;
    if (p.is_bf16 && units > kCUs && 2 * units <= 3 * kCUs && pages >= 128) s = 3;
    if (pages < (p.is_bf16 ? 40 : 32)) return 1;
    s = std::min<int64_t>(s, p.is_bf16 ? (pages + 19) / 20 : (pages + 7) / 8);
    return (int)std::max<int64_t>(1, std::min<int64_t>(s, kMaxSplits));
  }
  // Many rows: the split count of least estimated time.  The tiles are those that sequences of average length make of
  // the rows, half of one more each but for one alone; workgroups take the CUs in rounds, whose time per key tile was
  // measured (tile_us); 5 us for the set-up and end of a round's workgroups, 4 for the merge's launch, and partials
  // written and read at 6 TB/s.
  const double r = (double)tile_rows(p), per_seq = (double)p.n_rows * group / r / p.n_seqs;
  const double units = (p.n_seqs == 1 ? ceil(per_seq) : per_seq < 1. ? 1. : per_seq + 0.5) * p.n_seqs * p.n_kv_heads;
  const int64_t kt = p.head_dim == 256 ? 2 : 4, tiles = (pages + kt - 1) / kt;       // pages of a tile
  const double elems = (double)p.n_rows * p.n_q_heads * p.head_dim;
  int best = 1;
  double best_t = 1e30;
  for (int s = 1; s <= 16 && 4 * s <= tiles + 3; ++s) {
    const double round = p.head_dim == 64 ? 3 * kCUs : p.head_dim == 128 ? 2 * kCUs : kCUs;
    const double wgs = ceil(units * s), full = floor(wgs / round), left = wgs - full * round;
    const double steps = (double)((tiles + s - 1) / s);
    double t = full * (tile_us(p, round) * steps + 5.) + (left > 0. ? tile_us(p, left) * steps + 5. : 0.);
    if (s > 1) t += 4. + elems * (4. * s + 2.) / 6e6;
    if (t < 0.97 * best_t) {
      best_t = t;
      best = s;
    }
  }
  return best;
}

}  // namespace

bool plan_window(WindowLaunch &p) {
  p.n_splits = window_splits(p);
  // one grid dimension holds fewer than 2^32 threads: 512 a workgroup of window_d256_kernel (and of 8 fp32 waves, which
  // launches of up to 512 workgroups have), 256 of the others
  const bool wide = p.is_bf16 && p.q_start != nullptr && p.head_dim == 256;
  return window_units(p) * p.n_splits < (wide ? 1 << 23 : 1 << 24);
}

size_t window_workspace_bytes(const WindowLaunch &p) {
  const size_t s = (size_t)p.n_splits;
  return s == 1 ? 0 : s * p.n_rows * p.n_q_heads * (p.head_dim * (half_parts(p) ? 2 : 4) + sizeof(f32x4));
}

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
  a.n_splits = p.n_splits;
  a.n_cols = (uint32_t)p.n_phys_pages * 16u;
  a.n_units = (uint32_t)window_units(p);
  const bool half = half_parts(p);
  // Windows of 512 KB of keys and values a head and more are taken in the sequence's order (TileOrder): 1536 rows of 16
  // heads of 256, window 4096, transposed V 168 -> 161 us and 1034 -> 187 MB read; 4096 rows of 40 heads of 128, windows
  // of 1024 to 4096, 1 to 3% less; 8 x 512 such rows 3 to 7%.  Smaller ones from their start (16 sequences of up to 517
  // rows of 32 heads of 64, window 1024: 55 us, in the sequence's order 60).
  const int kt = p.head_dim == 256 ? 32 : 64;
  const int64_t tiles = ((int64_t)p.window + tile_rows(p) / a.group + 2 * kt) / kt + 1;
  a.period = (int64_t)p.window * p.head_dim * 4 >= 512 << 10 ? (int)tiles : kNoPeriod;
  a.part = p.workspace;
  a.part_ml = a.n_splits == 1 ? nullptr
                              : reinterpret_cast<f32x4 *>(reinterpret_cast<char *>(p.workspace) +
                                                          (size_t)a.n_splits * p.n_rows * p.n_q_heads * p.head_dim *
                                                              (half ? 2 : 4));
  const float log2e = 1.4426950408889634f;
  a.scale_log2 = p.scale * log2e;
  a.cap_in = p.softcap > 0.f ? p.scale / p.softcap : 0.f;
  a.cap_out = p.softcap * log2e;
  a.cap_k = p.softcap > 0.f ? 2.0f * p.scale * log2e / p.softcap : 0.f;
  const bool cap = p.softcap > 0.f;
  hipError_t e;
  if (!p.is_bf16) e = launch_window_f32(a, p.head_dim, p.v_transposed, cap, f32_waves(p), f32_blocks(p), stream);
  else if (p.q_start == nullptr) e = launch_window_decode(a, p.head_dim, p.v_transposed, cap, stream);
  else if (p.head_dim == 256) e = launch_window_d256(a, p.v_transposed, cap, stream);
  else e = launch_window_rows(a, p.head_dim, p.v_transposed, cap, stream);
  if (e != hipSuccess || a.n_splits == 1) return e;
  int lpr = 0, spr = 0;               // log2 of the lanes of a partial row, and of the groups that share its splits
  while ((half ? 8 : 4) << lpr < p.head_dim) ++lpr;
  // Up to eight splits of rows that fill two waves a CU: rows side by side, all of a row's loads in flight (with their
  // attention 192 rows of 40 heads of 128 in 4 splits 28.1 us, splits side by side 30.0; 64 rows 14.9, 15.4).  Few rows,
  // and more splits: the splits side by side (4 decode rows 11.2, rows side by side 12.2).
  const bool many = a.n_splits <= kPre && ((int64_t)p.n_rows * p.n_q_heads << lpr) >= 64 * 512;
  while (!many && lpr + spr < 6 && 1 << spr < a.n_splits) ++spr;
  const uint32_t per_wg = 4u << (6 - lpr - spr);
  const dim3 grid(((uint32_t)p.n_rows * p.n_q_heads + per_wg - 1) / per_wg);
  auto merge = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a, p.head_dim, lpr, spr);
  };
  if (half) merge(window_combine_kernel<true, true>);
  else if (p.is_bf16) merge(window_combine_kernel<true, false>);
  else merge(window_combine_kernel<false, false>);
  return hipGetLastError();
}

}  // namespace nexus
