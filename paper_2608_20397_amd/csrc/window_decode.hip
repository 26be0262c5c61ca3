// Windowed attention of a decode step, bf16: one query a sequence sees the last `window` keys of its cache and the
// first `sinks` ones.
//
// HBM-bound: window + sinks key and value rows a (sequence, KV head), read once for up to 16 query heads.  A workgroup
// is one (sequence, KV head, query group, split) and takes a run of the list of seen pages (sinks', then window's);
// its 4 waves take pairs of them in turn, S^T = K.Q^T and O^T += V^T.P^T on 16x16x32 MFMA straight from global memory
// as decode_bf16 does (layouts there), and merge their (m, l, O) through LDS.  Slots of a listed page that the query
// does not see are read as one that it sees (transposed V: zeroed) and masked, so that nothing in them matters; rows
// that come out not finite are formed key by key (row_again).
// 32 sequences of 17000 tokens, window 4096, 40 heads over 8 of 128: 85 us, 6.3 TB/s; one such sequence 14 us: 9 in 13
// splits (a chain of round trips: length, pages, keys) and the merge.  8 waves a workgroup were as fast there, slower
// with 64 sequences (43.5, 47.6) and at head_dim 256, where two buffers of a wave do not fit.  A page of a transposed V
// is 32 bytes of each feature's 128-byte lines, which come whole from memory (16 sequences of 4096, head_dim 256: 178
// us where the pages of a line are other sequences', 111 where they follow one another, row-major 90; 16 bytes a lane
// instead of 8 were no faster, runs of four pages a wave slower).
#include "attn_dma.h"
#include "decode_common.h"
#include "window_common.h"

#include <algorithm>
#include <type_traits>

namespace nexus {

namespace {

constexpr int kList = 2048;        // pages listed in LDS at a time
constexpr int kMinRun = 8;         // pages of a split at least

}  // namespace

template <int D, bool VT, bool CAP, bool NT>
__global__ __launch_bounds__(256, D == 64 ? 3 : D == 128 ? 2 : 1) void window_decode_kernel(const WindowArgs a) {
  constexpr int NW = kDecWaves;
  constexpr int NP = D == 256 ? 1 : 2;   // pages per step of a wave
  constexpr int KS = D / 32;          // S^T MFMA steps
  constexpr int DT = D / 16;          // O^T tiles
  constexpr int ROWB = 2 * D;         // bytes per key row
  constexpr int VL = VT ? 1 : D / 32; // 16-byte V loads per lane per row-major page
  constexpr int MO_LD = D + 4;        // padded row of the merge buffer (floats)
  constexpr int STAGE_BYTES = VT ? 0 : NW * NP * 16 * ROWB;
  constexpr int MERGE_BYTES = NW / 2 * 16 * (MO_LD * 4 + 2 * 4);
  constexpr int SMEM = STAGE_BYTES > MERGE_BYTES ? STAGE_BYTES : MERGE_BYTES;
  __shared__ __align__(1024) char smem[SMEM];
  __shared__ int32_t pgs[kList];
  __shared__ int32_t first[kList];      // first key of each listed page

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qn = lane & 15, grp = lane >> 4;
  const uint32_t n_hq = a.n_kv_heads * a.n_qgroups;
  const uint32_t rest = blockIdx.x / n_hq;
  int hg = blockIdx.x - rest * n_hq;
  hg = hg % a.n_kv_heads * a.n_qgroups + hg / a.n_kv_heads;   // KV heads vary fastest: an XCD keeps its heads
  const int split = rest % a.n_splits, b = rest / a.n_splits;
  const int qg = hg % a.n_qgroups, h = hg / a.n_qgroups;
  const int g_lo = qg * 16;
  const int g_cnt = min(16, a.group - g_lo);     // query heads of this workgroup
  const int hq0 = h * a.group + g_lo;            // first of them
  const bool direct = a.n_splits == 1;
  const bool q_ok = qn < g_cnt;
  const size_t row = (size_t)b * a.n_q_heads + hq0 + qn;
  const size_t slot = (size_t)split * a.n_rows * a.n_q_heads + row;
  uint16_t *out = reinterpret_cast<uint16_t *>(a.out);

  const int len = window_len(a, b);
  KeyList kl{};
  if (len > 0) kl = key_list(a.window, a.sinks, len - 1, len - 1);
  // the split's run of the list
  const int per = max((kl.n + a.n_splits - 1) / a.n_splits, kMinRun);
  const int e_begin = split * per, e_end = min(e_begin + per, kl.n);
  if (e_begin >= e_end) {
    if (direct) {
      for (int i = tid; i < g_cnt * D; i += 64 * NW) out[((size_t)b * a.n_q_heads + hq0) * D + i] = 0;
    } else if (tid < g_cnt) {
      a.part_ml[slot] = f32x4{-INFINITY, 0.f, 0.f, 0.f};
    }
    return;
  }

  // ---- queries: B operand of S^T = K.Q^T, column qn = query head hq0 + qn
  u32x4 qreg[KS];
  {
    const uint16_t *qrow = reinterpret_cast<const uint16_t *>(a.q) + row * D;
#pragma unroll
    for (int s = 0; s < KS; ++s)
      qreg[s] = q_ok ? *reinterpret_cast<const u32x4 *>(qrow + 32 * s + 8 * grp)
                     : u32x4{0u, 0u, 0u, 0u};
  }

  const int32_t *map = a.maps + (size_t)b * a.map_stride;
  const uint32_t page_elems = (uint32_t)a.n_kv_heads * 16u * D;
  const char *kbase = reinterpret_cast<const char *>(a.kc) + (size_t)h * 16 * ROWB;
  const char *vbase = VT ? reinterpret_cast<const char *>(a.vc) + (size_t)h * D * a.n_cols * 2
                         : reinterpret_cast<const char *>(a.vc) + (size_t)h * 16 * ROWB;
  char *vstage = smem + wave * NP * 16 * ROWB;

  struct Page {
    u32x4 k[KS];
    u32x4 v[VT ? 1 : VL];
    u32x2 vt[VT ? DT : 1];
  };
  auto read = [](const auto *p) {
    if constexpr (NT) return ld_stream(p);
    else return *p;
  };
  auto load_page = [&](int key0, uint32_t phys, Page &pg) {
    auto from = [&](int s) { return kl.stand_in(key0 + s) & (kPage - 1); };
    const char *kp = kbase + (size_t)phys * page_elems * 2;
    const int krow = from(qn);
#pragma unroll
    for (int s = 0; s < KS; ++s)
      pg.k[s] = read(reinterpret_cast<const u32x4 *>(kp + krow * ROWB + 64 * s + 16 * grp));
    if constexpr (!VT) {
      const char *vp = vbase + (size_t)phys * page_elems * 2;
#pragma unroll
      for (int j = 0; j < VL; ++j) {
        const int byte = 16 * lane + 1024 * j;
        pg.v[j] = read(reinterpret_cast<const u32x4 *>(vp + from(byte / ROWB) * ROWB + byte % ROWB));
      }
    } else {
      const char *vp = vbase + ((size_t)phys * 16 + 4 * grp) * 2;
#pragma unroll
      for (int t = 0; t < DT; ++t)
        pg.vt[t] = *reinterpret_cast<const u32x2 *>(vp + (size_t)(16 * t + qn) * a.n_cols * 2);
    }
  };

  f32x4 o[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_ref = -INFINITY;   // reference of query column qn (equal across the 4 lane groups)
  float lsum = 0.f;          // sum of this lane's rounded probabilities

  // Two pages at a time: 32 keys are the k extent of the 16x16x32 MFMA, lane group grp holding keys 4 grp .. +3 of
  // either page.  (head_dim 256: one page.)
  struct Pair {
    Page pg[NP];
  };
  auto compute_pair = [&](const int (&key0)[NP], bool two, const Pair &pr) {
    float x[4 * NP];
#pragma unroll
    for (int pp = 0; pp < NP; ++pp) {
      f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < KS; ++st)
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, pr.pg[pp].k[st]),
                                                    __builtin_bit_cast(bf16x8, qreg[st]), s, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float v = CAP ? a.cap_out * window_tanh(s[i] * a.cap_in) : s[i] * a.scale_log2;
        x[4 * pp + i] = kl.seen(key0[pp] + 4 * grp + i) && (pp == 0 || two) ? v : -INFINITY;
      }
    }
    float mx = x[0];
#pragma unroll
    for (int e = 1; e < 4 * NP; ++e) mx = fmaxf(mx, x[e]);
    mx = max_x32(max_x16(mx));
    const bool need = mx > m_ref + kDecSlack;
    if (__builtin_amdgcn_ballot_w64(need)) {
      const float nm = need ? mx : m_ref;
      const float alpha = nm == -INFINITY ? 1.f : fast_exp2(m_ref - nm);
#pragma unroll
      for (int t = 0; t < DT; ++t) o[t] *= alpha;
      lsum *= alpha;
      m_ref = nm;
    }
    const float nm = m_ref == -INFINITY ? 0.f : m_ref;
    uint32_t w[2 * NP];
#pragma unroll
    for (int e = 0; e < 2 * NP; ++e) {
      w[e] = pack_bf16x2(fast_exp2(x[2 * e] - nm), fast_exp2(x[2 * e + 1] - nm));
      lsum += __uint_as_float(w[e] << 16) + __uint_as_float(w[e] & 0xFFFF0000u);
    }
    // O^T tile += V^T.P^T with the lane's V of each page, 4 keys of one feature
    auto pv = [&](f32x4 &acc, const u32x2 (&v)[NP]) {
      if constexpr (NP == 2)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            __builtin_bit_cast(bf16x8, u32x4{v[0][0], v[0][1], v[NP - 1][0], v[NP - 1][1]}),
            __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2 * NP - 2], w[2 * NP - 1]}), acc, 0, 0, 0);
      else
        acc = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, v[0]),
                                                        __builtin_bit_cast(s16x4, u32x2{w[0], w[1]}),
                                                        acc, 0, 0, 0);
    };
    // (a page alone: the values beside it are zeros, for 0 x inf is NaN)
    if constexpr (!VT) {
#pragma unroll
      for (int pp = 0; pp < NP; ++pp)
#pragma unroll
        for (int j = 0; j < VL; ++j) {
          const int byte = 16 * lane + 1024 * j;
          const int r = byte / ROWB, c = (byte % ROWB) >> 4;
          *reinterpret_cast<u32x4 *>(vstage + pp * 16 * ROWB + r * ROWB + 16 * (c ^ vswz<D>(r))) =
              pp == 0 || two ? pr.pg[pp].v[j] : u32x4{0u, 0u, 0u, 0u};
        }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      const int r = 4 * grp + (qn >> 2);
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        const int c = 2 * t + ((qn & 3) >> 1);
        const char *src = vstage + r * ROWB + 16 * (c ^ vswz<D>(r)) + 8 * (qn & 1);
        u32x2 v[NP];
#pragma unroll
        for (int pp = 0; pp < NP; ++pp)
          v[pp] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                (lds_s16x4 *)(src + pp * 16 * ROWB)));
        pv(o[t], v);
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    } else {
      // slots that the query does not see may hold anything: zero this lane's keys among them
      u32x2 m[NP];
#pragma unroll
      for (int pp = 0; pp < NP; ++pp) {
        auto keep = [&](int i) { return (pp == 0 || two) && kl.seen(key0[pp] + 4 * grp + i); };
        m[pp][0] = (keep(0) ? 0xFFFFu : 0u) | (keep(1) ? 0xFFFF0000u : 0u);
        m[pp][1] = (keep(2) ? 0xFFFFu : 0u) | (keep(3) ? 0xFFFF0000u : 0u);
      }
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        u32x2 v[NP];
#pragma unroll
        for (int pp = 0; pp < NP; ++pp)
          v[pp] = u32x2{pr.pg[pp].vt[t][0] & m[pp][0], pr.pg[pp].vt[t][1] & m[pp][1]};
        pv(o[t], v);
      }
    }
  };

  for (int c0 = e_begin; c0 < e_end; c0 += kList) {
    const int n_sp = min(kList, e_end - c0);
    if (c0 > e_begin) __syncthreads();
    for (int i = tid; i < n_sp; i += 64 * NW) {
      const int p = kl.page(c0 + i);
      pgs[i] = map[p];
      first[i] = p * kPage;
    }
    __syncthreads();
    // this wave's pairs of list entries wave + NW k through two register buffers: a pair is loading while the other
    // is computed (entries past the list's end re-read its last page, masked or unused)
    const int n_pairs = (n_sp + NP - 1) / NP;
    const int n_mine = wave < n_pairs ? (n_pairs - wave + NW - 1) / NW : 0;
    if (n_mine > 0) {
      auto entry = [&](int k) { return NP * (wave + NW * k); };
      auto issue = [&](int k, Pair &pr) {
#pragma unroll
        for (int pp = 0; pp < NP; ++pp) {
          const int e = min(entry(min(k, n_mine - 1)) + pp, n_sp - 1);
          load_page(__builtin_amdgcn_readfirstlane(first[e]), (uint32_t)__builtin_amdgcn_readfirstlane(pgs[e]),
                    pr.pg[pp]);
        }
      };
      auto compute = [&](int k, const Pair &pr) {
        const int e = entry(k);
        int key0[NP];
#pragma unroll
        for (int pp = 0; pp < NP; ++pp) key0[pp] = __builtin_amdgcn_readfirstlane(first[min(e + pp, n_sp - 1)]);
        compute_pair(key0, e + 1 < n_sp, pr);
      };
      Pair b0, b1;
      issue(0, b0);
      // (the scheduling barriers keep a pair's loads ahead of the other pair's computation; one loop exit)
      int k = 0;
      for (; k + 1 < n_mine; k += 2) {
        issue(k + 1, b1);
        __builtin_amdgcn_sched_barrier(0);
        compute(k, b0);
        __builtin_amdgcn_sched_barrier(0);
        issue(k + 2, b0);
        __builtin_amdgcn_sched_barrier(0);
        compute(k + 1, b1);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (k < n_mine) compute(k, b0);
    }
  }

  // ---- merge the waves' (m, l, O^T) pairwise through LDS, the upper half into the lower, down to wave 0, which writes
  // the result
  lsum = sum_x32(sum_x16(lsum));
  float *mo = reinterpret_cast<float *>(smem);   // [NW / 2 slots][16 columns][MO_LD]
  float *mml = mo + NW / 2 * 16 * MO_LD;         // [NW / 2 slots][16 columns][m, l]
  auto store_state = [&](int s) {
#pragma unroll
    for (int t = 0; t < DT; ++t)
      *reinterpret_cast<f32x4 *>(mo + (s * 16 + qn) * MO_LD + 16 * t + 4 * grp) = o[t];
    if (grp == 0) {
      mml[2 * (s * 16 + qn)] = m_ref;
      mml[2 * (s * 16 + qn) + 1] = lsum;
    }
  };
  auto merge_state = [&](int s) {
    const float mb = mml[2 * (s * 16 + qn)];
    const float lb = mml[2 * (s * 16 + qn) + 1];
    const float M = fmaxf(m_ref, mb);
    // a wave that saw no page has m = -inf and contributes nothing (one that saw NaN scores alone has l = NaN)
    const float wa = m_ref > -INFINITY ? fast_exp2(m_ref - M) : m_ref == M ? 1.f : 0.f;
    const float wb = mb > -INFINITY ? fast_exp2(mb - M) : mb == M ? 1.f : 0.f;
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      const f32x4 ob = *reinterpret_cast<const f32x4 *>(mo + (s * 16 + qn) * MO_LD + 16 * t + 4 * grp);
      o[t] = o[t] * wa + ob * wb;
    }
    lsum = lsum * wa + lb * wb;
    m_ref = M;
  };
#pragma unroll
  for (int half = NW / 2; half > 0; half /= 2) {
    __syncthreads();   // the V staging slots, or the slots of the step before, are reused
    if (wave >= half && wave < 2 * half) store_state(wave - half);
    __syncthreads();
    if (wave < half) merge_state(wave);
  }
  if (wave != 0) return;
  const float inv = direct || lsum > 0.f ? 1.0f / lsum : 0.f;
  float check = 0.f;                             // NaN where a result is not finite
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[t][i] *= inv;
      check = fmaf(o[t][i], 0.f, check);
    }
  check = sum_x32(sum_x16(check));
  const bool bad = q_ok && (!(check == 0.f) || lsum != lsum);
  if (q_ok && !bad) {
    if (direct) {
#pragma unroll
      for (int t = 0; t < DT; ++t)
        *reinterpret_cast<u32x2 *>(out + row * D + 16 * t + 4 * grp) =
            u32x2{pack_bf16x2(o[t][0], o[t][1]), pack_bf16x2(o[t][2], o[t][3])};
    } else {
#pragma unroll
      for (int t = 0; t < DT; ++t)
        *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(a.part) + slot * D + 16 * t + 4 * grp) = o[t];
      if (grp == 0) a.part_ml[slot] = f32x4{part_max(m_ref, true, split), lsum, 0.f, 0.f};
    }
  }
  // a stand-in's value that is infinite times its probability 0 is NaN
  uint32_t left = (uint32_t)__builtin_amdgcn_ballot_w64(bad && grp == 0);
  while (left) {
    const int r = __builtin_ctz(left);
    left &= left - 1;
    const size_t rrow = (size_t)b * a.n_q_heads + hq0 + r;
    float res[D / 64], ma, la;
    row_again<uint16_t, D, VT, CAP>(a, kl, b, h, reinterpret_cast<const uint16_t *>(a.q) + rrow * D, len - 1,
                                    e_end - e_begin, [&](int i) { return e_begin + i; }, res, ma, la);
    store_again<uint16_t, D, false>(a, rrow, split, direct, res, ma, la);
  }
}

hipError_t launch_window_decode(const WindowArgs &a, int head_dim, bool vt, bool cap, hipStream_t stream) {
  const dim3 grid((uint32_t)a.n_kv_heads * a.n_qgroups * a.n_splits * a.n_seqs);
  // Keys and values that the 256 MB last-level cache cannot keep are read past it (32 sequences, window 4096, 538 MB:
  // 95.5 -> 85.0 us); of smaller launches it keeps some for the next one (64 sequences, window 1024, 269 MB, the same
  // layer again: 43.5, past it 49.1)  A transposed V never is: its lines serve several pages (the two
  // launches above 215 -> 178 and 176 -> 111).
  const int64_t keys = std::min<int64_t>((int64_t)a.window + a.sinks, a.max_len);
  const bool past = a.n_seqs * keys * a.n_kv_heads * head_dim * 4 > (int64_t)384 << 20;
  auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a);
    return hipGetLastError();
  };
  auto with_c = [&](auto d, auto v, auto c) {
    return past ? run(window_decode_kernel<d(), v(), c(), true>) : run(window_decode_kernel<d(), v(), c(), false>);
  };
  auto with_v = [&](auto d, auto v) {
    return cap ? with_c(d, v, std::true_type{}) : with_c(d, v, std::false_type{});
  };
  auto with_d = [&](auto d) { return vt ? with_v(d, std::true_type{}) : with_v(d, std::false_type{}); };
  if (head_dim == 64) return with_d(std::integral_constant<int, 64>{});
  if (head_dim == 128) return with_d(std::integral_constant<int, 128>{});
  return with_d(std::integral_constant<int, 256>{});
}

}  // namespace nexus
