// Decode step over an 8-bit paged cache (kv8_common.h has its format): one query for each of many
// sequences, each with its own page map and a length on the device; optional tanh soft cap.
//
// The work decomposition is that of the bf16 decode (decode_attn.hip): a workgroup takes one (sequence, KV
// head, group of up to 16 query heads, run of pages); its waves take the run's page pairs in turn, a
// pair in registers while the next one loads, and meet through LDS; a second kernel merges the runs.
//   * S^T = K.Q^T on v_mfma_scale_f32_16x16x128_f8f6f4, the keys' codes straight from global memory into
//     the A operand (lane l: row l % 16, 32 bytes from 32 (l / 16)); the query as two E4M3 terms
//     (split_query).  head_dim 64: one instruction.  Its lane group g takes k 16 g .. + 15 in the first
//     half of the operand and k 64 + 16 g .. + 15 in the second, and the scales of k < 64 from groups 0 and
//     1; so a lane's 16 bytes of codes stand in both halves, against hi in one and lo in the other.
//   * a lane holds the scores of keys 4 (l / 16) .. +3, whose 4 scale bytes are one word: the key's scale is
//     multiplied to the score, the value's to the probability that it is weighed with (a power of two:
//     exact), and V enters the PV product as its codes in bf16.
// Keys past a sequence's end re-read its last key and weigh nothing.  HBM-bound: head_dim + 1 bytes of K and of
// V per key and KV head, half the bf16 cache's.
//   * All heads of one (sequence, run) go to one XCD, side by side: a page's 16 scale bytes of 8 heads are one
//     cache line, which every XCD fetched for itself when heads were dealt to them (32 sequences of 17473
//     tokens: 1.19 GB fetched for 1.12 GB, 1.13 so).
//   * Launches over more bytes than the caches hold (STREAM) read the codes with non-temporal loads, except
//     where the next sequence maps the same page and may find it in a cache: 210 -> 192 us for those 32
//     sequences on pages of their own; on pages that all of them share, each read by all, 118 us with plain
//     loads, 162 without.
//   * Such launches look for a prefix that sequences share (a warm prefix): consecutive sequences form
//     groups, of as many as two blocks of 16 query columns hold (one block with head_dim 256), and the
//     leading pages that those sequences of a group which map the same 32nd page have in common, whole in each,
//     are read once for all of them: cut into ranges, one for a workgroup of the group, whose partials the
//     merge adds.  The other pages of each sequence are cut evenly over its workgroups.  Every workgroup finds
//     this out for itself from the maps (4 to 5 us where pages are shared, 1 to 2 where none are).  Against
//     every sequence on its own, 32 of 17473 tokens, 40 heads over 8 of 128: all shared 109 -> 48 us, 14000 tokens
//     104 -> 82, 8704 159 -> 127, 4096 188 -> 166; 64 of them, all shared 198 -> 77; 128 of 4000, none shared 170
//     -> 171; 48 of 9000 sharing 8000, 16 heads over 8 of 256, capped, 149 -> 88.  The shortest sharer bounds what a
//     group reads together: one of 520 tokens among 31 that share 17008 makes of 55 us 141.
// Probabilities are rounded to bf16 as in the suffix kernel, for the matrix instruction and, so that the weights sum to
// one, for the row sum; partials stay fp32.
#include "attn_common.h"
#include "attn_dma.h"
#include "decode_common.h"
#include "kv8_common.h"
#include "launch_kv8.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace nexus {

namespace {

// 16-query column blocks of a workgroup that serves shared pages.
__host__ __device__ constexpr int shared_blocks(int head_dim) { return head_dim == 256 ? 1 : 2; }
constexpr int kMinSharedPages = 32;    // leading pages in common from which on they are read together
constexpr int kMinRangePages = 16;     // of one workgroup's range of them
constexpr int kMaxGroupSeqs = 32;      // sequences of a group

template <int D, int NW>
constexpr int smem_bytes() {
  constexpr int stage = NW * (D == 256 ? 1 : 2) * 16 * 2 * D;
  constexpr int merge = NW * (16 * (D + 4) * 4 + 2 * 16 * 4);
  return stage > merge ? stage : merge;
}

// Attention of NCB blocks of 16 query columns over the n_sp pages listed in pgs[] (LDS; the last one holds
// last_keys keys), all of which every column sees.  row_of(i): the row [n_seqs * n_q_heads] of column i, -1 if
// it has none.  put(i, f0, acc, m, l) receives column i's unnormalised features f0 .. and its softmax state.
template <int D, bool CAP, int NW, int NCB, typename RowOf, typename Put>
__device__ __forceinline__ void attend(const DecodeArgs &a, int h, char *smem, const int32_t *pgs, int n_sp,
                                       int last_keys, bool non_temporal, RowOf row_of, Put put) {
  constexpr int NP = D == 256 ? 1 : 2;   // pages per step of a wave
  constexpr int KS = D == 256 ? 2 : 1;   // 128-feature steps of S^T
  constexpr int DT = D / 16;          // O^T tiles
  constexpr int ROWB = 2 * D;         // bytes of a staged V row (bf16)
  constexpr int KC = D == 64 ? 1 : 2;    // 16-byte loads of K codes per lane, page and step
  constexpr int VL = D / 64;          // 16-byte loads of V codes per lane and page
  constexpr int MO_LD = D + 4;        // padded row of the merge buffer (floats)
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qn = lane & 15, grp = lane >> 4;

  // ---- the queries (columns without a row are zero)
  i32x8 qhi[NCB][KS], qlo[NCB][KS];
  int qs_hi[NCB], qs_lo[NCB];
  float qmul[NCB];         // from a product with a key's value to log2 units (CAP: to the cap's argument)
#pragma unroll
  for (int cb = 0; cb < NCB; ++cb) {
    const int row = row_of(16 * cb + qn);
    const bool q_ok = row >= 0;
    const uint16_t *qrow = reinterpret_cast<const uint16_t *>(a.q) + (size_t)max(row, 0) * D;
    constexpr int QW = D == 64 ? 8 : 16 * KS;      // words of a lane
    uint32_t raw[QW];
#pragma unroll
    for (int i = 0; i < QW / 4; ++i) {
      const int f = D == 64 ? 16 * grp + 8 * i : 128 * (i >> 2) + 32 * grp + 8 * (i & 3);
      const u32x4 x = q_ok ? *reinterpret_cast<const u32x4 *>(qrow + f) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
      for (int w = 0; w < 4; ++w) raw[4 * i + w] = x[w];
    }
    uint32_t am = amax_bits_bf16<QW>(raw);
    am = max(am, (uint32_t)__shfl_xor((int)am, 16));
    am = max(am, (uint32_t)__shfl_xor((int)am, 32));
    const bool bad = am >= 0x7F800000u;
    const int e = row_exp(am);
    clamp_query<QW>(raw, am);
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int c = 0; c < (D == 64 ? 2 : 4); ++c) {
        uint32_t hi[2], lo[2];
        split_query<4>(raw + 16 * s + 4 * c, e, hi, lo);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          qhi[cb][s][2 * c + w] = hi[w];
          if (D == 64)
            qhi[cb][s][4 + 2 * c + w] = lo[w];
          else
            qlo[cb][s][2 * c + w] = lo[w];
        }
      }
    // The keys' scales come after the sum over features, which is at most 256 * 448 * 448 * 2^e = 2^(e + 25.6): of
    // queries past 2^96 * 448 a part of the scale, 2^32, waits for them
    const bool large = e > 96;
    const int eq = e + 127 - (large ? 32 : 0);
    qs_lo[cb] = bad ? (int)kBadScale : eq - 4;
    qs_hi[cb] = bad || (D == 64 && grp >= 2) ? qs_lo[cb] : eq;
    qmul[cb] = CAP ? a.cap_in : a.scale_log2;
    if (large) qmul[cb] = fminf(qmul[cb] * 0x1p32f, 3e38f);
  }
  __syncthreads();   // pgs[]

  // keys of entry i of the list
  auto keys_of = [&](int i) { return i == n_sp - 1 ? last_keys : 16; };
  const uint64_t page_bytes = (uint64_t)a.n_kv_heads * 16 * D;
  const uint64_t page_scales = (uint64_t)a.n_kv_heads * 16;
  const char *kbase = reinterpret_cast<const char *>(a.kc) + (size_t)h * 16 * D;
  const char *vbase = reinterpret_cast<const char *>(a.vc) + (size_t)h * 16 * D;
  const uint8_t *ksb = a.ks + h * 16, *vsb = a.vs + h * 16;
  char *vstage = smem + wave * NP * 16 * ROWB;

  struct Page {
    u32x4 k[KS][KC];
    u32x4 v[VL];
    uint32_t ks, vs;         // scale bytes of keys 4 grp .. +3
  };
  const uint32_t ko = D == 64 ? 16 * grp : 32 * grp;
  auto load_page = [&](int nvalid, uint32_t phys, Page &pg, auto stream) {
    auto ld = [&](const char *p) {
      const u32x4 *q = reinterpret_cast<const u32x4 *>(p);
      return decltype(stream)::value ? ld_stream(q) : *q;
    };
    // uniform page addresses, 32-bit lane offsets
    const char *kp = kbase + phys * page_bytes, *vp = vbase + phys * page_bytes;
    const uint32_t krow = (uint32_t)min(qn, nvalid - 1) * D + ko;
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int c = 0; c < KC; ++c)
        pg.k[s][c] = ld(kp + (uint32_t)(krow + 128 * s + 16 * c));
#pragma unroll
    for (int j = 0; j < VL; ++j) {
      const uint32_t row = min((16 * lane + 1024 * j) / D, nvalid - 1);
      pg.v[j] = ld(vp + (uint32_t)(row * D + 16 * lane % D));
    }
    const uint8_t *kq = ksb + phys * page_scales, *vq = vsb + phys * page_scales;
    pg.ks = *reinterpret_cast<const uint32_t *>(kq + (uint32_t)(4 * grp));
    pg.vs = *reinterpret_cast<const uint32_t *>(vq + (uint32_t)(4 * grp));
  };

  f32x4 o[NCB][DT];
  float m_ref[NCB];   // reference of query column qn (equal across the 4 lane groups)
  float lsum[NCB];    // sum of this lane's rounded probabilities
#pragma unroll
  for (int cb = 0; cb < NCB; ++cb) {
#pragma unroll
    for (int t = 0; t < DT; ++t) o[cb][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_ref[cb] = -INFINITY;
    lsum[cb] = 0.f;
  }

  struct Pair {
    Page pg[NP];
  };
  auto compute_pair = [&](const int (&keys)[NP], bool two, const Pair &pr) {
    uint32_t w[NCB][2 * NP];
#pragma unroll
    for (int cb = 0; cb < NCB; ++cb) {
      float x[4 * NP], vf[4 * NP];
#pragma unroll
      for (int pp = 0; pp < NP; ++pp) {
        f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < KS; ++st) {
          const u32x4 u = pr.pg[pp].k[st][0], w = pr.pg[pp].k[st][KC - 1];
          const i32x8 ka = {(int)u[0], (int)u[1], (int)u[2], (int)u[3],
                            (int)w[0], (int)w[1], (int)w[2], (int)w[3]};
          s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(ka, qhi[cb][st], s, 0, 0, 0, 127, 0, qs_hi[cb]);
          if constexpr (D != 64)
            s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(ka, qlo[cb][st], s, 0, 0, 0, 127, 0, qs_lo[cb]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool seen = 4 * grp + i < keys[pp] && (pp == 0 || two);
          const float kf = scale_value(pr.pg[pp].ks >> (8 * i) & 255);
          const float u = s[i] * kf * qmul[cb];
          const float v = CAP ? a.cap_out * tanh_fast(u) : u;
          x[4 * pp + i] = seen ? v : -INFINITY;
          vf[4 * pp + i] = seen ? scale_value(pr.pg[pp].vs >> (8 * i) & 255) : 0.f;
        }
      }
      float mx = x[0];
#pragma unroll
      for (int e = 1; e < 4 * NP; ++e) mx = fmaxf(mx, x[e]);
      mx = max_x32(max_x16(mx));
      const bool need = mx > m_ref[cb] + kDecSlack;
      if (__builtin_amdgcn_ballot_w64(need)) {
        const float nm = need ? mx : m_ref[cb];
        const float alpha = need ? fast_exp2(m_ref[cb] - nm) : 1.f;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[cb][t] *= alpha;
        lsum[cb] *= alpha;
        m_ref[cb] = nm;
      }
#pragma unroll
      for (int e = 0; e < 2 * NP; ++e) {
        const uint32_t p = pack_bf16x2(fast_exp2(x[2 * e] - m_ref[cb]), fast_exp2(x[2 * e + 1] - m_ref[cb]));
        const float p0 = __uint_as_float(p << 16), p1 = __uint_as_float(p & 0xFFFF0000u);
        lsum[cb] += p0 + p1;
        w[cb][e] = pack_bf16x2(p0 * vf[2 * e], p1 * vf[2 * e + 1]);
      }
    }
    // V codes as bf16 through the wave's own LDS slot (a page alone: zeros beside it, for 0 x NaN is NaN)
#pragma unroll
    for (int pp = 0; pp < NP; ++pp)
#pragma unroll
      for (int j = 0; j < VL; ++j) {
        const int byte = 16 * lane + 1024 * j;
        const int row = byte / D, c = 2 * ((byte % D) >> 4);
        u32x2 f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = codes_to_bf16(pp == 0 || two ? pr.pg[pp].v[j][i] : 0u, 1.f);
        char *dst = vstage + pp * 16 * ROWB + row * ROWB;
        *reinterpret_cast<u32x4 *>(dst + 16 * (c ^ vswz<D>(row))) =
            u32x4{f[0][0], f[0][1], f[1][0], f[1][1]};
        *reinterpret_cast<u32x4 *>(dst + 16 * ((c + 1) ^ vswz<D>(row))) =
            u32x4{f[2][0], f[2][1], f[3][0], f[3][1]};
      }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    const int r = 4 * grp + (qn >> 2);
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      const int c = 2 * t + ((qn & 3) >> 1);
      const char *src = vstage + r * ROWB + 16 * (c ^ vswz<D>(r)) + 8 * (qn & 1);
      if constexpr (NP == 2) {
        const bf16x8 v = tr_read_pair(src, src + 16 * ROWB);
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb)
          o[cb][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              v, __builtin_bit_cast(bf16x8, u32x4{w[cb][0], w[cb][1], w[cb][2 * NP - 2], w[cb][2 * NP - 1]}),
              o[cb][t], 0, 0, 0);
      } else {
        const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)src);
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb)
          o[cb][t] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(
              v, __builtin_bit_cast(s16x4, u32x2{w[cb][0], w[cb][1]}), o[cb][t], 0, 0, 0);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };

  // ---- this wave's steps (NP pages each) of the list, entries NP (wave + NW k), through two register
  // buffers, as decode_attn.hip: a step loads while the one before is computed
  auto run = [&](auto stream) {
    const int n_steps = (n_sp + NP - 1) / NP;
    const int n_mine = wave < n_steps ? (n_steps - wave + NW - 1) / NW : 0;
    if (n_mine == 0) return;
    auto entry = [&](int k) { return NP * (wave + NW * k); };
    auto issue = [&](int k, Pair &pr) {
#pragma unroll
      for (int pp = 0; pp < NP; ++pp) {
        const int e = min(entry(min(k, n_mine - 1)) + pp, n_sp - 1);
        load_page(keys_of(e), (uint32_t)__builtin_amdgcn_readfirstlane(pgs[e]), pr.pg[pp], stream);
      }
    };
    auto compute = [&](int k, const Pair &pr) {
      const int e = entry(k);
      int keys[NP];
#pragma unroll
      for (int pp = 0; pp < NP; ++pp) keys[pp] = keys_of(min(e + pp, n_sp - 1));
      compute_pair(keys, e + 1 < n_sp, pr);
    };
    Pair b0, b1;
    issue(0, b0);
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
  };
  if (non_temporal)
    run(std::true_type{});
  else
    run(std::false_type{});

  // ---- merge the waves' (m, l, O^T): every wave leaves its state in LDS, then a thread adds all of them for
  // NF features of one column (pairwise, with two barriers a level, 48 sequences of up to 700 tokens took 8.7
  // us instead of 8.0)
  float *mo = reinterpret_cast<float *>(smem);   // [NW][16 columns][MO_LD]
  float *mml = mo + NW * 16 * MO_LD;             // [16 columns][NW][m, l]
  constexpr int NF = 16 * D / (64 * NW);         // features of a thread
  const int col = tid * NF / D, f0 = tid * NF % D;
#pragma unroll
  for (int cb = 0; cb < NCB; ++cb) {
    const float ls = sum_x32(sum_x16(lsum[cb]));
    __syncthreads();   // the V staging slots, or the block before this one
#pragma unroll
    for (int t = 0; t < DT; ++t)
      *reinterpret_cast<f32x4 *>(mo + (wave * 16 + qn) * MO_LD + 16 * t + 4 * grp) = o[cb][t];
    if (grp == 0)
      *reinterpret_cast<f32x2 *>(mml + 2 * (qn * NW + wave)) = f32x2{m_ref[cb], ls};
    __syncthreads();
    if (row_of(16 * cb + col) < 0) continue;
    float mw[NW], M = -INFINITY, l_tot = 0.f, acc[NF];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      mw[w] = mml[2 * (col * NW + w)];
      M = fmaxf(M, mw[w]);
    }
#pragma unroll
    for (int i = 0; i < NF; ++i) acc[i] = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      // a wave that saw no page has m = -inf and contributes nothing
      const float f = mw[w] > -INFINITY ? fast_exp2(mw[w] - M) : 0.f;
      l_tot += f * mml[2 * (col * NW + w) + 1];
#pragma unroll
      for (int i = 0; i < NF; i += 2) {
        const f32x2 x = *reinterpret_cast<const f32x2 *>(mo + (w * 16 + col) * MO_LD + f0 + i);
        acc[i] += f * x[0];
        acc[i + 1] += f * x[1];
      }
    }
    put(16 * cb + col, f0, acc, M, l_tot);
  }
}

template <int D, int NF>
__device__ __forceinline__ void put_part(const DecodeArgs &a, int row, int slot_of_row, int f0,
                                         const float (&acc)[NF], float m, float l) {
  const size_t slot = (size_t)row * a.max_splits + slot_of_row;
#pragma unroll
  for (int i = 0; i < NF; i += 2)
    *reinterpret_cast<f32x2 *>(a.part + slot * D + f0 + i) = f32x2{acc[i], acc[i + 1]};
  if (f0 == 0) *reinterpret_cast<f32x2 *>(a.part_ml + 2 * slot) = f32x2{m, l};
}

// The sequences of a group g0 .. g1 - 1 (bits: index in the group) that map one physical page as page p of
// theirs, whole in each; the largest such set, empty if no two do.  min_whole: the least count of whole pages
// among them.
__device__ __forceinline__ uint32_t sharers(const DecodeArgs &a, int g0, int g1, int p, int &min_whole) {
  const int lane = threadIdx.x & 63;
  const int s = g0 + lane;
  const bool in = s < g1 && p < (a.max_len + 15) / 16;
  const int page = in ? a.maps[(size_t)s * a.map_stride + p] : -1;
  const int whole = in ? seq_len_of(a, s) >> 4 : 0;
  uint32_t best = 0;
  for (uint32_t c = (uint32_t)__builtin_amdgcn_ballot_w64(whole > p); c;) {
    const int pj = __builtin_amdgcn_readlane(page, __builtin_ctz(c));
    const uint32_t m = (uint32_t)__builtin_amdgcn_ballot_w64(whole > p && page == pj);
    if (__popc(m) > __popc(best)) best = m;
    c &= ~m;
  }
  if (__popc(best) < 2) return 0;
  min_whole = INT32_MAX;
  for (uint32_t c = best; c; c &= c - 1)
    min_whole = min(min_whole, __builtin_amdgcn_readlane(whole, __builtin_ctz(c)));
  return best;
}

// NW: waves of a workgroup.  STREAM: see the header comment.
template <int D, bool CAP, int NW, bool STREAM>
__global__ __launch_bounds__(64 * NW, 2) void decode_kv8_kernel(const DecodeArgs a) {
  __shared__ __align__(1024) char smem[smem_bytes<D, NW>()];
  __shared__ int32_t pgs[kMaxSplitPages];
  __shared__ int32_t ranks[STREAM ? kMaxGroupSeqs : 1];   // the sharers
  __shared__ int32_t n_shared;                            // leading pages that they share

  const int tid = threadIdx.x;
  // workgroups go to the 8 XCDs in turn
  const int unit = 8 * (int)(blockIdx.y + gridDim.y * blockIdx.z) + (blockIdx.x & 7), hg = blockIdx.x >> 3;
  if (unit >= a.n_seqs * a.own_splits) return;
  const int b = unit / a.own_splits, split = unit - b * a.own_splits;
  // The run's pages are loaded beside the length (a map row has max_len's pages; those past the sequence's
  // end are not used).
  const int32_t *map = a.maps + (size_t)b * a.map_stride;
  const int p_run = split * a.split_pages;
  const int n_map = min(a.split_pages, (a.max_len + 15) / 16 - p_run);
  for (int i = tid; i < n_map; i += 64 * NW) pgs[i] = map[p_run + i];
  bool next_shares = false;
  uint32_t members = 0;
  int g0 = 0, min_whole = 0;
  if constexpr (STREAM) {
    const int next = b + 1 < a.n_seqs ? b + 1 : 0, mid = p_run + n_map / 2;
    next_shares = next != b && map[mid] == a.maps[(size_t)next * a.map_stride + mid];
    if (a.n_groups > 0) {
      // groups of equal size, give or take one (six of 5 or 6 sequences: all of 17473 tokens shared 51 us,
      // five of 6 and one of 2: 70): group g starts at floor(g n_seqs / n_groups)
      const int g = (int)((((int64_t)b + 1) * a.n_groups - 1) / a.n_seqs);
      g0 = (int)((int64_t)g * a.n_seqs / a.n_groups);
      const int g1 = (int)((int64_t)(g + 1) * a.n_seqs / a.n_groups);
      members = sharers(a, g0, g1, kMinSharedPages - 1, min_whole);
      if (!(members >> (b - g0) & 1)) members = 0;
    }
  }
  const int len = seq_len_of(a, b);
  const int qg = hg % a.n_qgroups;
  const int h = hg / a.n_qgroups;
  const int g_lo = qg * 16;
  const int g_cnt = min(16, a.group - g_lo);     // query heads of this workgroup
  const int hq0 = h * a.group + g_lo;            // first of them
  uint16_t *out = reinterpret_cast<uint16_t *>(a.out);

  if (len == 0) {
    if (split == 0)
      for (int i = tid; i < g_cnt * D; i += 64 * NW)
        out[((size_t)b * a.n_q_heads + hq0) * D + i] = 0;
    return;
  }
  const int n_pages = (len + 15) >> 4;
  if (p_run >= n_pages) return;
  const int n_splits = (n_pages + a.split_pages - 1) / a.split_pages;
  const int row0 = b * a.n_q_heads + hq0;
  int p_begin = p_run, n_sp = min(a.split_pages, n_pages - p_run);

  // ---- the leading pages that the sharers have in common, cut into ranges, each of which one of their
  // workgroups takes for all of them; a sharer's other pages are cut evenly into as many runs as it has
  int n_sh = 0, rank = 0, n_ranges = 0, per = 0;
  const int n_mem = __popc(members);
  if constexpr (STREAM) {
    if (n_mem > 0) {
      if (tid < 32 && (members >> tid & 1)) ranks[__popc(members & ((1u << tid) - 1))] = g0 + tid;
      if (tid == 0) n_shared = min_whole;
      __syncthreads();
      int first = min_whole;                   // first page that some sharer maps elsewhere
      for (int i = tid; i < min_whole && first == min_whole; i += 64 * NW) {
        const int mine = map[i];
        bool same = true;
        for (int m = 0; m < n_mem; m += 8) {   // (eight loads in flight)
          int32_t other[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) other[e] = a.maps[(size_t)ranks[min(m + e, n_mem - 1)] * a.map_stride + i];
#pragma unroll
          for (int e = 0; e < 8; ++e) same &= other[e] == mine;
        }
        if (!same) first = i;
      }
      if (first < min_whole) atomicMin(&n_shared, first);
      __syncthreads();
      n_sh = __builtin_amdgcn_readfirstlane(n_shared);
      if (n_sh < kMinSharedPages) n_sh = 0;
    }
    if (n_sh > 0) {
      // (the shortest sharer has workgroups for its runs alone)
      const int min_runs = (min_whole + a.split_pages - 1) / a.split_pages;
      n_ranges = min(min(a.shared_splits, n_mem * min_runs), n_sh / kMinRangePages);
      n_sh = min(n_sh, n_ranges * kMaxSplitPages);   // what pgs[] holds
      per = (n_sh + n_ranges - 1) / n_ranges;
      n_ranges = (n_sh + per - 1) / per;
      rank = split * n_mem + __popc(members & ((1u << (b - g0)) - 1));
      const int n_own = n_pages - n_sh, per_own = (n_own + n_splits - 1) / n_splits;
      p_begin = min(n_sh + split * per_own, n_pages);
      n_sp = min(per_own, n_pages - p_begin);
    }
    if (a.n_groups > 0 && split == 0 && h == 0 && tid == 0) a.flags[b] = n_ranges;
  }
  // ---- the sequence's own pages first, then the shared ones: so all workgroups stream at the same time
  // (prefix of 4096 of 17473 tokens, 32 sequences: 169 us, the other way round 186, half of the workgroups
  // each way 180)
  if (n_sh > 0)
    for (int i = tid; i < n_sp; i += 64 * NW) pgs[i] = map[p_begin + i];
  if (n_sp > 0) {
    const bool direct = n_splits == 1 && n_sh == 0;
    const int last_keys = p_begin + n_sp == n_pages ? len - 16 * (n_pages - 1) : 16;
    attend<D, CAP, NW, 1>(
        a, h, smem, pgs, n_sp, last_keys, STREAM && (n_sh > 0 || !next_shares),
        [&](int i) { return i < g_cnt ? row0 + i : -1; },
        [&](int i, int f0, const auto &acc, float m, float l) {
          if (!direct) {
            put_part<D>(a, row0 + i, split, f0, acc, m, l);
            return;
          }
          constexpr int NF = sizeof(acc) / sizeof(float);
          const float inv = 1.0f / l;
#pragma unroll
          for (int j = 0; j < NF; j += 2)
            *reinterpret_cast<uint32_t *>(out + (size_t)(row0 + i) * D + f0 + j) =
                pack_bf16x2(acc[j] * inv, acc[j + 1] * inv);
        });
  } else {
    for (int g = tid; g < g_cnt; g += 64 * NW)
      *reinterpret_cast<f32x2 *>(a.part_ml + 2 * ((size_t)(row0 + g) * a.max_splits + split)) =
          f32x2{-INFINITY, 0.f};
    __syncthreads();   // pgs[] is written again
  }
  if constexpr (STREAM) {
    if (rank >= n_ranges) return;
    const int lo = rank * per, n = min(per, n_sh - lo);
    // (no wave still reads the other list: attend ends behind barriers)
    for (int i = tid; i < n; i += 64 * NW) pgs[i] = map[lo + i];
    const int per_block = 16 / a.group;
    auto row_of = [&](int i) {
      const int c = i & 15, m = (i >> 4) * per_block + c / a.group;
      if (c >= per_block * a.group || m >= n_mem) return -1;
      return ranks[m] * a.n_q_heads + hq0 + c % a.group;
    };
    attend<D, CAP, NW, shared_blocks(D)>(a, h, smem, pgs, n, 16, false, row_of,
                                         [&](int i, int f0, const auto &acc, float m, float l) {
                                           put_part<D>(a, row_of(i), a.own_splits + rank, f0, acc, m, l);
                                         });
  }
}

// Pages of a run, of lengths up to max_len that are taken to be alike (all figures are of equal lengths; the device's
// are not known here): the longest sequence decides a launch's time.  32 of 17473 tokens take 181 us, 32 evenly up to
// 17473 152 for half the bytes, one of 17473 and 31 of 500 135, over 8 heads of 128.
// A workgroup keeps its CU's memory pipe full by itself, so launches that have a workgroup per
// (sequence, KV head, query group) for half the CUs or more take whole sequences and need no merge, smaller ones
// as many runs as make one workgroup per CU (32 sequences of 17473 tokens, 40 heads over 8 of 128: one run 181
// us, two 186; 24: 154 and 170; 8 of 4000: four runs 17.8, eight 19.3; 2 of 17473: sixteen 19.2, 32 21.5).
//   * No more than the merge is worth: 8 pages and 0.7 sqrt(pages) a run (one sequence of 17473 tokens over one
//     head: 23 pages 12.7 us, 12 15.2, 46 14.1; of 70000: 46 19.5, 23 23.6, 92 22.0; of 1000 over 8: 8 pages
//     8.4, 12 9.1, 32 11.3); one run up to 32 pages, or 96 where there would be two (16 sequences of 1300: 14.0,
//     two runs 15.0).
//   * Between 256 and 512, two a CU: runs that fill whole rounds of 512 (36 sequences of 4000 over 8 heads:
//     three runs 55.6 us, one 66, two 60; 48 of 6000: two 102, one 114, three 111; 56 of 4000: one 82, two 92): three
//     while they fit two rounds (341 pairs), then two up to the middle of the two counts measured (384 and 448), then
//     one; the 96 pages below which there is one, and the 85 pairs from which 256 / pairs is two, are those above.
int kv8_split_pages(const DecodeLaunch &p, int n_qgroups) {
  const int64_t max_pages = ((int64_t)p.max_len + 15) / 16;
  const int64_t pairs = (int64_t)p.n_seqs * p.n_kv_heads * n_qgroups;
  if (max_pages <= 0 || pairs > 512) return decode_split_pages(p.n_seqs, p.n_kv_heads, n_qgroups, p.max_len);
  int64_t ns;
  if (pairs > 256)
    ns = max_pages < 96 || pairs > 416 ? 1 : 3 * pairs > 1024 ? 2 : 3;
  else
    ns = max_pages <= (pairs > 85 ? 96 : 32) ? 1 : 256 / pairs;
  int64_t sp = (max_pages + ns - 1) / ns;
  if (ns > 1) sp = std::max({sp, (int64_t)8, (int64_t)std::ceil(0.7 * std::sqrt((double)max_pages))});
  return (int)std::min<int64_t>(sp, kMaxSplitPages);
}

struct Shape {
  int split_pages, own_splits;         // pages per run, runs of the longest sequence
  int n_groups, group_seqs;            // 0 groups: shared pages are not looked for
  int shared_splits;                   // ranges of a group's shared pages at most
  bool stream;
  int slots() const { return own_splits + (n_groups ? shared_splits : 0); }
};

size_t part_bytes(const DecodeLaunch &p, int slots) {
  return (size_t)p.n_seqs * p.n_q_heads * slots * (p.head_dim + 2) * sizeof(float);
}

size_t shape_bytes(const DecodeLaunch &p, const Shape &s) {
  if (s.slots() <= 1) return 0;
  return part_bytes(p, s.slots()) + (s.n_groups ? (size_t)p.n_seqs * sizeof(int32_t) : 0);
}

// The shape of a launch that has ws_bytes of workspace (too few for shared pages: none are looked for).
Shape kv8_shape(const DecodeLaunch &p, size_t ws_bytes) {
  Shape s{};
  const int group = p.n_q_heads / p.n_kv_heads;
  const int n_qgroups = (group + 15) / 16;
  s.split_pages = kv8_split_pages(p, n_qgroups);
  const int64_t max_pages = ((int64_t)p.max_len + 15) / 16;
  s.own_splits = (int)std::max<int64_t>(1, (max_pages + s.split_pages - 1) / s.split_pages);
  // Non-temporal loads where the codes may pass twice the 256 MB last-level cache and a page is read by one
  // workgroup of a sequence (64 sequences of 2000 tokens, 0.26 GB: 46.9 us, 48.8 so).
  s.stream = n_qgroups == 1 &&
             (int64_t)p.n_seqs * p.max_len * p.n_kv_heads * p.head_dim * 2 >= (int64_t)512 << 20;
  // Shared pages are looked for in the same launches: in smaller ones the caches serve the repeated reads (16
  // sequences of 8000 tokens, 0.26 GB: all shared 42 -> 27 us, but half shared 42 -> 46 and none 47 -> 49).
  const int cap = n_qgroups == 1 ? std::min(kMaxGroupSeqs, shared_blocks(p.head_dim) * (16 / group)) : 1;
  if (!s.stream || p.n_seqs < 2 || cap < 2) return s;
  const int n_groups = (p.n_seqs + cap - 1) / cap;
  Shape t = s;
  t.n_groups = n_groups;
  t.group_seqs = (p.n_seqs + n_groups - 1) / n_groups;
  // a range for each workgroup of a group, as far as about 1024 in all, or 8 a group
  const int64_t want = std::max<int64_t>(8, 1024 / ((int64_t)n_groups * p.n_kv_heads));
  t.shared_splits = (int)std::min<int64_t>((int64_t)t.group_seqs * s.own_splits, want);
  while (t.shared_splits > 1 && shape_bytes(p, t) > ws_bytes) --t.shared_splits;
  return shape_bytes(p, t) <= ws_bytes ? t : s;
}

}  // namespace

size_t decode_kv8_workspace_bytes(const DecodeLaunch &p) { return shape_bytes(p, kv8_shape(p, SIZE_MAX)); }

size_t decode_kv8_workspace_min(const DecodeLaunch &p) { return shape_bytes(p, kv8_shape(p, 0)); }

hipError_t launch_decode_kv8(const DecodeLaunch &p, hipStream_t stream) {
  const int group = p.n_q_heads / p.n_kv_heads;
  const Shape sh = kv8_shape(p, p.workspace_bytes);
  const int ns = sh.own_splits;
  DecodeArgs a{};
  const size_t layer_rows = (size_t)p.layer * p.n_phys_pages * p.n_kv_heads * 16;
  a.q = p.q;
  a.out = p.out;
  a.kc = static_cast<const char *>(p.cache_k) + layer_rows * p.head_dim;
  a.vc = static_cast<const char *>(p.cache_v) + layer_rows * p.head_dim;
  a.ks = p.k_scale + layer_rows;
  a.vs = p.v_scale + layer_rows;
  a.maps = p.maps;
  a.lens = p.lens;
  float *ws = static_cast<float *>(p.workspace);
  if (sh.slots() > 1) {
    const size_t rows = (size_t)p.n_seqs * p.n_q_heads * sh.slots();
    a.part = ws;
    a.part_ml = ws + rows * p.head_dim;
    a.flags = reinterpret_cast<int32_t *>(a.part_ml + 2 * rows);
  }
  a.map_stride = p.map_stride;
  a.max_len = p.max_len;
  a.n_q_heads = p.n_q_heads;
  a.n_kv_heads = p.n_kv_heads;
  a.group = group;
  a.n_qgroups = (group + 15) / 16;
  a.split_pages = sh.split_pages;
  a.max_splits = sh.slots();
  a.own_splits = ns;
  a.n_groups = sh.n_groups;
  a.shared_splits = sh.shared_splits;
  a.n_seqs = p.n_seqs;
  const float log2e = 1.4426950408889634f;
  a.scale_log2 = p.scale * log2e;
  a.cap_in = p.softcap > 0.f ? p.scale / p.softcap : 0.f;
  a.cap_out = p.softcap * log2e;
  const bool cap = p.softcap > 0.f;
  // 8 units side by side, one per XCD; three grid dimensions, for one does not hold every launch
  const int64_t units8 = ((int64_t)p.n_seqs * ns + 7) / 8;
  const uint32_t gy = (uint32_t)std::min<int64_t>(units8, 32768);
  const int n_hq = p.n_kv_heads * a.n_qgroups;
  const dim3 grid(8 * n_hq, gy, (uint32_t)((units8 + gy - 1) / gy));
  // 8 waves where there are fewer workgroups than CUs and their runs give each wave two steps or more (4
  // sequences of 8000 over 8 heads of 128 in 128 workgroups 24.1 -> 21.2 us, in 256 17.8 -> 19.3; with 7 pages 6.2
  // becomes 7.2); up to 256 with head_dim 64, whose steps load half as much (32 of 4000: 29.9 -> 24.7), and where
  // pages may be shared (32 of 17473, all shared: 55 -> 48; none: 181 -> 183).  (head_dim 256 would spill.)
  const bool wide = p.head_dim != 256 && sh.split_pages >= 32 &&
                    (int64_t)n_hq * p.n_seqs * ns <= (p.head_dim == 64 || sh.n_groups > 0 ? 256 : 192);
  auto run = [&](auto kernel, int waves) {
    hipLaunchKernelGGL(kernel, grid, dim3(64 * waves), 0, stream, a);
    return hipGetLastError();
  };
  auto with_cap = [&](auto d, auto c) {
    constexpr int NW8 = d() == 256 ? 4 : 8;
    if (wide)
      return sh.stream ? run(decode_kv8_kernel<d(), c(), NW8, true>, NW8)
                          : run(decode_kv8_kernel<d(), c(), NW8, false>, NW8);
    return sh.stream ? run(decode_kv8_kernel<d(), c(), 4, true>, 4)
                        : run(decode_kv8_kernel<d(), c(), 4, false>, 4);
  };
  auto with_d = [&](auto d) { return cap ? with_cap(d, std::true_type{}) : with_cap(d, std::false_type{}); };
  const hipError_t e = p.head_dim == 64    ? with_d(std::integral_constant<int, 64>{})
                       : p.head_dim == 128 ? with_d(std::integral_constant<int, 128>{})
                                           : with_d(std::integral_constant<int, 256>{});
  if (e != hipSuccess || sh.slots() <= 1) return e;
  return launch_decode_combine(a, p.head_dim, true, stream);
}

}  // namespace nexus
