// Windowed attention of many rows, bf16, head_dim 256 (row-major and transposed V).
//
// The work of window_rows_kernel with the inner loop that head_dim 256 needs: O^T alone takes 128 of the 256 registers
// a wave has at two waves per SIMD, so a workgroup is 8 waves of 32 (token, head) pairs each on one CU, tiles are 32
// keys (two entries of the page list), and Q keeps k-steps 0..5 in registers and 6..15 in LDS.  Each iteration is two
// phases of 16 chunks - one MFMA, operand reads two MFMAs ahead, a few vector instructions - whose order is pinned by
// sched_barrier: S(t + 1) = K(t + 1) Q^T beside the exponentials of S(t), then O^T += V(t)^T P(t)^T beside the soft
// cap of S(t + 1) (in the form 1 / (2^(2 s scale log2(e) / cap) + 1), whose reciprocal is split over both phases).
// MFMA-bound by intensity.  1536 rows of 16 heads over 8 in a window of 4096, transposed V, capped: 150 us and 11 of
// merge, MFMA busy 44% (with the schedule of window_rows_kernel, 4 waves and 64-key tiles, 366 us).
// LDS tiles: K rows in pairs, pair p at 1056 p (32 bytes of padding), row r of a pair at 512 r, chunk c at c ^ r.
// Transposed V: 64-byte feature rows, chunk c at c ^ ((d >> 2) & 3), and K rows of a page permuted (bits 2 and 3 of the
// slot swapped) so that a lane's scores are 8 consecutive keys.  Row-major V: 512-byte key rows, chunk c at
// c ^ 4 (r & 3), read back transposed.  Operand reads are free of bank conflicts.
#include "attn_dma.h"
#include "window_common.h"

#include <type_traits>

namespace nexus {

namespace {

constexpr int kWideRing = 2048;    // entries of the page ring in LDS

}  // namespace

template <bool VT, bool CAP>
__global__ __launch_bounds__(512, 1) void window_d256_kernel(const WindowArgs a) {
  constexpr int W = 8;                        // waves
  static_assert(kWideRows == 32 * W, "a wave takes 32 pairs");
  constexpr int D = 256, KT = 32;
  constexpr int NS = D / 16;                  // k-steps of Q K^T
  constexpr int NSR = 6;                      // k-steps whose Q operand stays in registers
  constexpr int NDB = D / 32;                 // 32-row blocks of O^T
  constexpr int ROWB = D * 2;                 // bytes per K (and row-major V) row
  constexpr int VROWB = KT * 2;               // bytes per feature row of a transposed V tile
  constexpr int PAIRB = 2 * ROWB + 32;        // bytes per K row pair, padded
  constexpr int KTILEB = (KT / 2) * PAIRB;    // bytes per K tile
  constexpr int VTILEB = KT * ROWB;           // bytes per V tile
  constexpr int V0 = 2 * KTILEB;              // V buffers
  constexpr int QL0 = V0 + 2 * VTILEB;        // upper k-steps of Q
  constexpr int QLB = (NS - NSR) * 1024;      // per wave
  constexpr float kSlack = 8.0f;              // lazy rescale: p <= 2^8 between rescales
  __shared__ __align__(1024) char smem[QL0 + W * QLB];
  __shared__ __align__(16) int32_t pg[kWideRing];

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int j = lane & 31, hh = lane >> 5;
  const int kvh = blockIdx.x % a.n_kv_heads;
  const uint32_t rest = blockIdx.x / a.n_kv_heads;
  const int split = a.n_splits == 1 ? 0 : rest % a.n_splits;
  const uint32_t u = a.n_units / a.n_kv_heads - 1 - (a.n_splits == 1 ? rest : rest / a.n_splits);
  const RowTile rt = find_tile<kWideRows>(a, u);
  if (rt.b < 0) return;
  const int G = a.group;
  const bool direct = a.n_splits == 1;

  const int iw = rt.i0 + 32 * wave;
  const bool active = iw < rt.n;
  const int pair = min(iw + j, rt.n - 1);
  const int tok = pair / G, qhead = kvh * G + pair - tok * G;
  const size_t row = (size_t)(rt.row0 + tok) * a.n_q_heads + qhead;
  const int pos = rt.past + tok;
  const bool row_ok = iw + j < rt.n;
  const int p0 = rt.past + rt.i0 / G, p1 = rt.past + min(rt.i0 + kWideRows - 1, rt.n - 1) / G;
  const int pa = __builtin_amdgcn_readfirstlane(rt.past + min(iw, rt.n - 1) / G);
  const int pb_ = __builtin_amdgcn_readfirstlane(rt.past + min(iw + 31, rt.n - 1) / G);

  KeyList kl{};
  TileOrder<2> order{};
  if (p1 >= 0) {
    kl = key_list(a.window, a.sinks, p0, p1);
    order = tile_order<2>(kl, a.period, split, a.n_splits);
  }
  const int T = order.t1 - order.t0, n_le = 2 * T;                  // steps, and entries of the ring
  const int32_t *map = a.maps + (size_t)rt.b * a.map_stride;
  for (int i = tid; i < min(n_le, kWideRing); i += 64 * W) pg[i] = map[kl.page(min(order.entry(i), kl.n - 1))];

  // Q as B operands: lane (hh, j) holds Q[16 s + 8 hh .. + 7] of pair j; k-steps from NSR on in LDS (the offsets live in
  // registers, hidden from the compiler, so that buffer and block offsets fit the immediate of the LDS reads)
  bf16x8 qreg[NSR];
  const uint32_t qlds_off = QL0 + wave * QLB + 16 * lane;
  uint32_t oq = qlds_off;
  asm volatile("" : "+v"(oq));

  f32x16 o[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[db][v] = 0.f;
  float m_ref = -INFINITY;
  float l = 0.f;

  // ---- lane-invariant LDS read offsets.  K: row j, chunk 2s + hh at (2s + hh) ^ (j & 1)
  const uint32_t offk = (j >> 1) * PAIRB + (j & 1) * ROWB + 16 * (hh ^ (j & 1));
  // V.  Transposed: feature row 32 db + j, chunk 2 ks + hh.  Row-major: key row 4 h2 + e (and 8 more), features of
  // block db, whose low two bits the swizzle changes
  uint32_t offv[VT ? 2 : 4];
  if constexpr (VT) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) offv[ks] = V0 + j * VROWB + (((2 * ks + hh) ^ ((j >> 2) & 3)) * 16);
  } else {
    const int gg = lane >> 4, r = lane & 15, e = r >> 2, q = r & 3;
#pragma unroll
    for (int x = 0; x < 4; ++x)
      offv[x] = V0 + (4 * (gg >> 1) + e) * ROWB + 32 * (gg & 1) + 8 * q + 64 * (x ^ e);
  }
#pragma unroll
  for (auto &x : offv) asm volatile("" : "+v"(x));

  // ---- DMA.  K: wave w fills tile rows 4w .. 4w + 3 (two pairs, one an instruction) of the page of entry
  // 2t + w / 4; lane (h1, at) of instruction i fills row 4w + 2i + h1, position `at`, with chunk at ^ h1 of the row's
  // slot, kslot0 + 2i + h1.  Row-major V: the same rows, natural order, chunk at ^ 4 (2i + h1).
  const int at = lane & 31, h1 = lane >> 5;
  const uint32_t kdo = (uint32_t)h1 * ROWB + (uint32_t)((at ^ h1) * 16);
  const int kslot0 = VT ? 8 * (wave & 1) + 4 * ((wave >> 1) & 1) : 4 * (wave & 3);
  const int vslot0 = 4 * (wave & 3);
  const uint32_t vdo[2] = {(uint32_t)h1 * ROWB + (uint32_t)((at ^ (4 * h1)) * 16),
                           (uint32_t)h1 * ROWB + (uint32_t)((at ^ (4 * (2 + h1))) * 16)};
  // transposed V: wave w fills feature rows 32w .. 32w + 31, 16 an instruction; lane (r4 = lane / 4, q = lane % 4)
  // fills row 32w + 16i + r4, position q, with key chunk q ^ ((lane >> 4) & 3)
  const int vchunk = (lane & 3) ^ ((lane >> 4) & 3);
  const uint32_t vrow0 = (uint32_t)(32 * wave + (lane >> 2)) * a.n_cols * 2u;
  const uint32_t vrow_step = 16u * a.n_cols * 2u;                  // 16 feature rows
  const uint32_t smem_base = (uint32_t)(uintptr_t)smem;
  const uint64_t pbytes = (uint64_t)a.n_kv_heads * kPage * ROWB;   // one physical page
  const char *kbytes = reinterpret_cast<const char *>(a.kc) + (uint64_t)kvh * kPage * ROWB;
  const char *vbytes = reinterpret_cast<const char *>(a.vc) +
                       (VT ? (uint64_t)kvh * D * a.n_cols * 2u : (uint64_t)kvh * kPage * ROWB);
  auto kbuf = [&](int i) { return smem + i * KTILEB; };
  auto vbuf = [&](int i) { return smem + V0 + i * VTILEB; };
  auto vrd = [&](int i) { return smem + i * VTILEB; };             // as the reads see it: offv carries V0

  // the page list is waited for before any DMA is in flight (the compiler's own vmcnt bookkeeping must never count DMA
  // loads)
  wait_vm<0>();
  __syncthreads();   // pg[] visible

  auto ring = [&](int le) { return pg[max(min(le, n_le - 1), 0) & (kWideRing - 1)]; };
  auto k_page = [&](int it) { return ring(2 * it + (wave >> 2)); };
  auto v_page = [&](int it) { return VT ? ring(2 * it + (vchunk >> 1)) : 0; };
  auto tile_key = [&](int it) { return kl.page(2 * order.tile(it)) * kPage; };
  auto inner = [&](int it) {
    const int k = tile_key(it);
    return 2 * order.tile(it) >= kl.sp && k >= kl.lo && k + KT <= kl.hi;
  };
  // rows of this wave's page, into K (sel 0) or row-major V (sel 1)
  auto dma_rows = [&](int it, int sel, char *dstp, int page) {
    const uint32_t dst = smem_base + (uint32_t)(dstp - smem) + wave * 2 * (sel ? 2 * ROWB : PAIRB);
    const uint32_t step = sel ? 2 * ROWB : PAIRB;
    const char *ps = (sel ? vbytes : kbytes) + (uint32_t)__builtin_amdgcn_readfirstlane(page) * pbytes;
    const int s0 = sel ? vslot0 : kslot0;
    if (inner(it)) {
      dma_s<0>(dst, ps + s0 * ROWB, sel ? vdo[0] : kdo);
      dma_s<0>(dst + step, ps + (s0 + 2) * ROWB, sel ? vdo[1] : kdo);
    } else {
      const int key0 = kl.page(min(2 * order.tile(it) + (wave >> 2), kl.n - 1)) * kPage;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t from = (uint32_t)kl.stand_in(key0 + s0 + 2 * i + h1) & (kPage - 1);
        const uint32_t chunk = at ^ (sel ? 4 * (2 * i + h1) : h1);
        dma_s<0>(dst + i * step, ps, from * ROWB + chunk * 16);
      }
    }
  };
  auto dma_v = [&](int it, char *dstp, int kpage, int vpage) {
    if constexpr (VT) {
      const uint32_t dst = smem_base + (uint32_t)(dstp - smem) + wave * 32 * VROWB;
      const uint32_t vo = vrow0 + ((uint32_t)vpage * kPage + 8u * (vchunk & 1)) * 2u;
      dma_s<0>(dst, vbytes, vo);
      dma_s<0>(dst + 1024, vbytes, vo + vrow_step);
    } else {
      dma_rows(it, 1, dstp, kpage);
    }
  };
  auto group_key = [&](int it, int g) {
    const int e = 2 * order.tile(it) + g;
    return e < kl.n ? kl.page(e) * kPage : 1 << 30;
  };
  // transposed V: keys that no row sees, cleared in the feature rows that this wave loaded once they have landed
  auto clear_unseen = [&](int it, char *vl) {
    if (!VT || inner(it)) return;
    asm volatile("" ::: "memory");
    const int c = lane & 3;
    const int k0 = group_key(it, c >> 1) + 8 * (c & 1);
    u32x4 keep;
#pragma unroll
    for (int w = 0; w < 4; ++w)
      keep[w] = (kl.seen(k0 + 2 * w) ? 0xFFFFu : 0u) | (kl.seen(k0 + 2 * w + 1) ? 0xFFFF0000u : 0u);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int d = 32 * wave + 16 * i + (lane >> 2);
      u32x4 *x = reinterpret_cast<u32x4 *>(vl + d * VROWB + 16 * (c ^ ((d >> 2) & 3)));
      *x &= keep;
    }
  };

  const float c_scale = a.scale_log2;   // raw score -> log2 units (no cap)
  const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3F803F80u);
  constexpr float kMasked = CAP ? INFINITY : -INFINITY;   // a masked score (r = +inf with the cap)

  auto qk = [&](const char *kb, f32x16 &sc) __attribute__((always_inline)) {
#pragma unroll
    for (int v = 0; v < 16; ++v) sc[v] = 0.f;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const bf16x8 ka = *reinterpret_cast<const bf16x8 *>(kb + offk + 32 * s);
      const bf16x8 qs = s < NSR ? qreg[s < NSR ? s : 0]
                                : *reinterpret_cast<const bf16x8 *>(smem + oq + (s - NSR) * 1024);
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, qs, sc, 0, 0, 0);
    }
  };
  // Soft cap in two stages: the capped score is cap_out (1 - 2 r), r = 1 / e, e = 2^(s cap_k) + 1.  The first stage
  // leaves e in registers 8..15 and r in 0..7; the second takes the reciprocals of 8..15.  A masked score is r = +inf
  // (registers 0..7) or e = 0 (8..15).
  auto cap = [&](f32x16 &sc) __attribute__((always_inline)) {
    if constexpr (CAP) {
#pragma unroll
      for (int v = 0; v < 16; ++v) sc[v] = fast_exp2(sc[v] * a.cap_k) + 1.0f;
#pragma unroll
      for (int v = 0; v < 8; ++v) sc[v] = __builtin_amdgcn_rcpf(sc[v]);
    }
  };
  auto needs_mask = [&](int t) {
    const int k = tile_key(t);
    return !(inner(t) && k + KT - 1 <= pa && (k > pb_ - a.window || k + KT - 1 < a.sinks));
  };
  // register v of lane half hh: slot (v & 7) + 8 hh (transposed V), else 8 ((v >> 2) & 1) + (v & 3) + 4 hh, of the
  // tile's page v >> 3
  auto mask = [&](f32x16 &sc, int t) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int k0 = group_key(t, g) + (VT ? 8 : 4) * hh;
      const int up = pos - k0, low = pos - a.window - k0, snk = a.sinks - k0;
#pragma unroll
      for (int v = 0; v < 8; ++v) {
        const int off = VT ? v : 8 * (v >> 2) + (v & 3);
        if (off > up || (off <= low && off >= snk)) sc[8 * g + v] = (CAP && g == 1) ? 0.f : kMasked;
      }
    }
  };
  // row maximum in log2 units (-inf when every key is masked; with the cap, of scores after its first stage)
  auto row_max = [&](const f32x16 &sc) __attribute__((always_inline)) -> float {
    if constexpr (CAP) {
      float rmin = INFINITY, emax = 0.f;        // largest score = smallest r = 1 / largest e
#pragma unroll
      for (int v = 0; v < 8; ++v) rmin = fminf(rmin, sc[v]);
#pragma unroll
      for (int v = 8; v < 16; ++v) emax = fmaxf(emax, sc[v]);
      const float x = fmaxf(emax, __builtin_amdgcn_rcpf(rmin));
      return fmaf(__builtin_amdgcn_rcpf(max_halves(x)), -2.0f * a.cap_out, a.cap_out);
    } else {
      float mt = -INFINITY;
#pragma unroll
      for (int v = 0; v < 16; ++v) mt = fmaxf(mt, sc[v]);
      return max_halves(mt) * c_scale;
    }
  };
  // S^T of the K tile at `kb` into sn, beside P = 2^(score - m_ref) of the scores in sc (rounded to bf16 as V and the
  // output are, summed as rounded)
  auto qk_exp = [&](const char *kb_, f32x16 &sn, f32x16 &sc, float nm, bf16x8 *pb) __attribute__((always_inline)) {
    const float fa = CAP ? -2.0f * a.cap_out : c_scale;
    const float fc = CAP ? a.cap_out + nm : nm;
    auto kread = [&](int k) { return *reinterpret_cast<const bf16x8 *>(kb_ + offk + 32 * k); };
    auto qread = [&](int k) { return *reinterpret_cast<const bf16x8 *>(smem + oq + (k - NSR) * 1024); };
    bf16x8 kb[3], qb[3];
    kb[0] = kread(0);
    kb[1] = kread(1);
#pragma unroll
    for (int v = 0; v < 16; ++v) sn[v] = 0.f;
    uint32_t w[8];
    float p_even = 0.f;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      if (i + 2 < NS) {
        kb[(i + 2) % 3] = kread(i + 2);
        if (i + 2 >= NSR) qb[(i + 2) % 3] = qread(i + 2);
      }
      sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kb[i % 3], i < NSR ? qreg[i < NSR ? i : 0] : qb[i % 3], sn, 0, 0,
                                                   0);
      if constexpr (CAP) {
        if (i < 8) sc[8 + i] = __builtin_amdgcn_rcpf(sc[8 + i]);
      }
      const float p = fast_exp2(fmaf(sc[i], fa, fc));
      if (i & 1) {
        w[i >> 1] = pack_bf16x2(p_even, p);
        l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[i >> 1]), ones, l, false);
      } else {
        p_even = p;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    pb[0] = __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
    pb[1] = __builtin_bit_cast(bf16x8, u32x4{w[4], w[5], w[6], w[7]});
  };
  // O^T += V^T P^T over the V tile at `vl`, beside the first cap stage of sn
  auto pv_cap = [&](const char *vl, const bf16x8 *pb, f32x16 &sn) __attribute__((always_inline)) {
    constexpr int NM = NDB * 2;
    auto vread = [&](int i) {
      const int ks = i / NDB, db = i % NDB;
      if constexpr (VT) {
        return *reinterpret_cast<const bf16x8 *>(vl + offv[VT ? ks : 0] + db * 32 * VROWB);
      } else {
        const char *p = vl + offv[db & 3] + 256 * (db >> 2) + ks * 16 * ROWB;
        return tr_read_pair(p, p + 8 * ROWB);
      }
    };
    bf16x8 vb[3];
    vb[0] = vread(0);
    vb[1] = vread(1);
#pragma unroll
    for (int i = 0; i < NM; ++i) {
      if (i + 2 < NM) vb[(i + 2) % 3] = vread(i + 2);
      o[i % NDB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vb[i % 3], pb[i / NDB], o[i % NDB], 0, 0, 0);
      if constexpr (CAP) {
        sn[i] = fast_exp2(sn[i] * a.cap_k) + 1.0f;
        if (i < 8) sn[i] = __builtin_amdgcn_rcpf(sn[i]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  if (T > 0) {
    dma_rows(0, 0, kbuf(0), k_page(0));
    dma_v(0, vbuf(0), k_page(0), v_page(0));
  }
  if (T > 1) dma_rows(1, 0, kbuf(1), k_page(1));
  // pages of K(t + 2) and V(t + 1) at t = 0 (row-major V: this wave's page of a tile serves K and then V)
  int kp_next = k_page(2), kp_v = k_page(1), vp_next = v_page(1);
  // Q, behind the DMA: the compiler's waits for these loads count only loads issued after them, and the DMA loads,
  // issued earlier, complete first
  if (active) {
    const uint16_t *qrow = reinterpret_cast<const uint16_t *>(a.q) + row * D;
#pragma unroll
    for (int s = 0; s < NSR; ++s) qreg[s] = *reinterpret_cast<const bf16x8 *>(qrow + 16 * s + 8 * hh);
#pragma unroll
    for (int s = NSR; s < NS; ++s)
      *reinterpret_cast<bf16x8 *>(smem + qlds_off + (s - NSR) * 1024) =
          *reinterpret_cast<const bf16x8 *>(qrow + 16 * s + 8 * hh);
  }
  wait_vm<0>();
  if (T > 0) clear_unseen(0, vbuf(0));
  tile_barrier();

  f32x16 sa, sb;
  float mt_cur = -INFINITY;                     // row maximum of S(t), log2 units
  if (active && T > 0) {
    qk(kbuf(0), sa);
    cap(sa);
    mt_cur = row_max(sa);        // unmasked: iteration 0 masks S(0) and takes its maximum again
  }
  tile_barrier();                // every wave has read K(0): its buffer may be refilled

  auto step = [&](int t, auto par, f32x16 &s_cur, f32x16 &s_nxt) __attribute__((always_inline)) {
    constexpr int P = decltype(par)::value;     // t % 2
    if (t + 2 < T) dma_rows(t + 2, 0, kbuf(P), kp_next);
    if (t + 1 < T) dma_v(t + 1, vbuf(P ^ 1), kp_v, vp_next);
    if ((t & 511) == 0 && t > 0) {
      // the ring's half behind this tile takes the entries 1024 ahead
      for (int i = 2 * t + kWideRing / 2 + tid; i < min(2 * t + kWideRing, n_le); i += 64 * W)
        pg[i & (kWideRing - 1)] = map[kl.page(min(order.entry(i), kl.n - 1))];
    }
    kp_v = kp_next;
    kp_next = k_page(t + 3);
    vp_next = v_page(t + 2);
    if (active) {
      if (needs_mask(t)) {
        mask(s_cur, t);
        mt_cur = row_max(s_cur);
      }
      if (__builtin_amdgcn_ballot_w64(mt_cur > m_ref + kSlack) != 0) {
        const float m_new = fmaxf(m_ref, mt_cur);
        const float alpha = (m_new == -INFINITY) ? 1.f : fast_exp2(m_ref - m_new);
        l *= alpha;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[db][v] *= alpha;
        m_ref = m_new;
      }
      const float nm = (m_ref == -INFINITY) ? 0.f : -m_ref;
      bf16x8 pb[2];
      // (on the last tile S(t + 1) comes from a stale K buffer: a result never used)
      qk_exp(kbuf(P ^ 1), s_nxt, s_cur, nm, pb);
      pv_cap(vrd(P), pb, s_nxt);
      mt_cur = row_max(s_nxt);
    }
    wait_vm<0>();
    if (t + 1 < T) clear_unseen(t + 1, vbuf(P ^ 1));
    tile_barrier();
  };
  for (int t = 0; t < T; t += 2) {
    step(t, std::integral_constant<int, 0>{}, sa, sb);
    if (t + 1 < T) step(t + 1, std::integral_constant<int, 1>{}, sb, sa);
  }

  if (!active) return;
  store_rows<D, VT, CAP>(a, kl, order, rt, kvh, split, direct, pair, row, pos, row_ok, hh, m_ref, l, o);
}

hipError_t launch_window_d256(const WindowArgs &a, bool vt, bool cap, hipStream_t stream) {
  const dim3 grid(a.n_units * a.n_splits);
  auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(512), 0, stream, a);
    return hipGetLastError();
  };
  if (vt) return cap ? run(window_d256_kernel<true, true>) : run(window_d256_kernel<true, false>);
  return cap ? run(window_d256_kernel<false, true>) : run(window_d256_kernel<false, false>);
}

}  // namespace nexus
