// Windowed attention of many rows, bf16, head_dim 64 and 128 (MFMA): every row of a ragged batch sees the last `window`
// keys of its own sequence and the first `sinks` ones (Sec. III-A's attention, restricted as models with local layers
// do).
//
// softmax(s) V with s = scale q.k (soft-capped or not) over the keys that the row sees, in one pass with a running
// maximum and sum (log2 units), O^T += V^T.P^T and S^T = K.Q^T on 32x32x16 MFMA.
// Work: a workgroup is one KV head and 128 (token, head of the group) pairs of one sequence, token by token, 32 to a
// wave; it reads the keys that these pairs see together, window + 128 / group tokens and the sinks, once.  The keys
// come in tiles of 4 entries of a page list (sinks' pages, then the window's), one page a wave, so that the pages
// between them are never touched and the sinks cost one tile.  K[t + 2] and V[t + 1] travel global -> LDS (LDS DMA,
// swizzled by the lanes' source chunks) while S(t + 1) and O of tile t are computed: layouts, waits and schedule are
// those of attn_bf16_dma_kernel.
// 4096 rows of 40 heads over 8 of 128 at depth 12288, window 4096, 4 sinks: 331 us, 1040 TFLOP/s, MFMA busy 53%, 107 MB
// read (at the board's power limit; the loop is that of suffix attention).  head_dim 64, 16 sequences of up to 517 rows,
// 32 heads over 8, window 1024: 56 us, MFMA busy 31%.  Vector instructions, a fifth of them exponentials at a quarter
// rate, take some 30 us of it; 15 are rounds (four and a quarter workgroups a CU where three run together) and edges,
// which a prefill that fills the chip (757 TFLOP/s) does not have.
// Keys that no row of the tile sees (before the window, past the end, between sinks and window) are replaced by one
// that is seen (transposed V: zeroed) and masked; where a key is seen by some rows only and its value is not finite,
// row_again forms the rows that came out not finite.
#include "attn_dma.h"
#include "window_common.h"

#include <type_traits>

namespace nexus {

namespace {

constexpr int kRing = 2048;        // entries of the page ring in LDS

}  // namespace

template <int D, bool VT, bool CAP>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void window_rows_kernel(const WindowArgs a) {
  static_assert(D == 64 || D == 128, "head_dim");
  static_assert(kMfmaRows == 4 * 32, "4 waves of 32 pairs");
  constexpr int KT = 64;
  constexpr int NKB = KT / 32, NDB = D / 32, NS = D / 16;
  constexpr int ROWB = D * 2;                 // bytes per K or V row
  constexpr int TILEB = KT * ROWB;            // bytes per K or V tile
  constexpr int QTRB = TILEB / 4;             // a wave's quarter: one page
  constexpr int CH = D / 8;                   // 16-byte chunks per row
  constexpr int RPI = 64 / CH;                // rows of a DMA instruction
  constexpr int NI = QTRB / 1024;             // DMA instructions per quarter
  constexpr int VROWB = KT * 2;               // bytes per feature row of a transposed V tile
  constexpr float kSlack = 8.0f;              // lazy rescale: p <= 2^8 between rescales
  constexpr int kPrioPV = 2;                  // wave priority of the PV phase
  __shared__ __align__(1024) char smem[2 * 2 * TILEB];   // K buffers 0, 1, V buffers 0, 1
  __shared__ __align__(16) int32_t pg[kRing];

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int j = lane & 31, hh = lane >> 5;
  const int kvh = blockIdx.x % a.n_kv_heads;
  const uint32_t rest = blockIdx.x / a.n_kv_heads;
  const int split = a.n_splits == 1 ? 0 : rest % a.n_splits;
  // later tiles of a sequence see more keys (up to the window): the longest go first
  const uint32_t u = a.n_units / a.n_kv_heads - 1 - (a.n_splits == 1 ? rest : rest / a.n_splits);
  const RowTile rt = find_tile<kMfmaRows>(a, u);
  if (rt.b < 0) return;
  const int G = a.group;
  const bool direct = a.n_splits == 1;

  // this lane's pair, and the positions of the tile's and of the wave's rows
  const int iw = rt.i0 + 32 * wave;
  const bool active = iw < rt.n;
  const int pair = min(iw + j, rt.n - 1);
  const int tok = pair / G, qhead = kvh * G + pair - tok * G;
  const size_t row = (size_t)(rt.row0 + tok) * a.n_q_heads + qhead;
  const int pos = rt.past + tok;
  const bool row_ok = iw + j < rt.n;
  const int p0 = rt.past + rt.i0 / G, p1 = rt.past + min(rt.i0 + kMfmaRows - 1, rt.n - 1) / G;
  const int pa = __builtin_amdgcn_readfirstlane(rt.past + min(iw, rt.n - 1) / G);
  const int pb = __builtin_amdgcn_readfirstlane(rt.past + min(iw + 31, rt.n - 1) / G);

  KeyList kl{};
  TileOrder<4> order{};
  if (p1 >= 0) {
    kl = key_list(a.window, a.sinks, p0, p1);
    order = tile_order<4>(kl, a.period, split, a.n_splits);
  }
  const int n_tiles = order.t1 - order.t0, n_le = 4 * n_tiles;      // steps, and entries of the ring
  const int32_t *map = a.maps + (size_t)rt.b * a.map_stride;
  // the page ring: entries 0 .. kRing - 1 here, the next half every 256 tiles
  for (int i = tid; i < min(n_le, kRing); i += 256) pg[i] = map[kl.page(min(order.entry(i), kl.n - 1))];

  bf16x8 qreg[NS];
  if (active) {
    const uint16_t *qrow = reinterpret_cast<const uint16_t *>(a.q) + row * D;
#pragma unroll
    for (int s = 0; s < NS; ++s)
      qreg[s] = *reinterpret_cast<const bf16x8 *>(qrow + 16 * s + 8 * hh);
  }

  f32x16 o[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[db][v] = 0.f;
  float m_ref = -INFINITY;
  float l = 0.f;

  // ---- lane-invariant LDS read offsets; score row j belongs to key kj of its 32 (transposed V: bits 2 and 3
  // swapped, so that a lane's scores of 16 keys are 8 consecutive ones)
  const int kj = VT ? ((j & ~12) | ((j & 4) << 1) | ((j & 8) >> 1)) : j;
  uint32_t offk[NS];                          // S^T A operand: K row kj, chunk 2s + hh
#pragma unroll
  for (int s = 0; s < NS; ++s)
    offk[s] = kj * ROWB + (((2 * s + hh) ^ (D == 64 ? (kj >> 1) & 7 : kj & 15)) * 16);
  uint32_t offv[NDB];                         // PV A operand
  if constexpr (VT) {
#pragma unroll
    for (int db = 0; db < NDB; ++db) offv[db] = (32 * db + j) * VROWB;   // chunk added in pv_step
  } else {
    const int gg = lane >> 4, r = lane & 15, e = r >> 2, q = r & 3;
    const int h2 = gg >> 1, dh = gg & 1;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
      offv[db] = (4 * h2 + e) * ROWB + 32 * dh + 8 * q + 64 * (db ^ (D == 64 ? e >> 1 : e));
  }
  // ---- DMA: wave w fills tile rows 16 w .. 16 w + 15, the page of entry 4 t + w; instruction i covers slots
  // i RPI + lr, lane position lane % CH of the row; the source chunk undoes the swizzle
  const int lr = lane / CH;
  auto kswz = [](int r) { return D == 64 ? (r >> 1) & 7 : r & 15; };
  auto vswz = [](int r) { return D == 64 ? 4 * ((r >> 1) & 1) : 4 * (r & 3); };
  const uint32_t kdo = lr * ROWB + (((lane % CH) ^ kswz(lr)) * 16);
  const uint32_t vdo = lr * ROWB + (((lane % CH) ^ vswz(lr)) * 16);
  const uint32_t smem_base = (uint32_t)(uintptr_t)smem;
  const uint64_t pbytes = (uint64_t)a.n_kv_heads * kPage * ROWB;   // one physical page
  const char *kbytes = reinterpret_cast<const char *>(a.kc) + (uint64_t)kvh * kPage * ROWB;
  const char *vbytes = reinterpret_cast<const char *>(a.vc) +
                       (VT ? (uint64_t)kvh * D * a.n_cols * 2 : (uint64_t)kvh * kPage * ROWB);
  // transposed V: wave w fills feature rows w D / 4 .., 8 rows an instruction, lane position lane % 8; in
  // instruction i that is key chunk vc ^ 4 (i & 1), of the tile's page vp ^ 2 (i & 1)
  const int vc = (lane & 7) ^ (lane >> 4), vp = vc >> 1;
  const uint32_t vto = ((uint32_t)(wave * (D / 4) + (lane >> 3)) * a.n_cols + 8 * (vc & 1)) * 2;
  uint32_t vpg[2];                                                 // pages of the next V tile's DMA
  auto ring = [&](int le) { return (uint32_t)pg[min(le, n_le - 1) & (kRing - 1)]; };
  auto v_pages = [&](int it) {
    vpg[0] = ring(4 * it + vp);
    vpg[1] = ring(4 * it + (vp ^ 2));
  };
  auto kbuf = [&](int i) { return smem + i * TILEB; };
  auto vbuf = [&](int i) { return smem + (2 + i) * TILEB; };

  // The page list is there; Q may be on its way still: the wait for the first tiles covers it (no wait of the compiler's
  // for Q may stand in the tile loop, whose vmcnt would count DMA loads too).  43 sequences of 62 rows 31.7 -> 29.9 us.
  tile_barrier();    // pg[] visible

  auto page_of = [&](int it) -> uint32_t { return __builtin_amdgcn_readfirstlane(ring(4 * it + wave)); };
  // first key of tile `it`, and whether its 64 keys are neighbours that some row sees each
  auto tile_key = [&](int it) { return kl.page(4 * order.tile(it)) * kPage; };
  auto inner = [&](int it) {
    const int k = tile_key(it);
    return 4 * order.tile(it) >= kl.sp && k >= kl.lo && k + KT <= kl.hi;
  };
  // DMA of one K or V tile (`sel` 0 = K, 1 = V) of tile `it` into this wave's quarter of the buffer at `dstp`
  auto dma_tile = [&](int it, int sel, char *dstp, uint32_t page) {
    const char *src = sel ? vbytes : kbytes;
    const uint32_t dst = smem_base + (uint32_t)(dstp - smem) + wave * QTRB;
    auto go = [&](int i, const char *s, uint32_t voff) {
      if (i == 0) dma_s<0>(dst, s, voff);
      else if (i == 1) dma_s<1 * 1024>(dst, s, voff);
      else if (i == 2) dma_s<2 * 1024>(dst, s, voff);
      else dma_s<3 * 1024>(dst, s, voff);
    };
    if (VT && sel) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
        dma_s<0>(dst + i * 1024, src, vto + vpg[i & 1] * (2 * kPage) + (uint32_t)i * 16 * a.n_cols);
      return;
    }
    const char *ps = src + page * pbytes;
    if (inner(it)) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
        go(i, ps, sel ? vdo ^ (16u * vswz(i * RPI)) : kdo ^ (16u * kswz(i * RPI)));
    } else {
      const int key0 = kl.page(min(4 * order.tile(it) + wave, kl.n - 1)) * kPage;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int slot = i * RPI + lr;
        const uint32_t from = (uint32_t)kl.stand_in(key0 + slot) & (kPage - 1);
        const uint32_t c = (lane % CH) ^ (sel ? vswz(slot) : kswz(slot));
        dma_s<0>(dst + i * 1024, ps, from * ROWB + c * 16);
      }
    }
  };
  // first key of 16-key group g of tile `it`; past every position behind the list's end
  auto group_key = [&](int it, int g) {
    const int e = 4 * order.tile(it) + g;
    return e < kl.n ? kl.page(e) * kPage : 1 << 30;
  };
  // transposed V: slots that no row sees may hold anything; once such a tile has landed, the wave clears their keys
  // in its quarter
  auto clear_unseen = [&](int it, char *dstp) {
    if (!VT || inner(it)) return;
    asm volatile("" ::: "memory");            // the tile is read after the wait for it
    const int c = lane & 7;
    const int k0 = (c >> 1 == 0 ? group_key(it, 0) : c >> 1 == 1 ? group_key(it, 1)
                    : c >> 1 == 2 ? group_key(it, 2) : group_key(it, 3)) + 8 * (c & 1);
    u32x4 keep;
#pragma unroll
    for (int w = 0; w < 4; ++w)
      keep[w] = (kl.seen(k0 + 2 * w) ? 0xFFFFu : 0u) | (kl.seen(k0 + 2 * w + 1) ? 0xFFFF0000u : 0u);
    for (int x = lane >> 3; x < D / 4; x += 8) {
      const int r = wave * (D / 4) + x;
      u32x4 *at = reinterpret_cast<u32x4 *>(dstp + r * VROWB + 16 * (c ^ ((r >> 1) & 7)));
      *at &= keep;
    }
  };

  const float c_scale = CAP ? 1.0f : a.scale_log2;
  const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3F803F80u);

  // S^T of one tile from K buffer `kb` (raw scores)
  auto qk = [&](const char *kb_, f32x16 *sacc) {
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int v = 0; v < 16; ++v) sacc[kb][v] = 0.f;
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb) {
        const bf16x8 ka = *reinterpret_cast<const bf16x8 *>(kb_ + kb * 32 * ROWB + offk[s]);
        sacc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, qreg[s], sacc[kb], 0, 0, 0);
      }
  };
  // S(t) needs its mask unless every row of the wave sees all 64 keys
  auto needs_mask = [&](int t) {
    const int k = tile_key(t);
    return !(inner(t) && k + KT - 1 <= pa && (k > pb - a.window || k + KT - 1 < a.sinks));
  };
  auto cap = [&](f32x16 *sc) {
    if constexpr (CAP) {
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int v = 0; v < 16; ++v) sc[kb][v] = a.cap_out * window_tanh(sc[kb][v] * a.cap_in);
    }
  };
  // the mask of S(t), a page at a time: most edges of a wave's rows lie in one or two
  auto mask = [&](f32x16 *sc, int t) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int k = group_key(t, g), k0 = k + (VT ? 8 : 4) * hh;
      if (k + kPage - 1 > pa) {                                   // keys ahead of some row
        const int up = pos - k0;
#pragma unroll
        for (int v = 0; v < 8; ++v)
          if ((VT ? v : 8 * (v >> 2) + (v & 3)) > up) sc[g >> 1][8 * (g & 1) + v] = -INFINITY;
      }
      if (k <= pb - a.window && k + kPage - 1 >= a.sinks) {       // keys that left some row's window
        const int low = pos - a.window - k0, snk = a.sinks - k0;
#pragma unroll
        for (int v = 0; v < 8; ++v) {
          const int off = VT ? v : 8 * (v >> 2) + (v & 3);
          if (off <= low && off >= snk) sc[g >> 1][8 * (g & 1) + v] = -INFINITY;
        }
      }
    }
  };
  // row maximum of S(t) in log2 units
  auto row_max = [&](const f32x16 *sc) -> float {
    float mt = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int v = 0; v < 16; ++v) mt = fmaxf(mt, sc[kb][v]);
    return max_halves(mt) * c_scale;
  };
  // P of 16 keys of a score block as the B operand of a PV step, rounded to bf16 (8 bits, as V and the output have);
  // l adds the rounded values, so that the weights sum to what was multiplied
  auto softmax_half = [&](const f32x16 &sc, int hf, float nm, bf16x8 &pbo) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x0 = fast_exp2(fmaf(sc[8 * hf + 2 * e], c_scale, nm));
      const float x1 = fast_exp2(fmaf(sc[8 * hf + 2 * e + 1], c_scale, nm));
      w[e] = pack_bf16x2(x0, x1);
      l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[e]), ones, l, false);
    }
    pbo = __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
  };
  // O^T += V^T P^T over the 16 keys of step ks of the V tile at vl
  auto pv_step = [&](const char *vl, int ks, const bf16x8 &pbv) {
#pragma unroll
    for (int db = 0; db < NDB; ++db) {
      bf16x8 va;
      if constexpr (VT) {
        va = *reinterpret_cast<const bf16x8 *>(vl + offv[db] + 16 * ((2 * ks + hh) ^ ((j >> 1) & 7)));
      } else {
        const char *p = vl + ks * 16 * ROWB + offv[db];
        va = tr_read_pair(p, p + 8 * ROWB);
      }
      o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, pbv, o[db], 0, 0, 0);
    }
  };

  // Per iteration t: the DMA of K[t + 2] and V[t + 1] runs while the wave computes S(t + 1) = K[t + 1] Q^T and
  // O += V[t] P(t).  K buffers hold tiles t + 1 and t + 2, V buffers tiles t and t + 1.
  f32x16 sa[NKB], sb[NKB];
  uint32_t pgv = 0, pk = 0;
  if (n_tiles > 0) {
    const uint32_t pg0 = page_of(0);
    if constexpr (VT) v_pages(0);
    dma_tile(0, 0, kbuf(0), pg0);
    dma_tile(0, 1, vbuf(0), pg0);
    if constexpr (VT) v_pages(1);
    pgv = page_of(1);
    if (n_tiles > 1) dma_tile(1, 0, kbuf(1), pgv);
    pk = page_of(2);
  }
  wait_vm<0>();
  if (n_tiles > 0) clear_unseen(0, vbuf(0));
  tile_barrier();
  float mt_cur = -INFINITY;                     // row maximum of S(t), log2 units
  if (active && n_tiles > 0) {
    qk(kbuf(0), sa);
    cap(sa);
    mt_cur = row_max(sa);        // unmasked: step 0 masks S(0) and takes its maximum again
  }
  tile_barrier();    // K buffer 0 is refilled in iteration 0

  auto step = [&](int t, auto parity, f32x16 *s_cur, f32x16 *s_nxt) {
    constexpr int P = decltype(parity)::value;     // t & 1
    if (t + 2 < n_tiles) dma_tile(t + 2, 0, kbuf(P), pk);
    if (t + 1 < n_tiles) dma_tile(t + 1, 1, vbuf(P ^ 1), pgv);
    if ((t & 255) == 0 && t > 0) {
      // the ring's half behind this tile takes the entries 1024 ahead (looked up 254 iterations from here)
      for (int i = 4 * t + kRing / 2 + tid; i < min(4 * t + kRing, n_le); i += 256)
        pg[i & (kRing - 1)] = map[kl.page(min(order.entry(i), kl.n - 1))];
    }
    if (active) {
      // the maximum of S(t) was taken before its mask: where there is one, mask and take it again
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
      const char *vl = vbuf(P);
      bf16x8 pb[4];
      qk(kbuf(P ^ 1), s_nxt);
      softmax_half(s_cur[0], 0, nm, pb[0]);
      softmax_half(s_cur[0], 1, nm, pb[1]);
      softmax_half(s_cur[1], 0, nm, pb[2]);
      constexpr int VQ = D == 64 ? 10 : 5, VP = D == 64 ? 4 : 2, VM = D == 64 ? 12 : 6;
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
      for (int i = 0; i < NKB * NS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, VQ, 0);
      }
      // O += V P and what follows run at a raised wave priority: of the waves that share a SIMD, the one in this
      // phase issues first
      __builtin_amdgcn_s_setprio(kPrioPV);
      pv_step(vl, 0, pb[0]);
      pv_step(vl, 1, pb[1]);
      pv_step(vl, 2, pb[2]);
      softmax_half(s_cur[1], 1, nm, pb[3]);
      __builtin_amdgcn_sched_group_barrier(0x100, VT ? 2 : 4, 1);
#pragma unroll
      for (int i = 0; i < 3 * NDB; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
        __builtin_amdgcn_sched_group_barrier(0x100, VT ? 1 : 2, 1);
        __builtin_amdgcn_sched_group_barrier(0x002, VP, 1);
      }
      pv_step(vl, 3, pb[3]);
      cap(s_nxt);
      mt_cur = row_max(s_nxt);
#pragma unroll
      for (int i = 0; i < NDB; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 2);
        __builtin_amdgcn_sched_group_barrier(0x100, VT ? 1 : 2, 2);
        __builtin_amdgcn_sched_group_barrier(0x002, VM, 2);
      }
    }
    __builtin_amdgcn_s_setprio(0);
    // pages for the next iteration's DMA (the LDS read overlaps the wait below)
    pgv = pk;
    pk = page_of(t + 3);
    if constexpr (VT) v_pages(t + 2);
    // K[t + 2] and V[t + 1], issued above, are read in the next iteration
    wait_vm<0>();
    if (t + 1 < n_tiles) clear_unseen(t + 1, vbuf(P ^ 1));
    tile_barrier();
  };
  // (every iteration computes S(t + 1): on the last tile from a K buffer whose contents are stale, a result never used)
  for (int t = 0; t < n_tiles; t += 2) {
    step(t, std::integral_constant<int, 0>{}, sa, sb);
    if (t + 1 < n_tiles) step(t + 1, std::integral_constant<int, 1>{}, sb, sa);
  }

  if (!active) return;
  store_rows<D, VT, CAP>(a, kl, order, rt, kvh, split, direct, pair, row, pos, row_ok, hh, m_ref, l, o);
}

hipError_t launch_window_rows(const WindowArgs &a, int head_dim, bool vt, bool cap, hipStream_t stream) {
  const dim3 grid(a.n_units * a.n_splits);
  auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a);
    return hipGetLastError();
  };
  auto with_d = [&](auto d) {
    if (vt)
      return cap ? run(window_rows_kernel<d(), true, true>) : run(window_rows_kernel<d(), true, false>);
    return cap ? run(window_rows_kernel<d(), false, true>) : run(window_rows_kernel<d(), false, false>);
  };
  if (head_dim == 64) return with_d(std::integral_constant<int, 64>{});
  return with_d(std::integral_constant<int, 128>{});
}

}  // namespace nexus
