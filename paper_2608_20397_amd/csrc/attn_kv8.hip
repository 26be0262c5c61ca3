// Suffix attention over an 8-bit paged cache (kv8_common.h has its format): causal grouped-query
// softmax(Q K^T / sqrt d) V of many queries, optional tanh soft cap, row-major V, head_dim 64, 128 and 256.
//
// The work decomposition, plan and merge are those of the bf16 kernels (attn_bf16.hip): a workgroup serves
// one KV head, each wave one query head x 32 queries, tasks query-major, keys in tiles, the key axis split
// as the plan says, S^T = K.Q^T and O^T += V^T.P^T, online softmax in log2 units with a lazily moved reference.
//   * S^T on v_mfma_scale_f32_32x32x64_f8f6f4 with the keys as they are stored: each query is held as
//     two E4M3 terms hi + lo / 16 (split_query), whose products cost what one bf16 product does; the token's
//     scale byte is the instruction's own operand.  K tiles travel global -> LDS by DMA, 1 byte an element.
//   * V is converted to bf16 on its way to LDS, its scale applied by the conversion: exact.  P is rounded to
//     bf16 as in the bf16 kernels and the PV product is theirs (transposed LDS reads, 32x32x16 MFMA).
//   * A token whose key or value row is not finite (scale byte 255) gives NaN to the queries that see it
//     and nothing to the others: its scores are set to NaN, then masked like any other, and its values
//     enter the product as zeros.
//   * Slots past the last key of a workgroup are never read: their rows repeat the last key and are masked.
// LDS: K row r, 16-byte chunk c at c ^ kswz(r); V (bf16) chunk c at c ^ vswz(r), as the bf16 kernels.
#include "attn_common.h"
#include "attn_dma.h"
#include "kv8_common.h"
#include "launch_kv8.h"

namespace nexus {

template <int D, bool CAP>
__global__ __launch_bounds__(D == 256 ? 512 : 256, 2) void attn_kv8_kernel(const AttnArgs a,
                                                                           const AttnPlan plan) {
  static_assert(D == 64 || D == 128 || D == 256, "head_dim");
  constexpr int W = D == 256 ? kWavesWide : kWaves;
  constexpr int KT = D == 256 ? 32 : 64;
  constexpr int NT = 64 * W;                       // threads
  constexpr int NKB = KT / 32, NDB = D / 32, NS2 = D / 64;
  constexpr int CH = D / 16;                       // 16-byte chunks of a row of codes
  constexpr int KTILEB = KT * D;                   // bytes of a K tile (codes)
  constexpr int NI = KTILEB / 1024 / W;            // DMA instructions of a wave for one K tile
  constexpr int RPI = 1024 / D;                    // rows of one
  constexpr int VROWB = 2 * D;                     // bytes of a V tile row (bf16)
  constexpr int VTILEB = KT * VROWB;
  constexpr int NVC = KT * CH / NT;                // V chunks a thread converts
  constexpr float kSlack = 8.0f;                   // lazy rescale: p <= 2^8 between rescales
  static_assert(NI >= 1 && NVC >= 1 && RPI <= kPage, "tile shape");
  __shared__ __align__(1024) char smem[2 * KTILEB + 2 * VTILEB];
  __shared__ __align__(16) int32_t pg[kMaxSplitKeys / kPage + 8];

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int j = lane & 31, hh = lane >> 5;
  const int kvh = blockIdx.x % a.n_kv_heads;
  const UnitLoc loc = locate_unit(plan, blockIdx.x / a.n_kv_heads);
  const int b = loc.seq;
  const UnitWork uw = loc.w;
  const SeqPlan sp = plan.seq[b];
  const int tgrp = uw.tgrp, split = uw.split;
  const int G = a.group;

  const int task = tgrp * W + wave;
  const bool active = task < sp.n_tasks;
  const int qb = task / G;
  const int g = task - qb * G;
  const int q0 = qb * kQB;
  const int qhead = kvh * G + g;
  const int last_task = min(tgrp * W + W - 1, sp.n_tasks - 1);
  const int last_q = min((last_task / G + 1) * kQB, sp.len);
  const int wg_keys = (int)sp.n_past + last_q;
  const int k_begin = uw.k_begin;
  const int k_end = min(k_begin + uw.split_keys, wg_keys);
  const int qpos0 = (int)sp.n_past + q0;
  const int n_tiles = k_end > k_begin ? (k_end - k_begin + KT - 1) / KT : 0;

  const int pg0 = k_begin >> kPageShift;
  const int n_pg = n_tiles > 0 ? ((k_end - 1) >> kPageShift) - pg0 + 1 : 0;
  for (int i = tid; i < n_pg; i += NT) pg[i] = a.map[pg0 + i];

  // ---- the query as two E4M3 terms: lane (hh, j) holds features 64 s + 32 hh .. + 31 of query q0 + j
  i32x8 qhi[NS2], qlo[NS2];
  int qscale_hi = 127, qscale_lo = 127;
  {
    const int qi = min(q0 + j, sp.len - 1);
    const uint16_t *qrow = a.q + ((int64_t)(sp.q_start + qi) * a.n_q_heads + qhead) * D;
    u32x4 raw[NS2][4];
    uint32_t am = 0;
#pragma unroll
    for (int s = 0; s < NS2; ++s)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        raw[s][c] = active ? *reinterpret_cast<const u32x4 *>(qrow + 64 * s + 32 * hh + 8 * c)
                           : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          am = max(am, max((raw[s][c][e] << 16) & 0x7FFF0000u, raw[s][c][e] & 0x7FFF0000u));
      }
    const auto r = __builtin_amdgcn_permlane32_swap(am, am, false, false);
    am = max((uint32_t)r[0], (uint32_t)r[1]);
    const bool bad = am >= 0x7F800000u;
    const int e = row_exp(am);
    qscale_hi = e + 127;
    qscale_lo = e + 127 - 4;
#pragma unroll
    for (int s = 0; s < NS2; ++s)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float x[8];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          x[2 * w] = __uint_as_float(raw[s][c][w] << 16);
          x[2 * w + 1] = __uint_as_float(raw[s][c][w] & 0xFFFF0000u);
        }
        uint32_t hi[2], lo[2];
        split_query<8>(x, e, bad, hi, lo);
        qhi[s][2 * c] = hi[0];
        qhi[s][2 * c + 1] = hi[1];
        qlo[s][2 * c] = lo[0];
        qlo[s][2 * c + 1] = lo[1];
      }
  }

  f32x16 o[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[db][v] = 0.f;
  float m_ref = -INFINITY;
  float l = 0.f;

  // ---- LDS layouts
  auto kswz = [](int row) { return D == 64 ? (row >> 2) & 3 : D == 128 ? (row >> 1) & 7 : row & 15; };
  auto vswz = [](int row) { return D == 64 ? 4 * ((row >> 1) & 1) : 4 * (row & 3); };
  // S^T A operand: K row j (+ 32 kb, whose swizzle is the same), features 64 s + 32 hh .. + 31
  uint32_t offk[NS2][2];
#pragma unroll
  for (int s = 0; s < NS2; ++s)
#pragma unroll
    for (int c = 0; c < 2; ++c) offk[s][c] = j * D + 16 * ((4 * s + 2 * hh + c) ^ kswz(j));
  uint32_t offv[NDB];                          // PV A operand, as attn_bf16_dma.hip
  {
    const int gg = lane >> 4, r = lane & 15, e = r >> 2, q = r & 3;
    const int h2 = gg >> 1, dh = gg & 1;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
      offv[db] = (4 * h2 + e) * VROWB + 32 * dh + 8 * q + 64 * (db ^ (D == 64 ? e >> 1 : e));
  }
  auto kbuf = [&](int i) { return smem + i * KTILEB; };
  auto vbuf = [&](int i) { return smem + 2 * KTILEB + i * VTILEB; };
  const uint32_t smem_base = (uint32_t)(uintptr_t)smem;
  const uint64_t pbytes = (uint64_t)a.n_kv_heads * kPage * D;      // one physical page of codes
  const uint64_t sbytes = (uint64_t)a.n_kv_heads * kPage;          // and of scales
  const char *kbytes = reinterpret_cast<const char *>(a.kc) + (uint64_t)kvh * kPage * D;
  const char *vbytes = reinterpret_cast<const char *>(a.vc) + (uint64_t)kvh * kPage * D;
  const uint8_t *ksb = a.ks + kvh * kPage, *vsb = a.vs + kvh * kPage;

  // Q and the page table are waited for before any DMA is in flight (attn_bf16_dma.hip)
  wait_vm<0>();
  __syncthreads();   // pg[] visible

  auto page_at = [&](int lp) -> uint64_t {    // wave-uniform logical page, counted from pg0
    return (uint32_t)__builtin_amdgcn_readfirstlane(pg[lp]);
  };
  // DMA of K tile `it`: instruction i of the wave fills rows (wave NI + i) RPI ..
  auto dma_k = [&](int it) {
    const int kt = k_begin + it * KT;
    const uint32_t dst = smem_base + (it & 1) * KTILEB + wave * NI * 1024;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int row0 = (wave * NI + i) * RPI;
      const int row = row0 + lane / CH;
      const uint32_t c = (lane % CH) ^ kswz(row);
      if (kt + KT <= k_end) {
        const char *ps = kbytes + page_at(it * (KT / kPage) + row0 / kPage) * pbytes;
        dma_s<0>(dst + i * 1024, ps, (uint32_t)(row & (kPage - 1)) * D + 16 * c);
      } else {
        const int t = min(kt + row, k_end - 1);
        const uint64_t pp = (uint32_t)pg[(t >> kPageShift) - pg0];
        dma_v(dst + i * 1024, kbytes + pp * pbytes + (uint32_t)(t & (kPage - 1)) * D + 16 * c);
      }
    }
  };
  struct Stage {
    u32x4 v[NVC];                              // V codes on their way to LDS
    uint32_t vs[NVC];                          // their rows' scale bytes
    uint32_t ks, vt;                           // key and value scale bytes of token `lane` of the tile
  };
  auto load_tile = [&](int it, Stage &sg) {
    const int kt = k_begin + it * KT;
    const bool full = kt + KT <= k_end;
#pragma unroll
    for (int k = 0; k < NVC; ++k) {
      const int row0 = (64 * wave + NT * k) / CH;
      const int row = row0 + lane / CH;
      const int t = full ? kt + row : min(kt + row, k_end - 1);
      const uint64_t pp = full ? page_at(it * (KT / kPage) + row0 / kPage)
                               : (uint64_t)(uint32_t)pg[(t >> kPageShift) - pg0];
      const uint32_t slot = t & (kPage - 1);
      sg.v[k] = *reinterpret_cast<const u32x4 *>(vbytes + pp * pbytes + slot * D + 16 * (lane % CH));
      sg.vs[k] = vsb[pp * sbytes + slot];
    }
    const int t = min(kt + (lane & (KT - 1)), k_end - 1);
    const uint64_t pp = (uint32_t)pg[(t >> kPageShift) - pg0];
    sg.ks = ksb[pp * sbytes + (t & (kPage - 1))];
    sg.vt = vsb[pp * sbytes + (t & (kPage - 1))];
  };
  // V codes of a tile to bf16 in LDS; a row that is not finite as zeros
  auto store_v = [&](int it, const Stage &sg) {
    char *vl = vbuf(it & 1);
#pragma unroll
    for (int k = 0; k < NVC; ++k) {
      const int row = (64 * wave + NT * k) / CH + lane / CH;
      const int c = 2 * (lane % CH);
      const bool bad = sg.vs[k] == kBadScale;
      const float s = bad ? 1.f : exp2i((int)sg.vs[k] - 127);
      u32x2 w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = codes_to_bf16(bad ? 0u : sg.v[k][i], s);
      *reinterpret_cast<u32x4 *>(vl + row * VROWB + 16 * (c ^ vswz(row))) =
          u32x4{w[0][0], w[0][1], w[1][0], w[1][1]};
      *reinterpret_cast<u32x4 *>(vl + row * VROWB + 16 * ((c + 1) ^ vswz(row))) =
          u32x4{w[2][0], w[2][1], w[3][0], w[3][1]};
    }
  };

  const float c_scale = CAP ? 1.0f : a.scale_log2;
  const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3F803F80u);

  Stage sg{};
  if (n_tiles > 0) {
    dma_k(0);
    load_tile(0, sg);
  }
  for (int it = 0; it < n_tiles; ++it) {
    const int kt = k_begin + it * KT;
    wait_vm<0>();
    store_v(it, sg);
    // scales of this tile's tokens, and which of them are not finite
    const uint64_t bad = __builtin_amdgcn_ballot_w64(sg.ks == kBadScale || sg.vt == kBadScale);
    const auto ksw = __builtin_amdgcn_permlane32_swap(sg.ks, sg.ks, false, false);
    tile_barrier();   // K and V of tile `it` are in LDS; the other buffers are free
    if (it + 1 < n_tiles) {
      load_tile(it + 1, sg);
      dma_k(it + 1);
    }
    if (!active) continue;
    const char *kl = kbuf(it & 1), *vl = vbuf(it & 1);
    // ---- S^T = K . Q^T
    f32x16 sc[NKB];
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb) {
#pragma unroll
      for (int v = 0; v < 16; ++v) sc[kb][v] = 0.f;
#pragma unroll
      for (int s = 0; s < NS2; ++s) {
        const u32x4 x = *reinterpret_cast<const u32x4 *>(kl + kb * 32 * D + offk[s][0]);
        const u32x4 y = *reinterpret_cast<const u32x4 *>(kl + kb * 32 * D + offk[s][1]);
        const i32x8 ka = {(int)x[0], (int)x[1], (int)x[2], (int)x[3],
                          (int)y[0], (int)y[1], (int)y[2], (int)y[3]};
        const int ks = (int)ksw[kb];
        sc[kb] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ka, qhi[s], sc[kb], 0, 0, 0, ks, 0,
                                                                 qscale_hi);
        sc[kb] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ka, qlo[s], sc[kb], 0, 0, 0, ks, 0,
                                                                 qscale_lo);
      }
    }
    if constexpr (CAP) {
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int v = 0; v < 16; ++v) sc[kb][v] = a.cap_out * tanh_fast(sc[kb][v] * a.cap_in);
    }
    if (bad) {
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (bad >> (32 * kb + 8 * (v >> 2) + 4 * hh + (v & 3)) & 1) sc[kb][v] = __builtin_nanf("");
    }
    if ((kt + KT > k_end) || (kt + KT - 1 > qpos0)) {
      const int lim = min(qpos0 + j, k_end - 1) - kt - 4 * hh;   // last visible key - base
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (32 * kb + 8 * (v >> 2) + (v & 3) > lim) sc[kb][v] = -INFINITY;
    }
    // ---- online softmax (log2 units), lazily rescaled
    float mt = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int v = 0; v < 16; ++v) mt = fmaxf(mt, sc[kb][v]);
    mt = max_halves(mt) * c_scale;
    if (__builtin_amdgcn_ballot_w64(mt > m_ref + kSlack) != 0) {
      const float m_new = fmaxf(m_ref, mt);
      const float alpha = (m_new == -INFINITY) ? 1.f : fast_exp2(m_ref - m_new);
      l *= alpha;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[db][v] *= alpha;
      m_ref = m_new;
    }
    const float nm = (m_ref == -INFINITY) ? 0.f : -m_ref;
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p0 = fast_exp2(fmaf(sc[kb][8 * hf + 2 * e], c_scale, nm));
          const float p1 = fast_exp2(fmaf(sc[kb][8 * hf + 2 * e + 1], c_scale, nm));
          w[e] = pack_bf16x2(p0, p1);
          l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[e]), ones, l, false);
        }
        const bf16x8 pb = __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
        // ---- O^T += V^T . P^T over the 16 keys of this step
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
          const char *p = vl + (2 * kb + hf) * 16 * VROWB + offv[db];
          o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tr_read_pair(p, p + 8 * VROWB), pb, o[db], 0,
                                                          0, 0);
        }
      }
  }

  // ---- epilogue
  const float l_tot = sum_halves(l);
  float part_c = 0.f, part_sc = 0.f;
  if (uw.n_splits > 1) part_sc = part_scale(row_amax(o), l_tot, part_c);
  if (!active || q0 + j >= sp.len) return;
  const int row = q0 + j;
  if (uw.n_splits == 1) {
    const float inv = 1.0f / l_tot;
    uint16_t *orow = a.out + ((int64_t)(sp.q_start + row) * a.n_q_heads + qhead) * D;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int gq = 0; gq < 4; ++gq) {
        const int d0 = 32 * db + 8 * gq + 4 * hh;
        *reinterpret_cast<u32x2 *>(orow + d0) =
            u32x2{pack_bf16x2(o[db][4 * gq + 0] * inv, o[db][4 * gq + 1] * inv),
                  pack_bf16x2(o[db][4 * gq + 2] * inv, o[db][4 * gq + 3] * inv)};
      }
  } else {
    const int64_t prow = ((int64_t)split * sp.len + row) * a.n_q_heads + qhead;
    store_partial<NDB, D>(o, part_sc, m_ref, l_tot, part_c, hh, a.ws, sp, prow);
  }
}

size_t attn_kv8_workspace_bytes(const AttnLaunch &p) {
  AttnPlan plan;
  if (!plan_attention(p, plan)) return (size_t)-1;
  return plan.ws_bytes;
}

hipError_t launch_attention_kv8(const AttnLaunch &p, hipStream_t stream) {
  AttnPlan plan;
  if (!plan_attention(p, plan)) return hipErrorInvalidValue;
  if (plan.ws_bytes > p.workspace_bytes) return hipErrorInvalidValue;
  AttnArgs args{};
  const int64_t layer_rows = (int64_t)p.layer * p.n_phys_pages * p.n_kv_heads * kPage;
  args.q = (const uint16_t *)p.q;
  args.out = (uint16_t *)p.out;
  args.kc = (const uint16_t *)((const char *)p.cache_k + layer_rows * p.head_dim);
  args.vc = (const uint16_t *)((const char *)p.cache_v + layer_rows * p.head_dim);
  args.ks = p.k_scale + layer_rows;
  args.vs = p.v_scale + layer_rows;
  args.map = p.map;
  args.ws = (char *)p.workspace;
  args.n_q_heads = p.n_q_heads;
  args.n_kv_heads = p.n_kv_heads;
  args.group = p.n_q_heads / p.n_kv_heads;
  args.n_phys_pages = p.n_phys_pages;
  args.head_dim = p.head_dim;
  const float log2e = 1.4426950408889634f;
  args.scale_log2 = p.scale * log2e;
  args.cap_in = p.softcap > 0.f ? p.scale / p.softcap : 0.f;
  args.cap_out = p.softcap * log2e;
  const bool cap = p.softcap > 0.f;
  const int threads = p.head_dim == 256 ? 512 : 256;
  const int64_t blocks = (int64_t)plan.units_per_head * p.n_kv_heads;
  if (blocks * threads > (int64_t)UINT32_MAX) return hipErrorInvalidValue;
  auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((uint32_t)blocks), dim3(threads), 0, stream, args, plan);
    return hipGetLastError();
  };
  hipError_t e;
  switch (p.head_dim) {
    case 64: e = cap ? run(attn_kv8_kernel<64, true>) : run(attn_kv8_kernel<64, false>); break;
    case 128: e = cap ? run(attn_kv8_kernel<128, true>) : run(attn_kv8_kernel<128, false>); break;
    default: e = cap ? run(attn_kv8_kernel<256, true>) : run(attn_kv8_kernel<256, false>); break;
  }
  if (e != hipSuccess) return e;
  return launch_attn_combine(args, plan, p.head_dim, stream);
}

}  // namespace nexus
