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
//     bf16, which the matrix instruction takes beside such a V, and the PV product is the bf16 kernels' (transposed
//     LDS reads, 32x32x16 MFMA).  The row sum adds the rounded values, so that the weights sum to one.  Against 64
//     bits the outputs are off by 1.8e-3 (relative, rms), 1.7e-3 of it the rounding of the results themselves.
//   * A token whose key or value row is not finite (scale byte 255) gives NaN to the queries that see it
//     and nothing to the others: 255 is its keys' scale operand, which makes its scores NaN; they are masked
//     like any other, and its values enter the product as zeros.
//   * Slots past the last key of a workgroup are never read: their rows repeat the last key and are masked.
// LDS: K row r, 16-byte chunk c at c ^ kswz(r); V (bf16) chunk c at vchunk(c, r).
//
// What bounds it: the matrix and the vector units, about alike.  1088 queries at depth 16384, 40 heads over 8 of
// 128: 347 to 359 us (1.05 to 1.09 PFLOP/s; the bf16 kernel 343 to 357 on the same cards, from twice the
// cache), matrix pipe busy 50% of the cycles, vector instructions issuing in 48% (7.5 of them per MFMA: the
// softmax and the conversion of V).  Steps that led there from 436 us: the conversion beside the PV products instead of at
// the end of the iteration; MFMAs and vector work interleaved in the written order; a step without branches
// for whole, unmasked tiles.  head_dim 64, 16 x 256 queries at depths up to 15233, 32 heads over 8: 305 us
// (408 before), vector instructions in 66% and MFMA in 40% of the cycles: a score has half the products of
// head_dim 128 and the same exponential, and of 2560 workgroups, 10 a CU, three fit, so that the last round is a third
// full.  head_dim 256, capped, 512 queries at depth 8704, 16 heads over 8: 99 us (149
// before the lower query terms went to LDS and the kernel took the schedule of the others): one round of 256
// workgroups, matrix pipe busy 32% and vector instructions issuing in 43% of the cycles; without the cap 28%, 97 us.
// 4 waves of 32 queries, two workgroups a CU (head_dim 256: 8 waves, for K and V tiles of twice the width to be
// read by 8 tasks).  64 queries a wave, which would halve the operand reads, leave one wave a SIMD, and the
// accumulators then cost a copy per score between the register files.
#include "attn_common.h"
#include "attn_dma.h"
#include "kv8_common.h"
#include "launch_kv8.h"

#include <type_traits>

namespace nexus {

template <int D, bool CAP>
__global__ __launch_bounds__(D == 256 ? 512 : 256, D == 64 ? 3 : 2) void attn_kv8_kernel(const AttnArgs a,
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
  constexpr int kPrioPV = 2;                       // wave priority of the PV phase (attn_bf16_dma.hip)
  static_assert(NI >= 1 && NVC >= 1 && RPI <= kPage, "tile shape");
  // head_dim 256: O^T takes 128 of a wave's 256 registers and the scores 32, which leaves room for the upper
  // terms of Q's first 192 features; the others and the lower terms wait in LDS
  constexpr bool QLDS = D == 256;
  constexpr int NSR = QLDS ? 3 : NS2;              // steps whose upper terms stay in registers
  constexpr int QLB = QLDS ? 64 * 32 * (NS2 + 1) : 0;   // a wave's terms in LDS: lower, and upper of the last step
  __shared__ __align__(1024) char smem[2 * KTILEB + 2 * VTILEB + W * QLB];
  __shared__ __align__(16) int32_t pg[kMaxSplitKeys / kPage + 8];

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int j = lane & 31, hh = lane >> 5;
  const int kvh = blockIdx.x % a.n_kv_heads;
  // (one sequence: its plan is loaded at once, without the search for the unit's; 192 queries at depth 2432
  // 28.7 -> 28.0 us)
  const int unit = blockIdx.x / a.n_kv_heads;
  SeqPlan sp = plan.seq[0];
  UnitWork uw = unit_work(sp, unit);
  if (plan.n_seqs > 1) {
    const UnitLoc loc = locate_unit(plan, unit);
    uw = loc.w;
    sp = plan.seq[loc.seq];
  }
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
  i32x8 qhi[NSR], qlo[QLDS ? 1 : NS2];
  char *const ql_lds = smem + 2 * KTILEB + 2 * VTILEB + wave * QLB + 16 * lane;   // 16-byte piece i at + 1024 i
  int qscale;              // scale bytes of hi (byte 0) and lo (byte 1)
  {
    const int qi = min(q0 + j, sp.len - 1);
    const uint16_t *qrow = a.q + ((int64_t)(sp.q_start + qi) * a.n_q_heads + qhead) * D;
    uint32_t raw[16 * NS2];
#pragma unroll
    for (int s = 0; s < NS2; ++s)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const u32x4 x = active ? *reinterpret_cast<const u32x4 *>(qrow + 64 * s + 32 * hh + 8 * c)
                               : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int w = 0; w < 4; ++w) raw[16 * s + 4 * c + w] = x[w];
      }
    uint32_t am = amax_bits_bf16<16 * NS2>(raw);
    const auto r = __builtin_amdgcn_permlane32_swap(am, am, false, false);
    am = max((uint32_t)r[0], (uint32_t)r[1]);
    const int e = row_exp(am);
    qscale = am >= 0x7F800000u ? (int)(kBadScale | kBadScale << 8) : (e + 127) | (e + 127 - 4) << 8;
    clamp_query<16 * NS2>(raw, am);
#pragma unroll
    for (int s = 0; s < NS2; ++s)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t hi[2], lo[2];
        split_query<4>(raw + 16 * s + 4 * c, e, hi, lo);
        if (s < NSR) {
          qhi[s % NSR][2 * c] = hi[0];
          qhi[s % NSR][2 * c + 1] = hi[1];
        } else {
          *reinterpret_cast<u32x2 *>(ql_lds + 1024 * (2 * NS2 + (c >> 1)) + 8 * (c & 1)) = u32x2{hi[0], hi[1]};
        }
        if constexpr (QLDS) {
          *reinterpret_cast<u32x2 *>(ql_lds + 1024 * (2 * s + (c >> 1)) + 8 * (c & 1)) = u32x2{lo[0], lo[1]};
        } else {
          qlo[s][2 * c] = lo[0];
          qlo[s][2 * c + 1] = lo[1];
        }
      }
  }

  // (as one opaque value: kept as the parts it is made of, it cost head_dim 64 two reloads of spilled registers
  // an iteration, 317 -> 343 us for 16 x 256 queries at depths up to 15233)
  asm volatile("" : "+v"(qscale));

  f32x16 o[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[db][v] = 0.f;
  float m_ref = -INFINITY;
  float l = 0.f;

  // ---- LDS layouts
  auto kswz = [](int row) { return D == 64 ? (row >> 2) & 3 : D == 128 ? (row >> 1) & 7 : row & 15; };
  // V chunk c of row r.  Bits 2 and 3 put the rows of one transposed read on distinct banks; bit 0 does so
  // with the chunks of one conversion's writes, every second of a row, over 128 and over 256 bytes.
  auto vchunk = [](int c, int r) {
    return D == 64    ? c ^ (4 * ((r >> 1) & 1)) ^ ((r ^ (r >> 1)) & 1)
           : D == 128 ? c ^ (4 * (r & 3)) ^ ((r ^ (c >> 3)) & 1)
                      : c ^ (4 * (r & 3)) ^ (((c >> 3) ^ (c >> 4)) & 1);
  };
  // S^T A operand: K row j (+ 32 kb, whose swizzle is the same), features 64 s + 32 hh .. + 31,
  // in chunks 4 s + 2 hh + c: the XOR of one offset with constants (few registers hold offsets in the loop)
  const uint32_t offk = j * D + 16 * ((2 * hh) ^ kswz(j));
  // PV A operand, as attn_bf16_dma.hip: key 4 h2 + e of a half step, features 32 db + 16 dh + 4 q .. + 3;
  // head_dim 256: db and db + 4 differ by a constant XOR
  constexpr int NOV = NDB < 4 ? NDB : 4;
  uint32_t offv[NOV];
  {
    const int gg = lane >> 4, r = lane & 15, e = r >> 2, q = r & 3;
    const int h2 = gg >> 1, dh = gg & 1;
#pragma unroll
    for (int db = 0; db < NOV; ++db)
      offv[db] = (4 * h2 + e) * VROWB + 16 * vchunk(4 * db + 2 * dh + (q >> 1), e) + 8 * (q & 1);
  }
  auto kbuf = [&](int i) { return smem + i * KTILEB; };
  auto vbuf = [&](int i) { return smem + 2 * KTILEB + i * VTILEB; };
  const uint32_t smem_base = (uint32_t)(uintptr_t)smem;
  const uint64_t pbytes = (uint64_t)a.n_kv_heads * kPage * D;      // one physical page of codes
  const uint32_t sbytes = (uint32_t)a.n_kv_heads * kPage;          // and of scales
  const char *kbytes = reinterpret_cast<const char *>(a.kc) + (uint64_t)kvh * kPage * D;
  const char *vbytes = reinterpret_cast<const char *>(a.vc) + (uint64_t)kvh * kPage * D;
  const uint8_t *ksb = a.ks + kvh * kPage, *vsb = a.vs + kvh * kPage;

  // Q and the page table are waited for before any DMA is in flight (attn_bf16_dma.hip)
  wait_vm<0>();
  __syncthreads();   // pg[] visible

  auto page_at = [&](int lp) -> uint32_t {    // wave-uniform logical page, counted from pg0
    return (uint32_t)__builtin_amdgcn_readfirstlane(pg[lp]);
  };
  auto full = [&](int it) { return k_begin + it * KT + KT <= k_end; };
  // Pages of a wave's share of a whole tile: one per DMA instruction and per chunk of V codes.
  struct Pages {
    uint32_t k[NI], v[NVC];
  };
  auto k_pages = [&](int it, Pages &p) {
#pragma unroll
    for (int i = 0; i < NI; ++i) p.k[i] = page_at(it * (KT / kPage) + (wave * NI + i) * RPI / kPage);
  };
  auto v_pages = [&](int it, Pages &p) {
#pragma unroll
    for (int k = 0; k < NVC; ++k) p.v[k] = page_at(it * (KT / kPage) + (64 * wave + NT * k) / CH / kPage);
  };
  // (what the rare paths derive from the lane is derived there, not kept in registers for them)
  auto rare_lane = [&]() {
    int x = lane;
    asm volatile("" : "+v"(x));
    return x;
  };
  // DMA of K tile `it`: instruction i of the wave fills rows (wave NI + i) RPI ..
  uint32_t kdo[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int row = (wave * NI + i) * RPI + lane / CH;
    kdo[i] = (row & (kPage - 1)) * D + 16 * ((lane % CH) ^ kswz(row));
  }
  auto dma_k = [&](int it, const Pages &p, bool whole = false) {
    const uint32_t dst = smem_base + (it & 1) * KTILEB + wave * NI * 1024;
    if (whole || full(it)) {
#pragma unroll
      for (int i = 0; i < NI; ++i) dma_s<0>(dst + i * 1024, kbytes + p.k[i] * pbytes, kdo[i]);
    } else {
      const int x = rare_lane();
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int row = (wave * NI + i) * RPI + x / CH;
        const int t = min(k_begin + it * KT + row, k_end - 1);
        const uint64_t pp = (uint32_t)pg[(t >> kPageShift) - pg0];
        dma_v(dst + i * 1024, kbytes + pp * pbytes + (uint32_t)(t & (kPage - 1)) * D +
                                  16 * ((x % CH) ^ kswz(row)));
      }
    }
  };
  // V codes on their way to LDS: chunk lane % CH of rows (64 wave + NT k) / CH + lane / CH
  struct Codes {
    u32x4 v[NVC];
  };
  const uint32_t vdo = ((64 * wave / CH + lane / CH) & (kPage - 1)) * D + 16 * (lane % CH);
  auto load_v = [&](int it, const Pages &p, Codes &cd, bool whole = false) {
    if (whole || full(it)) {
#pragma unroll
      for (int k = 0; k < NVC; ++k)
        cd.v[k] = *reinterpret_cast<const u32x4 *>(vbytes + p.v[k] * pbytes + vdo);
      // (keeps these loads apart from the others below, whose addresses are the lanes' own)
      asm volatile("" ::: "memory");
    } else {
      const int x = rare_lane();
#pragma unroll
      for (int k = 0; k < NVC; ++k) {
        const int t = min(k_begin + it * KT + (64 * wave + NT * k) / CH + x / CH, k_end - 1);
        const uint64_t pp = (uint32_t)pg[(t >> kPageShift) - pg0];
        cd.v[k] = *reinterpret_cast<const u32x4 *>(vbytes + pp * pbytes +
                                                   (uint32_t)(t & (kPage - 1)) * D + 16 * (x % CH));
      }
    }
  };
  // key and value scale bytes of token `lane` of tile `it` (a layer's scales lie within 32-bit offsets)
  struct Scales {
    uint32_t k, v;
  };
  auto load_scales = [&](int it, Scales &s) {
    const int t = min(k_begin + it * KT + (lane & (KT - 1)), k_end - 1);
    const uint32_t at = (uint32_t)pg[(t >> kPageShift) - pg0] * sbytes + (t & (kPage - 1));
    s.k = ksb[at];
    s.v = vsb[at];
  };
  // the MFMA's scale operands of a tile's keys
  auto operands = [&](const Scales &s) -> int {      // of block kb in byte kb
    const uint32_t k = s.v == kBadScale ? kBadScale : s.k;
    const auto r = __builtin_amdgcn_permlane32_swap(k, k, false, false);
    return (int)(r[0] | r[1] << 8);
  };
  // V codes of a tile to bf16 in V buffer `buf`, `vs`: the value scale byte of token `lane`; a row that is
  // not finite as zeros
  // (the rows of a thread's chunks are 32 or 64 apart and swizzled alike)
  const uint32_t vrow = 64 * wave / CH + lane / CH;
  const uint32_t vdst[2] = {vrow * VROWB + 16 * vchunk(2 * (lane % CH), vrow),
                            vrow * VROWB + 16 * vchunk(2 * (lane % CH) + 1, vrow)};
  struct RowScales {
    uint32_t byte[NVC];
  };
  auto row_scales = [&](uint32_t vs, RowScales &rs) {
#pragma unroll
    for (int k = 0; k < NVC; ++k)
      rs.byte[k] = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (vrow + NT / CH * k), (int)vs);
  };
  auto clear_bad = [&](Codes &cd, uint32_t vs, RowScales &rs) {
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(vs == kBadScale) != 0, 0)) {
#pragma unroll
      for (int k = 0; k < NVC; ++k)
        if (rs.byte[k] == kBadScale) {
          cd.v[k] = u32x4{0u, 0u, 0u, 0u};
          rs.byte[k] = 127;
        }
    }
  };
  auto store_v = [&](int buf, const Codes &cd, const RowScales &rs) {
    char *vl = vbuf(buf);
#pragma unroll
    for (int k = 0; k < NVC; ++k) {
      const float s = __uint_as_float(rs.byte[k] << 23);
      u32x2 w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = codes_to_bf16(cd.v[k][i], s);
      *reinterpret_cast<u32x4 *>(vl + NT / CH * VROWB * k + vdst[0]) = u32x4{w[0][0], w[0][1], w[1][0], w[1][1]};
      *reinterpret_cast<u32x4 *>(vl + NT / CH * VROWB * k + vdst[1]) = u32x4{w[2][0], w[2][1], w[3][0], w[3][1]};
    }
  };
  auto convert_v = [&](int buf, Codes &cd, uint32_t vs) {
    RowScales rs;
    row_scales(vs, rs);
    clear_bad(cd, vs, rs);
    store_v(buf, cd, rs);
  };

  const float c_scale = CAP ? 1.0f : a.scale_log2;
  const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3F803F80u);

  // one product of 64 features: keys of block kb, whose scales are byte kb of ks, with hi (0) or lo (1)
  auto mfma8 = [&](const i32x8 &ka, const i32x8 &q, const f32x16 &c, int ks, int kb, int term) {
    // (the selectors are part of the instruction)
    if (kb == 0 && term == 0)
      return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ka, q, c, 0, 0, 0, ks, 0, qscale);
    if (kb == 0) return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ka, q, c, 0, 0, 0, ks, 1, qscale);
    if (term == 0)
      return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ka, q, c, 0, 0, 1, ks, 0, qscale);
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ka, q, c, 0, 0, 1, ks, 1, qscale);
  };
  auto two = [](const u32x4 &x, const u32x4 &y) {
    return i32x8{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)y[0], (int)y[1], (int)y[2], (int)y[3]};
  };
  // K operand q of a tile: block q % NKB, features 64 (q / NKB) ..; and the lower terms of those features
  constexpr int NQ = NS2 * NKB;
  auto k_operand = [&](const char *kl, uint32_t z, int q) {
    const char *at = kl + (q % NKB) * 32 * D;
    return two(*reinterpret_cast<const u32x4 *>(at + (offk ^ (64 * (q / NKB) + z))),
               *reinterpret_cast<const u32x4 *>(at + (offk ^ (64 * (q / NKB) + 16 + z))));
  };
  auto q_lds = [&](int s) {
    return two(*reinterpret_cast<const u32x4 *>(ql_lds + 2048 * s),
               *reinterpret_cast<const u32x4 *>(ql_lds + 2048 * s + 1024));
  };
  auto low = [&](int s) {
    if constexpr (QLDS)
      return q_lds(s);
    else
      return qlo[s];
  };
  auto high = [&](int s) { return s < NSR ? qhi[s % NSR] : q_lds(NS2); };
  f32x16 zero;
#pragma unroll
  for (int v = 0; v < 16; ++v) zero[v] = 0.f;
  // S^T of the tile in K buffer `kl`, whose tokens' scale bytes are the operands ks (raw scores)
  auto qk = [&](const char *kl, int ks, f32x16 *sc) {
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int kb = q % NKB, s = q / NKB;
      const i32x8 ka = k_operand(kl, 0, q);
      sc[kb] = mfma8(ka, high(s), q < NKB ? zero : sc[kb], ks, kb, 0);
      sc[kb] = mfma8(ka, low(s), sc[kb], ks, kb, 1);
    }
  };
  auto cap = [&](f32x16 *sc) {
    if constexpr (CAP) {
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int v = 0; v < 16; ++v) sc[kb][v] = a.cap_out * tanh_fast(sc[kb][v] * a.cap_in);
    }
  };
  // S(t) needs the causal / tail mask when its tile crosses this wave's diagonal or the split end
  auto needs_mask = [&](int t) {
    const int kt = k_begin + t * KT;
    return (kt + KT > k_end) || (kt + KT - 1 > qpos0);
  };
  auto mask = [&](f32x16 *sc, int t) {
    const int x = rare_lane();
    const int lim = min(qpos0 + (x & 31), k_end - 1) - (k_begin + t * KT) - 4 * (x >> 5);   // last visible key
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (32 * kb + 8 * (v >> 2) + (v & 3) > lim) sc[kb][v] = -INFINITY;
  };
  auto row_max = [&](const f32x16 *sc) -> float {
    float mt = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int v = 0; v < 16; ++v) mt = fmaxf(mt, sc[kb][v]);
    return max_halves(mt) * c_scale;
  };
  // moves the reference to a maximum that has left it behind; returns the exponent's addend
  auto rescale = [&](float mt) -> float {
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
    return (m_ref == -INFINITY) ? 0.f : -m_ref;
  };
  Codes cd{};
  Scales sn{};                               // scales of the tile that loads
  Pages pn{};                                // pages of the tiles to load next
  {
    // ---- the schedule of attn_bf16_dma.hip: per iteration t the wave computes S(t + 1) = K[t + 1] Q^T
    // beside the exponentials of S(t), then O += V[t] P(t) beside the maximum of S(t + 1), while K[t + 2]
    // travels by DMA.  The codes of V[t + 1], in registers since the iteration before, go to LDS as bf16
    // beside the PV products, which leave the vector units idle half their time (at the end of the
    // iteration, before its barrier, the conversion took 14% of the launch).
    f32x16 sa[NKB], sb[NKB];
    int ks = 0;                             // scale operands of tile t + 1's keys
    uint32_t vs = 127;                      // value scale of its token `lane`
    // what is asked for at the end of an iteration: codes of V[t], scales of tile s
    auto ask = [&](int t, int s, bool inner) {
      if (inner || t < n_tiles) {
        if (inner || full(t)) v_pages(t, pn);
        load_v(t, pn, cd, inner);
      }
      if (inner || s < n_tiles) load_scales(s, sn);
    };
    if (n_tiles > 0) {
      if (full(0)) k_pages(0, pn);
      ask(0, 0, false);
      dma_k(0, pn);
      wait_vm<0>();
      convert_v(0, cd, sn.v);
      ks = operands(sn);
      if (n_tiles > 1) {
        if (full(1)) k_pages(1, pn);
        dma_k(1, pn);
      }
      ask(1, 1, false);
    }
    tile_barrier();
    float mt_cur = -INFINITY;               // row maximum of S(t), log2 units
    if (active && n_tiles > 0) {
      qk(kbuf(0), ks, sa);
      cap(sa);
      mt_cur = row_max(sa);                 // unmasked: step 0 masks S(0) and takes its maximum again
    }
    wait_vm<0>();
    ks = operands(sn);
    vs = sn.v;
    if (n_tiles > 2) {
      load_scales(2, sn);
      if (full(2)) k_pages(2, pn);
    }
    tile_barrier();                         // K buffer 0 is refilled in iteration 0; K[1] has landed

    // INNER: the wave has a task, tile t needs no mask and tiles to t + 3 are whole: no branches but the
    // rescale's and the one for tokens that are not finite
    auto step = [&](int t, auto parity, auto inner, f32x16 *s_cur, f32x16 *s_nxt) {
      constexpr int P = decltype(parity)::value;     // t & 1
      constexpr bool INNER = decltype(inner)::value;
      if (INNER || t + 2 < n_tiles) dma_k(t + 2, pn, INNER);
      RowScales rs;
      row_scales(vs, rs);
      clear_bad(cd, vs, rs);
      if (INNER || active) {
        if (!INNER && needs_mask(t)) {
          mask(s_cur, t);
          mt_cur = row_max(s_cur);
        }
        const float nm = rescale(mt_cur);
        const char *kl = kbuf(P ^ 1), *vl = vbuf(P);
        // Both phases are chunks of one MFMA, the operand reads of a later one and a few vector
        // instructions, in the order written here (the sched_barriers hold it).
        // P(t), two scores of this lane at a time: pair i of 8 NKB, keys of 4 pairs per PV step
        uint32_t pw[8 * NKB];
        auto p_pair = [&](int i) {
          const float p0 = fast_exp2(fmaf(s_cur[i >> 3][2 * (i & 7)], c_scale, nm));
          const float p1 = fast_exp2(fmaf(s_cur[i >> 3][2 * (i & 7) + 1], c_scale, nm));
          pw[i] = pack_bf16x2(p0, p1);
          l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pw[i]), ones, l, false);
        };
        // ---- S(t + 1), beside the pairs of all PV steps but the last
        constexpr int NP = 8 * NKB, NPQ = NP - 4;   // pairs, and those here
        i32x8 ka[2], ql;
        // a zero that the compiler takes for anything: without it, the XORs of the operand offsets would be kept
        // in registers across the loop
        uint32_t z;
        asm volatile("s_mov_b32 %0, 0" : "=s"(z));
        ka[0] = k_operand(kl, z, 0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < 2 * NQ; ++c) {
          const int q = c >> 1, kb = q % NKB, s = q / NKB;
          if (c & 1) {
            s_nxt[kb] = mfma8(ka[q & 1], ql, s_nxt[kb], ks, kb, 1);
          } else {
            ql = low(s);
            if (q + 1 < NQ) ka[(q + 1) & 1] = k_operand(kl, z, q + 1);
            s_nxt[kb] = mfma8(ka[q & 1], high(s), q < NKB ? zero : s_nxt[kb], ks, kb, 0);
          }
#pragma unroll
          for (int i = NPQ * c / (2 * NQ); i < NPQ * (c + 1) / (2 * NQ); ++i) p_pair(i);
          __builtin_amdgcn_sched_barrier(0);
        }
        // ---- O += V P, beside the last 4 pairs, the conversion of V[t + 1] (past the last tile: to a
        // buffer that nothing reads any more) and the cap and maximum of S(t + 1)
        __builtin_amdgcn_s_setprio(kPrioPV);
        constexpr int NM = 2 * NKB * NDB;     // MFMA m: step m / NDB, features 32 (m % NDB) ..
        auto v_operand = [&](int m) {
          const int db = m % NDB;
          const char *at =
              vl + (m / NDB) * 16 * VROWB + (db < NOV ? offv[db % NOV] : offv[db % NOV] ^ (256 + 16 + z));
          return tr_read_pair(at, at + 8 * VROWB);
        };
        constexpr int VA = D == 256 ? 1 : 2;  // V operands read ahead
        bf16x8 va[VA + 1];
#pragma unroll
        for (int i = 0; i < VA; ++i) va[i] = v_operand(i);
        u32x2 cw[4];
        float mt = -INFINITY;
#pragma unroll
        for (int m = 0; m < NM; ++m) {
          const int step_m = m / NDB, db = m % NDB;
          if (m + VA < NM) va[(m + VA) % (VA + 1)] = v_operand(m + VA);
          o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              va[m % (VA + 1)],
              __builtin_bit_cast(bf16x8, u32x4{pw[4 * step_m], pw[4 * step_m + 1], pw[4 * step_m + 2],
                                               pw[4 * step_m + 3]}),
              o[db], 0, 0, 0);
          // the pairs before the step that takes them, then words of codes and scores
          constexpr int ML = NM - NDB;
#pragma unroll
          for (int i = 4 * m / ML; i < 4 * (m + 1) / ML && i < 4; ++i) p_pair(NPQ + i);
#pragma unroll
          for (int w = 4 * NVC * m / NM; w < 4 * NVC * (m + 1) / NM; ++w) {
            const int k = w >> 2, i = w & 3;
            cw[i] = codes_to_bf16(cd.v[k][i], __uint_as_float(rs.byte[k] << 23));
            if (i & 1)
              *reinterpret_cast<u32x4 *>(vbuf(P ^ 1) + NT / CH * VROWB * k + vdst[i >> 1]) =
                  u32x4{cw[i - 1][0], cw[i - 1][1], cw[i][0], cw[i][1]};
          }
          // (the last products of S(t + 1) are still on their way in the first chunks)
          constexpr int M0 = NM / 4;
#pragma unroll
          for (int i = m < M0 ? 0 : 16 * NKB * (m - M0) / (NM - M0);
               i < (m < M0 ? 0 : 16 * NKB * (m - M0 + 1) / (NM - M0)); ++i) {
            if constexpr (CAP)
              s_nxt[i >> 4][i & 15] = a.cap_out * tanh_fast(s_nxt[i >> 4][i & 15] * a.cap_in);
            mt = fmaxf(mt, s_nxt[i >> 4][i & 15]);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        mt_cur = max_halves(mt) * c_scale;
      } else {
        store_v(P ^ 1, cd, rs);
      }
      __builtin_amdgcn_s_setprio(0);
      if (INNER || (t + 3 < n_tiles && full(t + 3))) k_pages(t + 3, pn);
      // K[t + 2] and the scales of tile t + 2 have had the iteration to arrive
      wait_vm<0>();
      ks = operands(sn);
      vs = sn.v;
      ask(t + 2, t + 3, INNER);
      tile_barrier();
    };
    // Every iteration computes S(t + 1), on the last tile from a stale buffer, never used (a branch there
    // would split the scheduled region).
    const int n_inner =
        active ? min((k_end - k_begin) / KT - 3, (qpos0 + 1 - k_begin) / KT) : 0;
    const std::integral_constant<int, 0> even;
    const std::integral_constant<int, 1> odd;
    int t = 0;
    for (; t + 1 < n_inner; t += 2) {
      step(t, even, std::true_type{}, sa, sb);
      step(t + 1, odd, std::true_type{}, sb, sa);
    }
    for (; t < n_tiles; t += 2) {
      step(t, even, std::false_type{}, sa, sb);
      if (t + 1 < n_tiles) step(t + 1, odd, std::false_type{}, sb, sa);
    }
  }

  // ---- epilogue
  const int el = rare_lane(), ej = el & 31, eh = el >> 5;
  const float l_tot = sum_halves(l);
  float part_c = 0.f, part_sc = 0.f;
  if (uw.n_splits > 1) part_sc = part_scale(row_amax(o), l_tot, part_c);
  if (!active || q0 + ej >= sp.len) return;
  const int row = q0 + ej;
  if (uw.n_splits == 1) {
    const float inv = 1.0f / l_tot;
    uint16_t *orow = a.out + ((int64_t)(sp.q_start + row) * a.n_q_heads + qhead) * D;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int gq = 0; gq < 4; ++gq) {
        const int d0 = 32 * db + 8 * gq + 4 * eh;
        *reinterpret_cast<u32x2 *>(orow + d0) =
            u32x2{pack_bf16x2(o[db][4 * gq + 0] * inv, o[db][4 * gq + 1] * inv),
                  pack_bf16x2(o[db][4 * gq + 2] * inv, o[db][4 * gq + 3] * inv)};
      }
  } else {
    const int64_t prow = ((int64_t)split * sp.len + row) * a.n_q_heads + qhead;
    store_partial<NDB, D>(o, part_sc, m_ref, l_tot, part_c, eh, a.ws, sp, prow);
  }
}

hipError_t launch_attention_kv8(const AttnLaunch &p, const AttnPlan &plan, hipStream_t stream) {
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
