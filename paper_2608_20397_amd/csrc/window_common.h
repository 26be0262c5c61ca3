// Shared definitions of the windowed-attention kernels (internal, not part of the C ABI): the keys a row sees,
// the pages a tile of rows reads, the partial results of a split and the row that is taken again.
//
// The query at position p sees key k when k <= p and (k > p - window or k < sinks).  A tile of rows of one
// sequence, positions p0 .. p1, sees the union [0, sinks) and [p0 - window + 1, p1]; its pages are listed as
// entries: first the sinks' pages, then the window's (or one run from page 0 on, where they meet).
#pragma once

#include "device_common.h"
#include "launch_batch.h"

namespace nexus {

// (token, head) pairs of a workgroup, for the kernels and for the plan of their launches: window_rows_kernel,
// window_d256_kernel, and a block of window_f32_kernel
constexpr int kMfmaRows = 128, kWideRows = 256, kF32Rows = 16;
constexpr int kNoPeriod = 1 << 28;      // no list has as many tiles: each is taken from its start

struct WindowArgs {
  const void *q;
  void *out;
  const void *kc;         // layer base of the K cache [NPP][Hkv][16][D]
  const void *vc;         // layer base of V: as K, or [Hkv][D][NPP * 16] when transposed
  const int32_t *maps;    // [n_seqs][map_stride]
  const int32_t *q_start; // [n_seqs + 1], or null: row b is the one query of sequence b
  const int32_t *lens;    // [n_seqs]
  // partial results of a split, [n_splits][n_rows * Hq]: O / l, fp32 or, of window_rows and window_d256, fp16 scaled by
  // 2^-e so that the row's largest magnitude lies in [2^14, 2^15) (11 bits, three more than P and the output have; a
  // power of two costs no rounding and keeps any finite value in range); and (m, l, e, -), e = 0 in fp32
  void *part;
  f32x4 *part_ml;
  int32_t map_stride, max_len, n_seqs, n_rows;
  int32_t n_q_heads, n_kv_heads, group, n_qgroups;
  int32_t window, sinks, n_splits;
  uint32_t n_cols;        // transposed V: NPP * 16
  uint32_t n_units;       // (row tile, KV head) pairs of the launch
  int32_t period;         // key tiles of a window, or kNoPeriod (TileOrder)
  float scale_log2;       // scale * log2(e)
  float cap_in;           // scale / softcap
  float cap_out;          // softcap * log2(e)
  float cap_k;            // 2 * scale * log2(e) / softcap
};

// Rows of the launch's sequence b, clamped to the arrays: nothing the device holds leads out of them.
__device__ __forceinline__ int row_start(const WindowArgs &a, int b) {
  return min(max(a.q_start[b], 0), a.n_rows);
}
__device__ __forceinline__ int window_len(const WindowArgs &a, int b) {
  return min(max(a.lens[b], 0), a.max_len);
}

// A tile of rows: (token, head of the group) pairs i0 .. i0 + R - 1 of one sequence, token by token, so that one
// kernel serves a chunk of a prompt and a single token, and the heads that share keys share the tile.
struct RowTile {
  int b;          // sequence; -1: no such tile
  int row0;       // its first row
  int n;          // its (token, head) pairs: rows * group
  int i0;         // first pair of the tile
  int past;       // position of its first row (negative where the length is short)
};

// Tiles of R pairs: sequence b owns the tile numbers from floor(q_start[b] * group / R) + b on;
// floor(x + y) + 1 >= floor(x) + ceil(y) leaves it enough of them, so that no sum over the sequences is needed.
template <int R>
__host__ __device__ __forceinline__ uint32_t first_tile(uint32_t start, uint32_t group, uint32_t b) {
  return start * group / R + b;
}

// Tile u of a launch: the last b whose first number is not above u has it.  The wave looks through the sequences 64
// ways at a time.
template <int R>
__device__ __forceinline__ RowTile find_tile(const WindowArgs &a, uint32_t u) {
  RowTile t;
  if (a.q_start == nullptr) {          // one row a sequence
    const uint32_t per = (a.group + R - 1) / R;
    t.b = u / per;
    t.row0 = t.b;
    t.n = a.group;
    t.i0 = (u - t.b * per) * R;
    t.past = window_len(a, t.b) - 1;
    return t;
  }
  const int lane = threadIdx.x & 63;
  auto first = [&](int start, int b) { return first_tile<R>(start, a.group, b); };
  int lo = 0, n = a.n_seqs;
  while (n > 64) {
    const int step = (n + 63) >> 6;
    const int b = lo + lane * step;
    const uint64_t m = __builtin_amdgcn_ballot_w64(lane * step < n && first(row_start(a, b), b) <= u);
    const int k = max(__popcll(m) - 1, 0);
    lo += k * step;
    n = min(step, n - k * step);
  }
  // what the tile needs of its sequence comes with the last look, in one round trip
  const int b = min(lo + lane, a.n_seqs - 1);
  const int start = row_start(a, b), end = row_start(a, b + 1), len = window_len(a, b);
  const uint64_t m = __builtin_amdgcn_ballot_w64(lane < n && first(start, b) <= u);
  const int k = max(__popcll(m) - 1, 0);
  lo += k;
  t.row0 = __builtin_amdgcn_readlane(start, k);
  const int rows = max(__builtin_amdgcn_readlane(end, k) - t.row0, 0);
  t.n = rows * a.group;
  t.past = __builtin_amdgcn_readlane(len, k) - rows;
  const uint32_t f = first(t.row0, lo);
  const uint64_t i0 = u >= f ? (uint64_t)(u - f) * R : (uint64_t)INT32_MAX;
  t.b = i0 < (uint64_t)t.n ? lo : -1;
  t.i0 = (int)min(i0, (uint64_t)INT32_MAX);
  return t;
}

// The keys that the rows at positions p0 .. p1 (p1 >= 0) see together, and the list of their pages.
struct KeyList {
  int lo, hi;       // the window's part: [lo, hi)
  int sink_end;     // the sinks': [0, sink_end)
  int sp, wp;       // entry e is page e < sp ? e : wp + e - sp
  int n;            // entries

  __host__ __device__ __forceinline__ int page(int e) const { return e < sp ? e : wp + e - sp; }
  // whether some row sees key k of a listed page (without a branch, as the next)
  __host__ __device__ __forceinline__ bool seen(int k) const {
    return (int)(k < hi) & ((int)(k >= lo) | (int)(k < sink_end));
  }
  // a seen key of k's page, k itself if it is seen
  __host__ __device__ __forceinline__ int stand_in(int k) const {
    const int in_front = (lo >> kPageShift) == (k >> kPageShift) ? lo : sink_end - 1;
    const int other = k >= hi ? hi - 1 : in_front;
    return seen(k) ? k : other;
  }
};
__host__ __device__ __forceinline__ KeyList key_list(int window, int sinks, int p0, int p1) {
  KeyList l;
  l.hi = p1 + 1;
  l.lo = p0 - window + 1 > 0 ? p0 - window + 1 : 0;
  l.sink_end = sinks < l.hi ? sinks : l.hi;
  const int s_pages = (l.sink_end + kPage - 1) >> kPageShift, w_page = l.lo >> kPageShift;
  if (l.lo <= l.sink_end) l.lo = 0;                   // one run of keys
  const bool apart = s_pages < w_page;
  l.sp = apart ? s_pages : 0;
  l.wp = apart ? w_page : 0;
  l.n = l.sp + ((l.hi + kPage - 1) >> kPageShift) - l.wp;
  return l;
}

__device__ __forceinline__ float window_sum_halves(float x) {     // over lanes i and i ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The order in which a workgroup takes the tiles of PT entries that its list makes: from the first one whose place among
// the sequence's tiles is a multiple of the period (the tiles of a window, the same for the whole launch) to the list's
// end, then from its start.  The row tiles of a sequence, whose windows are shifted by some tokens each, then read the
// same keys at the same time and out of one another's L2 instead of in turn.  A split has a run of this order.
template <int PT>
struct TileOrder {
  int all, first, t0, t1;      // tiles of the list, the one taken first; the split's run
  __host__ __device__ __forceinline__ int tile(int t) const {     // of the split's step t
    const int x = t0 + t + first;
    return x >= all ? x - all : x;
  }
  __host__ __device__ __forceinline__ int entry(int i) const {    // PT a step
    return PT * tile(i / PT) + i % PT;
  }
};
template <int PT>
__host__ __device__ __forceinline__ TileOrder<PT> tile_order(const KeyList &l, int period, int split, int n_splits) {
  TileOrder<PT> o;
  o.all = (l.n + PT - 1) / PT;
  const int at = (l.wp / PT) % period;
  o.first = at == 0 ? 0 : period - at + l.sp / PT;
  if (l.wp == 0 || o.first >= o.all) o.first = 0;
  o.t0 = (int)((int64_t)o.all * split / n_splits);
  o.t1 = (int)((int64_t)o.all * (split + 1) / n_splits);
  return o;
}

// tanh x = 1 - 2 / (e^{2x} + 1); exp2 overflow to +inf gives 1, underflow to 0 gives -1.
__device__ __forceinline__ float window_tanh(float x) {
  return 1.0f - 2.0f * __builtin_amdgcn_rcpf(fast_exp2(x * 2.8853900817779268f) + 1.0f);
}

// A row's (m, l) as a split stores it.  l = 0 with m = -inf: the row sees none of the split's keys.  Split 0 of a row
// that sees any key keeps m finite, so that the merge tells a row without keys (zeros) from one all of whose scores
// are -inf (NaN, as 0 / 0).
__device__ __forceinline__ float part_max(float m, bool any, int split) {
  return any && split == 0 ? fmaxf(m, -3.0e38f) : m;
}

// One row taken again, key by key, from the list's entries entry(0) .. entry(n - 1): the way of rows whose result is not
// finite.  In a tile of several tokens a key that one row sees is hidden from another, and the matrix product of its
// probability 0 with a value that is infinite or NaN is NaN; so the tile's product may be used where it is finite, and
// where it is not the row is formed from the keys that it sees alone.  It costs about 1 us for 64 keys, which only such rows
// pay.
// Called by a whole wave; `res` gives lane l features l, l + 64, ... of O / l, then m and l.
template <typename T, int D, bool VT, bool CAP, typename Entry>
__device__ __forceinline__ void row_again(const WindowArgs &a, const KeyList &kl, int b, int h, const T *q, int pos,
                                          int n, Entry entry, float (&res)[(D + 63) / 64], float &m_out, float &l_out) {
  constexpr int N = (D + 63) / 64, E = 16 / (int)sizeof(T);
  const int lane = threadIdx.x & 63;
  const T *kc = reinterpret_cast<const T *>(a.kc), *vc = reinterpret_cast<const T *>(a.vc);
  const int32_t *map = a.maps + (size_t)b * a.map_stride;
  auto value = [](T x) {
    if constexpr (sizeof(T) == 2) return bf16_bits_to_float(x);
    else return x;
  };
  double o[N];
#pragma unroll
  for (int i = 0; i < N; ++i) o[i] = 0.;
  float m = -INFINITY;
  double l = 0.;
  for (int i = 0; i < n; i += 4) {
    const int e = entry(min(i + (lane >> 4), n - 1));
    const int page = kl.page(min(e, kl.n - 1)), key = page * kPage + (lane & 15);
    const bool vis = i + (lane >> 4) < n && e < kl.n && key <= pos && (key > pos - a.window || key < a.sinks);
    const uint32_t phys = vis ? (uint32_t)map[page] : 0u;
    float s = -INFINITY;
    if (vis) {
      const T *kr = kc + (((size_t)phys * a.n_kv_heads + h) * kPage + (key & 15)) * D;
      float acc = 0.f;
      for (int d = 0; d < D; d += E)
#pragma unroll
        for (int x = 0; x < E; ++x) acc = fmaf(value(q[d + x]), value(kr[d + x]), acc);
      s = CAP ? a.cap_out * (sizeof(T) == 2 ? window_tanh(acc * a.cap_in) : tanhf(acc * a.cap_in))
              : acc * a.scale_log2;
    }
    float mx = s;
    for (int off = 32; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off));
    const float m_new = fmaxf(m, mx);
    const float alpha = m_new == -INFINITY ? 1.f : fast_exp2(m - m_new);
    const float p = vis ? fast_exp2(s - (m_new == -INFINITY ? 0.f : m_new)) : 0.f;
    float ps = p;
    for (int off = 32; off > 0; off >>= 1) ps += __shfl_xor(ps, off);
    l = l * alpha + ps;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] *= alpha;
    m = m_new;
    uint64_t left = __builtin_amdgcn_ballot_w64(vis);
    while (left) {
      const int src = __builtin_ctzll(left);
      left &= left - 1;
      const float pk = __shfl(p, src);
      const uint32_t ph = __shfl(phys, src);
      const int slot = src & 15;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int d = lane + 64 * i;
        if (d >= D) continue;
        const T v = VT ? vc[((size_t)h * D + d) * a.n_cols + (size_t)ph * kPage + slot]
                       : vc[(((size_t)ph * a.n_kv_heads + h) * kPage + slot) * D + d];
        o[i] += (double)pk * (double)value(v);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) res[i] = (float)(o[i] / l);
  m_out = m;
  l_out = (float)l;
}

// e of a row's fp16 partial, from its largest finite magnitude: -141 (subnormal ones) .. 113, so that 2^e itself may be
// out of fp32's range; values take it by ldexpf, or where they are many by a product with two_to (-126 .. 127).
__device__ __forceinline__ int part_exponent(float amax) {
  return amax > 0.f ? (int)(__float_as_uint(amax) >> 23) - 127 - 14 : 0;
}
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

// Writes what row_again gave: to the output, or to the split's partial (HALF: in fp16).
template <typename T, int D, bool HALF>
__device__ __forceinline__ void store_again(const WindowArgs &a, size_t row, int split, bool direct,
                                            const float (&res)[(D + 63) / 64], float m, float l) {
  const int lane = threadIdx.x & 63;
  const size_t slot = (size_t)split * a.n_rows * a.n_q_heads + row;
  int e = 0;
  if (!direct && HALF) {
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < (D + 63) / 64; ++i)
      if (lane + 64 * i < D && fabsf(res[i]) <= 3.4e38f) amax = fmaxf(amax, fabsf(res[i]));
    for (int off = 32; off > 0; off >>= 1) amax = fmaxf(amax, __shfl_xor(amax, off));
    e = part_exponent(amax);
  }
#pragma unroll
  for (int i = 0; i < (D + 63) / 64; ++i) {
    const int d = lane + 64 * i;
    if (d >= D) continue;
    const float x = !direct && l == 0.f ? 0.f : res[i];
    if (direct && sizeof(T) == 2) reinterpret_cast<uint16_t *>(a.out)[row * D + d] = (uint16_t)pack_bf16x2(x, 0.f);
    else if (direct) reinterpret_cast<float *>(a.out)[row * D + d] = x;
    else if (HALF) reinterpret_cast<uint16_t *>(a.part)[slot * D + d] = (uint16_t)pack_f16x2(ldexpf(x, -e), 0.f);
    else reinterpret_cast<float *>(a.part)[slot * D + d] = x;
  }
  if (!direct && lane == 0) a.part_ml[slot] = f32x4{part_max(m, true, split), l, (float)e, 0.f};
}

// The end of the 32x32 MFMA kernels, for a wave with rows: lane pair (j, j + 32) holds a pair's row, feature
// 32 db + 8 gq + 4 hh + i in o[db][4 gq + i].  Rows that are not finite are taken again.
template <int D, bool VT, bool CAP, int PT>
__device__ __forceinline__ void store_rows(const WindowArgs &a, const KeyList &kl, const TileOrder<PT> &order,
                                           const RowTile &rt, int kvh, int split, bool direct, int pair, size_t row,
                                           int pos, bool row_ok, int hh, float m_ref, float l, f32x16 (&o)[D / 32]) {
  constexpr int NDB = D / 32;
  const int n_le = PT * (order.t1 - order.t0);
  const int G = a.group;
  const float l_tot = window_sum_halves(l);
  const bool empty = pos < 0 || n_le == 0;
  const float inv = direct ? (empty ? 0.f : 1.0f / l_tot) : l_tot > 0.f ? 1.0f / l_tot : 0.f;
  float check = 0.f;                             // NaN where an output is not finite
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      o[db][v] = empty ? 0.f : o[db][v] * inv;     // (0 x NaN is NaN)
      check = fmaf(o[db][v], 0.f, check);
    }
  check = window_sum_halves(check);
  const bool bad = row_ok && !empty && (!(check == 0.f) || l_tot != l_tot);
  int e = 0;
  if (!direct) {
    float amax = 0.f;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) amax = fmaxf(amax, fabsf(o[db][v]));
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(amax), __float_as_uint(amax), false, false);
    e = part_exponent(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
  }
  if (row_ok && !bad) {
    if (direct) {
      uint16_t *orow = reinterpret_cast<uint16_t *>(a.out) + row * D;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int gq = 0; gq < 4; ++gq)
          *reinterpret_cast<u32x2 *>(orow + 32 * db + 8 * gq + 4 * hh) =
              u32x2{pack_bf16x2(o[db][4 * gq + 0], o[db][4 * gq + 1]),
                    pack_bf16x2(o[db][4 * gq + 2], o[db][4 * gq + 3])};
    } else {
      const size_t slot = (size_t)split * a.n_rows * a.n_q_heads + row;
      const int e1 = min(-e, 127);
      const float s1 = two_to(e1), s2 = two_to(-e - e1);
      uint16_t *po = reinterpret_cast<uint16_t *>(a.part) + slot * D;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int gq = 0; gq < 4; ++gq)
          *reinterpret_cast<u32x2 *>(po + 32 * db + 8 * gq + 4 * hh) =
              u32x2{pack_f16x2(o[db][4 * gq + 0] * s1 * s2, o[db][4 * gq + 1] * s1 * s2),
                    pack_f16x2(o[db][4 * gq + 2] * s1 * s2, o[db][4 * gq + 3] * s1 * s2)};
      const float lw = empty ? 0.f : l_tot;
      if (hh == 0) a.part_ml[slot] = f32x4{part_max(m_ref, pos >= 0, split), lw, (float)e, 0.f};
    }
  }
  uint32_t left = (uint32_t)__builtin_amdgcn_ballot_w64(bad && hh == 0);
  while (left) {
    const int r = __builtin_ctz(left);
    left &= left - 1;
    const int rp = __builtin_amdgcn_readlane(pair, r), rtok = rp / G, rhead = kvh * G + rp - rtok * G;
    const size_t rrow = (size_t)(rt.row0 + rtok) * a.n_q_heads + rhead;
    float res[(D + 63) / 64], m, lr_;
    row_again<uint16_t, D, VT, CAP>(a, kl, rt.b, kvh, reinterpret_cast<const uint16_t *>(a.q) + rrow * D,
                                    rt.past + rtok, n_le, [&](int i) { return order.entry(i); }, res, m, lr_);
    store_again<uint16_t, D, true>(a, rrow, split, direct, res, m, lr_);
  }
}

// Kernel launches by type (window_attn.hip, window_decode.hip, window_f32.hip); the merge of the splits.
hipError_t launch_window_rows(const WindowArgs &a, int head_dim, bool vt, bool cap, hipStream_t stream);
hipError_t launch_window_d256(const WindowArgs &a, bool vt, bool cap, hipStream_t stream);
hipError_t launch_window_decode(const WindowArgs &a, int head_dim, bool vt, bool cap, hipStream_t stream);
hipError_t launch_window_f32(const WindowArgs &a, int head_dim, bool vt, bool cap, int waves, int blocks,
                             hipStream_t stream);

}  // namespace nexus
