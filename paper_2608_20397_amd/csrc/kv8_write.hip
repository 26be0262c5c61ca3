// Rows quantised on their way into an 8-bit paged cache, keys rotated first: the write side of the cache
// (kv8_common.h has the format).  Three uses share the kernel:
//   * kFixed: a compiled block re-anchored and spliced, every key turned by the same angle;
//   * kRange: freshly computed tokens, key j turned to its own position angle0 + j;
//   * kStep:  one new token of each of many sequences, positions and places from device lengths.
// The rotation is that of rope_math.h (angles in fp64, compensated fp32 products); its fp32 result is
// quantised directly, not rounded to bf16 between.  fp32 is what the conversion takes: its rounding moves a code where
// a border lies within 2^-24 of an element, 2 of 4 million elements at positions from 16384 on.
//
// A thread takes the feature pairs of two 16-byte chunks of a row (K and V alike); the threads of a row are
// neighbours in a wave and find its largest magnitude by lane exchanges.  HBM-bound: a row is read once
// and written once, at half (bf16) or a quarter (fp32) of its bytes.
//
// A workgroup takes a few tokens of one or two layers, all heads.  Its first loads go out before it forms its
// angles.  Angles that differ by token cost an fp64 sine and cosine per token and pair, more time than the
// rows of one layer take: such workgroups go through two layers with one table where there are enough of them.
#include "kv8_common.h"
#include "launch_kv8.h"
#include "rope_math.h"

#include <algorithm>

namespace nexus {

namespace {

constexpr int kTabEntries = 512;   // (token, pair) angles a workgroup keeps

// Lane exchanges within 16 lanes, without LDS.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xF, 0xF, true);
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E;          // quad permutations
constexpr int kMirror8 = 0x141, kMirror16 = 0x140;   // lane i and 7 - i, 15 - i

// Largest magnitude over the 2^shift lanes of a row (4 to 32).
__device__ __forceinline__ uint32_t row_max(uint32_t m, uint32_t shift) {
  m = max(m, dpp<kXor1>(m));
  m = max(m, dpp<kXor2>(m));
  if (shift >= 3) m = max(m, dpp<kMirror8>(m));      // (quads hold one value each, then eighths)
  if (shift >= 4) m = max(m, dpp<kMirror16>(m));
  if (shift >= 5) {
    const auto r = __builtin_amdgcn_permlane16_swap(m, m, false, false);
    m = max((uint32_t)r[0], (uint32_t)r[1]);
  }
  return m;
}

struct Kv8WriteArgs {
  Kv8Cache c;
  const void *src_k, *src_v;
  const int32_t *map, *lens;
  int64_t offset, angle0;
  double base;
  FastDiv div_heads, div_items, div_last;   // items of one layer: of a whole tile, of the last one
  uint32_t tpr_shift;          // log2 of the threads of a row
  int32_t n_tokens, map_stride, max_len;
  int32_t tile, layers;        // tokens and layers of a workgroup
};

}  // namespace

template <typename T, bool INTERLEAVED, int MODE>
__global__ __launch_bounds__(256) void kv8_write_kernel(const Kv8WriteArgs a, const RopeTab tab) {
  constexpr int N = Pack<T>::N;
  constexpr bool PER_TOKEN = MODE != Kv8WriteLaunch::kFixed;
  __shared__ float cs_tab[4][PER_TOKEN ? kTabEntries : kTabPairs];
  const int head_dim = a.c.head_dim, n_heads = a.c.n_heads;
  const int j0 = blockIdx.x * a.tile;
  const int l0 = blockIdx.y * a.layers;
  const int n_tok = min(a.tile, a.n_tokens - j0);
  const int n_pairs = head_dim / 2;
  const uint32_t items = (uint32_t)(n_tok * n_heads) << a.tpr_shift;   // of one layer
  const FastDiv div_items = n_tok == a.tile ? a.div_items : a.div_last;
  const uint32_t n_items = items * min(a.layers, a.c.n_layers - l0);
  const uint32_t tpr_mask = (1u << a.tpr_shift) - 1;
  const T *src_k = static_cast<const T *>(a.src_k), *src_v = static_cast<const T *>(a.src_v);

  // logical token of tile token t (kStep: -1, nothing to write)
  auto token_of = [&](int t) -> int64_t {
    if constexpr (MODE != Kv8WriteLaunch::kStep) return a.offset + j0 + t;
    const int len = a.lens[j0 + t];
    return len >= 1 && len <= a.max_len ? len - 1 : -1;
  };

  // Item = (layer, token, head, chunk c).  NEOX: chunk c covers pairs [N c, N c + N): elements [N c, + N) and
  // [D/2 + N c, + N); INTERLEAVED: elements [2 N c, 2 N c + 2 N) = those pairs.
  struct Item {
    u32x4 ka, kb, va, vb;
    int64_t row;                 // of the cache's codes and scales; -1: not written
    int t, c;
  };
  auto load = [&](uint32_t f, Item &x) {
    const uint32_t l = fdiv(f, div_items);
    const uint32_t it = f - l * items;
    x.c = it & tpr_mask;
    const uint32_t r = it >> a.tpr_shift;                    // t * n_heads + h
    x.t = fdiv(r, a.div_heads);
    const int h = r - x.t * n_heads;
    const int64_t tok = token_of(x.t);
    const int32_t *map =
        MODE == Kv8WriteLaunch::kStep ? a.map + (int64_t)(j0 + x.t) * a.map_stride : a.map;
    const int64_t page = (uint32_t)map[(tok < 0 ? 0 : tok) >> kPageShift];
    const int64_t row =
        (((int64_t)(l0 + l) * a.c.n_phys_pages + page) * n_heads + h) * kPage + (tok & (kPage - 1));
    x.row = tok < 0 ? -1 : row;
    const int64_t src =
        (((int64_t)(l0 + l) * a.n_tokens + j0) * n_heads + r) * head_dim + (INTERLEAVED ? 2 : 1) * N * x.c;
    const int64_t next = INTERLEAVED ? N : n_pairs;
    x.ka = ld_stream(reinterpret_cast<const u32x4 *>(src_k + src));
    x.kb = ld_stream(reinterpret_cast<const u32x4 *>(src_k + src + next));
    x.va = ld_stream(reinterpret_cast<const u32x4 *>(src_v + src));
    x.vb = ld_stream(reinterpret_cast<const u32x4 *>(src_v + src + next));
  };

  Item cur;
  uint32_t f = threadIdx.x;
  if (f < n_items) load(f, cur);

  if constexpr (PER_TOKEN) {
    const int i = threadIdx.x & (n_pairs - 1);
    const int step = blockDim.x / n_pairs;
    const double theta = pair_theta(a.base, i, head_dim);
    for (int t = threadIdx.x / n_pairs; t < n_tok; t += step) {
      const int64_t pos = MODE == Kv8WriteLaunch::kStep ? token_of(t) : a.angle0 + j0 + t;
      const int e = t * n_pairs + i;
      pair_cs_theta(pos < 0 ? 0 : pos, theta, cs_tab[0][e], cs_tab[1][e], cs_tab[2][e], cs_tab[3][e]);
    }
  } else {
    for (int i = threadIdx.x; i < n_pairs; i += blockDim.x) {
#pragma unroll
      for (int q = 0; q < 4; ++q) cs_tab[q][i] = tab.v[q][i];
    }
  }
  // LDS-only barrier: the loads above stay in flight
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");

  // a row's threads stay together: items and the stride are whole rows, and a row never leaves its wave
  for (; f < n_items; f += blockDim.x) {
    if (f != threadIdx.x) load(f, cur);
    const Item &x = cur;
    if (x.row < 0) continue;
    float y[2 * N], p[N], q[N];
    Pack<T>::unpack(x.ka, y);
    Pack<T>::unpack(x.kb, y + N);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      p[e] = INTERLEAVED ? y[2 * e] : y[e];
      q[e] = INTERLEAVED ? y[2 * e + 1] : y[N + e];
    }
    float ch[N], cl[N], sh[N], sl[N];
    const int e0 = (PER_TOKEN ? x.t * n_pairs : 0) + N * x.c;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      ch[e] = cs_tab[0][e0 + e];
      cl[e] = cs_tab[1][e0 + e];
      sh[e] = cs_tab[2][e0 + e];
      sl[e] = cs_tab[3][e0 + e];
    }
    rotate<N>(p, q, ch, cl, sh, sl);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      y[INTERLEAVED ? 2 * e : e] = p[e];
      y[INTERLEAVED ? 2 * e + 1 : N + e] = q[e];
    }
    // NEOX: neighbours exchange halves, so that a row's store instruction writes pieces of 16 bytes (fp32: 8),
    // the even lanes' in its first half and the odd lanes' in its second: whole cache lines at head_dim 128
    auto put = [&](const uint32_t *w, uint32_t am, uint8_t *codes, uint8_t *scales) {
      uint8_t *at = codes + x.row * head_dim;
      uint32_t o[N / 2];
      if constexpr (INTERLEAVED) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) o[i] = w[i];
        at += 2 * N * x.c;
      } else {
        const bool odd = x.c & 1;
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
          const uint32_t got = dpp<kXor1>(odd ? w[i] : w[N / 4 + i]);
          o[i] = odd ? got : w[i];
          o[N / 4 + i] = odd ? w[N / 4 + i] : got;
        }
        at += odd ? n_pairs + N * (x.c - 1) : N * x.c;
      }
      if constexpr (N == 8)
        st_stream(u32x4{o[0], o[1], o[N / 2 - 2], o[N / 2 - 1]}, reinterpret_cast<u32x4 *>(at));
      else
        st_stream(u32x2{o[0], o[1]}, reinterpret_cast<u32x2 *>(at));
      if (x.c == 0) scales[x.row] = (uint8_t)scale_byte(am);
    };
    uint32_t w[N / 2];
    const uint32_t ak = row_max(amax_bits<2 * N>(y), a.tpr_shift);
    quantise<2 * N>(y, ak, w);
    put(w, ak, a.c.k, a.c.ks);
    const uint32_t v[8] = {x.va[0], x.va[1], x.va[2], x.va[3], x.vb[0], x.vb[1], x.vb[2], x.vb[3]};
    uint32_t av;
    if constexpr (N == 8) {
      av = row_max(amax_bits_bf16<8>(v), a.tpr_shift);
      quantise_bf16<8>(v, av, w);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = __uint_as_float(v[e]);
      av = row_max(amax_bits<8>(y), a.tpr_shift);
      quantise<8>(y, av, w);
    }
    put(w, av, a.c.v, a.c.vs);
  }
}

hipError_t launch_kv8_write(const Kv8WriteLaunch &p, hipStream_t stream) {
  Kv8WriteArgs a{};
  a.c = p.c;
  a.src_k = p.src_k;
  a.src_v = p.src_v;
  a.map = p.map;
  a.lens = p.lens;
  a.offset = p.offset;
  a.angle0 = p.angle0;
  a.base = p.rope_base;
  a.div_heads = make_fastdiv((uint32_t)p.c.n_heads);
  const uint32_t tpr = (uint32_t)(p.c.head_dim / 2 / (16 / p.dtype_bytes));
  while ((1u << a.tpr_shift) < tpr) ++a.tpr_shift;
  a.n_tokens = p.n_tokens;
  a.map_stride = p.map_stride;
  a.max_len = p.max_len;
  RopeTab tab{};
  if (p.mode == Kv8WriteLaunch::kFixed) rope_tab_host(p.angle0, p.rope_base, p.c.head_dim, tab);
  // tokens of a workgroup: an item for each of its threads where the heads are few
  const int pairs = p.c.head_dim / 2, per_token = p.c.n_heads * (int)tpr;
  a.tile = std::min(kTabEntries / pairs, std::max(4, 256 / per_token));
  const int tiles = (p.n_tokens + a.tile - 1) / a.tile;
  // and layers: two where that leaves 8 workgroups a CU (1088 tokens x 48 layers: 71.0 us by one, 58.8 by two,
  // 59.9 by three; 512 tokens x 26 layers of head_dim 256, 3328 workgroups: 34.4, 44.1 by two)
  const int64_t all = (int64_t)tiles * p.c.n_layers;
  a.layers = p.mode == Kv8WriteLaunch::kFixed ? 1 : all >= 4096 ? 2 : 1;
  a.div_items = make_fastdiv((uint32_t)(a.tile * per_token));
  a.div_last = make_fastdiv((uint32_t)((p.n_tokens - (tiles - 1) * a.tile) * per_token));
  const dim3 grid(tiles, (p.c.n_layers + a.layers - 1) / a.layers);
  auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a, tab);
    return hipGetLastError();
  };
#define NEXUS_KV8_WRITE(T, IL)                                                              \
  (p.mode == Kv8WriteLaunch::kFixed   ? run(kv8_write_kernel<T, IL, Kv8WriteLaunch::kFixed>)   \
   : p.mode == Kv8WriteLaunch::kRange ? run(kv8_write_kernel<T, IL, Kv8WriteLaunch::kRange>)   \
                                      : run(kv8_write_kernel<T, IL, Kv8WriteLaunch::kStep>))
  if (p.dtype_bytes == 2)
    return p.interleaved ? NEXUS_KV8_WRITE(uint16_t, true) : NEXUS_KV8_WRITE(uint16_t, false);
  return p.interleaved ? NEXUS_KV8_WRITE(uint32_t, true) : NEXUS_KV8_WRITE(uint32_t, false);
#undef NEXUS_KV8_WRITE
}

}  // namespace nexus
