// Rows quantised on their way into an 8-bit paged cache, keys rotated first: the write side of the cache
// (kv8_common.h has the format).  Three uses share the kernel:
//   * kFixed: a compiled block re-anchored and spliced, every key turned by the same angle;
//   * kRange: freshly computed tokens, key j turned to its own position angle0 + j;
//   * kStep:  one new token of each of many sequences, positions and places from device lengths.
// The rotation is that of rope_math.h (angles in fp64, compensated fp32 products); its fp32 result is
// quantised directly, so an element is rounded once.
//
// A thread takes the feature pairs of two 16-byte chunks of a row (K and V alike); the threads of a row are
// neighbours in a wave and find its largest magnitude by lane exchanges.  HBM-bound: a row is read once
// and written once, at half (bf16) or a quarter (fp32) of its bytes.
#include "kv8_common.h"
#include "launch_kv8.h"
#include "rope_math.h"

namespace nexus {

namespace {

constexpr int kTileTokens = 4;   // tokens a workgroup takes, all heads of one layer

// Largest magnitude over the 2^shift lanes of a row.
__device__ __forceinline__ uint32_t row_max(uint32_t m, uint32_t shift) {
  for (uint32_t d = 1; d < 1u << shift; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, (int)d));
  return m;
}

struct Kv8WriteArgs {
  Kv8Cache c;
  const void *src_k, *src_v;
  const int32_t *map, *lens;
  int64_t offset, angle0;
  double base;
  FastDiv div_heads;
  uint32_t tpr_shift;          // log2 of the threads of a row
  int32_t n_tokens, map_stride, max_len;
};

}  // namespace

template <typename T, bool INTERLEAVED, int MODE>
__global__ __launch_bounds__(256) void kv8_write_kernel(const Kv8WriteArgs a, const RopeTab tab) {
  constexpr int N = Pack<T>::N;
  constexpr bool PER_TOKEN = MODE != Kv8WriteLaunch::kFixed;
  __shared__ float cs_tab[4][PER_TOKEN ? kTileTokens : 1][kTabPairs];
  const int head_dim = a.c.head_dim, n_heads = a.c.n_heads;
  const int j0 = blockIdx.x * kTileTokens;
  const int l = blockIdx.y;
  const int n_tok = min(kTileTokens, a.n_tokens - j0);
  const int n_pairs = head_dim / 2;
  const uint32_t items = (uint32_t)(n_tok * n_heads) << a.tpr_shift;
  const uint32_t tpr_mask = (1u << a.tpr_shift) - 1;
  const T *src_k = static_cast<const T *>(a.src_k), *src_v = static_cast<const T *>(a.src_v);
  const int64_t src0 = ((int64_t)l * a.n_tokens + j0) * n_heads * head_dim;

  // logical token of tile token t (kStep: -1, nothing to write)
  auto token_of = [&](int t) -> int64_t {
    if constexpr (MODE != Kv8WriteLaunch::kStep) return a.offset + j0 + t;
    const int len = a.lens[j0 + t];
    return len >= 1 && len <= a.max_len ? len - 1 : -1;
  };

  if constexpr (PER_TOKEN) {
    const int i = threadIdx.x & (n_pairs - 1);
    const int step = blockDim.x / n_pairs;
    const double theta = pair_theta(a.base, i, head_dim);
    for (int t = threadIdx.x / n_pairs; t < n_tok; t += step) {
      const int64_t pos = MODE == Kv8WriteLaunch::kStep ? token_of(t) : a.angle0 + j0 + t;
      pair_cs_theta(pos < 0 ? 0 : pos, theta, cs_tab[0][t][i], cs_tab[1][t][i], cs_tab[2][t][i],
                    cs_tab[3][t][i]);
    }
  } else {
    for (int i = threadIdx.x; i < n_pairs; i += blockDim.x) {
#pragma unroll
      for (int q = 0; q < 4; ++q) cs_tab[q][0][i] = tab.v[q][i];
    }
  }
  __syncthreads();

  // a row's threads stay together: items and the stride are whole rows, and a row never leaves its wave
  for (uint32_t it = threadIdx.x; it < items; it += blockDim.x) {
    const int c = it & tpr_mask;
    const uint32_t r = it >> a.tpr_shift;                    // t * n_heads + h
    const int t = fdiv(r, a.div_heads);
    const int h = r - t * n_heads;
    const int64_t tok = token_of(t);
    if (tok < 0) continue;
    const int64_t srow = src0 + (int64_t)r * head_dim;
    const int ea = INTERLEAVED ? 2 * N * c : N * c;
    const int eb = INTERLEAVED ? 2 * N * c + N : n_pairs + N * c;
    const u32x4 ka = ld_stream(reinterpret_cast<const u32x4 *>(src_k + srow + ea));
    const u32x4 kb = ld_stream(reinterpret_cast<const u32x4 *>(src_k + srow + eb));
    const u32x4 va = ld_stream(reinterpret_cast<const u32x4 *>(src_v + srow + ea));
    const u32x4 vb = ld_stream(reinterpret_cast<const u32x4 *>(src_v + srow + eb));
    const int32_t *map = MODE == Kv8WriteLaunch::kStep ? a.map + (int64_t)(j0 + t) * a.map_stride : a.map;
    const int64_t page = (uint32_t)map[tok >> kPageShift];
    const int64_t drow =
        (((int64_t)l * a.c.n_phys_pages + page) * n_heads + h) * kPage + (tok & (kPage - 1));

    float x[2 * N], p[N], q[N];
    Pack<T>::unpack(ka, x);
    Pack<T>::unpack(kb, x + N);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      p[e] = INTERLEAVED ? x[2 * e] : x[e];
      q[e] = INTERLEAVED ? x[2 * e + 1] : x[N + e];
    }
    float ch[N], cl[N], sh[N], sl[N];
    const int tt = PER_TOKEN ? t : 0;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      ch[e] = cs_tab[0][tt][N * c + e];
      cl[e] = cs_tab[1][tt][N * c + e];
      sh[e] = cs_tab[2][tt][N * c + e];
      sl[e] = cs_tab[3][tt][N * c + e];
    }
    rotate<N>(p, q, ch, cl, sh, sl);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      x[INTERLEAVED ? 2 * e : e] = p[e];
      x[INTERLEAVED ? 2 * e + 1 : N + e] = q[e];
    }
    auto put = [&](const float *y, uint8_t *codes, uint8_t *scales) {
      const uint32_t am = row_max(amax_bits<2 * N>(y), a.tpr_shift);
      uint32_t w[N / 2];
      quantise<2 * N>(y, am, w);
      if constexpr (N == 8) {
        *reinterpret_cast<u32x2 *>(codes + drow * head_dim + ea) = u32x2{w[0], w[1]};
        *reinterpret_cast<u32x2 *>(codes + drow * head_dim + eb) = u32x2{w[2], w[3]};
      } else {
        *reinterpret_cast<uint32_t *>(codes + drow * head_dim + ea) = w[0];
        *reinterpret_cast<uint32_t *>(codes + drow * head_dim + eb) = w[1];
      }
      if (c == 0) scales[drow] = (uint8_t)scale_byte(am);
    };
    put(x, a.c.k, a.c.ks);
    Pack<T>::unpack(va, x);
    Pack<T>::unpack(vb, x + N);
    put(x, a.c.v, a.c.vs);
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
  const dim3 grid((p.n_tokens + kTileTokens - 1) / kTileTokens, p.c.n_layers);
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
