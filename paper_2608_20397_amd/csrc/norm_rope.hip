// A layer's fresh rows on their way into the paged cache, in one pass: queries and keys normalised per head and
// rotated to their positions (RoPE, Sec. III-B), queries written out, keys and values written to their slots.
//
//   y = x / sqrt(mean(x^2) + eps) * w,   feature pair i turned by pos * base^(-2i/D)
//
// HBM-bound: every row is read once and written once.  A workgroup takes a few tokens: it issues the loads of its
// first items, forms the cosine and sine of the tokens' angles in LDS meanwhile (fp64 angle reduced modulo 2 pi, fp32
// head + tail, as every rotation of this library), then normalises, rotates and stores.  A row lies in D / 2N
// neighbouring lanes, N pairs each (N = 8 in bf16, 4 in fp32: both halves of a NEOX pair in one lane), so its sum of
// squares takes log2(D / 2N) lane swaps and its pairs none.  Sums and products are fp32; the result is rounded once.
#include "launch_batch.h"
#include "rope_math.h"

namespace nexus {

namespace {

// theta_i = a[i / 8] b[i % 8], off by three roundings of 2^-53
struct RopeFreq {
  double a[kTabPairs / 8], b[8];
};

struct NormRopeArgs {
  NormRopeLaunch p;
  RopeFreq f;
  uint32_t lane_shift;      // log2 of the lanes of a row
  FastDiv div_rows;         // by the rows of a token
  int32_t n_rows;           // n_q_heads + 2 n_kv_heads
};

}  // namespace

template <typename T, bool INTERLEAVED, bool NORM, bool VT, int TOK>
__global__ __launch_bounds__(256) void norm_rope_kernel(const NormRopeArgs a) {
  constexpr int N = Pack<T>::N;
  __shared__ float cs_tab[4][TOK][kTabPairs];
  __shared__ __align__(16) float w_tab[2][2 * kTabPairs];
  const NormRopeLaunch &p = a.p;
  const int D = p.head_dim, n_pairs = D / 2;
  // transposed V: neighbouring tokens are neighbours in a feature row, so runs of tokens go to one XCD (ids 8 apart),
  // whose L2 joins the elements to whole lines
  const int per = VT ? (gridDim.x + 7) / 8 : 0;
  const int tile = VT ? (blockIdx.x & 7) * per + (blockIdx.x >> 3) : blockIdx.x;
  const int t0 = tile * TOK;
  if (VT && t0 >= p.n_tokens) return;         // padding of the grid
  const int n_tok = min(TOK, p.n_tokens - t0);
  const uint32_t items = (uint32_t)(n_tok * a.n_rows) << a.lane_shift;
  const int c = threadIdx.x & ((1u << a.lane_shift) - 1);     // (the lanes of a row divide 256)
  const int ea = INTERLEAVED ? 2 * N * c : N * c;             // first element of the lane's two chunks
  const int eb = INTERLEAVED ? 2 * N * c + N : n_pairs + N * c;

  struct Item {
    u32x4 xa, xb;
    int t, r;
  };
  auto load = [&](uint32_t it_raw, Item &x) {
    const uint32_t it = min(it_raw, items - 1 - (~it_raw & ((1u << a.lane_shift) - 1)));   // past the end: the last row
    const uint32_t tr = it >> a.lane_shift;
    x.t = fdiv(tr, a.div_rows);
    x.r = tr - x.t * a.n_rows;
    const int64_t tok = t0 + x.t;
    const T *src = x.r < p.n_q_heads ? reinterpret_cast<const T *>(p.q) + tok * p.q_stride + (int64_t)x.r * D
                   : x.r < p.n_q_heads + p.n_kv_heads
                       ? reinterpret_cast<const T *>(p.k) + tok * p.k_stride + (int64_t)(x.r - p.n_q_heads) * D
                       : reinterpret_cast<const T *>(p.v) + tok * p.v_stride +
                             (int64_t)(x.r - p.n_q_heads - p.n_kv_heads) * D;
    x.xa = *reinterpret_cast<const u32x4 *>(src + ea);
    x.xb = *reinterpret_cast<const u32x4 *>(src + eb);
  };
  Item cur;
  load(threadIdx.x, cur);

  if constexpr (NORM) {
    for (int i = threadIdx.x; i < 2 * D; i += 256) {
      const float *w = i < D ? p.q_weight : p.k_weight;
      w_tab[i >= D][i < D ? i : i - D] = w ? w[i < D ? i : i - D] : 1.f;
    }
  }
  {
    // a thread keeps its pair (n_pairs is a power of two)
    const int i = threadIdx.x & (n_pairs - 1);
    const double theta = a.f.a[i >> 3] * a.f.b[i & 7];
    for (int t = threadIdx.x / n_pairs; t < n_tok; t += 256 / n_pairs)
      pair_cs_theta(p.pos[t0 + t], theta, cs_tab[0][t][i], cs_tab[1][t][i], cs_tab[2][t][i], cs_tab[3][t][i]);
  }
  // LDS-only barrier: the item loads above stay in flight
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");

  for (uint32_t it0 = 0; it0 < items; it0 += 256) {
    const Item x0 = cur;
    if (it0 + 256 < items) load(it0 + 256 + threadIdx.x, cur);
    const bool is_q = x0.r < p.n_q_heads, is_v = x0.r >= p.n_q_heads + p.n_kv_heads;
    const int slot = p.slot[t0 + x0.t];
    const bool live = it0 + threadIdx.x < items && (uint32_t)slot < (uint32_t)p.n_phys_pages * kPage;
    u32x4 ya = x0.xa, yb = x0.xb;
    if (!is_v) {
      float x[2 * N], u[N], v[N];
      Pack<T>::unpack(x0.xa, x);
      Pack<T>::unpack(x0.xb, x + N);
      if constexpr (NORM) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 2 * N; ++e) ss = fmaf(x[e], x[e], ss);
        for (uint32_t off = 1u << a.lane_shift >> 1; off > 0; off >>= 1) ss += __shfl_xor(ss, off);
        const float mean = ss / D + p.eps;
        const float *wa = w_tab[!is_q] + ea, *wb = w_tab[!is_q] + eb;
        if (mean > 1e-28f && mean < 1e36f) {
          const float r = 1.0f / sqrtf(mean);
#pragma unroll
          for (int e = 0; e < N; ++e) {
            x[e] = x[e] * r * wa[e];
            x[N + e] = x[N + e] * r * wb[e];
          }
        } else {
          // squares that leave fp32's range (rows past 1e18, or tiny ones beside a tiny eps): again in fp64
          double s2 = 0.;
#pragma unroll
          for (int e = 0; e < 2 * N; ++e) s2 += (double)x[e] * x[e];
          for (uint32_t off = 1u << a.lane_shift >> 1; off > 0; off >>= 1) s2 += __shfl_xor(s2, off);
          const double r = 1.0 / sqrt(s2 / D + (double)p.eps);
#pragma unroll
          for (int e = 0; e < N; ++e) {
            x[e] = (float)(x[e] * r) * wa[e];
            x[N + e] = (float)(x[N + e] * r) * wb[e];
          }
        }
      }
#pragma unroll
      for (int e = 0; e < N; ++e) {
        u[e] = INTERLEAVED ? x[2 * e] : x[e];
        v[e] = INTERLEAVED ? x[2 * e + 1] : x[N + e];
      }
      float ch[N], cl[N], sh[N], sl[N];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        ch[e] = cs_tab[0][x0.t][N * c + e];
        cl[e] = cs_tab[1][x0.t][N * c + e];
        sh[e] = cs_tab[2][x0.t][N * c + e];
        sl[e] = cs_tab[3][x0.t][N * c + e];
      }
      rotate<N>(u, v, ch, cl, sh, sl);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        x[INTERLEAVED ? 2 * e : e] = u[e];
        x[INTERLEAVED ? 2 * e + 1 : N + e] = v[e];
      }
      ya = Pack<T>::pack(x);
      yb = Pack<T>::pack(x + N);
    }
    if (!live) continue;
    const int h = is_q ? x0.r : is_v ? x0.r - p.n_q_heads - p.n_kv_heads : x0.r - p.n_q_heads;
    if (VT && is_v) {
      // one element a feature row
      const int64_t n_cols = (int64_t)p.n_phys_pages * kPage;
      T *dst = reinterpret_cast<T *>(p.cache_v) + (int64_t)h * D * n_cols + slot;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        constexpr int PER = 4 / (int)sizeof(T);
        dst[(ea + e) * n_cols] = (T)(ya[e / PER] >> (e % PER * 16));
        dst[(eb + e) * n_cols] = (T)(yb[e / PER] >> (e % PER * 16));
      }
      continue;
    }
    T *dst = is_q ? reinterpret_cast<T *>(p.q_out) + ((int64_t)(t0 + x0.t) * p.n_q_heads + h) * D
                  : reinterpret_cast<T *>(is_v ? p.cache_v : p.cache_k) +
                        (((int64_t)(slot >> kPageShift) * p.n_kv_heads + h) * kPage + (slot & (kPage - 1))) * D;
    *reinterpret_cast<u32x4 *>(dst + ea) = ya;
    *reinterpret_cast<u32x4 *>(dst + eb) = yb;
  }
}

hipError_t launch_norm_rope(const NormRopeLaunch &p, hipStream_t stream) {
  NormRopeArgs a{};
  a.p = p;
  // (powers by products of 64-bit mantissas: a call of pow for each took 1 us of host time)
  const long double r = powl((long double)p.rope_base, -2.0L / p.head_dim);
  long double x = 1.0L;
  for (int i = 0; i < 8; ++i, x *= r) a.f.b[i] = (double)x;
  const long double r8 = x;
  x = 1.0L;
  for (int i = 0; i < (p.head_dim / 2 + 7) / 8; ++i, x *= r8) a.f.a[i] = (double)x;
  const uint32_t lanes = (uint32_t)p.head_dim * p.dtype_bytes / 32;
  while ((1u << a.lane_shift) < lanes) ++a.lane_shift;
  a.n_rows = p.n_q_heads + 2 * p.n_kv_heads;
  a.div_rows = make_fastdiv((uint32_t)a.n_rows);
  constexpr int TOK = 4;
  const uint32_t tiles = (p.n_tokens + TOK - 1) / TOK;
  const dim3 grid(p.v_transposed ? (tiles + 7) / 8 * 8 : tiles);
  auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a);
    return hipGetLastError();
  };
#define NEXUS_NORM(T, IL, NO, VT) run(norm_rope_kernel<T, IL, NO, VT, TOK>)
#define NEXUS_NORM_V(T, IL, NO) (p.v_transposed ? NEXUS_NORM(T, IL, NO, true) : NEXUS_NORM(T, IL, NO, false))
#define NEXUS_NORM_N(T, IL) (p.eps > 0.f ? NEXUS_NORM_V(T, IL, true) : NEXUS_NORM_V(T, IL, false))
#define NEXUS_NORM_I(T) (p.interleaved ? NEXUS_NORM_N(T, true) : NEXUS_NORM_N(T, false))
  return p.dtype_bytes == 2 ? NEXUS_NORM_I(uint16_t) : NEXUS_NORM_I(uint32_t);
#undef NEXUS_NORM_I
#undef NEXUS_NORM_N
#undef NEXUS_NORM_V
#undef NEXUS_NORM
}

}  // namespace nexus
