// A layer's fresh rows on their way into the paged cache, in one pass: queries and keys normalised per head and
// rotated to their positions (RoPE, Sec. III-B), queries written out, keys and values written to their slots.
//
//   y = x / sqrt(mean(x^2) + eps) * w,   feature pair i turned by pos * base^(-2i/D)
//
// HBM-bound: every row is read once and written once.  A workgroup takes a few tokens: it issues the loads of its
// first items, forms the cosine and sine of the tokens' angles in LDS meanwhile, then normalises, rotates and stores.  A
// row lies in D / 2N neighbouring lanes, N pairs each (N = 8 in bf16, 4 in fp32: both halves of a NEOX pair in one
// lane), so its sum of squares takes log2(D / 2N) lane swaps and its pairs none.  Sums and products are fp32; the result
// is rounded once.
// Angles are formed and reduced modulo 2 pi in fp64.  fp32 rows take cosine and sine in fp64 and turn by head + tail
// pairs with compensated products, as every rotation of this library; bf16 rows, whose half step is 2^16 times the
// error of an fp32 product, take them in fp32 (within 2^-23) and turn by plain fp32 products.
// 4096 rows of 40 + 16 heads of 128 bf16 20.8 us (117 MB, 5.6 TB/s); 1001 such rows in fp32 with a transposed V 12.7 (57
// MB, 4.5 TB/s); one row 4.1.
// A transposed V is written by workgroups of its own, 16 tokens of two KV heads: through LDS, so that a thread has a
// feature of all of them and stores 16 bytes where their slots follow one another.
#include "launch_batch.h"
#include "rope_math.h"

#include <type_traits>

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
  int32_t n_rows;           // rows of a token that lie in rows of the cache or q_out: without a transposed V
  uint32_t v_tiles;         // workgroups of a transposed V (the first ones)
};

}  // namespace

constexpr int kVTok = 16, kVHeads = 2;      // tokens and KV heads of a workgroup that writes a transposed V

// Tokens [kVTok tile, ..) of heads [kVHeads hg, ..) into the feature rows of a transposed V.
template <typename T>
__device__ __forceinline__ void transposed_v(const NormRopeLaunch &p, int tile, int hg, char *smem) {
  constexpr int E = 16 / (int)sizeof(T);    // elements of 16 bytes
  __shared__ int32_t slots[kVTok];
  const int D = p.head_dim, t0 = tile * kVTok, n_tok = min(kVTok, p.n_tokens - t0);
  const int heads = min(kVHeads, p.n_kv_heads - hg * kVHeads);
  const int row = heads * D, ld = kVHeads * D + E;      // elements of a token here, and of its padded row in LDS
  T *buf = reinterpret_cast<T *>(smem);
  const T *src = reinterpret_cast<const T *>(p.v) + (int64_t)hg * kVHeads * D;
  for (int i = threadIdx.x * E; i < n_tok * row; i += 256 * E) {
    const int t = i / row, d = i - t * row;
    *reinterpret_cast<u32x4 *>(buf + t * ld + d) =
        *reinterpret_cast<const u32x4 *>(src + (int64_t)(t0 + t) * p.v_stride + d);
  }
  if (threadIdx.x < kVTok) {
    const int s = (int)threadIdx.x < n_tok ? p.slot[t0 + threadIdx.x] : -1;
    slots[threadIdx.x] = (uint32_t)s < (uint32_t)p.n_phys_pages * kPage ? s : -1;
  }
  __syncthreads();
  const int64_t n_cols = (int64_t)p.n_phys_pages * kPage;
  for (int d = threadIdx.x; d < row; d += 256) {
    T *dst = reinterpret_cast<T *>(p.cache_v) + ((int64_t)hg * kVHeads * D + d) * n_cols;
    for (int t = 0; t < n_tok;) {
      const int s = slots[t];
      bool run = s >= 0 && s % E == 0 && t + E <= n_tok;
#pragma unroll
      for (int e = 1; e < E; ++e) run = run && slots[min(t + e, kVTok - 1)] == s + e;
      if (run) {
        T x[E];
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = buf[(t + e) * ld + d];
        *reinterpret_cast<u32x4 *>(dst + s) = *reinterpret_cast<u32x4 *>(x);
        t += E;
      } else {
        if (s >= 0) dst[s] = buf[t * ld + d];
        ++t;
      }
    }
  }
}

template <typename T, bool INTERLEAVED, bool NORM, bool VT, int TOK>
__global__ __launch_bounds__(256) void norm_rope_kernel(const NormRopeArgs a) {
  constexpr int N = Pack<T>::N;
  constexpr bool TAIL = sizeof(T) == 4;        // cosines and sines as head + tail
  constexpr int TAB = (TAIL ? 4 : 2) * TOK * kTabPairs, WTAB = 4 * kTabPairs;
  constexpr int VBYTES = VT ? kVTok * (kVHeads * 2 * kTabPairs * (int)sizeof(T) + 16) : 0;
  constexpr int BYTES = 4 * (TAB + WTAB) > VBYTES ? 4 * (TAB + WTAB) : VBYTES;
  __shared__ __align__(16) char smem[BYTES];
  float *cs_tab = reinterpret_cast<float *>(smem);           // [cos, sin(, tails)][TOK][pairs]
  float *w_tab = cs_tab + TAB;                               // [q, k][head_dim]
  const NormRopeLaunch &p = a.p;
  uint32_t tile = blockIdx.x;
  if constexpr (VT) {
    if (tile < a.v_tiles) {
      const uint32_t groups = (p.n_kv_heads + kVHeads - 1) / kVHeads;
      transposed_v<T>(p, tile / groups, tile % groups, smem);
      return;
    }
    tile -= a.v_tiles;
  }
  const int D = p.head_dim, n_pairs = D / 2;
  const int t0 = tile * TOK;
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
      w_tab[i] = w ? w[i < D ? i : i - D] : 1.f;
    }
  }
  {
    // a thread keeps its pair (n_pairs is a power of two)
    const int i = threadIdx.x & (n_pairs - 1);
    const double theta = a.f.a[i >> 3] * a.f.b[i & 7];
    for (int t = threadIdx.x / n_pairs; t < n_tok; t += 256 / n_pairs) {
      float *at = cs_tab + t * kTabPairs + i;
      constexpr int P = TOK * kTabPairs;
      if constexpr (TAIL) {
        pair_cs_theta(p.pos[t0 + t], theta, at[0], at[2 * P], at[P], at[3 * P]);
      } else {
        const double ang = (double)p.pos[t0 + t] * theta;
        const double k = rint(ang / kTwoPiHi);
        sincosf((float)fma(-k, kTwoPiLo, fma(-k, kTwoPiHi, ang)), at + P, at);
      }
    }
  }
  // LDS-only barrier: the item loads above stay in flight
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");

  auto item = [&](uint32_t it, const Item &x0) {
    const bool is_q = x0.r < p.n_q_heads, is_v = x0.r >= p.n_q_heads + p.n_kv_heads;
    const int slot = p.slot[t0 + x0.t];
    const bool live = it < items && (uint32_t)slot < (uint32_t)p.n_phys_pages * kPage;
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
        const float *wa = w_tab + (is_q ? 0 : D) + ea, *wb = w_tab + (is_q ? 0 : D) + eb;
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
      const float *at = cs_tab + x0.t * kTabPairs + N * c;
      constexpr int P = TOK * kTabPairs;
      if constexpr (TAIL) {
        float ch[N], cl[N], sh[N], sl[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
          ch[e] = at[e];
          sh[e] = at[P + e];
          cl[e] = at[2 * P + e];
          sl[e] = at[3 * P + e];
        }
        rotate<N>(u, v, ch, cl, sh, sl);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float co = at[e], si = at[P + e], xu = u[e], xv = v[e];
          u[e] = fmaf(xu, co, -(xv * si));
          v[e] = fmaf(xv, co, xu * si);
        }
      }
#pragma unroll
      for (int e = 0; e < N; ++e) {
        x[INTERLEAVED ? 2 * e : e] = u[e];
        x[INTERLEAVED ? 2 * e + 1 : N + e] = v[e];
      }
      ya = Pack<T>::pack(x);
      yb = Pack<T>::pack(x + N);
    }
    if (!live) return;
    const int h = is_q ? x0.r : is_v ? x0.r - p.n_q_heads - p.n_kv_heads : x0.r - p.n_q_heads;
    T *dst = is_q ? reinterpret_cast<T *>(p.q_out) + ((int64_t)(t0 + x0.t) * p.n_q_heads + h) * D
                  : reinterpret_cast<T *>(is_v ? p.cache_v : p.cache_k) +
                        (((int64_t)(slot >> kPageShift) * p.n_kv_heads + h) * kPage + (slot & (kPage - 1))) * D;
    // (past the caches: 4096 rows of 40 + 16 heads of 128 bf16 after other data 28.2 -> 27.2 us, 1001 fp32 rows 20.0 ->
    // 17.8, the same rows over and over 20.9 -> 20.8 and 14.5 -> 12.7; the loads, often of what was just computed, are
    // not)
    st_stream(ya, reinterpret_cast<u32x4 *>(dst + ea));
    st_stream(yb, reinterpret_cast<u32x4 *>(dst + eb));
  };
  for (uint32_t it0 = 0; it0 < items; it0 += 256) {
    const Item x = cur;
    if (it0 + 256 < items) load(it0 + 256 + threadIdx.x, cur);
    item(it0 + threadIdx.x, x);
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
  a.n_rows = p.n_q_heads + (p.v_transposed ? 1 : 2) * p.n_kv_heads;
  a.div_rows = make_fastdiv((uint32_t)a.n_rows);
  a.v_tiles = p.v_transposed ? (uint32_t)((p.n_tokens + kVTok - 1) / kVTok) *
                                   ((p.n_kv_heads + kVHeads - 1) / kVHeads) : 0;
  // One token a workgroup, so that few tokens spread over the chip (32 rows of 40 + 16 heads of 128 bf16: 4.3 us, four
  // tokens a workgroup 8.6; 1001 rows in fp32, transposed V: 14.2, 17.9); four where bf16 rows fill it all the same
  // (4096 such rows 21.4 us, four 20.9; 8000 rows of 32 + 16 heads of 64: 19.7, 17.8).
  const bool four = p.dtype_bytes == 2 && p.n_tokens >= 2048;
  auto run = [&](auto kernel, int tok) {
    hipLaunchKernelGGL(kernel, dim3((p.n_tokens + tok - 1) / tok + a.v_tiles), dim3(256), 0, stream, a);
    return hipGetLastError();
  };
  auto with_v = [&](auto t, auto il, auto no, auto vt) {
    using T = decltype(t);
    if constexpr (sizeof(T) == 2) {
      if (four) return run(norm_rope_kernel<T, il(), no(), vt(), 4>, 4);
    }
    return run(norm_rope_kernel<T, il(), no(), vt(), 1>, 1);
  };
  using yes = std::true_type;
  using no = std::false_type;
  auto with_n = [&](auto t, auto il, auto n) {
    return p.v_transposed ? with_v(t, il, n, yes{}) : with_v(t, il, n, no{});
  };
  auto with_i = [&](auto t, auto il) { return p.eps > 0.f ? with_n(t, il, yes{}) : with_n(t, il, no{}); };
  auto with_t = [&](auto t) { return p.interleaved ? with_i(t, yes{}) : with_i(t, no{}); };
  return p.dtype_bytes == 2 ? with_t(uint16_t{}) : with_t(uint32_t{});
}

}  // namespace nexus
