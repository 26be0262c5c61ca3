// Tokens out of an 8-bit paged cache as the values that their codes stand for, code * 2^e (exact in bf16
// and fp32), in a block's layout [L][T][H][D]: the way back of kv8_write.hip.  A thread takes the codes of
// one 16-byte chunk of the output, of K and of V.  HBM-bound: 1 byte read and 2 (bf16) or 4 (fp32)
// written per element.
#include "kv8_common.h"
#include "launch_kv8.h"

namespace nexus {

namespace {

struct Kv8ReadArgs {
  Kv8Cache c;
  void *dst_k, *dst_v;
  const int32_t *map;
  int64_t offset;
  FastDiv div_heads;
  uint32_t cpr_shift;        // log2 of the chunks of a row
  uint32_t n_items;          // chunks of one layer
};

}  // namespace

// WIDE: fp32 (4 codes a chunk), else bf16 (8).
template <bool WIDE>
__global__ __launch_bounds__(256) void kv8_read_kernel(const Kv8ReadArgs a) {
  constexpr int N = WIDE ? 4 : 8;
  const uint32_t it = blockIdx.x * 256u + threadIdx.x;
  if (it >= a.n_items) return;
  const int l = blockIdx.y;
  const int head_dim = a.c.head_dim, n_heads = a.c.n_heads;
  const uint32_t c = it & ((1u << a.cpr_shift) - 1);
  const uint32_t r = it >> a.cpr_shift;                       // t * n_heads + h
  const uint32_t t = fdiv(r, a.div_heads);
  const uint32_t h = r - t * n_heads;
  const int64_t tok = a.offset + t;
  const int64_t page = (uint32_t)a.map[tok >> kPageShift];
  const int64_t row = (((int64_t)l * a.c.n_phys_pages + page) * n_heads + h) * kPage + (tok & (kPage - 1));
  const int64_t src = row * head_dim + N * c;
  const uint32_t kbyte = a.c.ks[row], vbyte = a.c.vs[row];
  uint32_t kw[N / 4], vw[N / 4];
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    kw[i] = reinterpret_cast<const uint32_t *>(a.c.k + src)[i];
    vw[i] = reinterpret_cast<const uint32_t *>(a.c.v + src)[i];
  }
  const int64_t out = ((int64_t)l * a.n_items + it);          // chunk index
  auto put = [&](const uint32_t *w, uint32_t byte, void *dst) {
    const float s = scale_value(byte);
    u32x4 o;
    if constexpr (WIDE) {
      const f32x2 x = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[0], false);
      const f32x2 y = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[0], true);
      o = u32x4{__float_as_uint(x[0] * s), __float_as_uint(x[1] * s), __float_as_uint(y[0] * s),
                __float_as_uint(y[1] * s)};
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const u32x2 b = codes_to_bf16(byte == kBadScale ? kBadCodes : w[i], exp2i((int)byte - 127));
        o[2 * i] = b[0];
        o[2 * i + 1] = b[1];
      }
    }
    st_stream(o, reinterpret_cast<u32x4 *>(dst) + out);
  };
  put(kw, kbyte, a.dst_k);
  put(vw, vbyte, a.dst_v);
}

hipError_t launch_kv8_read(const Kv8ReadLaunch &p, hipStream_t stream) {
  Kv8ReadArgs a{};
  a.c = p.c;
  a.dst_k = p.dst_k;
  a.dst_v = p.dst_v;
  a.map = p.map;
  a.offset = p.offset;
  a.div_heads = make_fastdiv((uint32_t)p.c.n_heads);
  const uint32_t cpr = (uint32_t)(p.c.head_dim * p.dtype_bytes / 16);
  while ((1u << a.cpr_shift) < cpr) ++a.cpr_shift;
  a.n_items = (uint32_t)p.n_tokens * (uint32_t)p.c.n_heads * cpr;
  const dim3 grid((a.n_items + 255) / 256, p.c.n_layers);
  if (p.dtype_bytes == 2)
    hipLaunchKernelGGL(kv8_read_kernel<false>, grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL(kv8_read_kernel<true>, grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace nexus
