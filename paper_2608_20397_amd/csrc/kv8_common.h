// The 8-bit cache's row format on the device (internal, not part of the C ABI).
//
// A row (one token, KV head and layer of K or V) is head_dim E4M3 codes under one scale 2^e, kept as
// the byte e + 127 (E8M0).  e is the least integer for which no element passes the largest code:
// amax <= 448 * 2^e, held within [kMinExp, kMaxExp].  The scale is a power of two because a code times it
// is then exact in bf16: what the attention multiplies is what a read returns, and the scale costs no
// instruction (the conversion to bf16 and the scaled MFMA both take it).  Against a scale amax / 448
// this loses nothing in the codes' normal range, from 2^-6 2^e up, where a code's relative error is that of its
// three mantissa bits whatever the scale.  (amax > 224 * 2^e, so that range begins below 2^-13.8 of amax, and
// what lies under it is off by at most 2^-10 2^e < 2^-17.8 of amax.)
#pragma once

#include "device_common.h"

namespace nexus {

constexpr int kMinExp = -100;    // keeps every value and scale a normal fp32 number
constexpr int kMaxExp = 119;     // 448 * 2^119 < 2^128: larger elements take the largest code
constexpr uint32_t kBadScale = 255;           // the row had an element that is not finite
constexpr uint32_t kBadCodes = 0x7F7F7F7Fu;   // its codes: NaN

typedef __attribute__((ext_vector_type(8))) int32_t i32x8;
typedef __attribute__((ext_vector_type(2))) short s16x2;
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;

// Exponent of a row from the bits of its largest magnitude (a finite one): adding 0x1FFFFF carries into
// the exponent field exactly when the mantissa passes 1.75.
__device__ __forceinline__ int row_exp(uint32_t amax_bits) {
  const int e = (int)((amax_bits + 0x1FFFFFu) >> 23) - 135;
  return min(max(e, kMinExp), kMaxExp);
}
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// The value of a scale byte.
__device__ __forceinline__ float scale_value(uint32_t byte) {
  return byte == kBadScale ? __uint_as_float(0x7FC00000u) : __uint_as_float(byte << 23);
}

// Largest magnitude as bits: what is not finite compares above everything finite.
template <int N>
__device__ __forceinline__ uint32_t amax_bits(const float *x) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) m = max(m, __float_as_uint(x[e]) & 0x7FFFFFFFu);
  return m;
}

// The same of bf16 pairs as they lie in words: the upper halves and the lower ones together.
template <int W>
__device__ __forceinline__ uint32_t amax_bits_bf16(const uint32_t *w) {
  u16x2 m = {0, 0};
#pragma unroll
  for (int i = 0; i < W; ++i)
    m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7FFF7FFFu));
  return (uint32_t)max(m[0], m[1]) << 16;
}

// Codes of N values (a multiple of 4) of a row whose largest magnitude has the bits `am`: x / 2^e, which the
// conversion divides by itself.
template <int N>
__device__ __forceinline__ void quantise(const float *x, uint32_t am, uint32_t *codes) {
  const float scale = exp2i(row_exp(am));
  float y[N];
#pragma unroll
  for (int e = 0; e < N; ++e) y[e] = x[e];
  if (am > 0x7F600000u) {   // past 448 * 2^kMaxExp, or not finite
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = fminf(fmaxf(y[e], -448.f * scale), 448.f * scale);
  }
#pragma unroll
  for (int e = 0; e < N / 4; ++e) {
    s16x2 w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, y[4 * e], y[4 * e + 1], scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, y[4 * e + 2], y[4 * e + 3], scale, true);
    codes[e] = am >= 0x7F800000u ? kBadCodes : __builtin_bit_cast(uint32_t, w);
  }
}
// ... of W words of bf16 pairs.
template <int W>
__device__ __forceinline__ void quantise_bf16(const uint32_t *x, uint32_t am, uint32_t *codes) {
  if (am > 0x7F600000u) {   // (the largest exponents take the clamps of the fp32 path)
    float y[2 * W];
#pragma unroll
    for (int i = 0; i < W; ++i) {
      y[2 * i] = __uint_as_float(x[i] << 16);
      y[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
    }
    quantise<2 * W>(y, am, codes);
    return;
  }
  const float scale = exp2i(row_exp(am));
#pragma unroll
  for (int i = 0; i < W / 2; ++i) {
    s16x2 w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, x[2 * i]), scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, x[2 * i + 1]), scale, true);
    codes[i] = __builtin_bit_cast(uint32_t, w);
  }
}
__device__ __forceinline__ uint32_t scale_byte(uint32_t am) {
  return am >= 0x7F800000u ? kBadScale : (uint32_t)(row_exp(am) + 127);
}

// Four codes (a word) times a power-of-two scale, as two words of bf16: exact.
__device__ __forceinline__ u32x2 codes_to_bf16(uint32_t w, float scale) {
  return u32x2{
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true))};
}

// A row's part of a bf16 query as two E4M3 terms, q = (hi + lo / 16) 2^e exactly where |q| is at least
// 2^-6 2^e, which is below 2^-13.8 of the row's largest magnitude, and to 2^-14 2^e, 2^-21.8 of that, below: a bf16
// has 8 significant bits, hi takes the upper 4 and the remainder needs no more than 4.  Two fp8 products with keys as they are
// stored then give the bf16 product at the matrix cores' same cost, with no conversion of the keys and
// half the bytes read from LDS.  x: W words of bf16 pairs (a multiple of 2); e: of the whole row (row_exp), whose
// magnitudes stay below 448 * 2^e (clamp_query).  A row that is not finite becomes NaN through the scale byte
// kBadScale, not here.  (The conversions scale by themselves, 7 instructions for 2 elements; scaled, clamped and
// converted apart, 16, one query over 16 keys took 10.7 us at head_dim 256 instead of 9.1, at 128 7.7 for 7.0.)
template <int W>
__device__ __forceinline__ void split_query(const uint32_t *x, int e, uint32_t *hi, uint32_t *lo) {
  const float s = exp2i(e), sl = exp2i(e - 4);
#pragma unroll
  for (int i = 0; i < W / 2; ++i) {
    s16x2 h = {0, 0}, l = {0, 0};
    h = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(h, __builtin_bit_cast(bf16x2, x[2 * i]), s, false);
    h = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(h, __builtin_bit_cast(bf16x2, x[2 * i + 1]), s, true);
    hi[i] = __builtin_bit_cast(uint32_t, h);
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi[i], s, false);
    const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi[i], s, true);
    const auto low = [](uint32_t w) { return __uint_as_float(w << 16); };
    const auto high = [](uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); };
    l = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(l, low(x[2 * i]) - a[0], high(x[2 * i]) - a[1], sl, false);
    l = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(l, low(x[2 * i + 1]) - b[0], high(x[2 * i + 1]) - b[1], sl,
                                                 true);
    lo[i] = __builtin_bit_cast(uint32_t, l);
  }
}
// Magnitudes past 448 * 2^kMaxExp (the last 1/8 of bf16's largest binade) become that; am: a row's amax bits.
template <int W>
__device__ __forceinline__ void clamp_query(uint32_t *x, uint32_t am) {
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(am > 0x7F600000u) != 0, 0)) {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const u16x2 m =
          __builtin_elementwise_min(__builtin_bit_cast(u16x2, x[i] & 0x7FFF7FFFu), u16x2{0x7F60, 0x7F60});
      x[i] = __builtin_bit_cast(uint32_t, m) | (x[i] & 0x80008000u);
    }
  }
}

}  // namespace nexus
