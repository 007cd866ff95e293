// Microscaled rows on gfx950: the record layout and the conversions shared by
// the store (mx_store.hip) and the product (mx_linear.hip).
//
// A row of `dim` elements is cut into blocks of 32.  Block b holds the scale
// 2^(c_b - 127), one byte c_b (255: not a number), and 32 elements of 4 bits
// (sign, then 0 .5 1 1.5 2 3 4 6) or of 8 bits (sign, 4 exponent bits of bias
// 7, 3 mantissa bits; 448 the largest).  A record is all blocks' elements,
// then all scales, then zeros up to a multiple of 16 bytes, so that a row is
// one address: its scales lie on the line after (or with) its elements.
//
// The block's scale is that of its largest magnitude, c = max(e - s, 0) with
// e the fp32 exponent field of that magnitude and s = 2 (4 bits) or 8 (8
// bits), the exponent of the format's largest value.  It is a power of two,
// so x / 2^(c - 127) is exact and an element takes one rounding, to nearest,
// ties to even; magnitudes past the largest value (6 or 448) become it.
#pragma once

#include "common.hpp"

namespace gmb {

typedef float mx_f32x2 __attribute__((ext_vector_type(2)));
typedef short mx_i16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kMxBlock = 32;

// The scale's code of a block whose largest magnitude has the fp32 bits
// `top` (sign cleared; infinities and NaN are above every number's bits).
template <int BITS>
__device__ __forceinline__ uint32_t mx_scale_code(uint32_t top) {
  const uint32_t e = top >> 23;
  constexpr uint32_t shift = BITS == 4 ? 2 : 8;
  return e == 255 ? 255u : (e > shift ? e - shift : 0u);
}

// The conversion instructions take the scale as the exponent field of an
// fp32 (field 0 stands for 2^-127, field 255 makes every result NaN).
__device__ __forceinline__ float mx_scale(uint32_t code) { return __uint_as_float(code << 23); }

// Eight values as elements at scale `code`: one word (4 bits) or two.
template <int BITS>
__device__ __forceinline__ void mx_pack8(const float (&v)[8], uint32_t code, uint32_t (&w)[BITS / 4]) {
  const float s = mx_scale(code);
  if constexpr (BITS == 4) {
    uint32_t x = 0;
    x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(x, v[0], v[1], s, 0);
    x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(x, v[2], v[3], s, 1);
    x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(x, v[4], v[5], s, 2);
    x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(x, v[6], v[7], s, 3);
    w[0] = code == 255 ? 0u : x;
  } else {
    // the 8-bit conversion turns what is past 448 into NaN: clamp to 448
    // scales first (1.75 * 2^8, at most 2^(246 + 8 - 127))
    const float most = __uint_as_float(((code + 8) << 23) | 0x600000u);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float c[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) c[j] = fminf(fmaxf(v[4 * i + j], -most), most);
      mx_i16x2 x = {0, 0};
      x = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(x, c[0], c[1], s, false);
      x = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(x, c[2], c[3], s, true);
      w[i] = code == 255 ? 0u : __builtin_bit_cast(uint32_t, x);
    }
  }
}

// What eight elements stand for.
template <int BITS>
__device__ __forceinline__ void mx_unpack8(const uint32_t (&w)[BITS / 4], uint32_t code, float (&v)[8]) {
  const float s = mx_scale(code);
  mx_f32x2 p[4];
  if constexpr (BITS == 4) {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], s, 0);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], s, 1);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], s, 2);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], s, 3);
  } else {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[0], s, false);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[0], s, true);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[1], s, false);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[1], s, true);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = p[i][0];
    v[2 * i + 1] = p[i][1];
  }
}

// Two values as bf16 bits, to nearest even (v_cvt_pk_bf16_f32).
__device__ __forceinline__ uint32_t mx_bf16x2_bits(float a, float b) {
  const mx_f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, mx_bf16x2));
}

// Eight values to p, fp32 or bf16; `count` of them (8 at once where whole).
__device__ __forceinline__ void mx_store8(float* p, const float (&v)[8], int count) {
  if (count >= 8) {
    const float4 a = make_float4(v[0], v[1], v[2], v[3]), b = make_float4(v[4], v[5], v[6], v[7]);
    __builtin_memcpy(p, &a, 16);
    __builtin_memcpy(p + 4, &b, 16);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < count) p[i] = v[i];
  }
}
__device__ __forceinline__ void mx_store8(uint16_t* p, const float (&v)[8], int count) {
  uint4 x;
  x.x = mx_bf16x2_bits(v[0], v[1]);
  x.y = mx_bf16x2_bits(v[2], v[3]);
  x.z = mx_bf16x2_bits(v[4], v[5]);
  x.w = mx_bf16x2_bits(v[6], v[7]);
  if (count >= 8) {
    __builtin_memcpy(p, &x, 16);
  } else {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < count) p[i] = static_cast<uint16_t>(w[i / 2] >> (16 * (i & 1)));
  }
}

}  // namespace gmb
