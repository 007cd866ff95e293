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

// N values (4, or a multiple of 8) as elements at scale `code`: N BITS / 32
// words, the first one's low half alone for four 4-bit elements.
template <int BITS, int N>
__device__ __forceinline__ void mx_pack(const float (&v)[N], uint32_t code, uint32_t (&w)[(N * BITS + 31) / 32]) {
  const float s = mx_scale(code);
  if constexpr (BITS == 4) {
#pragma unroll
    for (int i = 0; i < (N + 7) / 8; ++i) {
      uint32_t x = 0;
      x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(x, v[8 * i], v[8 * i + 1], s, 0);
      x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(x, v[8 * i + 2], v[8 * i + 3], s, 1);
      if constexpr (N >= 8) {
        x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(x, v[8 * i + 4], v[8 * i + 5], s, 2);
        x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(x, v[8 * i + 6], v[8 * i + 7], s, 3);
      }
      w[i] = code == 255 ? 0u : x;
    }
  } else {
    // the 8-bit conversion turns what is past 448 into NaN: clamp to 448
    // scales first (1.75 * 2^8, at most 2^(246 + 8 - 127))
    const float most = __uint_as_float(((code + 8) << 23) | 0x600000u);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
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

// What N elements stand for.
template <int BITS, int N>
__device__ __forceinline__ void mx_unpack(const uint32_t (&w)[(N * BITS + 31) / 32], uint32_t code, float (&v)[N]) {
  const float s = mx_scale(code);
  auto put = [&](int at, mx_f32x2 p) {
    v[at] = p[0];
    v[at + 1] = p[1];
  };
  if constexpr (BITS == 4) {
#pragma unroll
    for (int i = 0; i < (N + 7) / 8; ++i) {
      put(8 * i, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], s, 0));
      put(8 * i + 2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], s, 1));
      if constexpr (N >= 8) {
        put(8 * i + 4, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], s, 2));
        put(8 * i + 6, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], s, 3));
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      put(4 * i, __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], s, false));
      put(4 * i + 2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], s, true));
    }
  }
}

// The largest magnitude's fp32 bits among v.
template <int N>
__device__ __forceinline__ uint32_t mx_top(const float (&v)[N]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t m = __float_as_uint(v[i]) & 0x7FFFFFFFu;
    top = m > top ? m : top;
  }
  return top;
}

// The largest of the words of LANES (4 or 8) neighbouring lanes: their
// neighbour's, the other pair's, the other four's.
template <int LANES>
__device__ __forceinline__ uint32_t mx_lanes_max(uint32_t x) {
  auto with = [&](uint32_t o) { x = o > x ? o : x; };
  with(__builtin_amdgcn_mov_dpp(static_cast<int>(x), 0xB1, 0xF, 0xF, true));                           // 1 0 3 2
  with(__builtin_amdgcn_mov_dpp(static_cast<int>(x), 0x4E, 0xF, 0xF, true));                           // 2 3 0 1
  if constexpr (LANES == 8) with(__builtin_amdgcn_mov_dpp(static_cast<int>(x), 0x141, 0xF, 0xF, true));  // 7 .. 0
  return x;
}

// Two values as bf16 bits, to nearest even (v_cvt_pk_bf16_f32).
__device__ __forceinline__ uint32_t mx_bf16x2_bits(float a, float b) {
  const mx_f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, mx_bf16x2));
}

// BYTES bytes from or to p (any alignment).  STREAM: without a place in the
// caches (non-temporal).  (A template: behind a branch on a value the compiler
// joins the two stores into one plain one.)
template <int BYTES>
struct MxWords {
  typedef uint32_t Type __attribute__((ext_vector_type(BYTES / 4), aligned(2)));
};
template <int BYTES, bool STREAM>
__device__ __forceinline__ void mx_put(void* p, const void* v) {
  using Words = typename MxWords<BYTES>::Type;
  Words x;
  __builtin_memcpy(&x, v, BYTES);
  if constexpr (STREAM)
    __builtin_nontemporal_store(x, static_cast<Words*>(p));
  else
    *static_cast<Words*>(p) = x;
}
template <int BYTES>
__device__ __forceinline__ void mx_get(void* v, const void* p) {
  using Words = typename MxWords<BYTES>::Type;
  const Words x = *static_cast<const Words*>(p);
  __builtin_memcpy(v, &x, BYTES);
}
template <int BYTES>
__device__ __forceinline__ void mx_get_once(void* v, const void* p) {
  using Words = typename MxWords<BYTES>::Type;
  const Words x = __builtin_nontemporal_load(static_cast<const Words*>(p));
  __builtin_memcpy(v, &x, BYTES);
}

// 16 bytes of values to p, fp32 (4) or bf16 (8), or the first `count` of them.
template <bool STREAM>
__device__ __forceinline__ void mx_store(float* p, const float (&v)[4], int count) {
  if (count >= 4) {
    mx_put<16, STREAM>(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < count) p[i] = v[i];
  }
}
template <bool STREAM>
__device__ __forceinline__ void mx_store(uint16_t* p, const float (&v)[8], int count) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = mx_bf16x2_bits(v[2 * i], v[2 * i + 1]);
  if (count >= 8) {
    mx_put<16, STREAM>(p, w);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < count) p[i] = static_cast<uint16_t>(w[i / 2] >> (16 * (i & 1)));
  }
}

}  // namespace gmb
