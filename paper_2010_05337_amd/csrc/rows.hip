// Row operators of a residual model on gfx950: dropout whose mask is drawn
// again wherever it is needed, and the root-mean-square norm of a sum with
// its backward.
//
// A row is cut into pieces of eight columns, which share one Philox block
// (eight times 16 bits).  A row belongs to LANES neighbouring threads, lane o
// has the pieces o, o + LANES, ...  All of them read and write each row once and
// are bound by that (a large copy reaches 5.0 TB/s; what is still in the last-level
// cache comes faster).
#include "head_kernels.hpp"
#include "mx.hpp"
#include "mx_kernels.hpp"
#include "philox.hpp"

#include <type_traits>

namespace gmb {

namespace {

constexpr int kPiece = 8;           // columns

__device__ __forceinline__ int64_t count_rows(const int32_t* n_dev, int64_t n_cap) {
  if (!n_dev) return n_cap;
  const int64_t m = load_size(n_dev);
  return m < 0 ? 0 : (m < n_cap ? m : n_cap);
}

// Eight bf16 of which `left` (1 .. 8) are in the row, from p on; the others are 0.
// A row's last piece is read by one load that ends with the row, and shifted
// (26,420 x 1,270: element by element the norm took 90 us, this 61; 46 in rows of
// 1,272).
__device__ __forceinline__ void load_eight(const uint16_t* p, int left, bool first, uint32_t (&w)[4]) {
  if (left >= kPiece) {
    mx_get<16>(w, p);
  } else if (!first) {
    const int s = kPiece - left;
    uint32_t q[4];
    mx_get<16>(q, p - s);
    if (s & 1) {
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = (q[i] >> 16) | (i < 3 ? q[i + 1] << 16 : 0u);
    }
    if (s & 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = i < 3 ? q[i + 1] : 0u;
    }
    if (s & 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = i < 2 ? q[i + 2] : 0u;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = q[i];
  } else {                          // a row of fewer than eight
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = 2 * i < left ? p[2 * i] : 0u;
      if (2 * i + 1 < left) w[i] |= static_cast<uint32_t>(p[2 * i + 1]) << 16;
    }
  }
}

// Piece `o` of a row of `dim` columns; columns past dim are 0.  WHOLE: rows are whole
// pieces (said to the compiler: with the other cases behind a branch 350,000 x 128
// bf16 were dropped out in 49.7 us, without in 45.7).
template <typename T, bool WHOLE>
__device__ __forceinline__ void load_piece(const void* data, int64_t at, int o, int dim, float (&v)[kPiece]) {
  const T* p = static_cast<const T*>(data) + at + o * kPiece;
  const int left = WHOLE ? kPiece : dim - o * kPiece;
  if constexpr (sizeof(T) == 4) {
    if (left >= kPiece) {
      float w[kPiece];
      mx_get<16>(w, p);
      mx_get<16>(w + 4, p + 4);
#pragma unroll
      for (int i = 0; i < kPiece; ++i) v[i] = w[i];
    } else {
#pragma unroll
      for (int i = 0; i < kPiece; ++i) v[i] = i < left ? p[i] : 0.f;
    }
  } else {
    uint32_t w[4];
    load_eight(p, left, o == 0, w);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
}

// Piece `o` as it lies in memory; columns past dim (or `in` false) are 0.
template <typename T>
struct Raw {
  uint32_t w[2 * sizeof(T)];
};
template <typename T, bool WHOLE>
__device__ __forceinline__ void load_raw(const void* data, int64_t at, int o, int dim, bool in, Raw<T>& q) {
  const T* p = static_cast<const T*>(data) + at + o * kPiece;
  const int left = in ? (WHOLE ? kPiece : dim - o * kPiece) : 0;
  if (left <= 0) {
#pragma unroll
    for (int i = 0; i < static_cast<int>(2 * sizeof(T)); ++i) q.w[i] = 0u;
  } else if constexpr (WHOLE) {
    mx_get<16>(q.w, p);
    if constexpr (sizeof(T) == 4) mx_get<16>(q.w + 4, p + 4);
  } else if constexpr (sizeof(T) == 2) {
    load_eight(p, left, o == 0, q.w);
  } else if (left >= kPiece) {
    mx_get<16>(q.w, p);
    mx_get<16>(q.w + 4, p + 4);
  } else {
#pragma unroll
    for (int i = 0; i < kPiece; ++i) q.w[i] = i < left ? __builtin_bit_cast(uint32_t, p[i]) : 0u;
  }
}
template <typename T>
__device__ __forceinline__ void unpack(const Raw<T>& q, float (&v)[kPiece]) {
#pragma unroll
  for (int i = 0; i < kPiece; ++i) {
    if constexpr (sizeof(T) == 4) v[i] = __uint_as_float(q.w[i]);
    else v[i] = __uint_as_float((i & 1) ? q.w[i / 2] & 0xFFFF0000u : q.w[i / 2] << 16);
  }
}

// What a value is in T, as fp32.
template <typename T>
__device__ __forceinline__ void round_piece(float (&v)[kPiece]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < kPiece / 2; ++i) {
      const uint32_t w = mx_bf16x2_bits(v[2 * i], v[2 * i + 1]);
      v[2 * i] = __uint_as_float(w << 16);
      v[2 * i + 1] = __uint_as_float(w & 0xFFFF0000u);
    }
  }
}

template <typename T, bool WHOLE>
__device__ __forceinline__ void store_piece(void* data, int64_t at, int o, int dim, const float (&v)[kPiece]) {
  T* p = static_cast<T*>(data) + at + o * kPiece;
  const int left = WHOLE ? kPiece : dim - o * kPiece;
  if constexpr (sizeof(T) == 4) {
    if (left >= kPiece) {
      mx_put<16, false>(p, v);
      mx_put<16, false>(p + 4, v + 4);
    } else {
#pragma unroll
      for (int i = 0; i < kPiece; ++i)
        if (i < left) p[i] = v[i];
    }
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = mx_bf16x2_bits(v[2 * i], v[2 * i + 1]);
    if (left >= kPiece) {
      mx_put<16, false>(p, w);
    } else {
      if (left & 4) mx_put<8, false>(p, w);
      const uint32_t two = left & 4 ? w[2] : w[0];
      if (left & 2) mx_put<4, false>(p + (left & 4), &two);
      const uint32_t one = left & 4 ? (left & 2 ? w[3] : w[2]) : (left & 2 ? w[1] : w[0]);
      if (left & 1) p[left & 6] = static_cast<uint16_t>(one);
    }
  }
}

// Dropped elements become 0, whatever they hold; the others are scaled.
__device__ __forceinline__ void drop_piece(const DropArgs& d, uint32_t step, uint32_t key, int o, float (&v)[kPiece]) {
  // (the sampler's counters have a layer below 2^31 there)
  const Philox4 x = philox4x32_10(key, 0x80000000u | d.layer, static_cast<uint32_t>(o), step, d.k0, d.k1);
#pragma unroll
  for (int i = 0; i < kPiece; ++i) {
    const uint32_t u = (x.w[i / 2] >> (16 * (i & 1))) & 0xFFFFu;
    v[i] = u < d.below ? 0.f : v[i] * d.scale;
  }
}
__device__ __forceinline__ uint32_t row_key(const DropArgs& d, int64_t row) {
  return static_cast<uint32_t>(d.ids ? d.ids[row] : static_cast<int32_t>(row));
}

// ---- dropout --------------------------------------------------------------

// out = [residual +] keep x 65536 / (65536 - t).  Eight columns cost ten rounds of
// two 32 x 32 products, which hide behind the rows: 45,000 x 256 fp32 15.8 us (5.8
// TB/s), 350,000 x 128 bf16 with a residual 45.5 (5.9); 64 x 16 2.2, a launch.

template <typename T, int LANES, bool WHOLE>
__global__ __launch_bounds__(256) void k_dropout(DropoutArgs p) {
  constexpr int ROWS = 256 / LANES;
  const int64_t n = count_rows(p.n_dev, p.n_cap);
  const int lane = threadIdx.x % LANES, pieces = (p.dim + kPiece - 1) / kPiece;
  const uint32_t step = p.drop.step ? *p.drop.step : 0u;
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / LANES; row < n;
       row += static_cast<int64_t>(gridDim.x) * ROWS) {
    const uint32_t key = row_key(p.drop, row);
    for (int o = lane; o < pieces; o += LANES) {
      float v[kPiece];
      load_piece<T, WHOLE>(p.x.data, row * p.x.stride, o, p.dim, v);
      if (p.drop.below) drop_piece(p.drop, step, key, o, v);
      if (p.residual.data) {
        float r[kPiece];
        load_piece<T, WHOLE>(p.residual.data, row * p.residual.stride, o, p.dim, r);
#pragma unroll
        for (int i = 0; i < kPiece; ++i) v[i] += r[i];
      }
      store_piece<T, WHOLE>(p.out.data, row * p.out.stride, o, p.dim, v);
    }
  }
}

// ---- norm -----------------------------------------------------------------

// The sum of a value over the LANES threads of a row (every one gets it).
// Past a wave the waves' sums meet in LDS, in a fixed order.
template <int LANES, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float* lds) {
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int o = 1; o < (LANES < 64 ? LANES : 64); o <<= 1) v[k] += __shfl_xor(v[k], o, 64);
  if constexpr (LANES > 64) {
    constexpr int WAVES = LANES / 64;
    __syncthreads();                // the last row's reads
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int k = 0; k < N; ++k) lds[(threadIdx.x >> 6) * N + k] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) s += lds[(static_cast<int>(threadIdx.x) / LANES * WAVES + w) * N + k];
      v[k] = s;
    }
  }
}

// rsqrt of the mean square: 1 / sqrt is rounded to within an ulp or two; one
// step of Newton's from v_rsq_f32's result.
__device__ __forceinline__ float inverse_root(float x) {
  const float y = __builtin_amdgcn_rsqf(x);
  const float e = fmaf(-x * y, y, 1.f);
  return x < 3.0e38f ? fmaf(0.5f * y, e, y) : y;
}

// Block (LANES > 256: LANES) threads; OC pieces of the row a thread.
template <int LANES>
struct NormBlock {
  static constexpr int kThreads = LANES > 256 ? LANES : 256;
  static constexpr int kRows = kThreads / LANES;
};

// Piece `o` of the sum, as it is stored.
template <typename T, bool WHOLE>
__device__ __forceinline__ void load_sum(const NormArgs& p, int64_t row, int o, uint32_t step, uint32_t key,
                                         float (&v)[kPiece]) {
  load_piece<T, WHOLE>(p.x.data, row * p.x.stride, o, p.dim, v);
  if (p.drop.below) drop_piece(p.drop, step, key, o, v);
  if (p.residual.data) {
    float r[kPiece];
    load_piece<T, WHOLE>(p.residual.data, row * p.residual.stride, o, p.dim, r);
#pragma unroll
    for (int i = 0; i < kPiece; ++i) v[i] += r[i];
  }
  round_piece<T>(v);
}

// Piece `o` of the norm from the sum's; every lane takes part.
template <typename T, int BITS, bool WHOLE>
__device__ __forceinline__ void store_norm(const NormArgs& p, bool in, int64_t row, int o, int pieces, float inv,
                                           float (&v)[kPiece]) {
  if (in && o < pieces) {
    float g[kPiece];
    if (p.weight) {
      load_piece<float, WHOLE>(p.weight, 0, o, p.dim, g);
    } else {
#pragma unroll
      for (int i = 0; i < kPiece; ++i) g[i] = 1.f;
    }
#pragma unroll
    for (int i = 0; i < kPiece; ++i) v[i] = v[i] * inv * g[i];
    if constexpr (BITS == 0) store_piece<T, WHOLE>(p.out.data, row * p.out.stride, o, p.dim, v);
  }
  if constexpr (BITS != 0) {
    // four neighbouring lanes have a block of 32 columns
    const uint32_t code = mx_scale_code<BITS>(mx_lanes_max<4>(mx_top(v)));
    const int blocks = (p.dim + kMxBlock - 1) / kMxBlock, block = o / 4;
    if (in && block < blocks) {
      uint32_t w[BITS / 4];
      mx_pack<BITS>(v, code, w);
      uint8_t* rec = static_cast<uint8_t*>(p.out.data) + row * p.out.stride;
      __builtin_memcpy(rec + o * BITS, w, BITS);
      if (o % 4 == 0) rec[blocks * 4 * BITS + block] = static_cast<uint8_t>(code);
      if (block == blocks - 1)
        for (int b = blocks * (4 * BITS + 1) + o % 4; b < p.record; b += 4) rec[b] = 0;
    }
  }
}

// r = [residual +] dropout(x), y = g r / sqrt(mean r^2 + eps).  One pass: the row's
// threads keep its pieces while they add up its squares.  45,000 x 256 fp32 with
// dropout and a residual 30.9 us (6.0 TB/s), 8,192 x 4,096 bf16 into 8-bit records 45.0
// (5.3 TB/s, two pieces a thread), one row 2.4.
// HELD: the row stays in registers between its sum and its norm; else it is
// read again (from the stored sum where there is one).
template <typename T, int LANES, int OC, bool HELD, int BITS, bool WHOLE>
__global__ __launch_bounds__(NormBlock<LANES>::kThreads) void k_rms_norm(NormArgs p) {
  constexpr int ROWS = NormBlock<LANES>::kRows;
  __shared__ float lds[NormBlock<LANES>::kThreads / 64];
  const int64_t n = count_rows(p.n_dev, p.n_cap);
  const int lane = threadIdx.x % LANES, pieces = (p.dim + kPiece - 1) / kPiece;
  const uint32_t step = p.drop.step ? *p.drop.step : 0u;
  const float by = 1.f / static_cast<float>(p.dim);
  // (the loop's bound is the workgroup's: all its threads meet at row_sum's barriers)
  for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * ROWS; row0 < n;
       row0 += static_cast<int64_t>(gridDim.x) * ROWS) {
    const int64_t row = row0 + threadIdx.x / LANES;
    const bool in = row < n;
    const uint32_t key = in && p.drop.below ? row_key(p.drop, row) : 0u;
    float v[HELD ? OC : 1][kPiece];
    float ss[1] = {0.f};
#pragma unroll HELD ? OC : 1
    for (int k = 0; k < OC; ++k) {
      const int o = lane + k * LANES, at = HELD ? k : 0;
      if (in && o < pieces) {
        load_sum<T, WHOLE>(p, row, o, step, key, v[at]);
        if (p.sum.data) store_piece<T, WHOLE>(p.sum.data, row * p.sum.stride, o, p.dim, v[at]);
      } else {
#pragma unroll
        for (int i = 0; i < kPiece; ++i) v[at][i] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < kPiece; ++i) ss[0] = fmaf(v[at][i], v[at][i], ss[0]);
    }
    row_sum<LANES>(ss, lds);
    const float inv = inverse_root(fmaf(ss[0], by, p.eps));
#pragma unroll HELD ? OC : 1
    for (int k = 0; k < OC; ++k) {
      const int o = lane + k * LANES, at = HELD ? k : 0;
      if constexpr (!HELD) {
        if (in && o < pieces) {
          if (p.sum.data) load_piece<T, WHOLE>(p.sum.data, row * p.sum.stride, o, p.dim, v[0]);
          else load_sum<T, WHOLE>(p, row, o, step, key, v[0]);
        } else {
#pragma unroll
          for (int i = 0; i < kPiece; ++i) v[0][i] = 0.f;
        }
      }
      store_norm<T, BITS, WHOLE>(p, in, row, o, pieces, inv, v[at]);
    }
  }
}

// With s = 1 / sqrt(mean r^2 + eps): dr = carry + s (g dy - r s^2 mean(g dy r)),
// and d_weight = the sum over the rows of dy r s: a thread's rows in its
// registers, the rows of a workgroup in LDS, the workgroups' sums in 128 chains
// that meet in a fixed order (k_join_parts): no atomics, the same bits every time.
// HELD: a row's dy and r, and its carry, stay in registers as they lie in memory,
// and the next row's are on their way meanwhile (8,192 x 4,096 bf16: 63 us, 78
// without, when the sums of d_weight took 12.3 of them); else dy, r and g are read
// twice.  Now 8,192 x 4,096 bf16 49.2 us (5.5 TB/s), 45,000 x 256 fp32 with dropout
// 40.2 (5.7).
template <typename T, int LANES, int OC, bool HELD, bool WHOLE>
__global__ __launch_bounds__(NormBlock<LANES>::kThreads) void k_rms_norm_back(NormBackArgs p) {
  constexpr int ROWS = NormBlock<LANES>::kRows, KEPT = HELD ? OC : 1;
  __shared__ float lds[2 * (NormBlock<LANES>::kThreads / 64)];
  const int64_t n = count_rows(p.n_dev, p.n_cap);
  const int lane = threadIdx.x % LANES, pieces = (p.dim + kPiece - 1) / kPiece;
  const uint32_t step = p.drop.step ? *p.drop.step : 0u;
  const float by = 1.f / static_cast<float>(p.dim);
  float g[KEPT][kPiece], dw[OC][kPiece];
  Raw<T> r[KEPT], dy[KEPT], carry[KEPT];
  auto load_weight = [&](int o, float (&w)[kPiece]) {
#pragma unroll
    for (int i = 0; i < kPiece; ++i) w[i] = 1.f;
    if (p.weight && o < pieces) load_piece<float, WHOLE>(p.weight, 0, o, p.dim, w);
  };
  auto load = [&](int64_t row, int o, Raw<T>& a, Raw<T>& b) {
    const bool in = row < n && o < pieces;
    load_raw<T, WHOLE>(p.r.data, row * p.r.stride, o, p.dim, in, a);
    load_raw<T, WHOLE>(p.dy.data, row * p.dy.stride, o, p.dim, in, b);
  };
  auto load_carry = [&](int64_t row, int o, Raw<T>& a) {
    load_raw<T, WHOLE>(p.carry.data, row * p.carry.stride, o, p.dim, row < n && o < pieces, a);
  };
  const int64_t rows_each = static_cast<int64_t>(gridDim.x) * ROWS;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * ROWS;
#pragma unroll
  for (int k = 0; k < OC; ++k) {
    const int o = lane + k * LANES;
#pragma unroll
    for (int i = 0; i < kPiece; ++i) dw[k][i] = 0.f;
    if constexpr (HELD) {
      const int64_t row = first + threadIdx.x / LANES;
      load_weight(o, g[k]);
      load(row, o, r[k], dy[k]);
      if (p.carry.data) load_carry(row, o, carry[k]);
    }
  }
  for (int64_t row0 = first; row0 < n; row0 += rows_each) {
    const int64_t row = row0 + threadIdx.x / LANES;
    const bool in = row < n;
    Raw<T> next_r[KEPT], next_dy[KEPT], next_carry[KEPT];
    if constexpr (HELD) {
#pragma unroll
      for (int k = 0; k < OC; ++k) {
        load(row + rows_each, lane + k * LANES, next_r[k], next_dy[k]);
        if (p.carry.data) load_carry(row + rows_each, lane + k * LANES, next_carry[k]);
      }
    }
    float s[2] = {0.f, 0.f};        // r^2, g dy r
#pragma unroll HELD ? OC : 1
    for (int k = 0; k < OC; ++k) {
      const int at = HELD ? k : 0;
      if constexpr (!HELD) {
        load(row, lane + k * LANES, r[0], dy[0]);
        load_weight(lane + k * LANES, g[0]);
      }
      float a[kPiece], b[kPiece];
      unpack<T>(r[at], a);
      unpack<T>(dy[at], b);
#pragma unroll
      for (int i = 0; i < kPiece; ++i) {
        s[0] = fmaf(a[i], a[i], s[0]);
        s[1] = fmaf(g[at][i] * b[i], a[i], s[1]);
      }
    }
    row_sum<LANES>(s, lds);
    const float inv = inverse_root(fmaf(s[0], by, p.eps));
    // (squares past fp32's range: the row norms to 0 and nothing comes back through
    // it, however large the other sum is; a NaN stays one through inv)
    const float along = inv > 0.f ? s[1] * by * inv * inv : 0.f;
    const uint32_t key = in && p.drop.below ? row_key(p.drop, row) : 0u;
#pragma unroll
    for (int k = 0; k < OC; ++k) {
      const int o = lane + k * LANES, at = HELD ? k : 0;
      if constexpr (!HELD) {
        load(row, o, r[0], dy[0]);
        load_weight(o, g[0]);
        if (p.carry.data) load_carry(row, o, carry[0]);
      }
      if (in && o < pieces) {
        float a[kPiece], b[kPiece], d[kPiece];
        unpack<T>(r[at], a);
        unpack<T>(dy[at], b);
#pragma unroll
        for (int i = 0; i < kPiece; ++i) {
          dw[k][i] = fmaf(b[i], a[i] * inv, dw[k][i]);
          d[i] = inv * (g[at][i] * b[i] - a[i] * along);
        }
        if (p.carry.data) {
          float c[kPiece];
          unpack<T>(carry[at], c);
#pragma unroll
          for (int i = 0; i < kPiece; ++i) d[i] += c[i];
        }
        if (p.d_residual.data) store_piece<T, WHOLE>(p.d_residual.data, row * p.d_residual.stride, o, p.dim, d);
        if (p.dx.data) {
          if (p.drop.below) drop_piece(p.drop, step, key, o, d);
          store_piece<T, WHOLE>(p.dx.data, row * p.dx.stride, o, p.dim, d);
        }
      }
      if constexpr (HELD) {
        r[k] = next_r[k];
        dy[k] = next_dy[k];
        if (p.carry.data) carry[k] = next_carry[k];
      }
    }
  }
  if (!p.partial) return;
  if constexpr (ROWS > 1) {
    __shared__ float rows[ROWS][LANES * OC * kPiece];
#pragma unroll
    for (int k = 0; k < OC; ++k)
#pragma unroll
      for (int i = 0; i < kPiece; ++i) rows[threadIdx.x / LANES][(lane + k * LANES) * kPiece + i] = dw[k][i];
    __syncthreads();
    for (int c = threadIdx.x; c < p.dim; c += NormBlock<LANES>::kThreads) {
      float t = 0.f;
#pragma unroll
      for (int w = 0; w < ROWS; ++w) t += rows[w][c];
      p.partial[static_cast<int64_t>(blockIdx.x) * p.dim + c] = t;
    }
  } else {
#pragma unroll
    for (int k = 0; k < OC; ++k)
      if (lane + k * LANES < pieces)
        store_piece<float, WHOLE>(p.partial, static_cast<int64_t>(blockIdx.x) * p.dim, lane + k * LANES, p.dim, dw[k]);
  }
}

// out[c] = the sum over the parts of partial[part][c], in a fixed order: a
// workgroup has 32 columns, a thread four of them of every 128th part, a wave's
// sums meet by exchanges, the waves' in LDS.  A cache line belongs to one
// workgroup: with four columns a workgroup each of the eight L2s fetched all of
// them (512 parts of 4,096 columns: 4.9 us, so 12.3; 1,024 of 256: 4.6 and 4.9).
constexpr int kJoinThreads = 1024, kJoinColumns = 32;

__global__ __launch_bounds__(kJoinThreads) void k_join_parts(const float* partial, int parts, int dim, float* out) {
  constexpr int WAVES = kJoinThreads / 64, ACROSS = kJoinColumns / 4;
  __shared__ float lds[WAVES][kJoinColumns];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, a = lane % ACROSS;
  const int c = blockIdx.x * kJoinColumns + 4 * a, left = dim - c < 4 ? dim - c : 4;
  float t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int q = threadIdx.x / ACROSS; q < parts; q += kJoinThreads / ACROSS) {
    const float* from = partial + static_cast<int64_t>(q) * dim + c;
    float v[4];
    if (left == 4) {
      mx_get<16>(v, from);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = i < left ? from[i] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] += v[i];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int o = ACROSS; o < 64; o <<= 1) t[i] += __shfl_xor(t[i], o, 64);
    if (lane < ACROSS) lds[wave][4 * a + i] = t[i];
  }
  __syncthreads();
  const int i = threadIdx.x, at = blockIdx.x * kJoinColumns + i;
  if (i < kJoinColumns && at < dim) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += lds[w][i];
    out[at] = s;
  }
}

// ---- the gradients of the layers below a dropout --------------------------

__global__ __launch_bounds__(256) void k_scale(ScaleArgs a) {
  const int t = blockIdx.y;
  const int64_t n = a.n[t];
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n;
       i += static_cast<int64_t>(gridDim.x) * 256)
    a.w[t][i] *= a.by[t];
}

__global__ __launch_bounds__(256) void k_given_gradient(const float* from, int64_t rows, int cols, float* dz, int ldz,
                                                        int32_t* clear, int64_t clear_n) {
  const int64_t first = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int64_t step = static_cast<int64_t>(gridDim.x) * 256;
  for (int64_t i = first; i < rows * ldz; i += step) {
    const int64_t row = i / ldz;
    const int c = static_cast<int>(i - row * ldz);
    dz[i] = c < cols ? from[row * cols + c] : 0.f;
  }
  for (int64_t i = first; i < clear_n; i += step) clear[i] = 0;
}

// ---- dispatch -------------------------------------------------------------

// Workgroups: as many as the rows need, at most `most`.
unsigned grid_for(int64_t n, int rows, int64_t most) {
  const int64_t need = (n + rows - 1) / rows;
  return static_cast<unsigned>(need < most ? need : most);
}

constexpr int64_t kRowGrid = 16 * kComputeUnits;

template <typename T>
void dropout_as(const DropoutArgs& a, hipStream_t s) {
  const int pieces = (a.dim + kPiece - 1) / kPiece;
  auto run = [&](auto lanes) {
    constexpr int LANES = decltype(lanes)::value;
    const auto kernel = a.dim % kPiece == 0 ? k_dropout<T, LANES, true> : k_dropout<T, LANES, false>;
    hipLaunchKernelGGL(kernel, dim3(grid_for(a.n_cap, 256 / LANES, kRowGrid)), dim3(256), 0, s, a);
  };
  if (pieces <= 4) run(std::integral_constant<int, 4>{});
  else if (pieces <= 16) run(std::integral_constant<int, 16>{});
  else if (pieces <= 32) run(std::integral_constant<int, 32>{});
  else if (pieces <= 64) run(std::integral_constant<int, 64>{});
  else run(std::integral_constant<int, 256>{});
}

// LANES threads and OC pieces a thread for rows of `dim` columns (at most
// 65,536): calls f with the shape.
template <int LANES, int OC, bool HELD = true>
struct NormShape {
  static constexpr int kLanes = LANES, kOc = OC;
  static constexpr bool kHeld = HELD;
};
template <typename F>
void norm_shape(int dim, F&& f) {
  const int pieces = (dim + kPiece - 1) / kPiece;
  if (pieces <= 4) f(NormShape<4, 1>{});
  else if (pieces <= 16) f(NormShape<16, 1>{});
  else if (pieces <= 32) f(NormShape<32, 1>{});
  else if (pieces <= 64) f(NormShape<64, 1>{});
  else if (pieces <= 128) f(NormShape<64, 2>{});
  else if (pieces <= 256) f(NormShape<256, 1>{});
  else if (pieces <= 512) f(NormShape<256, 2>{});
  else if (pieces <= 1024) f(NormShape<256, 4>{});
  else if (pieces <= 2048) f(NormShape<1024, 2>{});
  else if (pieces <= 4096) f(NormShape<1024, 4>{});
  else f(NormShape<1024, 8, false>{});
}

// The backward's shapes: a piece a thread, as long as a workgroup has them.
template <typename F>
void back_shape(int dim, F&& f) {
  const int pieces = (dim + kPiece - 1) / kPiece;
  if (pieces <= 4) f(NormShape<4, 1>{});
  else if (pieces <= 16) f(NormShape<16, 1>{});
  else if (pieces <= 32) f(NormShape<32, 1>{});
  else if (pieces <= 64) f(NormShape<64, 1>{});
  else if (pieces <= 128) f(NormShape<128, 1>{});
  else if (pieces <= 256) f(NormShape<256, 1>{});
  else if (pieces <= 512) f(NormShape<512, 1>{});
  else if (pieces <= 1024) f(NormShape<1024, 1>{});
  else if (pieces <= 2048) f(NormShape<1024, 2, false>{});
  else if (pieces <= 4096) f(NormShape<1024, 4, false>{});
  else f(NormShape<1024, 8, false>{});
}

// Its workgroups: as many as are resident (four waves a SIMD), so that they end
// together (8,192 x 4,096 bf16, three for a CU resident: 78 us, four 104).
constexpr int64_t kNormBackThreads = 1024 * kComputeUnits;

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, int bf16, hipStream_t s) {
  bf16 ? dropout_as<uint16_t>(a, s) : dropout_as<float>(a, s);
  return hipGetLastError();
}

hipError_t launch_rms_norm(const NormArgs& a, int bf16, int bits, hipStream_t s) {
  norm_shape(a.dim, [&](auto shape) {
    using S = decltype(shape);
    using B = NormBlock<S::kLanes>;
    const dim3 grid(grid_for(a.n_cap, B::kRows, kRowGrid)), block(B::kThreads);
    auto run = [&](auto t, auto whole) {
      using T = decltype(t);
      constexpr bool WHOLE = decltype(whole)::value;
      const auto kernel = bits == 0   ? k_rms_norm<T, S::kLanes, S::kOc, S::kHeld, 0, WHOLE>
                          : bits == 4 ? k_rms_norm<T, S::kLanes, S::kOc, S::kHeld, 4, WHOLE>
                                      : k_rms_norm<T, S::kLanes, S::kOc, S::kHeld, 8, WHOLE>;
      hipLaunchKernelGGL(kernel, grid, block, 0, s, a);
    };
    if (a.dim % kPiece == 0) bf16 ? run(uint16_t{}, std::true_type{}) : run(float{}, std::true_type{});
    else bf16 ? run(uint16_t{}, std::false_type{}) : run(float{}, std::false_type{});
  });
  return hipGetLastError();
}

int norm_back_parts(int64_t n_cap, int dim) {
  int parts = 1;
  back_shape(dim, [&](auto shape) {
    using B = NormBlock<decltype(shape)::kLanes>;
    parts = static_cast<int>(grid_for(n_cap, B::kRows, kNormBackThreads / B::kThreads));
  });
  return parts;
}

hipError_t launch_rms_norm_backward(const NormBackArgs& a, int bf16, hipStream_t s) {
  NormBackArgs p = a;
  if (!p.d_weight) p.partial = nullptr;
  const int parts = norm_back_parts(p.n_cap, p.dim);
  back_shape(p.dim, [&](auto shape) {
    using S = decltype(shape);
    using B = NormBlock<S::kLanes>;
    auto run = [&](auto t) {
      using T = decltype(t);
      const auto kernel = p.dim % kPiece == 0 ? k_rms_norm_back<T, S::kLanes, S::kOc, S::kHeld, true>
                                              : k_rms_norm_back<T, S::kLanes, S::kOc, S::kHeld, false>;
      hipLaunchKernelGGL(kernel, dim3(parts), dim3(B::kThreads), 0, s, p);
    };
    bf16 ? run(uint16_t{}) : run(float{});
  });
  if (p.d_weight)
    hipLaunchKernelGGL(k_join_parts, dim3(static_cast<unsigned>((p.dim + kJoinColumns - 1) / kJoinColumns)),
                       dim3(kJoinThreads), 0, s, p.partial, parts, p.dim, p.d_weight);
  return hipGetLastError();
}

hipError_t launch_given_gradient(const float* from, int64_t rows, int cols, float* dz, int ldz, int32_t* clear,
                                 int64_t clear_n, hipStream_t s) {
  const int64_t work = rows * ldz > clear_n ? rows * ldz : clear_n;
  hipLaunchKernelGGL(k_given_gradient, dim3(grid_for(work, 1024, 4 * kComputeUnits)), dim3(256), 0, s, from, rows,
                     cols, dz, ldz, clear, clear_n);
  return hipGetLastError();
}

hipError_t launch_scale(const ScaleArgs& a, hipStream_t s) {
  int64_t most = 0;
  for (int t = 0; t < a.count; ++t) most = a.n[t] > most ? a.n[t] : most;
  if (a.count == 0 || most == 0) return hipSuccess;
  hipLaunchKernelGGL(k_scale, dim3(grid_for(most, 1024, kComputeUnits), static_cast<unsigned>(a.count)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace gmb
