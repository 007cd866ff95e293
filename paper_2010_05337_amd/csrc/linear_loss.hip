// Softmax cross-entropy of a linear head over many classes, and its gradients,
// without the logits: z = x W^T + b, L = (1 / n) sum_i (lse_i - z_i,y(i)),
// G = softmax(z) - onehot(y), dx = G W / n, dW = G^T x / n, db = G^T 1 / n.
//
//   k_amax, k_lay_out   x, and W where it cannot be read as it lies, as 16-bit
//                       rows padded with zeros; rows without a label as zeros
//   k_logits (stats)    a tile of logits in registers: every row's maximum and
//                       sum of exponentials over the tile's classes, its label's
//                       logit
//   k_join_rows         the tiles of a row: lse, the loss term
//   k_logits (grad)     the logits again, a piece of the classes at a time: G
//   k_products          dx += G W and dW = G^T x of the piece
//   k_join              sums that were split
//
// The logits are computed twice (8 n C d operations in all where keeping them
// would take 6) and never stored; G is, in 16 bits (kSplit: two times 16), for
// a piece of the classes.  Nothing is added by atomics: the same bits every time.
#include "head_kernels.hpp"
#include "mx.hpp"
#include "mx_kernels.hpp"
#include "tiles16.hpp"

namespace gmb {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kPadRows = 256, kPadCols = 64;
constexpr float kGradScale = 16384.f;   // kSplit: |G| <= 1 in the top of fp16's range

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// ---- 16-bit rows ----------------------------------------------------------

// The power of two that brings the largest magnitude (fp32 bits) into [2^14,
// 2^15), as far as it and its inverse are normal numbers.
__device__ __forceinline__ float split_scale(uint32_t top) {
  const int f = 268 - static_cast<int>(top >> 23);
  return __uint_as_float(static_cast<uint32_t>(f > 253 ? 253 : f) << 23);
}
__device__ __forceinline__ float inverse_of_power(float s) { return __uint_as_float((254u << 23) - __float_as_uint(s)); }

// The fp32 bits of a finite magnitude, 0 for others.
__device__ __forceinline__ uint32_t finite_bits(float v) {
  const uint32_t u = __float_as_uint(v) & 0x7FFFFFFFu;
  return u < 0x7F800000u ? u : 0u;
}

__device__ __forceinline__ bool has_label(const int32_t* labels, int64_t row, int classes) {
  const int32_t y = labels[row];
  return y >= 0 && y < classes;
}

struct AmaxArgs {
  const float* x;
  int64_t x_stride, rows;
  const int32_t* labels;
  int d, classes;
  uint32_t* row_top;               // [rows]
  uint32_t* x_top;                 // [x_blocks]
  const float* w;                  // w_rows rows of w_cols values, w_col apart
  int64_t w_stride, w_col, w_rows;
  int w_cols;
  uint32_t* w_top;                 // [w_blocks]
  int x_blocks, w_blocks;
};

// The largest finite magnitudes: of every row of x and of all of them (a word a
// workgroup), and of W (a word a workgroup).
__global__ __launch_bounds__(256) void k_amax(AmaxArgs p) {
  __shared__ uint32_t lds[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool of_x = static_cast<int>(blockIdx.x) < p.x_blocks;
  const int block = of_x ? blockIdx.x : blockIdx.x - p.x_blocks, blocks = of_x ? p.x_blocks : p.w_blocks;
  const float* data = of_x ? p.x : p.w;
  const int64_t rows = of_x ? p.rows : p.w_rows, stride = of_x ? p.x_stride : p.w_stride;
  const int64_t col = of_x ? 1 : p.w_col;
  const int cols = of_x ? p.d : p.w_cols;
  uint32_t all = 0;
  for (int64_t row = static_cast<int64_t>(block) * 4 + wave; row < rows; row += static_cast<int64_t>(blocks) * 4) {
    uint32_t top = 0;
    if (!of_x || has_label(p.labels, row, p.classes)) {
      for (int c = lane; c < cols; c += 64) {
        const uint32_t u = finite_bits(data[row * stride + c * col]);
        top = u > top ? u : top;
      }
    }
    if (of_x) {
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t u = __shfl_xor(top, o, 64);
        top = u > top ? u : top;
      }
      if (lane == 0) p.row_top[row] = top;
    }
    all = top > all ? top : all;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t u = __shfl_xor(all, o, 64);
    all = u > all ? u : all;
  }
  if (lane == 0) lds[wave] = all;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 4; ++w) all = lds[w] > all ? lds[w] : all;
    (of_x ? p.x_top : p.w_top)[block] = all;
  }
}

struct LayOutArgs {
  const void* src;                 // element (i, j) at i row + j col
  int64_t row, col;
  int64_t rows, out_rows;          // out_rows: with the rows of zeros behind
  int cols, out_cols;              // out_cols: a multiple of kPadCols
  int classes;
  const int32_t* labels;           // or NULL: rows without a label become zeros
  int32_t* kept_labels;            // with labels: [out_rows], -1 for none
  uint16_t* by_all;                // scaled alike (bf16: not scaled)
  uint16_t* by_row;                // kSplit: each row by its own scale, or NULL
  const uint32_t* row_top;
  const uint32_t* tops;            // kSplit: the largest magnitudes, `top_count` of them
  int top_count;
  float* row_inverse;              // with by_row: [out_rows]
  float* all_inverse;              // kSplit: one word
};

// Eight values as they are stored from column c of a row on.
template <T16Type TYPE>
__device__ __forceinline__ void put_split(uint16_t* row, int c, const float (&v)[8], float scale) {
  if constexpr (TYPE == kBf16) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = mx_bf16x2_bits(v[2 * i], v[2 * i + 1]);
    mx_put<16, false>(row + c, w);
  } else {
    uint16_t hi[8], lo[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = v[i] * scale;
      const _Float16 h = static_cast<_Float16>(x);
      const _Float16 l = static_cast<_Float16>(x - static_cast<float>(h));
      hi[i] = __builtin_bit_cast(uint16_t, h);
      lo[i] = __builtin_bit_cast(uint16_t, l);
    }
    uint16_t* at = row + (c / 32) * 64 + c % 32;
    mx_put<16, false>(at, hi);
    mx_put<16, false>(at + 32, lo);
  }
}

// A 64 x 64 tile of the source through LDS, read along whichever of its
// directions is contiguous, written as rows.
template <T16Type TYPE, typename T>
__global__ __launch_bounds__(256) void k_lay_out(LayOutArgs p) {
  __shared__ float tile[64][65];
  __shared__ uint32_t top_of[4];
  const int64_t r0 = static_cast<int64_t>(blockIdx.x) * 64;
  const int c0 = blockIdx.y * 64;
  const T* src = static_cast<const T*>(p.src);
  const int fast = threadIdx.x & 63, slow = threadIdx.x >> 6;
  const bool along_rows = p.col == 1 || p.row != 1;   // neighbouring threads: neighbouring columns
#pragma unroll 4
  for (int k = 0; k < 16; ++k) {
    const int i = along_rows ? 4 * k + slow : fast, j = along_rows ? fast : 4 * k + slow;
    float v = 0.f;
    if (r0 + i < p.rows && c0 + j < p.cols && (!p.labels || has_label(p.labels, r0 + i, p.classes))) {
      const T x = src[(r0 + i) * p.row + (c0 + j) * p.col];
      if constexpr (sizeof(T) == 4) v = x;
      else v = bf16_to_f32(x);
    }
    tile[i][j] = v;
  }
  float scale = 1.f;
  if constexpr (TYPE == kSplit) {
    uint32_t top = 0;
    for (int i = threadIdx.x; i < p.top_count; i += 256) top = p.tops[i] > top ? p.tops[i] : top;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t u = __shfl_xor(top, o, 64);
      top = u > top ? u : top;
    }
    if ((threadIdx.x & 63) == 0) top_of[threadIdx.x >> 6] = top;
    __syncthreads();
    for (int w = 0; w < 4; ++w) top = top_of[w] > top ? top_of[w] : top;
    scale = split_scale(top);
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.all_inverse = inverse_of_power(scale);
  } else {
    __syncthreads();
  }
  const int64_t ld = TYPE == kSplit ? 2 * static_cast<int64_t>(p.out_cols) : p.out_cols;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int i = 32 * k + (threadIdx.x >> 3), j = (threadIdx.x & 7) * 8;
    const int64_t row = r0 + i;
    if (row >= p.out_rows) continue;
    float v[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = tile[i][j + q];
    put_split<TYPE>(p.by_all + row * ld, c0 + j, v, scale);
    const bool first = blockIdx.y == 0 && j == 0;
    if (TYPE == kSplit && p.by_row) {
      const float s = split_scale(row < p.rows ? p.row_top[row] : 0u);
      put_split<TYPE>(p.by_row + row * ld, c0 + j, v, s);
      if (first) p.row_inverse[row] = inverse_of_power(s);
    }
    if (first && p.labels)
      p.kept_labels[row] = row < p.rows && has_label(p.labels, row, p.classes) ? p.labels[row] : -1;
  }
}

// ---- logits ---------------------------------------------------------------

struct LogitsArgs {
  T16Side w, x;                    // W's rows: A, those of x: B (`first` is set by the kernel)
  int64_t stages;
  int m_tiles, n_tiles;            // classes, rows
  int c0;                          // the first class
  int classes;
  const float* bias;               // or NULL
  const float* row_inverse;        // kSplit
  const float* w_inverse;          // kSplit: one word
  const int32_t* labels;           // [padded rows], -1 for none
  int64_t pad_rows;
  float2* stats;                   // [m_tiles][pad_rows]: maximum, sum of exponentials
  float* label_logit;              // [pad_rows]
  const float2* rows;              // [pad_rows]: maximum, 1 / sum
  uint16_t* g;                     // [pad_rows][ldg]
  int64_t ldg;
  float* db;                       // [n_tiles][ld_db] at the piece's first class, or NULL
  int64_t ld_db;
};

// Workgroup ids go round the eight XCDs: each takes a contiguous run of tiles.
__device__ __forceinline__ int64_t xcd_id(int64_t tiles) {
  const int64_t per = (tiles + 7) / 8, id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  return (blockIdx.x >> 3) < per && id < tiles ? id : -1;
}

// The sum of v over the sixteen lanes r of a group g: four turns of a row.
__device__ __forceinline__ float sum16(float v) {
  v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x128, 0xF, 0xF, true));
  v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x124, 0xF, 0xF, true));
  v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x122, 0xF, 0xF, true));
  v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x121, 0xF, 0xF, true));
  return v;
}

enum LogitsMode { kStats, kGrad };

template <T16Type TYPE, LogitsMode MODE, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void k_logits(LogitsArgs p) {
  using Tile = T16Tile<TYPE, kByRow, kByRow, TM, TN, WM, WN>;
  constexpr int RT = Tile::RT, CT = Tile::CT;
  __shared__ __attribute__((aligned(1024))) char lds[2 * Tile::kStage];
  const int64_t id = xcd_id(static_cast<int64_t>(p.m_tiles) * p.n_tiles);
  if (id < 0) return;
  // eight row tiles wide, so that an L2 holds what neighbours share
  const int band = static_cast<int>(id / (8 * static_cast<int64_t>(p.m_tiles)));
  const int64_t in_band = id - static_cast<int64_t>(band) * 8 * p.m_tiles;
  const int width = p.n_tiles - 8 * band < 8 ? p.n_tiles - 8 * band : 8;
  const int nt = 8 * band + static_cast<int>(in_band % width), mt = static_cast<int>(in_band / width);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, r = lane & 15;
  const int wm = wave / WN, wn = wave % WN;
  T16Side a = p.w, b = p.x;
  a.first = p.c0 + static_cast<int64_t>(mt) * TM;
  b.first = static_cast<int64_t>(nt) * TN;
  t16_f32x4 acc[RT][CT];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int j = 0; j < CT; ++j) acc[i][j] = t16_f32x4{0.f, 0.f, 0.f, 0.f};
  Tile::run(a, b, 0, p.stages, lds, acc);

  // logits: class c0 + c(i) + e, row row(j)
  const int cw = mt * TM + 16 * RT * wm + 4 * g;      // of the piece
  const int64_t row0 = static_cast<int64_t>(nt) * TN + 16 * CT * wn + r;
  float by[CT];
#pragma unroll
  for (int j = 0; j < CT; ++j) by[j] = TYPE == kSplit ? p.row_inverse[row0 + 16 * j] * *p.w_inverse : 1.f;
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = p.c0 + cw + 16 * i + e;
      const bool in = c < p.classes;
      const float bias = in && p.bias ? p.bias[c] : 0.f;
#pragma unroll
      for (int j = 0; j < CT; ++j)
        acc[i][j][e] = in ? (TYPE == kSplit ? fmaf(acc[i][j][e], by[j], bias) : acc[i][j][e] + bias) : -INFINITY;
    }
  if constexpr (MODE == kStats) {
    float* top_of = reinterpret_cast<float*>(lds);               // [WM][TN]
    float* sum_of = top_of + WM * TN;
#pragma unroll
    for (int j = 0; j < CT; ++j) {
      float top = -INFINITY;
      const int y = p.labels[row0 + 16 * j] - p.c0 - cw;
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float z = acc[i][j][e];
          top = z > top || z != z ? z : top;
          if (y == 16 * i + e) p.label_logit[row0 + 16 * j] = z;
        }
      // (a NaN stays one: the row's loss is NaN then)
      for (int o = 16; o < 64; o <<= 1) {
        const float t = __shfl_xor(top, o, 64);
        top = t > top || t != t ? t : top;
      }
      float sum = 0.f;
      const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += exp2_fast((acc[i][j][e] - base) * kLog2e);
      for (int o = 16; o < 64; o <<= 1) sum += __shfl_xor(sum, o, 64);
      if (g == 0) {
        top_of[wm * TN + 16 * (CT * wn + j) + r] = top;
        sum_of[wm * TN + 16 * (CT * wn + j) + r] = sum;
      }
    }
    __syncthreads();
    for (int q = threadIdx.x; q < TN; q += 64 * WM * WN) {
      float top = top_of[q];
#pragma unroll
      for (int w = 1; w < WM; ++w) {
        const float t = top_of[w * TN + q];
        top = t > top || t != t ? t : top;
      }
      const float base = top == -INFINITY ? 0.f : top;
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < WM; ++w) sum += sum_of[w * TN + q] * exp2_fast((top_of[w * TN + q] - base) * kLog2e);
      p.stats[static_cast<int64_t>(mt) * p.pad_rows + static_cast<int64_t>(nt) * TN + q] = make_float2(top, sum);
    }
  } else {
    float db[RT][4];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) db[i][e] = 0.f;
#pragma unroll
    for (int j = 0; j < CT; ++j) {
      const int64_t row = row0 + 16 * j;
      const int32_t y = p.labels[row];
      const float2 of = p.rows[row];
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int c = p.c0 + cw + 16 * i + e;
          const float q = exp2_fast((acc[i][j][e] - of.x) * kLog2e) * of.y;
          v[e] = y < 0 ? 0.f : (c == y ? q - 1.f : q);
          db[i][e] += v[e];
        }
        const int64_t at = row * p.ldg;
        const int col = cw + 16 * i;
        if constexpr (TYPE == kBf16) {
          const uint32_t w[2] = {mx_bf16x2_bits(v[0], v[1]), mx_bf16x2_bits(v[2], v[3])};
          mx_put<8, false>(p.g + at + col, w);
        } else {
          uint16_t hi[4], lo[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = v[e] * kGradScale;
            const _Float16 h = static_cast<_Float16>(x);
            const _Float16 l = static_cast<_Float16>(x - static_cast<float>(h));
            hi[e] = __builtin_bit_cast(uint16_t, h);
            lo[e] = __builtin_bit_cast(uint16_t, l);
          }
          uint16_t* to = p.g + at + (col / 32) * 64 + col % 32;
          mx_put<8, false>(to, hi);
          mx_put<8, false>(to + 32, lo);
        }
      }
    }
    if (p.db) {
      float* part = reinterpret_cast<float*>(lds);               // [WN][TM]
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float t = sum16(db[i][e]);
          if (r == 0) part[wn * TM + 16 * (RT * wm + i) + 4 * g + e] = t;
        }
      __syncthreads();
      for (int q = threadIdx.x; q < TM; q += 64 * WM * WN) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < WN; ++w) t += part[w * TM + q];
        if (p.c0 + mt * TM + q < p.classes) p.db[static_cast<int64_t>(nt) * p.ld_db + mt * TM + q] = t;
      }
    }
  }
}

// ---- the rows' statistics -------------------------------------------------

struct JoinRowsArgs {
  const float2* stats;             // [tiles][pad_rows]
  int tiles;
  int64_t rows, pad_rows;
  int32_t* labels;                 // a row whose logits are all -inf loses its label
  const float* label_logit;
  float2* out;                     // [pad_rows]
  float* loss_rows;                // [rows]
};

// 32 rows a workgroup, the tiles of a row dealt to eight threads.
__global__ __launch_bounds__(256) void k_join_rows(JoinRowsArgs p) {
  __shared__ float2 lds[8][32];
  const int q = threadIdx.x & 31, part = threadIdx.x >> 5;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * 32 + q;
  float top = -INFINITY, sum = 0.f;
  auto add = [&](float2 s) {
    const float m = s.x > top || s.x != s.x ? s.x : top;
    const float base = m == -INFINITY ? 0.f : m;
    sum = sum * exp2_fast((top - base) * kLog2e) + s.y * exp2_fast((s.x - base) * kLog2e);
    top = m;
  };
  for (int t = part; t < p.tiles; t += 8) add(p.stats[static_cast<int64_t>(t) * p.pad_rows + row]);
  lds[part][q] = make_float2(top, sum);
  __syncthreads();
  if (part) return;
  for (int w = 1; w < 8; ++w) add(lds[w][q]);
  const bool on = p.labels[row] >= 0 && top != -INFINITY;
  if (!on) p.labels[row] = -1;
  p.out[row] = make_float2(top, 1.f / sum);
  if (row < p.rows) p.loss_rows[row] = on ? (top - p.label_logit[row]) + logf(sum) : 0.f;
}

// ---- products -------------------------------------------------------------

struct Product {
  T16Side a, b;                    // `first` is set by the kernel
  int64_t m, n;                    // out: n rows of m contiguous values
  int m_tiles, n_tiles, splits;
  int64_t stages;                  // of k
  void* out;                       // the result, or NULL: sums go to `slab`
  int64_t ld;
  float factor;                    // result = sum factor inverse
  const float* inverse;            // or NULL
  float* slab;                     // [splits][n][ld_slab]
  int64_t ld_slab;
  int more;                        // add to what the slab holds
};

// Four contiguous values of a row, `left` of them.
template <bool BF16>
__device__ __forceinline__ void put_four(void* out, int64_t at, t16_f32x4 v, int64_t left) {
  if constexpr (BF16) {
    uint16_t* o = static_cast<uint16_t*>(out) + at;
    const uint32_t w[2] = {mx_bf16x2_bits(v[0], v[1]), mx_bf16x2_bits(v[2], v[3])};
    if (left >= 4) {
      mx_put<8, false>(o, w);
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (e < left) o[e] = static_cast<uint16_t>(w[e / 2] >> (16 * (e & 1)));
    }
  } else {
    float* o = static_cast<float*>(out) + at;
    if (left >= 4) {
      mx_put<16, false>(o, &v);
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (e < left) o[e] = v[e];
    }
  }
}

template <T16Type TYPE, T16Form FA, T16Form FB, int TM, int TN, int WM, int WN>
__device__ __forceinline__ void product_tile(const Product& p, int64_t id, char* lds) {
  using Tile = T16Tile<TYPE, FA, FB, TM, TN, WM, WN>;
  constexpr int RT = Tile::RT, CT = Tile::CT;
  const int mt = static_cast<int>(id % p.m_tiles);
  const int64_t rest = id / p.m_tiles;
  const int nt = static_cast<int>(rest % p.n_tiles), split = static_cast<int>(rest / p.n_tiles);
  T16Side a = p.a, b = p.b;
  a.first = static_cast<int64_t>(mt) * TM;
  b.first = static_cast<int64_t>(nt) * TN;
  t16_f32x4 acc[RT][CT];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int j = 0; j < CT; ++j) acc[i][j] = t16_f32x4{0.f, 0.f, 0.f, 0.f};
  Tile::run(a, b, p.stages * split / p.splits, p.stages * (split + 1) / p.splits, lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, r = lane & 15;
  const int wm = wave / WN, wn = wave % WN;
  const int64_t m0 = a.first + 16 * RT * wm + 4 * g, n0 = b.first + 16 * CT * wn + r;
  const float inverse = p.inverse ? *p.inverse : 1.f;
#pragma unroll
  for (int j = 0; j < CT; ++j) {
    const int64_t row = n0 + 16 * j;
    if (row >= p.n) continue;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int64_t col = m0 + 16 * i;
      if (col >= p.m) continue;
      t16_f32x4 v = acc[i][j];
      if (p.out) {
        v = v * p.factor * inverse;   // (their product alone may be no normal number)
        put_four<TYPE == kBf16>(p.out, row * p.ld + col, v, p.m - col);
      } else {
        float* to = p.slab + (split * p.n + row) * p.ld_slab + col;
        t16_f32x4 had = {0.f, 0.f, 0.f, 0.f};
        if (p.more) mx_get<16>(&had, to);
        v += had;
        mx_put<16, false>(to, &v);
      }
    }
  }
}

// dx = G W (A: W by its rows of k, B: G by its rows), then dW = G^T x, its rows
// those of W (A: x, B: G) or, turned, those of W's transpose (A: G, B: x).
template <T16Type TYPE, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void k_products(Product dx, Product dw) {
  __shared__ __attribute__((aligned(1024))) char lds[2 * t16_stage_bytes<TM, TN>()];
  const int64_t of_dx = static_cast<int64_t>(dx.m_tiles) * dx.n_tiles * dx.splits;
  const int64_t of_dw = static_cast<int64_t>(dw.m_tiles) * dw.n_tiles * dw.splits;
  const int64_t id = xcd_id(of_dx + of_dw);
  if (id < 0) return;
  if (id < of_dx) product_tile<TYPE, kByK, kByRow, TM, TN, WM, WN>(dx, id, lds);
  else product_tile<TYPE, kByK, kByK, TM, TN, WM, WN>(dw, id - of_dx, lds);
}

struct JoinArgs {
  const float* slab;               // [parts][rows][ld_slab]
  int parts;
  int64_t rows, cols, ld_slab;
  float factor;
  const float* inverse;
  void* out;
  int64_t ld;
};

// out = factor inverse times the sum of the parts, in a fixed order.
template <bool BF16>
__global__ __launch_bounds__(256) void k_join(JoinArgs p) {
  const int64_t fours = (p.cols + 3) / 4, all = p.rows * fours;
  const float inverse = p.inverse ? *p.inverse : 1.f;
  for (int64_t q = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; q < all;
       q += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t row = q / fours, col = (q - row * fours) * 4;
    t16_f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < p.parts; ++s) {
      t16_f32x4 x;
      mx_get<16>(&x, p.slab + (s * p.rows + row) * p.ld_slab + col);
      v += x;
    }
    v = v * p.factor * inverse;
    put_four<BF16>(p.out, row * p.ld + col, v, p.cols - col);
  }
}

// ---- plan -----------------------------------------------------------------

constexpr int kTile = 128;
// G of a piece of the classes.
constexpr int64_t kGradBytes = int64_t{256} << 20;
constexpr int kMostTops = 1024;

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

struct Plan {
  int es;                          // 16-bit words of a value
  int64_t pad_rows, pad_d;
  bool copy_w;
  int64_t piece, pieces;           // classes of a piece (a multiple of kPadRows)
  int m_tiles, n_tiles;            // classes (of all), rows
  int dx_splits, dw_splits;
  bool dx_slab;
  int64_t ld_dw;                   // the contiguous extent of dw, padded to four
  // offsets
  size_t x_all, x_row, w, row_top, tops, row_inverse, inverses, labels, stats, label_logit, rows, loss_rows, g, db, dx_sums, dw_sums, total;
};

Plan plan(const LinearLossArgs& a, int bf16) {
  Plan p{};
  p.es = bf16 ? 1 : 2;
  p.pad_rows = round_up(a.rows, kPadRows);
  p.pad_d = round_up(a.d, kPadCols);
  // bf16 weights are read as they lie if their rows are whole stages
  p.copy_w = !(bf16 && a.w_col == 1 && a.d % kPadCols == 0 && a.w_row % 8 == 0 &&
               reinterpret_cast<uintptr_t>(a.w) % 16 == 0);
  const int64_t pad_classes = round_up(a.classes, kPadRows);
  const bool grad = a.dx || a.dw || a.db;
  int64_t piece = kGradBytes / (p.pad_rows * 2 * p.es) / kPadRows * kPadRows;
  piece = piece < kPadRows ? kPadRows : (piece > pad_classes ? pad_classes : piece);
  p.pieces = (pad_classes + piece - 1) / piece;
  p.piece = round_up((pad_classes + p.pieces - 1) / p.pieces, kPadRows);
  p.pieces = (pad_classes + p.piece - 1) / p.piece;
  p.m_tiles = static_cast<int>((a.classes + kTile - 1) / kTile);
  p.n_tiles = static_cast<int>(p.pad_rows / kTile);
  auto splits = [&](int64_t tiles, int64_t stages) {
    int64_t s = (2 * kComputeUnits + tiles - 1) / tiles;
    const int64_t most = stages / 4;
    s = s > most ? most : s;
    return static_cast<int>(s < 1 ? 1 : s);
  };
  const int64_t d_tiles = (a.d + kTile - 1) / kTile, k = 64 / p.es;
  p.dx_splits = splits(d_tiles * ((a.rows + kTile - 1) / kTile), p.piece / k);
  p.dx_slab = p.dx_splits > 1 || p.pieces > 1;
  p.dw_splits = splits(d_tiles * (p.piece / kTile), p.pad_rows / k);
  p.ld_dw = round_up(a.turned ? a.classes : a.d, 4);
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t here = at;
    at += static_cast<size_t>(round_up(bytes, 256));
    return here;
  };
  const int64_t x_bytes = p.pad_rows * p.pad_d * 2 * p.es;
  p.x_all = take(x_bytes);
  p.x_row = bf16 ? p.x_all : take(x_bytes);
  p.w = p.copy_w ? take(static_cast<int64_t>(a.classes) * p.pad_d * 2 * p.es) : 0;
  p.row_top = bf16 ? 0 : take(p.pad_rows * 4);
  p.tops = bf16 ? 0 : take(2 * kMostTops * 4);
  p.row_inverse = bf16 ? 0 : take(p.pad_rows * 4);
  p.inverses = bf16 ? 0 : take(8);
  p.labels = take(p.pad_rows * 4);
  p.stats = take(p.m_tiles * p.pad_rows * 8);
  p.label_logit = take(p.pad_rows * 4);
  p.rows = take(p.pad_rows * 8);
  p.loss_rows = take(p.pad_rows * 4);
  if (grad) {
    p.g = take(p.pad_rows * p.piece * 2 * p.es);
    p.db = a.db ? take(static_cast<int64_t>(p.n_tiles) * pad_classes * 4) : 0;
    p.dx_sums = a.dx && p.dx_slab ? take(p.dx_splits * a.rows * round_up(a.d, 4) * 4) : 0;
    p.dw_sums = a.dw && p.dw_splits > 1 ? take(p.dw_splits * (a.turned ? a.d * p.ld_dw : p.piece * p.ld_dw) * 4) : 0;
  }
  p.total = at;
  return p;
}

unsigned grid8(int64_t tiles) { return static_cast<unsigned>((tiles + 7) / 8 * 8); }

template <T16Type TYPE, typename T>
hipError_t run(const LinearLossArgs& a, hipStream_t s) {
  constexpr bool kLo = TYPE == kBf16;
  const Plan p = plan(a, kLo);
  char* ws = a.ws;
  auto at = [&](size_t off) { return ws + off; };
  uint16_t* x_all = reinterpret_cast<uint16_t*>(at(p.x_all));
  uint16_t* x_row = reinterpret_cast<uint16_t*>(at(p.x_row));
  int32_t* labels = reinterpret_cast<int32_t*>(at(p.labels));
  float* inverses = kLo ? nullptr : reinterpret_cast<float*>(at(p.inverses));
  uint32_t* tops = kLo ? nullptr : reinterpret_cast<uint32_t*>(at(p.tops));
  const bool w_rows = a.w_col == 1 || a.w_row != 1;    // W's rows are contiguous (or nothing is)
  int x_blocks = 0, w_blocks = 0;
  if constexpr (!kLo) {
    AmaxArgs m{};
    m.x = static_cast<const float*>(a.x);
    m.x_stride = a.x_stride;
    m.rows = a.rows;
    m.labels = a.labels;
    m.d = a.d;
    m.classes = a.classes;
    m.row_top = reinterpret_cast<uint32_t*>(at(p.row_top));
    m.x_top = tops;
    m.w = static_cast<const float*>(a.w);
    m.w_stride = w_rows ? a.w_row : a.w_col;
    m.w_col = w_rows ? a.w_col : a.w_row;
    m.w_rows = w_rows ? a.classes : a.d;
    m.w_cols = w_rows ? a.d : a.classes;
    m.w_top = tops + kMostTops;
    auto blocks = [](int64_t rows) { return static_cast<int>(rows < 4 * kMostTops ? (rows + 3) / 4 : kMostTops); };
    m.x_blocks = x_blocks = blocks(a.rows);
    m.w_blocks = w_blocks = blocks(m.w_rows);
    hipLaunchKernelGGL(k_amax, dim3(static_cast<unsigned>(x_blocks + w_blocks)), dim3(256), 0, s, m);
  }
  auto lay_out = [&](const LayOutArgs& l) {
    const dim3 grid(static_cast<unsigned>((l.out_rows + 63) / 64), static_cast<unsigned>(l.out_cols / 64));
    hipLaunchKernelGGL((k_lay_out<TYPE, T>), grid, dim3(256), 0, s, l);
  };
  LayOutArgs l{};
  l.src = a.x;
  l.row = a.x_stride;
  l.col = 1;
  l.rows = a.rows;
  l.out_rows = p.pad_rows;
  l.cols = a.d;
  l.out_cols = static_cast<int>(p.pad_d);
  l.classes = a.classes;
  l.labels = a.labels;
  l.kept_labels = labels;
  l.by_all = x_all;
  if constexpr (!kLo) {
    l.by_row = x_row;
    l.row_top = reinterpret_cast<const uint32_t*>(at(p.row_top));
    l.tops = tops;
    l.top_count = x_blocks;
    l.row_inverse = reinterpret_cast<float*>(at(p.row_inverse));
    l.all_inverse = inverses;
  }
  lay_out(l);
  T16Side w{static_cast<const uint16_t*>(a.w), a.w_row, a.classes, static_cast<int>(p.pad_d), 0};
  if (p.copy_w) {
    LayOutArgs lw{};
    lw.src = a.w;
    lw.row = a.w_row;
    lw.col = a.w_col;
    lw.rows = lw.out_rows = a.classes;
    lw.cols = a.d;
    lw.out_cols = static_cast<int>(p.pad_d);
    lw.by_all = reinterpret_cast<uint16_t*>(at(p.w));
    if constexpr (!kLo) {
      lw.tops = tops + kMostTops;
      lw.top_count = w_blocks;
      lw.all_inverse = inverses + 1;
    }
    lay_out(lw);
    w.data = lw.by_all;
    w.ld = p.pad_d * p.es;
  }
  const T16Side x_by_row{x_row, p.pad_d * p.es, p.pad_rows, static_cast<int>(p.pad_d), 0};
  const T16Side x_by_all{x_all, p.pad_d * p.es, p.pad_rows, static_cast<int>(p.pad_d), 0};
  const int64_t k = 64 / p.es;                          // of a stage
  LogitsArgs g{};
  g.w = w;
  g.x = x_by_row;
  g.stages = p.pad_d / k;
  g.m_tiles = p.m_tiles;
  g.n_tiles = p.n_tiles;
  g.classes = a.classes;
  g.bias = a.bias;
  g.row_inverse = kLo ? nullptr : reinterpret_cast<const float*>(at(p.row_inverse));
  g.w_inverse = kLo ? nullptr : inverses + 1;
  g.labels = labels;
  g.pad_rows = p.pad_rows;
  g.stats = reinterpret_cast<float2*>(at(p.stats));
  g.label_logit = reinterpret_cast<float*>(at(p.label_logit));
  g.rows = reinterpret_cast<const float2*>(at(p.rows));
  // (a launch's threads fit 31 bits)
  const int most = static_cast<int>((kLaunchThreads / 1024) / g.n_tiles);
  for (int t = 0; t < p.m_tiles; t += most) {
    g.c0 = t * kTile;
    g.m_tiles = p.m_tiles - t < most ? p.m_tiles - t : most;
    g.stats = reinterpret_cast<float2*>(at(p.stats)) + t * p.pad_rows;
    hipLaunchKernelGGL((k_logits<TYPE, kStats, kTile, kTile, 2, 2>),
                       dim3(grid8(static_cast<int64_t>(g.m_tiles) * g.n_tiles)), dim3(256), 0, s, g);
  }
  JoinRowsArgs j{};
  j.stats = reinterpret_cast<const float2*>(at(p.stats));
  j.tiles = p.m_tiles;
  j.rows = a.rows;
  j.pad_rows = p.pad_rows;
  j.labels = labels;
  j.label_logit = g.label_logit;
  j.out = reinterpret_cast<float2*>(at(p.rows));
  j.loss_rows = reinterpret_cast<float*>(at(p.loss_rows));
  hipLaunchKernelGGL(k_join_rows, dim3(static_cast<unsigned>(p.pad_rows / 32)), dim3(256), 0, s, j);
  const hipError_t e = launch_loss_mean(j.loss_rows, a.rows, a.loss, s);
  if (e != hipSuccess || (!a.dx && !a.dw && !a.db)) return e;

  const float mean = static_cast<float>((kLo ? 1.0 : 1.0 / kGradScale) / static_cast<double>(a.rows));
  auto join = [&](const float* slab, int parts, int64_t rows, int64_t cols, int64_t ld_slab, float factor,
                  const float* inverse, void* out, int64_t ld, bool lo) {
    JoinArgs q{slab, parts, rows, cols, ld_slab, factor, inverse, out, ld};
    const int64_t need = (rows * ((cols + 3) / 4) + 255) / 256;
    const dim3 grid(static_cast<unsigned>(need < 8 * kComputeUnits ? need : 8 * kComputeUnits));
    if (lo) hipLaunchKernelGGL(k_join<true>, grid, dim3(256), 0, s, q);
    else hipLaunchKernelGGL(k_join<false>, grid, dim3(256), 0, s, q);
  };
  const int64_t pad_classes = round_up(a.classes, kPadRows), ld_dx = round_up(a.d, 4);
  g.g = reinterpret_cast<uint16_t*>(at(p.g));
  g.ldg = p.piece * p.es;
  g.ld_db = pad_classes;
  const int d_tiles = (a.d + kTile - 1) / kTile;
  for (int64_t c0 = 0; c0 < a.classes; c0 += p.piece) {
    const int64_t left = a.classes - c0, have = left < p.piece ? left : p.piece;
    g.c0 = static_cast<int>(c0);
    g.m_tiles = static_cast<int>(round_up(have, kPadRows) / kTile);   // G's padding is written too
    g.db = a.db ? reinterpret_cast<float*>(at(p.db)) + c0 : nullptr;
    hipLaunchKernelGGL((k_logits<TYPE, kGrad, kTile, kTile, 2, 2>),
                       dim3(grid8(static_cast<int64_t>(g.m_tiles) * g.n_tiles)), dim3(256), 0, s, g);
    if (!a.dx && !a.dw) continue;
    const T16Side grad{g.g, g.ldg, p.pad_rows, static_cast<int>(p.piece), 0};
    Product dx{}, dw{};
    if (a.dx) {
      dx.a = w;
      dx.a.data = w.data + c0 * w.ld;
      dx.a.rows = left;
      dx.b = grad;
      dx.m = a.d;
      dx.n = a.rows;
      dx.m_tiles = d_tiles;
      dx.n_tiles = static_cast<int>((a.rows + kTile - 1) / kTile);
      dx.splits = p.dx_splits;
      dx.stages = (have + k - 1) / k;
      dx.factor = mean;
      dx.inverse = kLo ? nullptr : inverses + 1;
      dx.out = p.dx_slab ? nullptr : a.dx;
      dx.ld = a.d;
      dx.slab = reinterpret_cast<float*>(at(p.dx_sums));
      dx.ld_slab = ld_dx;
      dx.more = c0 > 0;
    }
    if (a.dw) {
      dw.a = a.turned ? grad : x_by_all;
      dw.b = a.turned ? x_by_all : grad;
      dw.m = a.turned ? have : a.d;
      dw.n = a.turned ? a.d : have;
      dw.m_tiles = static_cast<int>((dw.m + kTile - 1) / kTile);
      dw.n_tiles = static_cast<int>((dw.n + kTile - 1) / kTile);
      dw.splits = p.dw_splits;
      dw.stages = (a.rows + k - 1) / k;
      dw.factor = mean;
      dw.inverse = kLo ? nullptr : inverses;
      const int64_t skip = a.turned ? c0 : c0 * a.d;
      dw.out = p.dw_splits > 1 ? nullptr : static_cast<T*>(a.dw) + skip;
      dw.ld = a.turned ? a.classes : a.d;
      dw.slab = reinterpret_cast<float*>(at(p.dw_sums));
      dw.ld_slab = p.ld_dw;
    }
    const int64_t tiles = static_cast<int64_t>(dx.m_tiles) * dx.n_tiles * dx.splits +
                          static_cast<int64_t>(dw.m_tiles) * dw.n_tiles * dw.splits;
    hipLaunchKernelGGL((k_products<TYPE, kTile, kTile, 2, 2>), dim3(grid8(tiles)), dim3(256), 0, s, dx, dw);
    if (a.dw && p.dw_splits > 1)
      join(dw.slab, dw.splits, dw.n, dw.m, dw.ld_slab, mean, dw.inverse,
           static_cast<T*>(a.dw) + (a.turned ? c0 : c0 * a.d), dw.ld, kLo);
  }
  if (a.dx && p.dx_slab)
    join(reinterpret_cast<const float*>(at(p.dx_sums)), p.dx_splits, a.rows, a.d, ld_dx, mean,
         kLo ? nullptr : inverses + 1, a.dx, a.d, kLo);
  if (a.db)
    join(reinterpret_cast<const float*>(at(p.db)), p.n_tiles, 1, a.classes, pad_classes,
         static_cast<float>(1.0 / static_cast<double>(a.rows)), nullptr, a.db, a.classes, false);
  return hipGetLastError();
}

__global__ __launch_bounds__(256) void k_zero(uint16_t* p, int64_t n) {
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n;
       i += static_cast<int64_t>(gridDim.x) * 256)
    p[i] = 0;
}

}  // namespace

size_t linear_loss_bytes(const LinearLossArgs& a, int bf16) { return plan(a, bf16).total; }

hipError_t launch_linear_loss(const LinearLossArgs& a, int bf16, hipStream_t s) {
  if (a.rows > 0) return bf16 ? run<kBf16, uint16_t>(a, s) : run<kSplit, float>(a, s);
  // no rows: the loss and the gradients of W and b are 0
  auto zero = [&](void* p, int64_t bytes) {
    const int64_t need = (bytes / 2 + 255) / 256;
    if (p) hipLaunchKernelGGL(k_zero, dim3(static_cast<unsigned>(need < 8 * kComputeUnits ? need : 8 * kComputeUnits)),
                              dim3(256), 0, s, static_cast<uint16_t*>(p), bytes / 2);
  };
  zero(a.loss, 4);
  zero(a.dw, static_cast<int64_t>(a.classes) * a.d * (bf16 ? 2 : 4));
  zero(a.db, static_cast<int64_t>(a.classes) * 4);
  return hipGetLastError();
}

}  // namespace gmb
