// Softmax cross-entropy of a linear head over many classes, and its gradients,
// without the logits: z = x W^T + b, L = (1 / n) sum_i (lse_i - z_i,y(i)),
// G = softmax(z) - onehot(y), dx = G W / n, dW = G^T x / n, db = G^T 1 / n.
//
//   k_amax, k_lay_out   x, and W where it cannot be read as it lies, as 16-bit
//                       rows padded with zeros; rows without a label as zeros
//   k_logits (kStats)   tiles of logits in registers: every row's maximum and
//                       sum of exponentials over a chunk of the classes, its
//                       label's logit
//   k_logits (kGrad)    the chunks of a row joined, the logits again, a piece of
//                       the classes at a time: G; few classes (kBoth): at once
//   k_products          dx += G W and dW = G^T x of the piece
//   k_join_piece        dW and db of a piece, where their sums were split
//   k_finish            the same of the last piece, and dx; the mean
//   k_stream_head       few rows, or few classes: all of it on W as it lies
//
// The logits are computed twice (8 n C d operations in all where keeping them
// would take 6) and never stored; G is, in 16 bits (kSplit: two times 16), for
// a piece of the classes.  Nothing is added by atomics: the same bits every time.
// bf16: G is rounded to bf16 (half a step of each entry) so that its products take
// one matrix instruction; two parts of it would take two, half as much again for
// the whole call.  What shows is the label's entry, p - 1: dx and dw are 0.0019 of
// their size from 64 bits where their own rounding to bf16 alone is 0.0017 (0.0010
// of G's, in quadrature).  dbias adds G up before it is rounded.
// The figures below are times of kernels; a large product of the library's reaches
// 1,210 TFLOP/s in bf16 on random values (here the power it may draw is the bound:
// 8,192 x 1,024 x 32,768 takes it 514 us, with zeros 336).
#include "head_kernels.hpp"
#include "mx.hpp"
#include "mx_kernels.hpp"
#include "tiles16.hpp"

#include <algorithm>

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
  int64_t w_all;                   // values in all if they lie one behind the other, or 0
  uint32_t* w_top;                 // [w_blocks]
  int x_blocks, w_blocks;
};

// The largest finite magnitudes: of every row of x and of all of them (a word a
// workgroup), and of W (a word a workgroup).  A wave has a row (W, if its rows
// lie one behind the other: a piece of the whole), 16 bytes a lane.  Bound by the
// reading: 4,000 and 20,011 rows of 256, 25 MB, 8.9 us.
__global__ __launch_bounds__(256) void k_amax(AmaxArgs p) {
  __shared__ uint32_t lds[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool of_x = static_cast<int>(blockIdx.x) < p.x_blocks;
  const int block = of_x ? blockIdx.x : blockIdx.x - p.x_blocks, blocks = of_x ? p.x_blocks : p.w_blocks;
  const float* data = of_x ? p.x : p.w;
  const int64_t rows = of_x ? p.rows : p.w_rows, stride = of_x ? p.x_stride : p.w_stride;
  const int64_t col = of_x ? 1 : p.w_col;
  uint32_t all = 0;
  for (int64_t row = static_cast<int64_t>(block) * 4 + wave; row < rows; row += static_cast<int64_t>(blocks) * 4) {
    uint32_t top = 0;
    int cols = of_x ? p.d : p.w_cols;
    if (!of_x && p.w_all && p.w_all - row * stride < cols) cols = static_cast<int>(p.w_all - row * stride);
    if (!of_x || has_label(p.labels, row, p.classes)) {
      const float* from = data + row * stride;
      int c = 4 * lane;
      if (col == 1) {
#pragma unroll 4
        for (; c + 4 <= cols; c += 256) {
          float v[4];
          mx_get<16>(v, from + c);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t u = finite_bits(v[i]);
            top = u > top ? u : top;
          }
        }
      }
      for (; c < cols; c += 256) {
        for (int i = 0; i < 4 && c + i < cols; ++i) {
          const uint32_t u = finite_bits(from[(c + i) * col]);
          top = u > top ? u : top;
        }
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

// A 64 x 64 tile of the source: rows with contiguous columns eight values a
// thread; else through LDS, read along the direction that is contiguous.  (The
// first `first` workgroups lay out x, the others W.)  Bound by memory: 25 MB read
// and 29 written, 11.8 us.
template <T16Type TYPE, typename T>
__global__ __launch_bounds__(256) void k_lay_out(LayOutArgs x, LayOutArgs w, int64_t first) {
  __shared__ float tile[64][65];
  __shared__ uint32_t top_of[4];
  const bool of_x = static_cast<int64_t>(blockIdx.x) < first;
  const LayOutArgs& p = of_x ? x : w;
  const int64_t id = of_x ? blockIdx.x : blockIdx.x - first;
  const int across = p.out_cols / 64;
  const int64_t r0 = id / across * 64;
  const int c0 = static_cast<int>(id % across) * 64;
  const T* src = static_cast<const T*>(p.src);
  const bool direct = p.col == 1;
  float v[2][8];
  bool on[2];
  if (direct) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int64_t row = r0 + 32 * k + (threadIdx.x >> 3);
      const int c = c0 + (threadIdx.x & 7) * 8, left = p.cols - c;
      on[k] = row < p.rows && (!p.labels || has_label(p.labels, row, p.classes));
#pragma unroll
      for (int i = 0; i < 8; ++i) v[k][i] = 0.f;
      if (row >= p.rows || left <= 0) continue;     // (a row without a label is read and thrown away)
      const T* from = src + row * p.row + c;
      if constexpr (sizeof(T) == 4) {
        if (left >= 8) {
          mx_get<16>(v[k], from);
          mx_get<16>(v[k] + 4, from + 4);
        } else {
#pragma unroll
          for (int i = 0; i < 7; ++i)
            if (i < left) v[k][i] = from[i];
        }
      } else {
        if (left >= 8) {
          uint32_t q[4];
          mx_get<16>(q, from);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[k][2 * i] = __uint_as_float(q[i] << 16);
            v[k][2 * i + 1] = __uint_as_float(q[i] & 0xFFFF0000u);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 7; ++i)
            if (i < left) v[k][i] = bf16_to_f32(from[i]);
        }
      }
    }
  } else {
    const int fast = threadIdx.x & 63, slow = threadIdx.x >> 6;
    const bool along_rows = p.row != 1;                // neighbouring threads: neighbouring columns
#pragma unroll 4
    for (int k = 0; k < 16; ++k) {
      const int i = along_rows ? 4 * k + slow : fast, j = along_rows ? fast : 4 * k + slow;
      float z = 0.f;
      if (r0 + i < p.rows && c0 + j < p.cols) {
        const T q = src[(r0 + i) * p.row + (c0 + j) * p.col];
        if constexpr (sizeof(T) == 4) z = q;
        else z = bf16_to_f32(q);
      }
      tile[i][j] = z;
    }
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
    for (int w4 = 0; w4 < 4; ++w4) top = top_of[w4] > top ? top_of[w4] : top;
    scale = split_scale(top);
    if (id == 0 && threadIdx.x == 0) *p.all_inverse = inverse_of_power(scale);
  } else if (!direct) {
    __syncthreads();
  }
  const int64_t ld = TYPE == kSplit ? 2 * static_cast<int64_t>(p.out_cols) : p.out_cols;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int i = 32 * k + (threadIdx.x >> 3), j = (threadIdx.x & 7) * 8;
    const int64_t row = r0 + i;
    if (row >= p.out_rows) continue;
    if (!direct) {
      on[k] = true;                                    // (W: no labels)
#pragma unroll
      for (int q = 0; q < 8; ++q) v[k][q] = tile[i][j + q];
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) v[k][q] = on[k] ? v[k][q] : 0.f;
    put_split<TYPE>(p.by_all + row * ld, c0 + j, v[k], scale);
    const bool lead = c0 == 0 && j == 0;
    if (TYPE == kSplit && p.by_row) {
      const float s = split_scale(row < p.rows ? p.row_top[row] : 0u);
      put_split<TYPE>(p.by_row + row * ld, c0 + j, v[k], s);
      if (lead) p.row_inverse[row] = inverse_of_power(s);
    }
    if (lead && p.labels) p.kept_labels[row] = on[k] ? p.labels[row] : -1;
  }
}

// ---- logits ---------------------------------------------------------------

struct LogitsArgs {
  T16Side w, x;                    // W's rows: A, those of x: B (`first` is set by the kernel)
  int d_values;                    // of a row, with the padding
  int c0, m_tiles, n_tiles;        // the first class, tiles of classes from it on, of rows
  int chunks;                      // workgroups of a row tile
  int classes;
  const float* bias;               // or NULL
  const float* row_inverse;        // kSplit
  const float* w_inverse;          // kSplit: one word
  const int32_t* labels;           // [padded rows], -1 for none
  int64_t rows, pad_rows;
  float2* stats;                   // [stat_chunks][pad_rows]: maximum, sum of exponentials, in powers of two
  int stat_chunks;
  float* label_logit;              // [pad_rows], times log2(e)
  float* loss_rows;                // [rows], or NULL
  uint16_t* g;                     // [pad_rows][ldg], or NULL
  int64_t ldg;
  float* db;                       // [n_tiles][ld_db] from the first class on, or NULL
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

// A maximum and the sum of 2^(u - maximum) of some of a row's u = z log2(e),
// joined with others'.  -inf: nothing yet.  A NaN among the u makes the sum NaN.
// SUM is double where a chain is as long as the classes or their chunks are many:
// 50,000 equal terms added up in fp32 round the same way one after the other (a
// row's loss over 400,000 classes was off by 7e-5).
template <typename SUM>
__device__ __forceinline__ void join_stats(float& top, SUM& sum, float t, float s) {
  const float m = fmaxf(top, t), base = m == -INFINITY ? 0.f : m;
  sum = sum * static_cast<SUM>(exp2_fast(top - base)) + static_cast<SUM>(s) * static_cast<SUM>(exp2_fast(t - base));
  top = m;
}
// Every logit is -inf (a sum that is no number has a NaN among them).
__device__ __forceinline__ bool row_empty(float top, float sum) { return top == -INFINITY && sum == 0.f; }
constexpr float kLn2 = 0.6931471805599453f;
// A row's loss and probabilities go by the distance to its maximum, 2^(u - top) /
// sum, not to the logarithm of its sum: top + log2(sum) in 32 bits has lost what the
// sum says where logits are far from 0 (equal ones at 1e5: probabilities 0.3% off, at
// 1e9 all 1).
__device__ __forceinline__ float row_loss(float top, float sum, float of_label) {
  return ((top - of_label) + log2f(sum)) * kLn2;
}

// kStats: a row's statistics over a chunk of the classes.  kGrad: G of the
// classes' piece, from the statistics of all chunks.  kBoth: at most TM classes:
// statistics and G at once.
enum LogitsMode { kStats, kGrad, kBoth };

// Stages in LDS.  256 x 256: two of 64 elements, 128 KB (bf16, four of 32: 535 us
// for 494, statistics of 8,192 x 1,024 x 32,768; 128 x 256 in three of 32, two
// workgroups a CU: 561 for 515).  64 x 64: four for logits, whose sums are short
// (1,000 x 256 x 47 fp32: 9.0 us, two 11.1), two for products, which have more
// code than time (6.5 us, four 12.2).
constexpr int logits_stages(int tm) { return tm > 64 ? 2 : 4; }

template <int TM, int TN, int WM, int WN>
struct LogitsLds {
  static constexpr int kStages = logits_stages(TM) * t16_stage_bytes<TM, TN, 64>();
  static constexpr int kRows = kStages;                        // [2][WM][TN]: statistics; maximum, 1 / sum; [TN]: label's logit
  static constexpr int kClasses = kRows + (2 * WM + 1) * TN * 4;   // [WN][TM]: sums of G
  static constexpr int kBytes = kClasses + WN * TM * 4;
};

// A workgroup has a tile of rows and goes over its chunk of the classes, tile by
// tile, without a pause in the loads between two; a lane has eight neighbouring
// classes of a row, so that G leaves in 16 bytes.  256 x 256: bound by the matrix
// instructions (busy 0.49; the library's product takes as long), and where d is
// short by the exponentials behind every tile's d / 64 stages of them.  bf16,
// statistics and G:
// 8,192 x 1,024 x 32,768 502 and 602 us (1,096 and 912 TFLOP/s), 4,000 x 256 x 100,000 250
// and 369 (820 and 555); fp32 4,000 x 256 x 20,011 128 and 164 (three part products: 959
// and 750).
template <T16Type TYPE, LogitsMode MODE, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void k_logits(LogitsArgs p) {
  using Tile = T16Tile<TYPE, kByRow, kByRow, TM, TN, WM, WN, logits_stages(TM), 64, true>;
  using Lds = LogitsLds<TM, TN, WM, WN>;
  constexpr int NST = Tile::STAGES;
  constexpr int RT = Tile::RT, CT = Tile::CT, THREADS = 64 * WM * WN;
  static_assert(RT % 2 == 0, "classes are dealt to pairs of tiles");
  __shared__ __attribute__((aligned(1024))) char lds[Lds::kBytes];
  float* row_a = reinterpret_cast<float*>(lds + Lds::kRows);
  float* row_b = row_a + WM * TN;
  float* row_label = row_b + WM * TN;
  const int64_t id = xcd_id(static_cast<int64_t>(p.n_tiles) * p.chunks);
  if (id < 0) return;
  // bands of eight row tiles: what an XCD's workgroups read together is few tiles
  // of x and few chunks of W
  const int band = static_cast<int>(id / (8 * static_cast<int64_t>(p.chunks)));
  const int in_band = static_cast<int>(id - static_cast<int64_t>(band) * 8 * p.chunks);
  const int width = p.n_tiles - 8 * band < 8 ? p.n_tiles - 8 * band : 8;
  const int nt = 8 * band + in_band % width, chunk = in_band / width;
  const int t0 = static_cast<int>(static_cast<int64_t>(p.m_tiles) * chunk / p.chunks);
  const int t1 = static_cast<int>(static_cast<int64_t>(p.m_tiles) * (chunk + 1) / p.chunks);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, r = lane & 15;
  const int wm = wave / WN, wn = wave % WN;
  const int64_t tile_row = static_cast<int64_t>(nt) * TN, row0 = tile_row + 16 * CT * wn + r;
  typename Tile::LoadA la;
  typename Tile::LoadB lb;
  T16Side a = p.w, b = p.x;
  b.first = tile_row;
  lb.init(b, wave, lane);
  a.first = p.c0 + static_cast<int64_t>(t0) * TM;
  la.init(a, wave, lane);
  // the stages of all tiles, one after the other: `left` are to be fetched, the
  // next one is stage `next` of its tile (la's)
  const int stages = p.d_values / Tile::K;
  int left = (t1 - t0) * stages, next = 0, rest = left;   // rest: to be used
  auto fetched = [&] {
    --left;
    if (++next == stages) {
      next = 0;
      la.advance();
    }
  };
#pragma unroll
  for (int s = 0; s < NST - 1; ++s)
    if (left > 0) {
      Tile::fetch(la, lb, next, lds + s * Tile::kStage);
      fetched();
    }
  // the rows' labels, scales and, for G, statistics
  float scale[CT];
  int label[CT];
#pragma unroll
  for (int j = 0; j < CT; ++j) {
    scale[j] = kLog2e;
    if constexpr (TYPE == kSplit) scale[j] *= p.row_inverse[row0 + 16 * j] * *p.w_inverse;
    label[j] = p.labels[row0 + 16 * j];
  }
  float base[CT], over[CT];         // G: 2^(u - base) over - onehot
  if constexpr (MODE == kGrad) {
    constexpr int PARTS = THREADS / TN > 0 ? THREADS / TN : 1;
    static_assert(PARTS * TN <= THREADS || PARTS == 1, "");
    float* part = reinterpret_cast<float*>(lds + (NST - 1) * Tile::kStage);   // (the last stage is still empty)
    for (int q = threadIdx.x; q < PARTS * TN; q += THREADS) {
      const int row = q % TN;
      float top = -INFINITY;
      double sum = 0.0;
#pragma unroll 8
      for (int c = q / TN; c < p.stat_chunks; c += PARTS) {
        const float2 s = p.stats[c * p.pad_rows + tile_row + row];
        join_stats(top, sum, s.x, s.y);
      }
      part[2 * q] = top;
      part[2 * q + 1] = static_cast<float>(sum);
    }
    __syncthreads();
    for (int row = threadIdx.x; row < TN; row += THREADS) {
      float top = part[2 * row], sum = part[2 * row + 1];
#pragma unroll
      for (int w = 1; w < PARTS; ++w) join_stats(top, sum, part[2 * (w * TN + row)], part[2 * (w * TN + row) + 1]);
      const bool on = p.labels[tile_row + row] >= 0 && !row_empty(top, sum);
      row_a[row] = top;
      row_b[row] = on ? 1.f / sum : 0.f;
      if (p.loss_rows && chunk == 0 && tile_row + row < p.rows)
        p.loss_rows[tile_row + row] = on ? row_loss(top, sum, p.label_logit[tile_row + row]) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < CT; ++j) {
      const int q = 16 * (CT * wn + j) + r;
      over[j] = row_b[q];
      base[j] = over[j] == 0.f ? INFINITY : row_a[q];   // (G is 0 there)
      if (over[j] == 0.f) label[j] = -1;
    }
  }
  float top[CT];
  double long_sum[CT];              // (tiles follow one another: as many links as the chunk has)
#pragma unroll
  for (int j = 0; j < CT; ++j) {
    top[j] = -INFINITY;
    long_sum[j] = 0.0;
  }
  __syncthreads();
  int at = 0;
  for (int t = t0; t < t1; ++t) {
    t16_f32x4 acc[RT][CT];
    Tile::clear(acc);
    for (int k = 0; k < stages; ++k) {
      Tile::wait(--rest >= NST - 2);
      const int to = at == 0 ? NST - 1 : at - 1;
      const bool more = left > 0;
      Tile::step(la, lb, next, more, lds + at * Tile::kStage, lds + to * Tile::kStage, wave, lane, acc);
      if (more) fetched();
      at = at == NST - 1 ? 0 : at + 1;
    }
    // u = z log2(e) = acc by[j], in place where there is more to it than that; the
    // registers of tiles i and i + 1 (i even) are classes c0 + 16 i .. + 7, -inf past
    // the last class
    const int cw = t * TM + 16 * RT * wm + 8 * g;       // of the piece
    const int c0 = p.c0 + cw;
    const bool whole = p.c0 + t * TM + TM <= p.classes;
    float by[CT];
#pragma unroll
    for (int j = 0; j < CT; ++j) by[j] = scale[j];
    if (p.bias || !whole) {
#pragma unroll
      for (int j = 0; j < CT; ++j) by[j] = 1.f;
#pragma unroll
      for (int i = 0; i < RT; i += 2) {
        float bias[8] = {};
        const int c = c0 + 16 * i;
        if (whole) {
          mx_get<16>(bias, p.bias + c);
          mx_get<16>(bias + 4, p.bias + c + 4);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) bias[e] = c + e >= p.classes ? -INFINITY : (p.bias ? p.bias[c + e] : 0.f);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          bias[e] *= kLog2e;
#pragma unroll
          for (int j = 0; j < CT; ++j) acc[i + e / 4][j][e % 4] = fmaf(acc[i + e / 4][j][e % 4], scale[j], bias[e]);
        }
      }
    }
    if constexpr (MODE != kGrad) {
#pragma unroll
      for (int j = 0; j < CT; ++j) {
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) most = fmaxf(most, acc[i][j][e]);
        most = fmaxf(top[j], most * by[j]);
        const float from = most == -INFINITY ? 0.f : most;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) s += exp2_fast(fmaf(acc[i][j][e], by[j], -from));
        long_sum[j] = long_sum[j] * static_cast<double>(exp2_fast(top[j] - from)) + static_cast<double>(s);
        top[j] = most;
        // the label's logit, where it is one of this lane's
        const int y = label[j] - c0;
        if (y >= 0 && y < 16 * RT && (y & 31) < 8) {
          float z = 0.f;
#pragma unroll
          for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) z = y == 16 * (i & ~1) + 4 * (i & 1) + e ? acc[i][j][e] : z;
          z *= by[j];
          if constexpr (MODE == kBoth) row_label[16 * (CT * wn + j) + r] = z;
          else p.label_logit[row0 + 16 * j] = z;
        }
      }
    }
    if constexpr (MODE == kBoth) {
      // all classes are here: the lanes' and waves' statistics joined
#pragma unroll
      for (int j = 0; j < CT; ++j) {
        float sum = static_cast<float>(long_sum[j]);
        for (int o = 16; o < 64; o <<= 1) join_stats(top[j], sum, __shfl_xor(top[j], o, 64), __shfl_xor(sum, o, 64));
        if (g == 0) {
          row_a[wm * TN + 16 * (CT * wn + j) + r] = top[j];
          row_b[wm * TN + 16 * (CT * wn + j) + r] = sum;
        }
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < CT; ++j) {
        const int q = 16 * (CT * wn + j) + r;
        float m = row_a[q], s = row_b[q];
#pragma unroll
        for (int w = 1; w < WM; ++w) join_stats(m, s, row_a[w * TN + q], row_b[w * TN + q]);
        if (row_empty(m, s)) label[j] = -1;
        base[j] = label[j] < 0 ? INFINITY : m;            // (G is 0 there)
        over[j] = label[j] < 0 ? 0.f : 1.f / s;
        if (wm == 0 && g == 0 && row0 + 16 * j < p.rows)
          p.loss_rows[row0 + 16 * j] = label[j] >= 0 ? row_loss(m, s, row_label[q]) : 0.f;
      }
      if (!p.g) return;
    }
    if constexpr (MODE != kStats) {
      float* part = reinterpret_cast<float*>(lds + Lds::kClasses);
#pragma unroll
      for (int i = 0; i < RT; i += 2) {
        float db[8] = {};
#pragma unroll
        for (int j = 0; j < CT; ++j) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            v[e] = exp2_fast(fmaf(acc[i + e / 4][j][e % 4], by[j], -base[j])) * over[j];
          }
          const int y = label[j] - c0 - 16 * i;
          if (y >= 0 && y < 8) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] -= y == e ? 1.f : 0.f;
          }
          put_split<TYPE>(p.g + (row0 + 16 * j) * p.ldg, cw + 16 * i, v, kGradScale);
          if (p.db) {
#pragma unroll
            for (int e = 0; e < 8; ++e) db[e] += v[e];
          }
        }
        if (p.db) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float s = sum16(db[e]);
            if (r == 0) part[wn * TM + 16 * RT * wm + 16 * i + 8 * g + e] = s;
          }
        }
      }
      if (p.db) {
        __syncthreads();
        for (int q = threadIdx.x; q < TM; q += THREADS) {
          float s = 0.f;
#pragma unroll
          for (int w = 0; w < WN; ++w) s += part[w * TM + q];
          if (p.c0 + t * TM + q < p.classes) p.db[static_cast<int64_t>(nt) * p.ld_db + t * TM + q] = s;
        }
        // (the next tile's sums come behind the barriers of its stages)
      }
    }
  }
  if constexpr (MODE == kStats) {
#pragma unroll
    for (int j = 0; j < CT; ++j) {
      float sum = static_cast<float>(long_sum[j]);
      for (int o = 16; o < 64; o <<= 1) join_stats(top[j], sum, __shfl_xor(top[j], o, 64), __shfl_xor(sum, o, 64));
      if (g == 0) {
        row_a[wm * TN + 16 * (CT * wn + j) + r] = top[j];
        row_b[wm * TN + 16 * (CT * wn + j) + r] = sum;
      }
    }
    __syncthreads();
    for (int q = threadIdx.x; q < TN; q += THREADS) {
      float m = row_a[q], s = row_b[q];
#pragma unroll
      for (int w = 1; w < WM; ++w) join_stats(m, s, row_a[w * TN + q], row_b[w * TN + q]);
      p.stats[chunk * p.pad_rows + tile_row + q] = make_float2(m, s);
    }
  }
}

// ---- the rows' losses, where no gradient is wanted --------------------------

// As k_logits (kGrad) joins them, so that the loss alone has the same bits: the
// chunks of a row dealt to PARTS threads.
template <int PARTS>
__global__ __launch_bounds__(256) void k_join_rows(const float2* stats, int chunks, int64_t rows, int64_t pad_rows,
                                                   const int32_t* labels, const float* label_logit, float* loss_rows,
                                                   int classes) {
  constexpr int ROWS = 256 / PARTS;
  __shared__ float2 lds[PARTS][ROWS];
  const int q = threadIdx.x % ROWS, part = threadIdx.x / ROWS;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + q;
  float top = -INFINITY;
  double long_sum = 0.0;
#pragma unroll 8
  for (int c = part; c < chunks; c += PARTS) {
    const float2 s = stats[c * pad_rows + row];
    join_stats(top, long_sum, s.x, s.y);
  }
  float sum = static_cast<float>(long_sum);
  lds[part][q] = make_float2(top, sum);
  __syncthreads();
  if (part || row >= rows) return;
#pragma unroll
  for (int w = 1; w < PARTS; ++w) join_stats(top, sum, lds[w][q].x, lds[w][q].y);
  loss_rows[row] = has_label(labels, row, classes) && !row_empty(top, sum) ? row_loss(top, sum, label_logit[row]) : 0.f;
}

// ---- products -------------------------------------------------------------

struct Product {
  T16Side a, b;                    // `first` is set by the kernel
  int64_t m, n;                    // out: n rows of m contiguous values
  int m_tiles, n_tiles, splits;
  int64_t k;
  void* out;                       // the result, or NULL: sums go to `slab`
  int64_t ld;
  float factor;                    // result = sum factor inverse
  const float* inverse;            // or NULL
  float* slab;                     // row i of split q at q part + i ld_slab
  int64_t ld_slab, part;
  int more;                        // add to what the slab holds
};

__host__ __device__ inline int64_t product_tiles(const Product& p) {
  return static_cast<int64_t>(p.m_tiles) * p.n_tiles * p.splits;
}

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
  using Tile = T16Tile<TYPE, FA, FB, TM, TN, WM, WN, 2, 64>;
  constexpr int RT = Tile::RT, CT = Tile::CT;
  const int mt = static_cast<int>(id % p.m_tiles);
  const int64_t rest = id / p.m_tiles;
  const int nt = static_cast<int>(rest % p.n_tiles), split = static_cast<int>(rest / p.n_tiles);
  T16Side a = p.a, b = p.b;
  a.first = static_cast<int64_t>(mt) * TM;
  b.first = static_cast<int64_t>(nt) * TN;
  t16_f32x4 acc[RT][CT];
  Tile::clear(acc);
  const int64_t stages = (p.k + Tile::K - 1) / Tile::K;
  Tile::run(a, b, stages * split / p.splits, stages * (split + 1) / p.splits, lds, acc);
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
        float* to = p.slab + split * p.part + row * p.ld_slab + col;
        t16_f32x4 had = {0.f, 0.f, 0.f, 0.f};
        if (p.more) mx_get<16>(&had, to);
        v += had;
        mx_put<16, false>(to, &v);
      }
    }
  }
}

// dx = G W (A: W by its rows of k, B: G by its rows), then dW = G^T x, its rows
// those of W (A: x, B: G) or, turned, those of W's transpose (A: G, B: x).  One
// launch, so that the ends of one fill the other's.  256 x 256: matrix instructions,
// and G from the last-level cache (loss of 8,192 x 1,024 x 32,768 bf16: 1,001 us, 1,099
// TFLOP/s; 4,000 x 256 x 100,000 bf16 509, 805; 4,000 x 256 x 20,011 fp32 279, 880 of part
// products).  Four waves of 128 x 128 instead of eight, their operands read a stage
// ahead: 535 us a piece for 531, and the logits' kernels spilled.
template <T16Type TYPE, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void k_products(Product dx, Product dw) {
  __shared__ __attribute__((aligned(1024))) char lds[2 * t16_stage_bytes<TM, TN, 64>()];
  // workgroup ids go round the eight XCDs: each has an eighth of either product
  const int64_t of_dx = product_tiles(dx), of_dw = product_tiles(dw);
  const int64_t dx_each = (of_dx + 7) / 8, dw_each = (of_dw + 7) / 8, xcd = blockIdx.x & 7;
  int64_t id = blockIdx.x >> 3;
  if (id < dx_each) {
    id += xcd * dx_each;
    if (id < of_dx) product_tile<TYPE, kByK, kByRow, TM, TN, WM, WN>(dx, id, lds);
  } else if (id < dx_each + dw_each) {
    id += xcd * dw_each - dx_each;
    if (id < of_dw) product_tile<TYPE, kByK, kByK, TM, TN, WM, WN>(dw, id, lds);
  }
}

// ---- sums that were split, and the mean ------------------------------------

struct JoinArgs {
  const float* slab;               // [parts][rows][ld_slab]
  int parts;
  int64_t rows, cols, ld_slab;
  float factor;
  const float* inverse;            // or NULL
  void* out;
  int64_t ld;
  int blocks;                      // workgroups of the launch that have it
};
struct FinishArgs {
  JoinArgs dx, dw, db;
  const float* loss_rows;
  int64_t rows;
  float* loss;
};

// Parts from which on a workgroup has 16 times four columns and 16 threads share
// the parts of each (63 parts of 47 x 256: one thread for all, 16 us; 16, 4).
constexpr int kManyParts = 8;
constexpr int join_columns(int parts) { return parts > kManyParts ? 16 : 256; }   // fours of a workgroup

// out = factor inverse times the sum of the parts, in a fixed order.
template <bool BF16>
__device__ __forceinline__ void join_parts(const JoinArgs& p, int block) {
  const int64_t fours = (p.cols + 3) / 4, all = p.rows * fours;
  const float inverse = p.inverse ? *p.inverse : 1.f;
  const int64_t step = p.rows * p.ld_slab;
  if (p.parts > kManyParts) {
    __shared__ t16_f32x4 lds[16][16];
    const int q0 = threadIdx.x & 15, mine = threadIdx.x >> 4;
    for (int64_t first = static_cast<int64_t>(block) * 16; first < all; first += static_cast<int64_t>(p.blocks) * 16) {
      const int64_t q = first + q0, row = q / fours, col = (q - row * fours) * 4;
      t16_f32x4 v = {0.f, 0.f, 0.f, 0.f};
      if (q < all) {
        const float* from = p.slab + row * p.ld_slab + col;
#pragma unroll 8
        for (int s = mine; s < p.parts; s += 16) {
          t16_f32x4 x;
          mx_get<16>(&x, from + s * step);
          v += x;
        }
      }
      __syncthreads();              // the last turn's reads
      lds[mine][q0] = v;
      __syncthreads();
      if (mine == 0 && q < all) {
#pragma unroll
        for (int w = 1; w < 16; ++w) v += lds[w][q0];
        put_four<BF16>(p.out, row * p.ld + col, v * p.factor * inverse, p.cols - col);
      }
    }
    return;
  }
  for (int64_t q = static_cast<int64_t>(block) * 256 + threadIdx.x; q < all; q += static_cast<int64_t>(p.blocks) * 256) {
    const int64_t row = q / fours, col = (q - row * fours) * 4;
    t16_f32x4 v = {0.f, 0.f, 0.f, 0.f};
    const float* from = p.slab + row * p.ld_slab + col;
#pragma unroll 4
    for (int s = 0; s < p.parts; ++s) {
      t16_f32x4 x;
      mx_get<16>(&x, from + s * step);
      v += x;
    }
    put_four<BF16>(p.out, row * p.ld + col, v * p.factor * inverse, p.cols - col);
  }
}

// dW and db of a piece behind which others come: their sums' memory is one piece's
// (for all classes it would grow with the rows, whose number makes pieces small and
// splits many: 20 GB for 16,384 rows over 2.4M classes of 256).
template <bool BF16>
__global__ __launch_bounds__(256) void k_join_piece(JoinArgs dw, JoinArgs db) {
  const int block = blockIdx.x;
  if (block < dw.blocks) join_parts<BF16>(dw, block);
  else join_parts<false>(db, block - dw.blocks);
}

// The last workgroup adds the rows' losses, in 64 bits and a fixed order; the
// others join sums, bound by reading them (4,000 x 256 x 20,011 fp32: 33 us).
template <bool BF16>
__global__ __launch_bounds__(256) void k_finish(FinishArgs p) {
  int block = blockIdx.x;
  if (block < p.dx.blocks) return join_parts<BF16>(p.dx, block);
  block -= p.dx.blocks;
  if (block < p.dw.blocks) return join_parts<BF16>(p.dw, block);
  block -= p.dw.blocks;
  if (block < p.db.blocks) return join_parts<false>(p.db, block);
  __shared__ double lds[4];
  double s = 0.0;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < p.rows; i += 256) s += p.loss_rows[i];
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) *p.loss = static_cast<float>((((lds[0] + lds[1]) + lds[2]) + lds[3]) / static_cast<double>(p.rows));
}

// ---- few rows, small heads -------------------------------------------------

// v_mfma_f32_16x16x4_f32 (exact products, fp32 sums) on W as it lies, with its own
// strides and type, read once a pass: no rows are laid out, nothing is cut, and G
// never leaves the workgroup, which has sixteen rows (in LDS) and goes over tiles
// of the classes of its chunk.  A tile has up to 16,384 values of W, sixteen a
// thread: the next one is on its way in registers while this one is used.  LDS
// rows are a multiple of four words that is odd in fours apart: sixteen rows'
// reads of four words, and four rows' of sixteen, fall on different banks.  Code
// is kept short: a launch starts with an empty instruction cache, and the first
// form, its loops unrolled, took 22 us for 12.8.
//   kBoth   all classes are one tile (1,000 x 256 x 47 fp32: 17 us in two launches,
//           through k_logits and k_products 29 in five)
//   kStats, kGrad   as in k_logits (5 x 226 x 147,879 fp32: 73 and 128 us traced, the
//           call 186, for 134 MB read and 268 read and written)
// 128 registers a thread are few: kBoth spills 17 (and 58 scalar ones), kGrad 9 (47).
constexpr int kStreamThreads = 1024, kStreamWaves = 16;
constexpr int kStreamClasses = 256, kStreamCells = 16384, kStreamD = 1024;   // a tile's classes, values; d

struct StreamArgs {
  const void* x;
  int64_t x_stride;
  const void* w;
  int64_t w_row, w_col;
  const float* bias;               // or NULL
  const int32_t* labels;
  int64_t rows;
  int d, classes;
  int tile;                        // classes of a tile, a multiple of 16
  int tiles, row_blocks, chunks;
  int turned;
  float mean;                      // 1 / rows
  float2* stats;                   // [chunks][16 row_blocks]
  float* label_logit;              // [16 row_blocks]
  float* loss_rows;                // [rows]
  int grad;                        // kBoth: whether G is wanted
  // Results, or (sums) parts of sums: dx's one a chunk, the others' one a row block.
  void* dx;
  int dx_sums;
  int64_t ld_dx, part_dx;
  void* dw;
  float* db;
  int dw_sums;
  int64_t ld_dw, part_dw, part_db;
};

template <typename T>
__device__ __forceinline__ float as_float(T v) {
  if constexpr (sizeof(T) == 4) return v;
  else return bf16_to_f32(v);
}
template <typename T>
__device__ __forceinline__ t16_f32x4 get_four(const T* p) {
  t16_f32x4 v;
  if constexpr (sizeof(T) == 4) {
    mx_get<16>(&v, p);
  } else {
    uint32_t q[2];
    mx_get<8>(q, p);
    v = t16_f32x4{__uint_as_float(q[0] << 16), __uint_as_float(q[0] & 0xFFFF0000u), __uint_as_float(q[1] << 16),
                  __uint_as_float(q[1] & 0xFFFF0000u)};
  }
  return v;
}

__device__ __forceinline__ t16_f32x4 mfma4(float a, float b, t16_f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// A thread's fours of a block of LDS rows [rows][4 across] (at most sixteen values
// a thread): four m is row row[m], columns 4 at[m] .. + 3.
struct Fours {
  int row[4], at[4];               // row -1: none
  // by_row: neighbouring threads have neighbouring fours; else neighbouring rows
  __device__ __forceinline__ void init(int rows, int across, bool by_row) {
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const int q = threadIdx.x + m * kStreamThreads;
      const int a = q / (by_row ? across : rows), b = q - a * (by_row ? across : rows);
      row[m] = q < rows * across ? (by_row ? a : b) : -1;
      at[m] = by_row ? b : a;
    }
  }
  // The values from element (row, column) at row r + column c; rows from `have` on
  // and columns from `cols` on are 0.  No load is behind a branch: what is past the
  // end is read where there is something, and left out.
  template <typename T>
  __device__ __forceinline__ void load(const T* from, int64_t r, int64_t c, int have, int cols, t16_f32x4 (&v)[4]) const {
    if (c == 1 && cols % 4 == 0) {
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const bool in = row[m] >= 0 && row[m] < have && 4 * at[m] < cols;
        v[m] = get_four<T>(from + (in ? row[m] * r + 4 * at[m] : 0));
#pragma unroll
        for (int e = 0; e < 4; ++e) v[m][e] = in ? v[m][e] : 0.f;
      }
    } else {
#pragma unroll
      for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool in = row[m] >= 0 && row[m] < have && 4 * at[m] + e < cols;
          const float z = as_float(from[in ? row[m] * r + (4 * at[m] + e) * c : 0]);
          v[m][e] = in ? z : 0.f;
        }
    }
  }
  __device__ __forceinline__ void store(float* lds, int stride, const t16_f32x4 (&v)[4]) const {
#pragma unroll
    for (int m = 0; m < 4; ++m)
      if (row[m] >= 0) *reinterpret_cast<t16_f32x4*>(lds + row[m] * stride + 4 * at[m]) = v[m];
  }
};

template <typename T, LogitsMode MODE>
__global__ __launch_bounds__(kStreamThreads) void k_stream_head(StreamArgs p) {
  constexpr int kWords = (kStreamCells + 4 * kStreamClasses) + 16 * (kStreamD + 4) + 16 * (kStreamClasses + 4);
  __shared__ __attribute__((aligned(16))) float lds[kWords];
  __shared__ float row_top[kStreamWaves][16], row_sum[kStreamWaves][16], row_label[16];
  __shared__ int32_t row_y[16];
  const int ct = p.tile / 16, dt = (p.d + 15) / 16;
  const int sd = 16 * dt + 4, sc = p.tile + 4;
  float* lw = lds;                                       // [tile][sd]
  float* lx = lw + p.tile * sd;                          // [16][sd]
  float* lg = lx + 16 * sd;                              // [16][sc]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, r = lane & 15;
  const int block = blockIdx.x % p.row_blocks, chunk = blockIdx.x / p.row_blocks;
  const int t0 = static_cast<int>(static_cast<int64_t>(p.tiles) * chunk / p.chunks);
  const int t1 = static_cast<int>(static_cast<int64_t>(p.tiles) * (chunk + 1) / p.chunks);
  const int64_t row0 = 16 * static_cast<int64_t>(block);
  const int rows = p.rows - row0 < 16 ? static_cast<int>(p.rows - row0) : 16;
  const T* w = static_cast<const T*>(p.w);
  Fours of_w;
  t16_f32x4 next[4];
  of_w.init(p.tile, 4 * dt, p.w_col == 1 || p.w_row != 1);
  auto fetch = [&](int t) {
    const int64_t c = static_cast<int64_t>(t) * p.tile;
    const int have = p.classes - c < p.tile ? static_cast<int>(p.classes - c) : p.tile;
    of_w.load(w + c * p.w_row, p.w_row, p.w_col, have, p.d, next);
  };
  fetch(t0);
  if (threadIdx.x < 16) {
    const int32_t y = static_cast<int>(threadIdx.x) < rows ? p.labels[row0 + threadIdx.x] : -1;
    row_y[threadIdx.x] = y >= 0 && y < p.classes ? y : -1;
  }
  {
    Fours of_x;
    t16_f32x4 v[4];
    of_x.init(16, 4 * dt, true);
    of_x.load(static_cast<const T*>(p.x) + row0 * p.x_stride, p.x_stride, 1, rows, p.d, v);
    __syncthreads();                                     // the labels
#pragma unroll
    for (int m = 0; m < 4; ++m)                          // (a row without a label is read, and left out)
      if (of_x.row[m] >= 0 && row_y[of_x.row[m]] < 0) v[m] = t16_f32x4{0.f, 0.f, 0.f, 0.f};
    of_x.store(lx, sd, v);
  }
  const int y = row_y[r];
  float top = -INFINITY, sum = 0.f, over = 0.f;
  double long_sum = 0.0;
  bool on = y >= 0;
  if constexpr (MODE == kGrad) {
    if (threadIdx.x < 256) {
      const int q = threadIdx.x & 15, part = threadIdx.x >> 4;
#pragma unroll 4
      for (int c = part; c < p.chunks; c += 16) {
        const float2 s = p.stats[(static_cast<int64_t>(c) * p.row_blocks + block) * 16 + q];
        join_stats(top, long_sum, s.x, s.y);
      }
      row_top[part][q] = top;
      row_sum[part][q] = static_cast<float>(long_sum);
    }
    __syncthreads();
    top = row_top[0][r];
    sum = row_sum[0][r];
    for (int v = 1; v < 16; ++v) join_stats(top, sum, row_top[v][r], row_sum[v][r]);
    over = 1.f / sum;
    on = on && !row_empty(top, sum);
    if (chunk == 0 && wave == 0 && g == 0 && r < rows)
      p.loss_rows[row0 + r] = on ? row_loss(top, sum, p.label_logit[row0 + r]) : 0.f;
  }
  t16_f32x4 dx[4];                                       // d tiles wave, wave + 16, ...
#pragma unroll
  for (int m = 0; m < 4; ++m) dx[m] = t16_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int t = t0; t < t1; ++t) {
    const int c_tile = t * p.tile;
    if (t > t0) __syncthreads();                         // the last tile is used
    of_w.store(lw, sd, next);
    if (t + 1 < t1) fetch(t + 1);
    __syncthreads();
    // logits: wave i has 16 classes of the tile; a step of sixteen of d is four
    // instructions, lane group g having d 4 g .. 4 g + 3 of them
    t16_f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    const int c0 = 16 * wave + 4 * g;
    if (wave < ct) {
      for (int k = 0; k < dt; ++k) {
        const t16_f32x4 b = *reinterpret_cast<const t16_f32x4*>(lx + r * sd + 16 * k + 4 * g);
        const t16_f32x4 a = *reinterpret_cast<const t16_f32x4*>(lw + (16 * wave + r) * sd + 16 * k + 4 * g);
#pragma unroll
        for (int s = 0; s < 4; ++s) acc = mfma4(a[s], b[s], acc);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = c_tile + c0 + e;
        const float bias = p.bias ? p.bias[c < p.classes ? c : 0] : 0.f;
        acc[e] = c < p.classes ? fmaf(acc[e], kLog2e, bias * kLog2e) : -INFINITY;
      }
      if constexpr (MODE != kGrad) {
        const float most = fmaxf(fmaxf(fmaxf(acc[0], acc[1]), fmaxf(acc[2], acc[3])), top);
        const float base = most == -INFINITY ? 0.f : most;
        sum = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sum += exp2_fast(acc[e] - base);
          if (c_tile + c0 + e == y) {
            if constexpr (MODE == kBoth) row_label[r] = acc[e];
            else p.label_logit[row0 + r] = acc[e];
          }
        }
        // (kBoth has one tile; else the chunk's tiles follow one another)
        if constexpr (MODE == kStats)
          long_sum = long_sum * static_cast<double>(exp2_fast(top - base)) + static_cast<double>(sum);
        top = most;
      }
    }
    if constexpr (MODE == kBoth) {
      for (int o = 16; o < 64; o <<= 1) join_stats(top, sum, __shfl_xor(top, o, 64), __shfl_xor(sum, o, 64));
      if (g == 0) {
        row_top[wave][r] = top;
        row_sum[wave][r] = sum;
      }
      __syncthreads();
      top = row_top[0][r];
      sum = row_sum[0][r];
      for (int v = 1; v < ct; ++v) join_stats(top, sum, row_top[v][r], row_sum[v][r]);
      over = 1.f / sum;
      on = on && !row_empty(top, sum);
      if (wave == 0 && g == 0 && r < rows) p.loss_rows[row0 + r] = on ? row_loss(top, sum, row_label[r]) : 0.f;
      if (!p.grad) return;
    }
    if constexpr (MODE != kStats) {
      if (wave < ct) {
        t16_f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float q = exp2_fast(acc[e] - top) * over;
          v[e] = on ? (c_tile + c0 + e == y ? q - 1.f : q) : 0.f;
        }
        *reinterpret_cast<t16_f32x4*>(lg + r * sc + c0) = v;
      }
      __syncthreads();
      if (const int c = threadIdx.x; p.db && c < p.tile && c_tile + c < p.classes) {
        float s = 0.f;
#pragma unroll 4
        for (int i = 0; i < 16; ++i) s += lg[i * sc + c];
        p.db[block * p.part_db + c_tile + c] = p.dw_sums ? s : s * p.mean;
      }
      if (p.dx) {
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const int q = wave + 16 * m;
          if (q < dt) {
            for (int k = 0; k < ct; ++k) {
              const t16_f32x4 b = *reinterpret_cast<const t16_f32x4*>(lg + r * sc + 16 * k + 4 * g);
#pragma unroll
              for (int s = 0; s < 4; ++s) dx[m] = mfma4(lw[(16 * k + 4 * g + s) * sd + 16 * q + r], b[s], dx[m]);
            }
          }
        }
      }
      if (p.dw) {
        for (int q = wave; q < ct * dt; q += kStreamWaves) {
          const int tc = q / dt, tj = q - tc * dt;
          t16_f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            const float a = lx[(4 * g + s) * sd + 16 * tj + r], b = lg[(4 * g + s) * sc + 16 * tc + r];
            v = p.turned ? mfma4(b, a, v) : mfma4(a, b, v);
          }
          // a row of the result, and four of its columns
          const int row = p.turned ? 16 * tj + r : c_tile + 16 * tc + r;
          const int col = p.turned ? c_tile + 16 * tc + 4 * g : 16 * tj + 4 * g;
          const int left = (p.turned ? p.classes : p.d) - col;
          if (row >= (p.turned ? p.d : p.classes) || left <= 0) continue;
          const int64_t at = row * p.ld_dw + col;
          if (p.dw_sums) mx_put<16, false>(static_cast<float*>(p.dw) + block * p.part_dw + at, &v);   // (rows of whole fours)
          else put_four<sizeof(T) == 2>(p.dw, at, v * p.mean, left);
        }
      }
    }
  }
  if constexpr (MODE == kStats) {
    sum = static_cast<float>(long_sum);
    for (int o = 16; o < 64; o <<= 1) join_stats(top, sum, __shfl_xor(top, o, 64), __shfl_xor(sum, o, 64));
    if (g == 0) {
      row_top[wave][r] = top;
      row_sum[wave][r] = sum;
    }
    __syncthreads();
    if (threadIdx.x < 16) {
      for (int v = 1; v < ct; ++v) join_stats(top, sum, row_top[v][r], row_sum[v][r]);
      p.stats[(static_cast<int64_t>(chunk) * p.row_blocks + block) * 16 + r] = make_float2(top, sum);
    }
  } else if (p.dx && r < rows) {
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const int col = 16 * (wave + 16 * m) + 4 * g;
      if (col >= p.d) continue;
      const int64_t at = (row0 + r) * p.ld_dx + col;
      if (p.dx_sums) mx_put<16, false>(static_cast<float*>(p.dx) + chunk * p.part_dx + at, &dx[m]);
      else put_four<sizeof(T) == 2>(p.dx, at, dx[m] * p.mean, p.d - col);
    }
  }
}

// ---- plan -----------------------------------------------------------------

// Tiles: 256 x 256 (eight waves of 128 x 64, one workgroup a CU), 64 x 64 (four of 32 x
// 32).
constexpr int kLarge = 256, kSmall = 64;
// G of a piece of the classes: less costs launches whose tiles do not fill the GPU
// and sums that are stored in between (4,000 x 256 x 100,000 bf16 at 64, 128, 256, 512
// and 1,024 MB: 1,455, 1,241, 1,150, 1,133, 1,122 us; 4,000 x 256 x 20,011 fp32, 331
// MB in one piece: 636, 595, 593, 559, 560; 8,192 x 1,024 x 32,768 bf16: 2,128, 1,956,
// 1,978, 2,038, 2,032), more only memory.
constexpr int64_t kGradBytes = int64_t{384} << 20;
constexpr int kMostTops = 1024;

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
int64_t tiles_of(int64_t x, int tile) { return (x + tile - 1) / tile; }

struct Plan {
  int es;                          // 16-bit words of a value
  int64_t pad_rows, pad_d, pad_classes;
  bool copy_w, grad, both;         // both: statistics and G in one launch
  // k_stream_head: row blocks (0: not taken), chunks and tiles of the classes
  int row_blocks, stream_chunks, stream_tile, stream_tiles;
  bool one_tile;
  int64_t piece, pieces;           // classes of a piece (a multiple of kPadRows)
  int tile;                        // of the logits
  int chunks, piece_chunks;        // workgroups of a row tile, for the statistics and for G
  int product_tile, dx_splits, dw_splits;
  bool dx_slab;
  int64_t ld_dw;                   // the contiguous extent of a piece's dw, padded to four
  int64_t dw_rows, dw_cols;        // of a piece's dw (k_stream_head: of all of it)
  // offsets
  size_t x_all, x_row, w, row_top, tops, row_inverse, inverses, labels, stats, label_logit, loss_rows, g, db, dx_sums,
      dw_sums, total;
};

// Which tiles k_products takes, and how many splits of k, by when an XCD's
// workgroups end: its tiles are an eighth of dx's first, each `long_` stages, then
// dw's; done in t if what fits until then is enough.  A kind of tile: its edge,
// workgroups of a CU, microseconds of a stage and of a tile of sums that is stored
// (bf16 and kSplit alike, in stages of 64 elements).  The whole call, us, with 256 /
// with 64, * the rule's: 784 x 631 x 4,132 fp32 150 / 111 *; 1,000 x 256 x 5,000 bf16 79 / 48
// *; 445 x 8 x 73,341 fp32 196 / 134 *; 8,192 x 1,024 x 2,048 bf16 167 * / 195; 4,000 x 256 x
// 20,011 fp32 583 * / 650; 4,000 x 256 x 100,000 bf16 1,079 * / 1,440.  (128 x 128, two a CU:
// 118, 64, 150, 169, 575, 1,194.)
struct TileKind {
  int edge, each;
  double stage, sums;
};
constexpr TileKind kTileKinds[] = {{kLarge, 1, 1.9, 20.0}, {kSmall, 4, 0.8, 3.0}};

void plan_products(const LinearLossArgs& a, Plan* p) {
  const int64_t have = p->piece < a.classes ? p->piece : a.classes, k = 64 / p->es;
  const int64_t dx_stages = tiles_of(have, k), dw_stages = tiles_of(a.rows, k);
  auto most_splits = [](int64_t stages) { return stages < 8 ? int64_t{1} : stages / 4; };
  double best = -1.0;
  for (const TileKind& kind : kTileKinds) {
    // (tiles that are mostly padding)
    if (kind.edge > kSmall && (a.rows <= kind.edge / 4 || a.d <= kind.edge / 4 || have <= kind.edge / 4)) continue;
    const int64_t slots = kind.each * kComputeUnits / 8, slab = static_cast<int64_t>(kind.sums / kind.stage + 0.5);
    const int64_t d_tiles = tiles_of(a.d, kind.edge);
    const int64_t dx_tiles = a.dx ? d_tiles * tiles_of(a.rows, kind.edge) : 0;
    const int64_t dw_tiles = a.dw ? d_tiles * tiles_of(have, kind.edge) : 0;
    for (int sw = 1; sw <= 64 && sw <= most_splits(dw_stages) && dw_tiles * (sw / 2) < 8 * slots; sw *= 2) {
      const int64_t short_ = tiles_of(dw_stages, sw) + (sw > 1 ? slab : 0), shorts = tiles_of(dw_tiles * sw, 8);
      for (int sx = 1; sx <= 256 && sx <= most_splits(dx_stages) && dx_tiles * (sx - 1) < 8 * slots; sx += sx < 8 ? 1 : sx / 4) {
        const bool sums = sx > 1 || p->pieces > 1;
        const int64_t long_ = tiles_of(dx_stages, sx) + (sums ? slab : 0), longs = tiles_of(dx_tiles * sx, 8);
        const int64_t rounds = longs / slots, more = longs % slots;
        auto fits = [&](int64_t t) {
          const int64_t a0 = t - rounds * long_, a1 = a0 - long_;
          if (a0 < 0 || (more && a1 < 0)) return false;
          return (slots - more) * (a0 / short_) + (more ? more * (a1 / short_) : 0) >= shorts;
        };
        int64_t lo = (rounds + (more ? 1 : 0)) * long_, hi = lo + (shorts / slots + 2) * short_;
        while (lo < hi) {
          const int64_t mid = (lo + hi) / 2;
          if (fits(mid)) hi = mid;
          else lo = mid + 1;
        }
        // (sums are joined by the whole GPU: 4.5 TB/s)
        const double joined = ((sw > 1 ? dw_tiles * sw : 0) + (sx > 1 ? dx_tiles * sx : 0)) *
                              (static_cast<double>(kind.edge) * kind.edge * 4 / 4.5e6);
        const double cost = static_cast<double>(lo) * kind.stage + joined;
        if (best < 0 || cost < best) {
          best = cost;
          p->product_tile = kind.edge;
          p->dx_splits = sx;
          p->dw_splits = sw;
        }
      }
    }
  }
}

// Whether k_stream_head takes it, and how (us of the whole call, with it / by
// k_logits and k_products):
//   - fp32, sixteen rows at most: its fp32 products (157 TFLOP/s) hide behind
//     reading W (5 x 226 x 147,879: 186 / 268; 1 x 128 x 5,000: 25 / 30), or a short
//     pass (1,000 x 256 x 47: 20 / 29; 300 x 32 x 2,000: 27 / 29; but 165 x 177 x 1,577,
//     2^25.7 products: 43 / 34), its sums of dW 64 MB at most;
//   - bf16, where nothing else need be laid out, only short passes of one tile
//     (64 x 16 x 8: 20 / 28; but 1,000 x 128 x 172, two tiles: 32 / 28), or few rows
//     whose W would be copied (16 x 100 x 100,000: 54 / 68; x 256 x 100,000: 101 / 82).
constexpr int64_t kStreamWork = int64_t{1} << 25, kStreamSums = int64_t{16} << 20;

bool plan_stream(const LinearLossArgs& a, int bf16, Plan* p) {
  if (a.d > kStreamD) return false;
  const int64_t blocks = tiles_of(a.rows, 16), pad_d = round_up(a.d, 16);
  int64_t tile = kStreamCells / pad_d / 16 * 16;
  tile = std::min<int64_t>(std::min<int64_t>(tile, kStreamClasses), round_up(a.classes, 16));
  const int64_t tiles = tiles_of(a.classes, static_cast<int>(tile));
  int64_t chunks = tiles_of(kComputeUnits, blocks);
  chunks = std::min(chunks, tiles);
  if (blocks > kComputeUnits) return false;
  const bool brief = 16 * blocks * pad_d * a.classes <= kStreamWork;
  if (blocks > 1 && (!brief || blocks * a.classes * static_cast<int64_t>(a.d) > kStreamSums)) return false;
  if (bf16 && !(tiles == 1 && brief) &&
      !(blocks == 1 && a.d % kPadCols != 0 && static_cast<int64_t>(a.classes) * a.d >= int64_t{1} << 20))
    return false;
  p->row_blocks = static_cast<int>(blocks);
  p->stream_tile = static_cast<int>(tile);
  p->stream_tiles = static_cast<int>(tiles);
  p->stream_chunks = static_cast<int>(chunks);
  p->one_tile = tiles == 1;
  return true;
}

Plan plan(const LinearLossArgs& a, int bf16) {
  Plan p{};
  p.es = bf16 ? 1 : 2;
  p.pad_rows = round_up(a.rows, kPadRows);
  p.pad_d = round_up(a.d, kPadCols);
  p.pad_classes = round_up(a.classes, kPadRows);
  // bf16 weights are read as they lie if their rows are whole stages
  p.copy_w = !(bf16 && a.w_col == 1 && a.d % kPadCols == 0 && a.w_row % 8 == 0 && a.w_row * 2 <= kT16MostBytes &&
               reinterpret_cast<uintptr_t>(a.w) % 16 == 0);
  p.grad = a.dx || a.dw || a.db;
  p.dw_rows = a.turned ? a.d : a.classes;
  p.dw_cols = a.turned ? a.classes : a.d;
  p.ld_dw = round_up(p.dw_cols, 4);
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t here = at;
    at += static_cast<size_t>(round_up(bytes, 256));
    return here;
  };
  if (plan_stream(a, bf16, &p)) {
    const int64_t pad = 16 * static_cast<int64_t>(p.row_blocks);
    p.stats = p.one_tile ? 0 : take(p.stream_chunks * pad * 8);
    p.label_logit = p.one_tile ? 0 : take(pad * 4);
    p.loss_rows = take(a.rows * 4);
    p.db = a.db && p.row_blocks > 1 ? take(p.row_blocks * round_up(a.classes, 4) * 4) : 0;
    p.dw_sums = a.dw && p.row_blocks > 1 ? take(p.row_blocks * p.dw_rows * p.ld_dw * 4) : 0;
    p.dx_sums = a.dx && p.stream_chunks > 1 ? take(p.stream_chunks * a.rows * round_up(a.d, 4) * 4) : 0;
    p.total = at;
    return p;
  }
  int64_t piece = kGradBytes / (p.pad_rows * 2 * p.es) / kPadRows * kPadRows;
  piece = piece < kPadRows ? kPadRows : (piece > p.pad_classes ? p.pad_classes : piece);
  p.pieces = tiles_of(p.pad_classes, piece);
  p.piece = round_up(tiles_of(p.pad_classes, p.pieces), kPadRows);
  p.pieces = tiles_of(p.pad_classes, p.piece);
  const int64_t of_piece = p.piece < a.classes ? p.piece : a.classes;
  (a.turned ? p.dw_cols : p.dw_rows) = of_piece;
  p.ld_dw = round_up(p.dw_cols, 4);
  // Large tiles of logits where there are enough, few of their rows are padding, and
  // rows or products many (256 / 64, us of the whole call: 4,000 x 64 x 10,000 bf16 82.6 /
  // 87.8, 8,192 x 1,024 x 2,048 164 / 201; but 300 x 100 x 50,000 75 / 66, 1,000 x 128 x
  // 20,000 71 / 69, 784 x 631 x 4,132 fp32, 68 tiles, 155 / 112)
  p.tile = tiles_of(a.rows, kLarge) * tiles_of(a.classes, kLarge) >= kComputeUnits / 2 &&
                   8 * a.rows >= 7 * p.pad_rows && (a.rows > 1024 || a.d >= 256)
               ? kLarge
               : kSmall;
  p.both = a.classes <= kSmall;
  if (p.both) p.tile = kSmall;
  // workgroups of a row tile: one for each CU (two for small tiles) where the
  // classes' tiles allow
  auto chunks = [&](int64_t classes) {
    const int64_t n = tiles_of(a.rows, p.tile), m = tiles_of(classes, p.tile);
    const int64_t want = (p.tile == kLarge ? 1 : 2) * kComputeUnits / n;
    return static_cast<int>(want < 1 ? 1 : (want > m ? m : want));
  };
  p.chunks = chunks(a.classes);
  p.piece_chunks = chunks(of_piece);
  plan_products(a, &p);
  p.dx_slab = p.dx_splits > 1 || p.pieces > 1;
  const int64_t x_bytes = p.pad_rows * p.pad_d * 2 * p.es;
  p.x_all = take(x_bytes);
  p.x_row = bf16 ? p.x_all : take(x_bytes);
  p.w = p.copy_w ? take(static_cast<int64_t>(a.classes) * p.pad_d * 2 * p.es) : 0;
  p.row_top = bf16 ? 0 : take(p.pad_rows * 4);
  p.tops = bf16 ? 0 : take(2 * kMostTops * 4);
  p.row_inverse = bf16 ? 0 : take(p.pad_rows * 4);
  p.inverses = bf16 ? 0 : take(8);
  p.labels = take(p.pad_rows * 4);
  p.stats = p.both ? 0 : take(p.chunks * p.pad_rows * 8);
  p.label_logit = p.both ? 0 : take(p.pad_rows * 4);
  p.loss_rows = take(p.pad_rows * 4);
  if (p.grad) {
    p.g = take(p.pad_rows * p.piece * 2 * p.es);
    p.db = a.db ? take(tiles_of(a.rows, p.tile) * p.piece * 4) : 0;
    p.dx_sums = a.dx && p.dx_slab ? take(p.dx_splits * a.rows * round_up(a.d, 4) * 4) : 0;
    p.dw_sums = a.dw && p.dw_splits > 1 ? take(p.dw_splits * p.dw_rows * p.ld_dw * 4) : 0;
  }
  // (a launch's threads fit 31 bits; else there is no plan: 0 bytes)
  const int64_t across = p.pad_d / 64, tile = p.product_tile;
  const int64_t laid_out = (p.pad_rows / 64 + (p.copy_w ? tiles_of(a.classes, 64) : 0)) * across;
  const int64_t products = tiles_of(a.d, tile) * (tiles_of(a.rows, tile) * p.dx_splits + tiles_of(of_piece, tile) * p.dw_splits);
  p.total = laid_out > kLaunchThreads / 256 || (p.grad && products + 16 > kLaunchThreads / 512) ? 0 : at;
  return p;
}

unsigned grid8(int64_t tiles) { return static_cast<unsigned>((tiles + 7) / 8 * 8); }

template <T16Type TYPE, LogitsMode MODE>
void launch_logits(const LogitsArgs& g, int tile, hipStream_t s) {
  const dim3 grid(grid8(static_cast<int64_t>(g.n_tiles) * g.chunks));
  if constexpr (MODE != kBoth) {
    if (tile == kLarge) {
      hipLaunchKernelGGL((k_logits<TYPE, MODE, kLarge, kLarge, 2, 4>), grid, dim3(512), 0, s, g);
      return;
    }
  }
  hipLaunchKernelGGL((k_logits<TYPE, MODE, kSmall, kSmall, 2, 2>), grid, dim3(256), 0, s, g);
}

JoinArgs join_of(const float* slab, int parts, int64_t rows, int64_t cols, int64_t ld_slab, float factor,
                 const float* inverse, void* out, int64_t ld) {
  const int64_t need = tiles_of(rows * tiles_of(cols, 4), join_columns(parts));
  return JoinArgs{slab, parts, rows, cols, ld_slab, factor, inverse, out, ld,
                  static_cast<int>(need < 8 * kComputeUnits ? need : 8 * kComputeUnits)};
}

template <bool BF16>
hipError_t finish(FinishArgs f, const LinearLossArgs& a, const float* loss_rows, hipStream_t s) {
  f.loss_rows = loss_rows;
  f.rows = a.rows;
  f.loss = a.loss;
  hipLaunchKernelGGL(k_finish<BF16>, dim3(static_cast<unsigned>(f.dx.blocks + f.dw.blocks + f.db.blocks + 1)), dim3(256), 0,
                     s, f);
  return hipGetLastError();
}

template <typename T>
hipError_t run_stream(const LinearLossArgs& a, const Plan& p, hipStream_t s) {
  auto floats = [&](size_t off) { return reinterpret_cast<float*>(a.ws + off); };
  const float mean = static_cast<float>(1.0 / static_cast<double>(a.rows));
  const int64_t ld_dx = round_up(a.d, 4);
  StreamArgs m{};
  m.x = a.x;
  m.x_stride = a.x_stride;
  m.w = a.w;
  m.w_row = a.w_row;
  m.w_col = a.w_col;
  m.bias = a.bias;
  m.labels = a.labels;
  m.rows = a.rows;
  m.d = a.d;
  m.classes = a.classes;
  m.tile = p.stream_tile;
  m.tiles = p.stream_tiles;
  m.row_blocks = p.row_blocks;
  m.chunks = p.stream_chunks;
  m.turned = a.turned;
  m.mean = mean;
  m.stats = reinterpret_cast<float2*>(a.ws + p.stats);
  m.label_logit = floats(p.label_logit);
  m.loss_rows = floats(p.loss_rows);
  m.grad = p.grad;
  m.dx_sums = p.stream_chunks > 1;
  m.dx = a.dx && m.dx_sums ? floats(p.dx_sums) : a.dx;
  m.ld_dx = m.dx_sums ? ld_dx : a.d;
  m.part_dx = a.rows * ld_dx;
  m.dw_sums = p.row_blocks > 1;
  m.dw = a.dw && m.dw_sums ? floats(p.dw_sums) : a.dw;
  m.db = a.db && m.dw_sums ? floats(p.db) : a.db;
  m.ld_dw = m.dw_sums ? p.ld_dw : p.dw_cols;
  m.part_dw = p.dw_rows * p.ld_dw;
  m.part_db = round_up(a.classes, 4);
  const dim3 grid(static_cast<unsigned>(p.row_blocks * p.stream_chunks)), threads(kStreamThreads);
  if (p.one_tile) {
    hipLaunchKernelGGL((k_stream_head<T, kBoth>), grid, threads, 0, s, m);
  } else {
    hipLaunchKernelGGL((k_stream_head<T, kStats>), grid, threads, 0, s, m);
    if (p.grad) hipLaunchKernelGGL((k_stream_head<T, kGrad>), grid, threads, 0, s, m);
    else
      hipLaunchKernelGGL(k_join_rows<16>, dim3(static_cast<unsigned>(p.row_blocks)), dim3(256), 0, s, m.stats, m.chunks,
                         a.rows, 16 * static_cast<int64_t>(p.row_blocks), a.labels, m.label_logit, m.loss_rows, a.classes);
  }
  FinishArgs f{};
  if (a.dx && m.dx_sums) f.dx = join_of(floats(p.dx_sums), m.chunks, a.rows, a.d, ld_dx, mean, nullptr, a.dx, a.d);
  if (a.dw && m.dw_sums)
    f.dw = join_of(floats(p.dw_sums), m.row_blocks, p.dw_rows, p.dw_cols, p.ld_dw, mean, nullptr, a.dw, p.dw_cols);
  if (a.db && m.dw_sums) f.db = join_of(floats(p.db), m.row_blocks, 1, a.classes, m.part_db, mean, nullptr, a.db, a.classes);
  return finish<sizeof(T) == 2>(f, a, m.loss_rows, s);
}

template <T16Type TYPE, typename T>
hipError_t run(const LinearLossArgs& a, hipStream_t s) {
  constexpr bool kLo = TYPE == kBf16;
  const Plan p = plan(a, kLo);
  if (p.row_blocks) return run_stream<T>(a, p, s);
  auto at = [&](size_t off) { return a.ws + off; };
  auto floats = [&](size_t off) { return reinterpret_cast<float*>(a.ws + off); };
  uint16_t* x_all = reinterpret_cast<uint16_t*>(at(p.x_all));
  uint16_t* x_row = reinterpret_cast<uint16_t*>(at(p.x_row));
  int32_t* labels = reinterpret_cast<int32_t*>(at(p.labels));
  float* inverses = kLo ? nullptr : floats(p.inverses);
  uint32_t* tops = kLo ? nullptr : reinterpret_cast<uint32_t*>(at(p.tops));
  int x_blocks = 0, w_blocks = 0;
  if constexpr (!kLo) {
    const bool w_rows = a.w_col == 1 || a.w_row != 1;    // W's rows are contiguous (or nothing is)
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
    if (m.w_col == 1 && m.w_stride == m.w_cols) {
      // one behind the other: in rows of 1,024 values, and the rest as one more
      const int64_t all = m.w_rows * m.w_cols;
      m.w_cols = static_cast<int>(all < 1024 ? all : 1024);
      m.w_stride = m.w_cols;
      m.w_rows = tiles_of(all, m.w_cols);
      m.w_all = all;
    }
    auto blocks = [](int64_t rows) { return static_cast<int>(rows < 4 * kMostTops ? (rows + 3) / 4 : kMostTops); };
    m.x_blocks = x_blocks = blocks(a.rows);
    m.w_blocks = w_blocks = blocks(m.w_rows);
    hipLaunchKernelGGL(k_amax, dim3(static_cast<unsigned>(x_blocks + w_blocks)), dim3(256), 0, s, m);
  }
  LayOutArgs l{}, lw{};
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
    l.row_inverse = floats(p.row_inverse);
    l.all_inverse = inverses;
  }
  T16Side w{static_cast<const uint16_t*>(a.w), a.w_row, a.classes, static_cast<int>(p.pad_d), 0};
  const int64_t across = p.pad_d / 64, x_tiles = p.pad_rows / 64 * across;
  int64_t w_tiles = 0;
  if (p.copy_w) {
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
    w_tiles = tiles_of(a.classes, 64) * across;
    w.data = lw.by_all;
    w.ld = p.pad_d * p.es;
  }
  hipLaunchKernelGGL((k_lay_out<TYPE, T>), dim3(static_cast<unsigned>(x_tiles + w_tiles)), dim3(256), 0, s, l, lw, x_tiles);
  const T16Side x_by_row{x_row, p.pad_d * p.es, p.pad_rows, static_cast<int>(p.pad_d), 0};
  const T16Side x_by_all{x_all, p.pad_d * p.es, p.pad_rows, static_cast<int>(p.pad_d), 0};
  LogitsArgs g{};
  g.w = w;
  g.x = x_by_row;
  g.d_values = static_cast<int>(p.pad_d);
  g.m_tiles = static_cast<int>(tiles_of(a.classes, p.tile));
  g.n_tiles = static_cast<int>(tiles_of(a.rows, p.tile));
  g.chunks = p.chunks;
  g.classes = a.classes;
  g.bias = a.bias;
  g.row_inverse = kLo ? nullptr : floats(p.row_inverse);
  g.w_inverse = kLo ? nullptr : inverses + 1;
  g.labels = labels;
  g.rows = a.rows;
  g.pad_rows = p.pad_rows;
  g.stats = reinterpret_cast<float2*>(at(p.stats));
  g.stat_chunks = p.chunks;
  g.label_logit = floats(p.label_logit);
  g.loss_rows = floats(p.loss_rows);
  g.g = p.grad ? reinterpret_cast<uint16_t*>(at(p.g)) : nullptr;
  g.ldg = p.piece * p.es;
  g.ld_db = p.piece;
  if (!p.both) {
    launch_logits<TYPE, kStats>(g, p.tile, s);
    if (!p.grad) {
      const auto join = p.tile == kLarge ? k_join_rows<2> : k_join_rows<4>;
      hipLaunchKernelGGL(join, dim3(static_cast<unsigned>(p.pad_rows / (p.tile == kLarge ? 128 : 64))), dim3(256), 0, s,
                         g.stats, p.chunks, a.rows, p.pad_rows, labels, g.label_logit, g.loss_rows, a.classes);
    }
  }
  const float mean = static_cast<float>((kLo ? 1.0 : 1.0 / kGradScale) / static_cast<double>(a.rows));
  const float mean_db = static_cast<float>(1.0 / static_cast<double>(a.rows));
  const int64_t ld_dx = round_up(a.d, 4);
  const float* w_inverse = kLo ? nullptr : inverses + 1;
  FinishArgs f{};
  for (int64_t c0 = 0; c0 < a.classes && (p.grad || p.both); c0 += p.piece) {
    const int64_t left = a.classes - c0, have = left < p.piece ? left : p.piece;
    g.c0 = static_cast<int>(c0);
    // (so G's padding is written as far as a stage of dx's product reads)
    g.m_tiles = static_cast<int>(tiles_of(have, p.tile));
    g.chunks = p.piece_chunks < g.m_tiles ? p.piece_chunks : g.m_tiles;
    g.db = a.db ? floats(p.db) : nullptr;
    if (p.both) launch_logits<TYPE, kBoth>(g, p.tile, s);
    else launch_logits<TYPE, kGrad>(g, p.tile, s);
    g.loss_rows = nullptr;
    if (a.db) f.db = join_of(floats(p.db), g.n_tiles, 1, have, p.piece, mean_db, nullptr, a.db + c0, have);
    if (a.dx || a.dw) {
      const T16Side grad{g.g, g.ldg, round_up(a.rows, p.tile), static_cast<int>(p.piece), 0};
      const int tile = p.product_tile;
      Product dx{}, dw{};
      if (a.dx) {
        dx.a = w;
        dx.a.data = w.data + c0 * w.ld;
        dx.a.rows = left;
        dx.b = grad;
        dx.m = a.d;
        dx.n = a.rows;
        dx.m_tiles = static_cast<int>(tiles_of(a.d, tile));
        dx.n_tiles = static_cast<int>(tiles_of(a.rows, tile));
        dx.splits = p.dx_splits;
        dx.k = have;
        dx.factor = mean;
        dx.inverse = w_inverse;
        dx.out = p.dx_slab ? nullptr : a.dx;
        dx.ld = a.d;
        dx.slab = floats(p.dx_sums);
        dx.ld_slab = ld_dx;
        dx.more = c0 > 0;
      }
      if (a.dw) {
        T* out = static_cast<T*>(a.dw) + (a.turned ? c0 : c0 * a.d);
        dw.a = a.turned ? grad : x_by_all;
        dw.b = a.turned ? x_by_all : grad;
        dw.a.rows = dw.b.rows = grad.rows;
        dw.m = a.turned ? have : a.d;
        dw.n = a.turned ? a.d : have;
        dw.m_tiles = static_cast<int>(tiles_of(dw.m, tile));
        dw.n_tiles = static_cast<int>(tiles_of(dw.n, tile));
        dw.splits = p.dw_splits;
        dw.k = a.rows;
        dw.factor = mean;
        dw.inverse = kLo ? nullptr : inverses;
        dw.ld = a.turned ? a.classes : a.d;
        dw.ld_slab = p.ld_dw;
        dw.part = dw.n * dw.ld_slab;
        if (p.dw_splits > 1) {
          dw.slab = floats(p.dw_sums);
          f.dw = join_of(dw.slab, p.dw_splits, dw.n, dw.m, p.ld_dw, mean, dw.inverse, out, dw.ld);
        } else {
          dw.out = out;
        }
      }
      dx.part = dx.n * dx.ld_slab;
      const int64_t tiles = round_up(product_tiles(dx), 8) + round_up(product_tiles(dw), 8);
      if (tile == kLarge) hipLaunchKernelGGL((k_products<TYPE, kLarge, kLarge, 2, 4>), dim3(grid8(tiles)), dim3(512), 0, s, dx, dw);
      else hipLaunchKernelGGL((k_products<TYPE, kSmall, kSmall, 2, 2>), dim3(grid8(tiles)), dim3(256), 0, s, dx, dw);
    }
    if (c0 + p.piece < a.classes && f.dw.blocks + f.db.blocks > 0) {
      hipLaunchKernelGGL(k_join_piece<kLo>, dim3(static_cast<unsigned>(f.dw.blocks + f.db.blocks)), dim3(256), 0, s, f.dw, f.db);
      f.dw = f.db = JoinArgs{};
    }
  }
  if (a.dx && p.dx_slab) f.dx = join_of(floats(p.dx_sums), p.dx_splits, a.rows, a.d, ld_dx, mean, w_inverse, a.dx, a.d);
  return finish<kLo>(f, a, floats(p.loss_rows), s);
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
