// Host-side launchers of the row operators (rows.hip: dropout and the
// root-mean-square norm) and of the cross-entropy over many classes
// (linear_loss.hip); called by the C ABI in api_head.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gmb.h"

namespace gmb {

// Rows in memory: `stride` in elements (records: bytes).
struct RowsIn {
  const void* data;
  int64_t stride;
};
struct RowsOut {
  void* data;
  int64_t stride;
};

// A dropout as the kernels take it: an element is dropped where its 16 bits
// are below `below` (0: none is), the others are scaled.
struct DropArgs {
  uint32_t below;
  float scale;
  uint32_t k0, k1, layer;
  const uint32_t* step;             // or NULL: 0
  const int32_t* ids;               // the rows' keys, or NULL: their positions
};

// round(65536 p), and what kept elements are scaled by (0 if there are none).
inline uint32_t drop_below(float p) { return static_cast<uint32_t>(65536.0 * p + 0.5); }
inline float drop_scale(uint32_t below) {
  return below >= 65536u ? 0.f : static_cast<float>(65536.0 / (65536.0 - below));
}

struct DropoutArgs {
  RowsIn x, residual;               // residual.data may be NULL
  RowsOut out;
  DropArgs drop;
  const int32_t* n_dev;
  int64_t n_cap;
  int dim;
};
hipError_t launch_dropout(const DropoutArgs& a, int bf16, hipStream_t s);

struct NormArgs {
  RowsIn x, residual;               // residual.data may be NULL
  DropArgs drop;
  const int32_t* n_dev;
  int64_t n_cap;
  int dim;
  const float* weight;              // or NULL: ones
  float eps;
  RowsOut sum;                      // data may be NULL
  RowsOut out;
  int record;                       // bytes of a record
};
// bits: 0 (rows of the inputs' type), 4 or 8 (records)
hipError_t launch_rms_norm(const NormArgs& a, int bf16, int bits, hipStream_t s);

struct NormBackArgs {
  RowsIn dy, r, carry;              // carry.data may be NULL
  DropArgs drop;
  const int32_t* n_dev;
  int64_t n_cap;
  int dim;
  const float* weight;              // or NULL: ones
  float eps;
  RowsOut d_residual, dx;           // data may be NULL
  float* d_weight;                  // or NULL
  float* partial;                   // [norm_back_parts][dim], with d_weight
};
// Workgroups of the backward, each with a row of partial sums of d_weight.
int norm_back_parts(int64_t n_cap, int dim);
hipError_t launch_rms_norm_backward(const NormBackArgs& a, int bf16, hipStream_t s);

// ---- the cross-entropy over many classes ----------------------------------

struct LinearLossArgs {
  const void* x;                    // [rows, d] at x_stride
  int64_t x_stride;
  const void* w;                    // element j of class c at c w_row + j w_col
  int64_t w_row, w_col;
  const float* bias;                // or NULL
  const int32_t* labels;
  int64_t rows;
  int d, classes;
  void* dx;                         // [rows, d], or NULL
  void* dw;                         // [classes, d], turned: [d, classes], or NULL
  int turned;
  float* db;                        // or NULL
  float* loss;
  char* ws;
};
constexpr int64_t kLinearLossRows = int64_t{1} << 22;
// Bytes of workspace; grads: dx, dw and db are looked at for being NULL only.
size_t linear_loss_bytes(const LinearLossArgs& a, int bf16);
hipError_t launch_linear_loss(const LinearLossArgs& a, int bf16, hipStream_t s);

// w[t][0 .. n[t]) *= by[t]
struct ScaleArgs {
  int count;
  float* w[3 * GMB_MAX_LAYERS];
  int64_t n[3 * GMB_MAX_LAYERS];
  float by[3 * GMB_MAX_LAYERS];
};
hipError_t launch_scale(const ScaleArgs& a, hipStream_t s);
// dz[i, 0 .. cols) = from[i, :], dz[i, cols .. ldz) = 0; clear[0 .. clear_n) = 0
hipError_t launch_given_gradient(const float* from, int64_t rows, int cols, float* dz, int ldz, int32_t* clear,
                                 int64_t clear_n, hipStream_t s);

}  // namespace gmb
