// Host-side launchers of the microscaled store, its mean and product
// (mx_store.hip, mx_linear.hip) and of the distillation loss (distill.hip);
// called by the C ABI in api_mx.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gmb.h"

namespace gmb {

// What a launcher writes: fp32 rows, bf16 rows, or 4-bit records.
constexpr int kMxOutF32 = 0, kMxOutBf16 = 1, kMxOutRecords = 2;

// Outputs of at least this many bytes are stored past the caches: the L2s (32
// MB together) could not keep them for a reader, and writing them there costs
// what it evicts.  Plain against streaming stores: reads of the store, 16 MB of
// fp32 rows 6.4 / 6.2 us, 64 MB 20.4 / 16.8, 138 MB 42.1 / 33.2, 205 MB 61.0 / 48.2;
// the linear layer, 23 MB 12.4 / 10.4, 56 MB 30.9 / 25.2, 102 MB 64.4 / 51.5;
// means (25 neighbours of 500), 120 MB 184 / 183.  Smaller ones stay where the next
// kernel finds them.  (The linear layer has a further condition.)
constexpr int64_t kStreamBytes = 16 << 20;

// Threads of one launch: a grid counts them in 32 bits.
constexpr int64_t kLaunchThreads = int64_t{1} << 31;

inline int64_t mx_blocks(int64_t dim) { return (dim + 31) / 32; }
inline int64_t mx_record(int64_t dim, int bits) {
  return (mx_blocks(dim) * (4 * bits + 1) + 15) / 16 * 16;
}

struct MxWriteArgs {
  const void* x;
  int64_t row_stride, col_stride;   // in elements
  const int32_t* n_dev;
  int64_t n_cap;
  int dim, blocks, record;
  const int32_t* ids;               // or NULL: row i is record i
  uint8_t* table;
  int64_t table_rows, table_stride;
  uint32_t* status;
  const uint32_t* slots;            // set by the launcher
};

struct MxReadArgs {
  const int32_t* ids;
  const int32_t* n_dev;
  int64_t n_cap;
  int dim, blocks;
  const uint8_t* table;
  int64_t table_rows, table_stride;
  void* out;
  uint32_t* status;
};

struct MxMeanArgs {
  const int32_t* indptr;
  const int32_t* ids;
  const int32_t* n_dev;
  int64_t n_cap;
  int dim, blocks;
  const uint8_t* table;
  int64_t table_rows, table_stride;
  void* out;
  int64_t out_stride;               // records: bytes
  int out_record;
  uint32_t* status;                 // or NULL: not told of an id outside the table
  int64_t row0;                     // set by the launcher: the launch's first row
};

// slots: the sampler state's table (the last row written to a vertex wins),
// or NULL (the ids are distinct)
hipError_t launch_mx_write(const MxWriteArgs& a, int bf16, int bits, uint32_t* slots, hipStream_t s);
hipError_t launch_mx_read(const MxReadArgs& a, int bf16, int bits, hipStream_t s);
hipError_t launch_mx_mean(const MxMeanArgs& a, int bf16, int bits, hipStream_t s);
// 4 bits to 4 bits
hipError_t launch_mx_mean_records(const MxMeanArgs& a, hipStream_t s);

// One pair of a product: rows of `a` (row ids[i] of rows `a_rows`, or row i)
// by the records of `w`.
struct MxPair {
  const uint8_t* a;
  int64_t a_rows, a_stride;
  const int32_t* ids;
  const uint8_t* w;
  int64_t w_stride;
};
struct MxLinearArgs {
  MxPair pair[2];
  int pairs;
  const int32_t* n_dev;
  int64_t n_cap;
  int d_in, blocks, d_out;
  const float* bias;                // or NULL
  int relu;
  void* out;
  int64_t out_stride;               // records: bytes
  int out_record;
  uint32_t* status;
};
hipError_t launch_mx_linear(const MxLinearArgs& a, int out, hipStream_t s);

// ---- distillation ---------------------------------------------------------

struct DistillArgs {
  const void* logits;
  int64_t rows;
  int classes;
  const float* top;
  const int32_t* top_ids;
  int k;
  const int32_t* labels;            // or NULL
  float alpha, temperature;
  void* grad;                       // or NULL
  int64_t ld_grad;                  // its row stride; columns classes .. ld_grad - 1 become 0
  float* loss_rows;                 // [rows]
  float* stats;                     // shared rows' statistics, 3 words a row and part, or NULL
  int parts;                        // workgroups of a row, with stats
  int32_t* clear;                   // cleared by the launch, clear_n words
  int64_t clear_n;
  int64_t row0;                     // set by the launcher: the launch's first row
};
// Classes that a launch without stats can hold.
constexpr int kDistillHeld = 32768;
// Workgroups that share a row (0: none do, the row is held and no stats are needed).
int distill_parts(int64_t rows, int64_t classes);
hipError_t launch_distill(const DistillArgs& a, int bf16, hipStream_t s);
// *loss = (1 / rows) sum of loss_rows, in a fixed order
hipError_t launch_loss_mean(const float* loss_rows, int64_t rows, float* loss, hipStream_t s);

}  // namespace gmb
