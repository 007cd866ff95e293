// What the ABI's translation units (api.hip, api_mx.hip) share.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "gmb.h"

namespace gmb {

constexpr size_t kAbiAlign = 256;
constexpr size_t kAbiStateHeader = 256;   // sampler state: header, then one slot per vertex

// Sets the thread's error message and returns `status`.
int abi_fail(int status, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int abi_check_blocks(const gmb_blocks* b);

// The loss that a backward starts from: writes dZ [num_seeds, ldz] of the
// last layer (columns past the classes 0) and the rows' loss terms, and
// clears clear[0 .. clear_n).
struct LossLaunch {
  hipError_t (*launch)(const void* what, float* dz, int ldz, float* loss_rows, int32_t* clear, int64_t clear_n,
                       hipStream_t s);
  const void* what;
};

// gmb_sage_backward (table NULL) or gmb_sage_backward_embedding with that
// loss.
int abi_backward_from(const LossLaunch& how, const gmb_blocks* blocks, const void* x,
                      const gmb_sage_weights* weights, const float* logits, const void* fwd_ws, size_t fwd_ws_bytes,
                      const gmb_sage_grads* grads, float* loss, void* ws, size_t ws_bytes, float* table,
                      int64_t num_nodes, float emb_lr, void* stream);

// What is done to a hidden layer's output `rows` (the first *blk.sizes[0] of
// blk.cap_dst rows of `dim`) before the next layer reads it.
struct HiddenLaunch {
  hipError_t (*launch)(const void* what, int layer, const gmb_block& blk, void* rows, int dim, int bf16,
                       hipStream_t s);
  const void* what;
};

// gmb_sage_forward (feats NULL) or gmb_sage_forward_fused (x: its x_dst) with
// that.
int abi_forward_with(const HiddenLaunch& then, const gmb_blocks* blocks, void* x, const void* feats, int64_t num_nodes,
                     const gmb_sage_weights* weights, float* logits, void* ws, size_t ws_bytes, uint32_t* status,
                     void* stream);

}  // namespace gmb
