// C ABI of dropout, the root-mean-square norm and the cross-entropy over many
// classes (declared in include/gmb.h): argument validation, workspace planning
// and kernel launches.  No C++ exception crosses the ABI; every entry point
// returns a gmb_status.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "api_common.hpp"
#include "gmb.h"
#include "head_kernels.hpp"
#include "kernels.hpp"
#include "mx_kernels.hpp"

namespace {

using gmb::abi_fail;

constexpr int64_t kMaxInt32 = 0x7FFFFFFF;
constexpr int32_t kMaxDim = 65536, kMaxClasses = 1 << 27;

int hip_fail(hipError_t e, const char* what) { return abi_fail(GMB_EDEVICE, "%s: %s", what, hipGetErrorString(e)); }
hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }

int check_dtype(int32_t dtype) {
  if (dtype != GMB_F32 && dtype != GMB_BF16) return abi_fail(GMB_EINVAL, "dtype=%d unknown", dtype);
  return GMB_OK;
}

int check_shape(int64_t n_cap, int32_t dim) {
  if (dim < 1 || dim > kMaxDim) return abi_fail(GMB_EINVAL, "dim=%d outside 1..%d", dim, kMaxDim);
  if (n_cap < 0 || n_cap > kMaxInt32)
    return abi_fail(GMB_EINVAL, "n_cap=%lld outside 0..2^31-1", static_cast<long long>(n_cap));
  return GMB_OK;
}

// Rows that have to be there (`need`), or may be NULL.
int check_rows(const gmb_rows* r, int32_t dim, bool need, const char* what) {
  if (!r) return need ? abi_fail(GMB_EINVAL, "%s is NULL", what) : GMB_OK;
  if (!r->data) return abi_fail(GMB_EINVAL, "%s: data is NULL", what);
  if (r->stride < dim)
    return abi_fail(GMB_EINVAL, "%s: stride %lld below dim=%d", what, static_cast<long long>(r->stride), dim);
  return GMB_OK;
}

// An output that starts where an input does has to have its rows there too.
int check_in_place(const gmb_rows* out, const gmb_rows* in, const char* what) {
  if (out && in && out->data == in->data && out->stride != in->stride)
    return abi_fail(GMB_EINVAL, "%s in place with another stride", what);
  return GMB_OK;
}

gmb::RowsIn rows_in(const gmb_rows* r) { return r ? gmb::RowsIn{r->data, r->stride} : gmb::RowsIn{nullptr, 0}; }
gmb::RowsOut rows_out(const gmb_rows* r) { return r ? gmb::RowsOut{r->data, r->stride} : gmb::RowsOut{nullptr, 0}; }

// (the kernels' root takes normal numbers)
int check_eps(float eps) {
  if (!(eps >= 1.17549435e-38f) || eps > 3.0e38f)
    return abi_fail(GMB_EINVAL, "eps=%g is no positive normal number", static_cast<double>(eps));
  return GMB_OK;
}

int check_head(const gmb_linear_head* h) {
  if (!h) return abi_fail(GMB_EINVAL, "head is NULL");
  int st = check_dtype(h->dtype);
  if (st != GMB_OK) return st;
  if (h->rows < 0 || h->rows > gmb::kLinearLossRows)
    return abi_fail(GMB_EINVAL, "rows=%lld outside 0..2^22", static_cast<long long>(h->rows));
  if (h->d < 1 || h->d > kMaxDim) return abi_fail(GMB_EINVAL, "d=%d outside 1..%d", h->d, kMaxDim);
  if (h->classes < 1 || h->classes > kMaxClasses)
    return abi_fail(GMB_EINVAL, "classes=%d outside 1..2^27", h->classes);
  if (h->rows > 0 && h->x_stride < h->d)
    return abi_fail(GMB_EINVAL, "x_stride=%lld below d=%d", static_cast<long long>(h->x_stride), h->d);
  if (h->w_row_stride < 0 || h->w_col_stride < 0) return abi_fail(GMB_EINVAL, "a negative stride");
  return GMB_OK;
}

gmb::LinearLossArgs head_args(const gmb_linear_head* h, const gmb_linear_grads* g) {
  gmb::LinearLossArgs a{};
  a.x = h->x;
  a.x_stride = h->x_stride;
  a.w = h->w;
  // (the stride along an extent of one says nothing)
  a.w_row = h->classes == 1 ? h->d : h->w_row_stride;
  a.w_col = h->d == 1 ? 1 : h->w_col_stride;
  a.bias = h->bias;
  a.labels = h->labels;
  a.rows = h->rows;
  a.d = h->d;
  a.classes = h->classes;
  if (g) {
    a.dx = g->dx;
    a.dw = g->dw;
    a.db = g->dbias;
    a.turned = g->turned != 0;
  }
  return a;
}

int check_dropout(const gmb_dropout* d) {
  if (!d) return abi_fail(GMB_EINVAL, "dropout is NULL");
  if (!(d->p >= 0.f && d->p <= 1.f)) return abi_fail(GMB_EINVAL, "p=%g outside 0..1", static_cast<double>(d->p));
  if (d->layer < 0) return abi_fail(GMB_EINVAL, "layer=%d is negative", d->layer);
  return GMB_OK;
}

// As the kernels take it (NULL: nothing is dropped).
gmb::DropArgs drop_args(const gmb_dropout* d, const int32_t* ids) {
  gmb::DropArgs a{};
  if (!d) return a;
  a.below = gmb::drop_below(d->p);
  a.scale = gmb::drop_scale(a.below);
  a.k0 = static_cast<uint32_t>(d->seed);
  a.k1 = static_cast<uint32_t>(d->seed >> 32);
  a.layer = static_cast<uint32_t>(d->layer);
  a.step = d->step;
  a.ids = ids;
  return a;
}

// The dropout of layer `layer`'s output, in place, by vertex.  (A bf16 model's rows
// are rounded as the layer stores them and again here, half a step each: the
// layers' kernels stay without dropout.  At p = 1/2 the factor is 2 and exact.)
hipError_t drop_hidden(const void* what, int layer, const gmb_block& blk, void* rows, int dim, int bf16,
                       hipStream_t s) {
  gmb::DropoutArgs a{};
  a.x = {rows, dim};
  a.out = {rows, dim};
  a.drop = drop_args(static_cast<const gmb_dropout*>(what), blk.src_ids);   // (the first sources are the destinations)
  a.drop.layer += static_cast<uint32_t>(layer);
  a.n_dev = blk.sizes + gmb::kNDst;
  a.n_cap = blk.cap_dst;
  a.dim = dim;
  return gmb::launch_dropout(a, bf16, s);
}

// The "loss" of gmb_sage_backward_from: the gradient that the caller has.
struct GivenGradient {
  const float* d_logits;
  int64_t rows;
  int cols;
};
hipError_t given_gradient(const void* what, float* dz, int ldz, float*, int32_t* clear, int64_t clear_n,
                          hipStream_t s) {
  const GivenGradient& g = *static_cast<const GivenGradient*>(what);
  return gmb::launch_given_gradient(g.d_logits, g.rows, g.cols, dz, ldz, clear, clear_n, s);
}

}  // namespace

extern "C" {

int gmb_dropout_rows(const gmb_rows* x, const gmb_rows* residual, const gmb_dropout* drop, const int32_t* ids,
                     const int32_t* n_dev, int64_t n_cap, int32_t dim, int32_t dtype, const gmb_rows* out,
                     void* stream) {
  int st = check_shape(n_cap, dim);
  if (st == GMB_OK) st = check_dtype(dtype);
  if (st == GMB_OK) st = check_dropout(drop);
  if (st != GMB_OK) return st;
  if (n_cap == 0) return GMB_OK;
  st = check_rows(x, dim, true, "x");
  if (st == GMB_OK) st = check_rows(residual, dim, false, "residual");
  if (st == GMB_OK) st = check_rows(out, dim, true, "out");
  if (st == GMB_OK) st = check_in_place(out, x, "out");
  if (st == GMB_OK) st = check_in_place(out, residual, "out");
  if (st != GMB_OK) return st;
  gmb::DropoutArgs a{};
  a.x = rows_in(x);
  a.residual = rows_in(residual);
  a.out = rows_out(out);
  a.drop = drop_args(drop, ids);
  a.n_dev = n_dev;
  a.n_cap = n_cap;
  a.dim = dim;
  const hipError_t e = gmb::launch_dropout(a, dtype == GMB_BF16, as_stream(stream));
  if (e != hipSuccess) return hip_fail(e, "dropout launch");
  return GMB_OK;
}

int gmb_rms_norm(const gmb_rows* x, const gmb_rows* residual, const gmb_dropout* drop, const int32_t* ids,
                 const int32_t* n_dev, int64_t n_cap, int32_t dim, int32_t dtype, const float* weight, float eps,
                 const gmb_rows* sum, int32_t format, const gmb_rows* out, void* stream) {
  int st = check_shape(n_cap, dim);
  if (st == GMB_OK) st = check_dtype(dtype);
  if (st == GMB_OK) st = check_eps(eps);
  if (st == GMB_OK && drop) st = check_dropout(drop);
  if (st != GMB_OK) return st;
  if (format != 0 && format != GMB_MXFP4 && format != GMB_MXFP8) return abi_fail(GMB_EINVAL, "format=%d unknown", format);
  if (n_cap == 0) return GMB_OK;
  st = check_rows(x, dim, true, "x");
  if (st == GMB_OK) st = check_rows(residual, dim, false, "residual");
  if (st == GMB_OK) st = check_rows(sum, dim, false, "sum");
  if (st == GMB_OK) st = check_rows(out, format ? 0 : dim, true, "out");
  if (st == GMB_OK) st = check_in_place(sum, x, "sum");
  if (st == GMB_OK) st = check_in_place(sum, residual, "sum");
  if (st != GMB_OK) return st;
  gmb::NormArgs a{};
  if (format == 0) {
    st = check_in_place(out, x, "out");
    if (st == GMB_OK) st = check_in_place(out, residual, "out");
    if (st != GMB_OK) return st;
  } else {
    a.record = static_cast<int>(gmb::mx_record(dim, format));
    if (reinterpret_cast<uintptr_t>(out->data) % 16 || out->stride % 16)
      return abi_fail(GMB_EINVAL, "out: the address and the row stride of records must be multiples of 16 bytes");
    if (out->stride < a.record)
      return abi_fail(GMB_EINVAL, "out: row stride %lld below the record's %d bytes",
                      static_cast<long long>(out->stride), a.record);
    if (out->data == x->data || (residual && out->data == residual->data))
      return abi_fail(GMB_EINVAL, "records in place of rows");
  }
  if (sum && sum->data == out->data) return abi_fail(GMB_EINVAL, "sum and out are the same rows");
  a.x = rows_in(x);
  a.residual = rows_in(residual);
  a.drop = drop_args(drop, ids);
  a.n_dev = n_dev;
  a.n_cap = n_cap;
  a.dim = dim;
  a.weight = weight;
  a.eps = eps;
  a.sum = rows_out(sum);
  a.out = rows_out(out);
  const hipError_t e = gmb::launch_rms_norm(a, dtype == GMB_BF16, format, as_stream(stream));
  if (e != hipSuccess) return hip_fail(e, "norm launch");
  return GMB_OK;
}

size_t gmb_rms_norm_workspace_bytes(int64_t n_cap, int32_t dim) {
  if (check_shape(n_cap, dim) != GMB_OK) return 0;
  return static_cast<size_t>(gmb::norm_back_parts(std::max<int64_t>(n_cap, 1), dim)) * dim * 4;
}

int gmb_rms_norm_backward(const gmb_rows* dy, const gmb_rows* r, const gmb_rows* carry, const gmb_dropout* drop,
                          const int32_t* ids, const int32_t* n_dev, int64_t n_cap, int32_t dim, int32_t dtype,
                          const float* weight, float eps, const gmb_rows* d_residual, const gmb_rows* dx,
                          float* d_weight, void* ws, size_t ws_bytes, void* stream) {
  int st = check_shape(n_cap, dim);
  if (st == GMB_OK) st = check_dtype(dtype);
  if (st == GMB_OK) st = check_eps(eps);
  if (st == GMB_OK && drop) st = check_dropout(drop);
  if (st != GMB_OK) return st;
  if (n_cap == 0) {   // a sum over no rows
    if (!d_weight) return GMB_OK;
    gmb::SgdArgs z{};
    z.w[0] = d_weight;
    z.n[0] = dim;
    z.count = 1;
    const hipError_t e = gmb::launch_zero(z, nullptr, as_stream(stream));
    if (e != hipSuccess) return hip_fail(e, "zero-fill launch");
    return GMB_OK;
  }
  st = check_rows(dy, dim, true, "dy");
  if (st == GMB_OK) st = check_rows(r, dim, true, "r");
  if (st == GMB_OK) st = check_rows(carry, dim, false, "carry");
  if (st == GMB_OK) st = check_rows(d_residual, dim, false, "d_residual");
  if (st == GMB_OK) st = check_rows(dx, dim, false, "dx");
  const gmb_rows* in[] = {dy, r, carry};
  for (const gmb_rows* i : in) {
    if (st == GMB_OK) st = check_in_place(d_residual, i, "d_residual");
    if (st == GMB_OK) st = check_in_place(dx, i, "dx");
  }
  if (st != GMB_OK) return st;
  if (dx && d_residual && dx->data == d_residual->data)
    return abi_fail(GMB_EINVAL, "dx and d_residual are the same rows");
  gmb::NormBackArgs a{};
  if (d_weight) {
    if (!ws) return abi_fail(GMB_EINVAL, "workspace is NULL");
    if (reinterpret_cast<uintptr_t>(ws) % gmb::kAbiAlign)
      return abi_fail(GMB_EINVAL, "workspace is not 256-byte aligned");
    const size_t need = gmb_rms_norm_workspace_bytes(n_cap, dim);
    if (ws_bytes < need) return abi_fail(GMB_ENOSPC, "workspace holds %zu bytes, %zu needed", ws_bytes, need);
  }
  a.dy = rows_in(dy);
  a.r = rows_in(r);
  a.carry = rows_in(carry);
  a.drop = drop_args(drop, ids);
  a.n_dev = n_dev;
  a.n_cap = n_cap;
  a.dim = dim;
  a.weight = weight;
  a.eps = eps;
  a.d_residual = rows_out(d_residual);
  a.dx = rows_out(dx);
  a.d_weight = d_weight;
  a.partial = static_cast<float*>(ws);
  const hipError_t e = gmb::launch_rms_norm_backward(a, dtype == GMB_BF16, as_stream(stream));
  if (e != hipSuccess) return hip_fail(e, "norm backward launch");
  return GMB_OK;
}

size_t gmb_linear_loss_workspace_bytes(const gmb_linear_head* head, const gmb_linear_grads* grads) {
  if (check_head(head) != GMB_OK) return 0;
  gmb::LinearLossArgs a = head_args(head, grads);
  a.rows = std::max<int64_t>(a.rows, 1);
  return gmb::linear_loss_bytes(a, head->dtype == GMB_BF16);
}

int gmb_linear_loss(const gmb_linear_head* head, const gmb_linear_grads* grads, float* loss, void* ws,
                    size_t ws_bytes, void* stream) {
  const int st = check_head(head);
  if (st != GMB_OK) return st;
  if (!loss) return abi_fail(GMB_EINVAL, "loss is NULL");
  gmb::LinearLossArgs a = head_args(head, grads);
  a.loss = loss;
  const int bf16 = head->dtype == GMB_BF16;
  if (a.rows > 0) {
    if (!a.x || !a.w || !a.labels) return abi_fail(GMB_EINVAL, "x, w or labels is NULL");
    // the gradients apart from what they are computed from
    const uintptr_t es = bf16 ? 2 : 4, d = static_cast<uintptr_t>(a.d), c = static_cast<uintptr_t>(a.classes);
    const uintptr_t n = static_cast<uintptr_t>(a.rows);
    const auto at = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
    struct Span { uintptr_t first, bytes; };
    const Span in[] = {{at(a.x), ((n - 1) * a.x_stride + d) * es},
                       {at(a.w), ((c - 1) * a.w_row + (d - 1) * a.w_col + 1) * es},
                       {at(a.bias), a.bias ? c * 4 : 0},
                       {at(a.labels), n * 4}};
    const Span out[] = {{at(a.dx), a.dx ? n * d * es : 0}, {at(a.dw), a.dw ? c * d * es : 0}, {at(a.db), a.db ? c * 4 : 0}};
    for (const Span& o : out)
      for (const Span& i : in)
        if (o.bytes && i.bytes && o.first < i.first + i.bytes && i.first < o.first + o.bytes)
          return abi_fail(GMB_EINVAL, "a gradient overlaps an input");
    if (!ws) return abi_fail(GMB_EINVAL, "workspace is NULL");
    if (reinterpret_cast<uintptr_t>(ws) % gmb::kAbiAlign)
      return abi_fail(GMB_EINVAL, "workspace is not 256-byte aligned");
    const size_t need = gmb_linear_loss_workspace_bytes(head, grads);
    if (!need)
      return abi_fail(GMB_EINVAL, "rows=%lld, d=%d and classes=%d are too many together", static_cast<long long>(a.rows),
                      a.d, a.classes);
    if (ws_bytes < need) return abi_fail(GMB_ENOSPC, "workspace holds %zu bytes, %zu needed", ws_bytes, need);
    a.ws = static_cast<char*>(ws);
  }
  const hipError_t e = gmb::launch_linear_loss(a, bf16, as_stream(stream));
  if (e != hipSuccess) return hip_fail(e, "linear loss launch");
  return GMB_OK;
}

int gmb_sage_forward_dropout(const gmb_blocks* blocks, void* x, const void* feats, int64_t num_nodes,
                             const gmb_sage_weights* weights, const gmb_dropout* drop, float* logits, void* ws,
                             size_t ws_bytes, uint32_t* status, void* stream) {
  const int st = check_dropout(drop);
  if (st != GMB_OK) return st;
  if (drop->layer > kMaxInt32 - GMB_MAX_LAYERS)
    return abi_fail(GMB_EINVAL, "layer=%d leaves no room for the model's", drop->layer);
  return gmb::abi_forward_with({drop_hidden, drop}, blocks, x, feats, num_nodes, weights, logits, ws, ws_bytes, status,
                               stream);
}

int gmb_sage_backward_from(const gmb_blocks* blocks, const void* x, const gmb_sage_weights* weights,
                           const float* d_logits, const gmb_dropout* drop, const void* fwd_ws, size_t fwd_ws_bytes,
                           const gmb_sage_grads* grads, void* ws, size_t ws_bytes, float* table, int64_t num_nodes,
                           float emb_lr, void* stream) {
  int st = gmb::abi_check_blocks(blocks);
  if (st == GMB_OK && drop) st = check_dropout(drop);
  if (st != GMB_OK) return st;
  if (!weights) return abi_fail(GMB_EINVAL, "weights is NULL");
  if (weights->num_layers != blocks->num_layers)
    return abi_fail(GMB_EINVAL, "weights have %d layers, blocks %d", weights->num_layers, blocks->num_layers);
  if (table) {
    if (num_nodes < 1 || num_nodes > kMaxInt32)
      return abi_fail(GMB_EINVAL, "num_nodes=%lld outside 1..2^31-1", static_cast<long long>(num_nodes));
    if (reinterpret_cast<uintptr_t>(table) % 16) return abi_fail(GMB_EINVAL, "table must be 16-byte aligned");
  }
  // A dropped hidden value is 0, so the backward's mask (outputs above 0) stops
  // its gradient already; what passes lacks the dropout's factor once for every
  // hidden layer above, which a layer's gradients (and the embeddings' step)
  // take at the end: they are linear in it.
  const int L = weights->num_layers;
  const gmb::DropArgs d = drop_args(drop, nullptr);
  gmb::ScaleArgs a{};
  float by = 1.f;
  for (int l = L - 2; l >= 0 && d.below > 0 && blocks->num_seeds > 0; --l) {
    by *= d.scale;
    if (!grads || !grads->d_self[l] || !grads->d_neigh[l] || !grads->d_bias[l]) break;   // (refused below)
    const int64_t n = static_cast<int64_t>(weights->dims[l]) * weights->dims[l + 1];
    float* const w[] = {grads->d_self[l], grads->d_neigh[l], grads->d_bias[l]};
    for (int i = 0; i < 3; ++i) {
      a.w[a.count] = w[i];
      a.n[a.count] = i < 2 ? n : weights->dims[l + 1];
      a.by[a.count++] = by;
    }
  }
  const GivenGradient given{d_logits, blocks->num_seeds, weights->dims[L]};
  const gmb::LossLaunch how{given_gradient, &given};
  st = gmb::abi_backward_from(how, blocks, x, weights, d_logits, fwd_ws, fwd_ws_bytes, grads, nullptr, ws, ws_bytes,
                              table, num_nodes, emb_lr * by, stream);
  if (st != GMB_OK || a.count == 0) return st;
  const hipError_t e = gmb::launch_scale(a, as_stream(stream));
  if (e != hipSuccess) return hip_fail(e, "scale launch");
  return GMB_OK;
}

}  // extern "C"
