// C ABI of the microscaled store and model and of the distillation loss
// (declared in include/gmb.h): argument validation, workspace planning and
// kernel launches.  No C++ exception crosses the ABI; every entry point
// returns a gmb_status.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "api_common.hpp"
#include "gmb.h"
#include "kernels.hpp"
#include "mx_kernels.hpp"

namespace {

using gmb::abi_fail;

constexpr int64_t kMaxInt32 = 0x7FFFFFFF;
constexpr int32_t kMaxDim = 65536;
constexpr int64_t kMaxLinearRows = kMaxInt32 - 1023;   // in tiles of 64, one launch's threads fit 32 bits

int hip_fail(hipError_t e, const char* what) { return abi_fail(GMB_EDEVICE, "%s: %s", what, hipGetErrorString(e)); }
hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }
size_t align_up(size_t x) { return (x + gmb::kAbiAlign - 1) / gmb::kAbiAlign * gmb::kAbiAlign; }

int check_shape(int32_t dim, int32_t bits) {
  if (dim < 1 || dim > kMaxDim) return abi_fail(GMB_EINVAL, "dim=%d outside 1..%d", dim, kMaxDim);
  if (bits != GMB_MXFP4 && bits != GMB_MXFP8) return abi_fail(GMB_EINVAL, "format=%d unknown", bits);
  return GMB_OK;
}

// A table of records: its address, rows and stride.
int check_table(const void* table, int64_t rows, int64_t stride, int32_t dim, int32_t bits, const char* what) {
  if (!table) return abi_fail(GMB_EINVAL, "%s is NULL", what);
  if (rows < 1 || rows > kMaxInt32)
    return abi_fail(GMB_EINVAL, "%s: %lld rows outside 1..2^31-1", what, static_cast<long long>(rows));
  if (reinterpret_cast<uintptr_t>(table) % 16 || stride % 16)
    return abi_fail(GMB_EINVAL, "%s: the address and the row stride must be multiples of 16 bytes", what);
  if (stride < gmb::mx_record(dim, bits))
    return abi_fail(GMB_EINVAL, "%s: row stride %lld below the record's %lld bytes", what,
                    static_cast<long long>(stride), static_cast<long long>(gmb::mx_record(dim, bits)));
  return GMB_OK;
}

int check_count(int64_t n_cap) {
  if (n_cap < 0 || n_cap > kMaxInt32)
    return abi_fail(GMB_EINVAL, "n_cap=%lld outside 0..2^31-1", static_cast<long long>(n_cap));
  return GMB_OK;
}

int check_dtype(int32_t dtype) {
  if (dtype != GMB_F32 && dtype != GMB_BF16) return abi_fail(GMB_EINVAL, "dtype=%d unknown", dtype);
  return GMB_OK;
}

}  // namespace

extern "C" {

int64_t gmb_mx_row_bytes(int32_t dim, int32_t format) {
  if (check_shape(dim, format) != GMB_OK) return 0;
  return gmb::mx_record(dim, format);
}

int gmb_mx_quantise(const void* x, int32_t dtype, int64_t row_stride, int64_t col_stride, const int32_t* ids,
                 const int32_t* n_dev, int64_t n_cap, int32_t dim, int32_t format, void* table, int64_t num_rows,
                 int64_t table_stride, void* state, size_t state_bytes, uint32_t* status, void* stream) {
  int st = check_shape(dim, format);
  if (st == GMB_OK) st = check_dtype(dtype);
  if (st == GMB_OK) st = check_count(n_cap);
  if (st != GMB_OK) return st;
  if (row_stride < 0 || col_stride < 0) return abi_fail(GMB_EINVAL, "a negative stride");
  if (n_cap == 0) return GMB_OK;
  st = check_table(table, num_rows, table_stride, dim, format, "table");
  if (st != GMB_OK) return st;
  if (!x) return abi_fail(GMB_EINVAL, "x is NULL");
  if (!ids && n_cap > num_rows)
    return abi_fail(GMB_EINVAL, "%lld rows into a table of %lld", static_cast<long long>(n_cap),
                    static_cast<long long>(num_rows));
  uint32_t* slots = nullptr;
  if (state) {
    if (!ids) return abi_fail(GMB_EINVAL, "a state without ids");
    if (reinterpret_cast<uintptr_t>(state) % gmb::kAbiAlign)
      return abi_fail(GMB_EINVAL, "state must be 256-byte aligned");
    const size_t need = gmb_sampler_state_bytes(num_rows);
    if (state_bytes < need) return abi_fail(GMB_ENOSPC, "state holds %zu bytes, %zu needed", state_bytes, need);
    slots = reinterpret_cast<uint32_t*>(static_cast<char*>(state) + gmb::kAbiStateHeader);
    if (!status) status = static_cast<uint32_t*>(state);
  }
  gmb::MxWriteArgs a{};
  a.x = x;
  a.row_stride = row_stride;
  a.col_stride = dim == 1 ? 1 : col_stride;
  a.n_dev = n_dev;
  a.n_cap = n_cap;
  a.dim = dim;
  a.blocks = static_cast<int>(gmb::mx_blocks(dim));
  a.record = static_cast<int>(gmb::mx_record(dim, format));
  a.ids = ids;
  a.table = static_cast<uint8_t*>(table);
  a.table_rows = num_rows;
  a.table_stride = table_stride;
  a.status = status;
  const hipError_t e = gmb::launch_mx_write(a, dtype == GMB_BF16, format, slots, as_stream(stream));
  if (e != hipSuccess) return hip_fail(e, "store write launch");
  return GMB_OK;
}

int gmb_mx_gather(const int32_t* ids, const int32_t* n_dev, int64_t n_cap, const void* table, int64_t num_rows,
                int64_t table_stride, int32_t dim, int32_t format, void* out, int32_t dtype, uint32_t* status,
                void* stream) {
  int st = check_shape(dim, format);
  if (st == GMB_OK) st = check_dtype(dtype);
  if (st == GMB_OK) st = check_count(n_cap);
  if (st != GMB_OK) return st;
  if (n_cap == 0) return GMB_OK;
  st = check_table(table, num_rows, table_stride, dim, format, "table");
  if (st != GMB_OK) return st;
  if (!out) return abi_fail(GMB_EINVAL, "out is NULL");
  if (!ids && n_cap > num_rows)
    return abi_fail(GMB_EINVAL, "%lld rows of a table of %lld", static_cast<long long>(n_cap),
                    static_cast<long long>(num_rows));
  gmb::MxReadArgs a{};
  a.ids = ids;
  a.n_dev = n_dev;
  a.n_cap = n_cap;
  a.dim = dim;
  a.blocks = static_cast<int>(gmb::mx_blocks(dim));
  a.table = static_cast<const uint8_t*>(table);
  a.table_rows = num_rows;
  a.table_stride = table_stride;
  a.out = out;
  a.status = status;
  const hipError_t e = gmb::launch_mx_read(a, dtype == GMB_BF16, format, as_stream(stream));
  if (e != hipSuccess) return hip_fail(e, "store read launch");
  return GMB_OK;
}

int gmb_mx_mean(const int32_t* indptr, const int32_t* ids, const int32_t* n_dev, int64_t n_cap, const void* table,
                int64_t num_rows, int64_t table_stride, int32_t dim, int32_t format, void* out, int32_t dtype,
                void* stream) {
  int st = check_shape(dim, format);
  if (st == GMB_OK) st = check_dtype(dtype);
  if (st == GMB_OK) st = check_count(n_cap);
  if (st != GMB_OK) return st;
  if (n_cap == 0) return GMB_OK;
  st = check_table(table, num_rows, table_stride, dim, format, "table");
  if (st != GMB_OK) return st;
  if (!indptr || !ids || !out) return abi_fail(GMB_EINVAL, "a NULL array");
  gmb::MxMeanArgs a{};
  a.indptr = indptr;
  a.ids = ids;
  a.n_dev = n_dev;
  a.n_cap = n_cap;
  a.dim = dim;
  a.blocks = static_cast<int>(gmb::mx_blocks(dim));
  a.table = static_cast<const uint8_t*>(table);
  a.table_rows = num_rows;
  a.table_stride = table_stride;
  a.out = out;
  const hipError_t e = gmb::launch_mx_mean(a, dtype == GMB_BF16, format, as_stream(stream));
  if (e != hipSuccess) return hip_fail(e, "store mean launch");
  return GMB_OK;
}

int gmb_mx_linear(const gmb_mx_operand* a, const gmb_mx_operand* a2, const int32_t* n_dev, int64_t n_cap,
                  int32_t d_in, int32_t d_out, const float* bias, int32_t relu, void* out, int32_t dtype,
                  uint32_t* status, void* stream) {
  int st = check_shape(d_in, GMB_MXFP4);
  if (st == GMB_OK) st = check_shape(d_out, GMB_MXFP4);
  if (st == GMB_OK) st = check_dtype(dtype);
  if (st == GMB_OK) st = check_count(n_cap);
  if (st != GMB_OK) return st;
  if (!a) return abi_fail(GMB_EINVAL, "a is NULL");
  if (n_cap > kMaxLinearRows)
    return abi_fail(GMB_EINVAL, "n_cap=%lld above 2^31 - 1024", static_cast<long long>(n_cap));
  if (n_cap == 0) return GMB_OK;
  gmb::MxLinearArgs p{};
  p.pairs = a2 ? 2 : 1;
  for (int i = 0; i < p.pairs; ++i) {
    const gmb_mx_operand& o = i ? *a2 : *a;
    st = check_table(o.rows, o.num_rows, o.row_stride, d_in, GMB_MXFP4, i ? "a2 rows" : "a rows");
    if (st == GMB_OK) st = check_table(o.weights, d_out, o.weight_stride, d_in, GMB_MXFP4, i ? "a2 weights" : "a weights");
    if (st != GMB_OK) return st;
    if (i && o.ids) return abi_fail(GMB_EINVAL, "only the first operand's rows may go by id");
    if (!o.ids && n_cap > o.num_rows)
      return abi_fail(GMB_EINVAL, "%lld rows of a table of %lld", static_cast<long long>(n_cap),
                      static_cast<long long>(o.num_rows));
    p.pair[i] = gmb::MxPair{static_cast<const uint8_t*>(o.rows), o.num_rows, o.row_stride, o.ids,
                            static_cast<const uint8_t*>(o.weights), o.weight_stride};
  }
  if (!out) return abi_fail(GMB_EINVAL, "out is NULL");
  p.n_dev = n_dev;
  p.n_cap = n_cap;
  p.d_in = d_in;
  p.blocks = static_cast<int>(gmb::mx_blocks(d_in));
  p.d_out = d_out;
  p.bias = bias;
  p.relu = relu ? 1 : 0;
  p.out = out;
  p.status = status;
  const hipError_t e =
      gmb::launch_mx_linear(p, dtype == GMB_BF16 ? gmb::kMxOutBf16 : gmb::kMxOutF32, as_stream(stream));
  if (e != hipSuccess) return hip_fail(e, "microscaled linear launch");
  return GMB_OK;
}

}  // extern "C"

// ---- a model in microscaled form ------------------------------------------

namespace {

struct MxForwardPlan {
  size_t off_mean[GMB_MAX_LAYERS], off_hidden[GMB_MAX_LAYERS];
  size_t total;
};

int plan_mx_forward(const gmb_blocks* b, const gmb_sage_mx_weights* w, MxForwardPlan* plan) {
  int st = gmb::abi_check_blocks(b);
  if (st != GMB_OK) return st;
  if (!w) return abi_fail(GMB_EINVAL, "weights is NULL");
  if (w->num_layers != b->num_layers)
    return abi_fail(GMB_EINVAL, "weights have %d layers, blocks %d", w->num_layers, b->num_layers);
  for (int l = 0; l <= w->num_layers; ++l) {
    st = check_shape(w->dims[l], GMB_MXFP4);
    if (st != GMB_OK) return st;
  }
  for (int l = 0; l < w->num_layers; ++l) {
    if (b->blk[l].cap_dst > kMaxLinearRows)
      return abi_fail(GMB_EINVAL, "block %d: %lld destinations above 2^31 - 1024", l,
                      static_cast<long long>(b->blk[l].cap_dst));
    const int64_t rec = gmb::mx_record(w->dims[l], GMB_MXFP4);
    st = check_table(w->w_self[l], w->dims[l + 1], rec, w->dims[l], GMB_MXFP4, "w_self");
    if (st == GMB_OK) st = check_table(w->w_neigh[l], w->dims[l + 1], rec, w->dims[l], GMB_MXFP4, "w_neigh");
    if (st != GMB_OK) return st;
    if (!w->bias[l]) return abi_fail(GMB_EINVAL, "layer %d bias is NULL", l);
    if (l > 0 && b->blk[l].cap_src != b->blk[l - 1].cap_dst)
      return abi_fail(GMB_EINVAL, "block %d sources (cap %lld) are not block %d destinations (cap %lld)", l,
                      static_cast<long long>(b->blk[l].cap_src), l - 1,
                      static_cast<long long>(b->blk[l - 1].cap_dst));
  }
  MxForwardPlan p{};
  size_t off = 0;
  for (int l = 0; l < w->num_layers; ++l) {
    const size_t rows = static_cast<size_t>(std::max<int64_t>(b->blk[l].cap_dst, 1));
    p.off_mean[l] = off;
    off = align_up(off + rows * gmb::mx_record(w->dims[l], GMB_MXFP4));
    if (l + 1 < w->num_layers) {
      p.off_hidden[l] = off;
      off = align_up(off + rows * gmb::mx_record(w->dims[l + 1], GMB_MXFP4));
    }
  }
  p.total = off;
  *plan = p;
  return GMB_OK;
}

}  // namespace

extern "C" {

size_t gmb_mx_forward_workspace_bytes(const gmb_blocks* blocks, const gmb_sage_mx_weights* weights) {
  MxForwardPlan p;
  if (plan_mx_forward(blocks, weights, &p) != GMB_OK) return 0;
  return p.total;
}

int64_t gmb_mx_forward_offset(const gmb_blocks* blocks, const gmb_sage_mx_weights* weights, int32_t layer,
                              int32_t hidden) {
  MxForwardPlan p;
  if (plan_mx_forward(blocks, weights, &p) != GMB_OK) return -1;
  if (layer < 0 || layer + (hidden ? 1 : 0) >= weights->num_layers) return -1;
  return static_cast<int64_t>(hidden ? p.off_hidden[layer] : p.off_mean[layer]);
}

int gmb_sage_forward_mx(const gmb_blocks* blocks, const void* table, int64_t num_nodes, int64_t table_stride,
                        const gmb_sage_mx_weights* weights, float* logits, void* ws, size_t ws_bytes,
                        uint32_t* status, void* stream) {
  MxForwardPlan p;
  int st = plan_mx_forward(blocks, weights, &p);
  if (st != GMB_OK) return st;
  st = check_table(table, num_nodes, table_stride, weights->dims[0], GMB_MXFP4, "table");
  if (st != GMB_OK) return st;
  if (!ws) return abi_fail(GMB_EINVAL, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(ws) % gmb::kAbiAlign)
    return abi_fail(GMB_EINVAL, "workspace is not 256-byte aligned");
  if (ws_bytes < p.total) return abi_fail(GMB_ENOSPC, "workspace holds %zu bytes, %zu needed", ws_bytes, p.total);
  if (blocks->num_seeds == 0) return GMB_OK;   // an empty batch: no rows anywhere
  if (!logits) return abi_fail(GMB_EINVAL, "logits is NULL");
  const hipStream_t s = as_stream(stream);
  uint8_t* base = static_cast<uint8_t*>(ws);
  const int L = weights->num_layers;
  const uint8_t* h = static_cast<const uint8_t*>(table);   // the layer's input records
  for (int l = 0; l < L; ++l) {
    const gmb_block& bk = blocks->blk[l];
    const int d_in = weights->dims[l], d_out = weights->dims[l + 1];
    const int64_t rec_in = gmb::mx_record(d_in, GMB_MXFP4), rec_out = gmb::mx_record(d_out, GMB_MXFP4);
    const bool last = l == L - 1;
    // layer 0 reads the store by the vertices' ids, the others the layer
    // below by position
    const int64_t h_stride = l == 0 ? table_stride : rec_in;
    const int64_t h_rows = l == 0 ? num_nodes : std::max<int64_t>(bk.cap_src, 1);
    if (bk.cap_dst == 0) return abi_fail(GMB_EINVAL, "block %d has no destinations for %d seeds", l, blocks->num_seeds);
    gmb::MxMeanArgs m{};
    m.indptr = bk.indptr;
    m.ids = l == 0 ? bk.nbr : bk.indices;
    if (!m.ids) return abi_fail(GMB_EINVAL, "block %d has a NULL array", l);
    m.n_dev = bk.sizes + gmb::kNDst;
    m.n_cap = bk.cap_dst;
    m.dim = d_in;
    m.blocks = static_cast<int>(gmb::mx_blocks(d_in));
    m.table = h;
    m.table_rows = h_rows;
    m.table_stride = h_stride;
    m.out = base + p.off_mean[l];
    m.out_stride = rec_in;
    m.out_record = static_cast<int>(rec_in);
    m.status = l == 0 ? status : nullptr;   // (above, positions in the layer below)
    hipError_t e = gmb::launch_mx_mean_records(m, s);
    if (e != hipSuccess) return hip_fail(e, "store mean launch");
    gmb::MxLinearArgs a{};
    a.pairs = 2;
    a.pair[0] = gmb::MxPair{h, h_rows, h_stride, l == 0 ? bk.src_ids : nullptr,
                            static_cast<const uint8_t*>(weights->w_self[l]), rec_in};
    a.pair[1] = gmb::MxPair{base + p.off_mean[l], std::max<int64_t>(bk.cap_dst, 1), rec_in, nullptr,
                            static_cast<const uint8_t*>(weights->w_neigh[l]), rec_in};
    a.n_dev = bk.sizes + gmb::kNDst;
    a.n_cap = bk.cap_dst;
    a.d_in = d_in;
    a.blocks = m.blocks;
    a.d_out = d_out;
    a.bias = weights->bias[l];
    a.relu = last ? 0 : 1;
    a.out = last ? static_cast<void*>(logits) : static_cast<void*>(base + p.off_hidden[l]);
    a.out_stride = rec_out;
    a.out_record = static_cast<int>(rec_out);
    a.status = status;
    e = gmb::launch_mx_linear(a, last ? gmb::kMxOutF32 : gmb::kMxOutRecords, s);
    if (e != hipSuccess) return hip_fail(e, "microscaled linear launch");
    if (!last) h = base + p.off_hidden[l];
  }
  return GMB_OK;
}

}  // extern "C"

// ---- distillation ---------------------------------------------------------

namespace {

int check_teacher(const gmb_teacher* t) {
  if (!t) return abi_fail(GMB_EINVAL, "teacher is NULL");
  if (t->top < 1 || t->top > GMB_MAX_TEACHER)
    return abi_fail(GMB_EINVAL, "teacher->top=%d outside 1..%d", t->top, GMB_MAX_TEACHER);
  if (!(t->alpha >= 0.f && t->alpha <= 1.f)) return abi_fail(GMB_EINVAL, "teacher->alpha outside 0..1");
  if (!(t->temperature >= 1e-3f && t->temperature <= 1e3f))
    return abi_fail(GMB_EINVAL, "teacher->temperature outside 0.001..1000");
  if (!t->logits || !t->classes) return abi_fail(GMB_EINVAL, "teacher has a NULL array");
  return GMB_OK;
}

int check_rows(int64_t rows, int32_t classes) {
  if (rows < 0 || rows > kMaxInt32)
    return abi_fail(GMB_EINVAL, "rows=%lld outside 0..2^31-1", static_cast<long long>(rows));
  if (classes < 1) return abi_fail(GMB_EINVAL, "classes=%d < 1", classes);
  return GMB_OK;
}

size_t loss_rows_bytes(int64_t rows) { return align_up(4 * static_cast<size_t>(std::max<int64_t>(rows, 1))); }

gmb::DistillArgs distill_args(const void* logits, int64_t rows, int classes, const gmb_teacher* t,
                              const int32_t* labels) {
  gmb::DistillArgs a{};
  a.logits = logits;
  a.rows = rows;
  a.classes = classes;
  a.top = t->logits;
  a.top_ids = t->classes;
  a.k = t->top;
  a.labels = labels;
  a.alpha = t->alpha;
  a.temperature = t->temperature;
  return a;
}

// The last layer's loss of a backward (LossLaunch): one launch, no room for
// split statistics.
hipError_t distill_into(const void* what, float* dz, int ldz, float* loss_rows, int32_t* clear, int64_t clear_n,
                        hipStream_t s) {
  gmb::DistillArgs a = *static_cast<const gmb::DistillArgs*>(what);
  a.grad = dz;
  a.ld_grad = ldz;
  a.loss_rows = loss_rows;
  a.clear = clear;
  a.clear_n = clear_n;
  return gmb::launch_distill(a, 0, s);
}

}  // namespace

extern "C" {

size_t gmb_distill_workspace_bytes(int64_t rows, int32_t classes) {
  if (check_rows(rows, classes) != GMB_OK) return 0;
  const int64_t r = std::max<int64_t>(rows, 1);
  return loss_rows_bytes(rows) + align_up(12 * static_cast<size_t>(r) * gmb::distill_parts(r, classes));
}

int gmb_distill_loss(const void* logits, int32_t dtype, int64_t rows, int32_t classes, const gmb_teacher* teacher,
                     const int32_t* labels, void* dlogits, float* loss, void* ws, size_t ws_bytes, void* stream) {
  int st = check_rows(rows, classes);
  if (st == GMB_OK) st = check_dtype(dtype);
  if (st != GMB_OK) return st;
  if (!loss) return abi_fail(GMB_EINVAL, "loss is NULL");
  const hipStream_t s = as_stream(stream);
  if (rows == 0) {   // a mean over no rows is taken as 0
    const hipError_t e = gmb::launch_zero(gmb::SgdArgs{}, loss, s);
    if (e != hipSuccess) return hip_fail(e, "zero-fill launch");
    return GMB_OK;
  }
  st = check_teacher(teacher);
  if (st != GMB_OK) return st;
  if (!logits) return abi_fail(GMB_EINVAL, "logits is NULL");
  const uintptr_t from = reinterpret_cast<uintptr_t>(logits), to = reinterpret_cast<uintptr_t>(dlogits);
  const uintptr_t size = static_cast<uintptr_t>(rows) * classes * (dtype == GMB_BF16 ? 2 : 4);
  if (dlogits && from < to + size && to < from + size)
    return abi_fail(GMB_EINVAL, "dlogits overlaps the logits");
  if (!ws) return abi_fail(GMB_EINVAL, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(ws) % gmb::kAbiAlign)
    return abi_fail(GMB_EINVAL, "workspace is not 256-byte aligned");
  const size_t need = gmb_distill_workspace_bytes(rows, classes);
  if (ws_bytes < need) return abi_fail(GMB_ENOSPC, "workspace holds %zu bytes, %zu needed", ws_bytes, need);
  gmb::DistillArgs a = distill_args(logits, rows, classes, teacher, labels);
  a.grad = dlogits;
  a.ld_grad = classes;
  a.loss_rows = static_cast<float*>(ws);
  a.parts = gmb::distill_parts(rows, classes);
  a.stats = a.parts > 0 ? reinterpret_cast<float*>(static_cast<char*>(ws) + loss_rows_bytes(rows)) : nullptr;
  hipError_t e = gmb::launch_distill(a, dtype == GMB_BF16, s);
  if (e != hipSuccess) return hip_fail(e, "distillation launch");
  e = gmb::launch_loss_mean(a.loss_rows, rows, loss, s);
  if (e != hipSuccess) return hip_fail(e, "loss launch");
  return GMB_OK;
}

int gmb_sage_backward_distill(const gmb_blocks* blocks, const void* x, const gmb_sage_weights* weights,
                              const float* logits, const gmb_teacher* teacher, const int32_t* labels,
                              const void* fwd_ws, size_t fwd_ws_bytes, const gmb_sage_grads* grads, float* loss,
                              void* ws, size_t ws_bytes, float* table, int64_t num_nodes, float emb_lr,
                              void* stream) {
  int st = gmb::abi_check_blocks(blocks);
  if (st != GMB_OK) return st;
  if (!weights) return abi_fail(GMB_EINVAL, "weights is NULL");
  if (weights->num_layers != blocks->num_layers)
    return abi_fail(GMB_EINVAL, "weights have %d layers, blocks %d", weights->num_layers, blocks->num_layers);
  if (blocks->num_seeds > 0) {
    st = check_teacher(teacher);
    if (st != GMB_OK) return st;
    if (weights->dims[weights->num_layers] > gmb::kDistillHeld)
      return abi_fail(GMB_EINVAL, "%d classes above %d", weights->dims[weights->num_layers], gmb::kDistillHeld);
  }
  if (table) {
    if (num_nodes < 1 || num_nodes > kMaxInt32)
      return abi_fail(GMB_EINVAL, "num_nodes=%lld outside 1..2^31-1", static_cast<long long>(num_nodes));
    if (reinterpret_cast<uintptr_t>(table) % 16) return abi_fail(GMB_EINVAL, "table must be 16-byte aligned");
  }
  gmb::DistillArgs a{};
  if (blocks->num_seeds > 0)
    a = distill_args(logits, blocks->num_seeds, weights->dims[weights->num_layers], teacher, labels);
  const gmb::LossLaunch how{distill_into, &a};
  return gmb::abi_backward_from(how, blocks, x, weights, logits, fwd_ws, fwd_ws_bytes, grads, loss, ws, ws_bytes,
                                table, num_nodes, emb_lr, stream);
}

}  // extern "C"
