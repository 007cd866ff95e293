// Distillation loss on gfx950: a student's logits against the top logits of a
// teacher and, optionally, against labels, with the gradient in the logits.
//
// Row i has logits z, teacher entries (class c_j, logit t_j), a label y, the
// temperature T and the weight alpha.  With p = softmax(t / T) over the row's
// valid entries, q^T = softmax(z / T) and q = softmax(z) over all classes:
//   loss_i = alpha T^2 sum_j p_j (log p_j - log q^T_{c_j}) - (1 - alpha) log q_y
//   n dz_c = alpha T (q^T_c - sum_{j: c_j = c} p_j) + (1 - alpha) (q_c - [c = y])
// (n rows; the loss is the mean of loss_i).  T^2 keeps the gradient's size
// over T.  An entry is valid if its class is in [0, C) and its logit is not
// -inf; without one the first term is nothing, without a label in [0, C) the
// second, and a row whose logits are all -inf adds nothing at all.
//
//   k_distill_held   a wave (C up to 1,024) or a workgroup holds the row in
//                    registers: one read, one write of the logits' size
//   k_distill_stats, k_distill_grad
//                    rows too long for that, and few rows: workgroups share a
//                    row, each with a range of classes; the first kernel
//                    leaves their maxima and sums, the second joins them
//   k_loss_mean      the mean over the rows, in a fixed order
// The statistics are fp32: the running maximum m, sum exp((z - m) / T) and
// sum exp(z - m).
#include "common.hpp"
#include "mx_kernels.hpp"
#include "mx.hpp"

namespace gmb {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kSplitThreads = 256;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float load_logit(const float* p) { return *p; }
__device__ __forceinline__ float load_logit(const uint16_t* p) { return bf16_to_f32(*p); }

template <typename T>
struct Chunk;
template <>
struct Chunk<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void load(const float* p, float (&v)[4]) {
    float4 x;
    __builtin_memcpy(&x, p, 16);
    v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
  }
  static __device__ __forceinline__ void store(float* p, const float (&v)[4]) {
    const float4 x = make_float4(v[0], v[1], v[2], v[3]);
    __builtin_memcpy(p, &x, 16);
  }
  static __device__ __forceinline__ void store1(float* p, float v) { *p = v; }
};
template <>
struct Chunk<uint16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void load(const uint16_t* p, float (&v)[8]) {
    uint4 x;
    __builtin_memcpy(&x, p, 16);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ void store(uint16_t* p, const float (&v)[8]) { mx_store8(p, v, 8); }
  static __device__ __forceinline__ void store1(uint16_t* p, float v) {
    *p = static_cast<uint16_t>(mx_bf16x2_bits(v, 0.f));
  }
};

// Reductions over the TH threads of a row (a wave, or the workgroup).
struct Max {
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Sum {
  __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
template <int TH, typename Op>
__device__ __forceinline__ float row_reduce(float x, Op op, float* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = op(x, __shfl_xor(x, o, 64));
  if constexpr (TH > 64) {
    constexpr int W = TH / 64;
    const int wave = threadIdx.x >> 6;
    __syncthreads();   // the last reduction's reads of red
    if ((threadIdx.x & 63) == 0) red[wave] = x;
    __syncthreads();
    x = red[0];
#pragma unroll
    for (int w = 1; w < W; ++w) x = op(x, red[w]);
  }
  return x;
}

// What a row's gradient and loss are made of.
struct RowTerms {
  float m;          // the largest logit (0 where all are -inf)
  float kt, k1;     // log2(e) / T, log2(e)
  float ft, f1;     // factors of exp((z - m) / T) and exp(z - m) in the gradient
  float fp;         // a teacher probability's share of the gradient: alpha T / n
  float fy;         // the label's: (1 - alpha) / n
  int label;        // -1: none
};

// The teacher's entries of a row in LDS (classes in `ids`, -1 for an invalid
// one; probabilities in `ps`), then the loss and the gradient's factors; m,
// st and s1 are the row's statistics.  Every thread of the row calls it.
template <typename T, int TH>
__device__ __forceinline__ RowTerms row_terms(const DistillArgs& a, int64_t row, bool live, const T* z, float m,
                                              float st, float s1, int t, int32_t* ids, float* ps, float* red,
                                              float& loss) {
  RowTerms r;
  const float inv_t = 1.f / a.temperature;
  const float inv_n = 1.f / static_cast<float>(a.rows);
  r.m = m;
  r.kt = kLog2e * inv_t;
  r.k1 = kLog2e;
  const bool some = !(st == 0.f);   // not: every logit is -inf
  // the teacher
  float mt = -INFINITY;
  const bool taught = live && some && a.alpha > 0.f;
  for (int j = t; j < a.k; j += TH) {
    int32_t id = -1;
    float v = -INFINITY;
    if (taught) {
      id = a.top_ids[row * a.k + j];
      v = a.top[row * a.k + j] * inv_t;
      if (id < 0 || id >= a.classes || v == -INFINITY) {
        id = -1;
        v = -INFINITY;
      }
    }
    ids[j] = id;
    ps[j] = v;
    mt = fmaxf(mt, v);
  }
  mt = row_reduce<TH>(mt, Max(), red);
  mt = mt == -INFINITY ? 0.f : mt;
  float sum = 0.f;
  for (int j = t; j < a.k; j += TH) sum += exp2_((ps[j] - mt) * kLog2e);
  sum = row_reduce<TH>(sum, Sum(), red);
  const bool any = !(sum == 0.f);
  const float log_sum = logf(sum), log_st = logf(st), inv_sum = any ? 1.f / sum : 0.f;
  float kl = 0.f;
  if (any) {
    for (int j = t; j < a.k; j += TH) {
      const int32_t id = ids[j];
      const float u = ps[j] - mt;
      const float p = exp2_(u * kLog2e) * inv_sum;
      ps[j] = p;
      if (id >= 0 && !(p == 0.f)) kl += p * ((u - log_sum) - ((load_logit(z + id) - m) * inv_t - log_st));
    }
  }
  kl = row_reduce<TH>(kl, Sum(), red);
  r.ft = any ? a.alpha * a.temperature * inv_n / st : 0.f;
  r.fp = a.alpha * a.temperature * inv_n;
  // the label
  r.label = -1;
  if (live && some && a.labels && a.alpha < 1.f) {
    const int32_t y = a.labels[row];
    if (y >= 0 && y < a.classes) r.label = y;
  }
  r.fy = (1.f - a.alpha) * inv_n;
  r.f1 = r.label >= 0 ? r.fy / s1 : 0.f;
  loss = any ? a.alpha * a.temperature * a.temperature * kl : 0.f;
  if (r.label >= 0) loss += (1.f - a.alpha) * (logf(s1) - (load_logit(z + r.label) - m));
  return r;
}

// The classes that the teacher's entries name, in [lo, hi): the whole
// gradient again with their probabilities taken off.  Entries of one class
// add up in the entries' order and all write the same value.
template <typename T, int TH>
__device__ __forceinline__ void correct_entries(const DistillArgs& a, const RowTerms& r, const T* z, T* grad, int t,
                                                const int32_t* ids, const float* ps, int64_t lo, int64_t hi) {
  if (r.ft == 0.f) return;
  for (int j = t; j < a.k; j += TH) {
    const int32_t id = ids[j];
    if (id < lo || id >= hi) continue;
    float p = 0.f;
    for (int i = 0; i < a.k; ++i) p += ids[i] == id ? ps[i] : 0.f;
    const float d = load_logit(z + id) - r.m;
    float g = r.ft * exp2_(d * r.kt) - r.fp * p;
    if (r.label >= 0) g += r.f1 * exp2_(d * r.k1) - (id == r.label ? r.fy : 0.f);
    Chunk<T>::store1(grad + id, g);
  }
}

// TH threads hold a row of up to TH * V classes, V values each.
template <typename T, int TH, int V>
__global__ __launch_bounds__(TH < 256 ? 256 : TH) void k_distill_held(DistillArgs a) {
  constexpr int E = Chunk<T>::N, K = V / E;
  constexpr int ROWS = TH < 256 ? 256 / TH : 1;
  extern __shared__ uint32_t lds[];
  __shared__ float red[16];
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < a.clear_n;
       i += static_cast<int64_t>(gridDim.x) * blockDim.x)
    a.clear[i] = 0;
  const int sub = threadIdx.x / TH, t = threadIdx.x % TH;
  int32_t* ids = reinterpret_cast<int32_t*>(lds) + sub * a.k;
  float* ps = reinterpret_cast<float*>(lds + ROWS * a.k) + sub * a.k;
  int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + sub;
  const bool live = row < a.rows;
  if (!live) row = a.rows - 1;
  const T* z = static_cast<const T*>(a.logits) + row * a.classes;
  float v[K][E];
  float m = -INFINITY;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = (k * TH + t) * E;
    if (c + E <= a.classes) {
      Chunk<T>::load(z + c, v[k]);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) v[k][e] = c + e < a.classes ? load_logit(z + c + e) : -INFINITY;
    }
  }
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) m = fmaxf(m, v[k][e]);
  m = row_reduce<TH>(m, Max(), red);
  m = m == -INFINITY ? 0.f : m;
  const float kt = kLog2e / a.temperature;
  float st = 0.f, s1 = 0.f;
  const bool hard = a.labels && a.alpha < 1.f;
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      st += exp2_((v[k][e] - m) * kt);
      if (hard) s1 += exp2_((v[k][e] - m) * kLog2e);
    }
  st = row_reduce<TH>(st, Sum(), red);
  if (hard) s1 = row_reduce<TH>(s1, Sum(), red);
  float loss;
  const RowTerms r = row_terms<T, TH>(a, row, live, z, m, st, s1, t, ids, ps, red, loss);
  if (live && t == 0) a.loss_rows[row] = loss;
  if (!a.grad) return;
  T* grad = static_cast<T*>(a.grad) + row * a.ld_grad;
  if (live) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * TH + t) * E;
      float g[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float d = v[k][e] - m;
        g[e] = r.ft == 0.f ? 0.f : r.ft * exp2_(d * r.kt);
        if (r.label >= 0) g[e] += r.f1 * exp2_(d * r.k1) - (c + e == r.label ? r.fy : 0.f);
      }
      if (c + E <= a.classes) {
        Chunk<T>::store(grad + c, g);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (c + e < a.classes) Chunk<T>::store1(grad + c + e, g[e]);
      }
    }
    for (int64_t c = a.classes + t; c < a.ld_grad; c += TH) Chunk<T>::store1(grad + c, 0.f);
  }
  __syncthreads();   // the entries' classes are written again
  if (live) correct_entries<T, TH>(a, r, z, grad, t, ids, ps, 0, a.classes);
}

// The range of classes of part `part`: whole chunks.
__device__ __forceinline__ void part_range(int classes, int parts, int part, int64_t& lo, int64_t& hi) {
  const int64_t per = ((static_cast<int64_t>(classes) + parts - 1) / parts + 7) / 8 * 8;
  lo = per * part;
  hi = lo + per < classes ? lo + per : classes;
}

// stats[(row * parts + part) * 3 ..]: the part's m, st, s1.
template <typename T>
__global__ __launch_bounds__(kSplitThreads) void k_distill_stats(DistillArgs a) {
  constexpr int E = Chunk<T>::N;
  __shared__ float red[16];
  const int64_t row = blockIdx.x / a.parts;
  const int part = static_cast<int>(blockIdx.x % a.parts);
  const T* z = static_cast<const T*>(a.logits) + row * a.classes;
  int64_t lo, hi;
  part_range(a.classes, a.parts, part, lo, hi);
  const float kt = kLog2e / a.temperature;
  const bool hard = a.labels && a.alpha < 1.f;
  float m = -INFINITY, st = 0.f, s1 = 0.f;   // the thread's own, joined at the end
  for (int64_t c = lo + threadIdx.x * E; c < hi; c += kSplitThreads * E) {
    float v[E];
    if (c + E <= hi) {
      Chunk<T>::load(z + c, v);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = c + e < hi ? load_logit(z + c + e) : -INFINITY;
    }
    float top = v[0];
#pragma unroll
    for (int e = 1; e < E; ++e) top = fmaxf(top, v[e]);
    if (top > m) {   // (m = -inf: st = s1 = 0, and exp2(-inf) is 0)
      st *= exp2_((m - top) * kt);
      s1 *= exp2_((m - top) * kLog2e);
      m = top;
    }
    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      st += exp2_((v[e] - base) * kt);
      if (hard) s1 += exp2_((v[e] - base) * kLog2e);
    }
  }
  const float all = row_reduce<kSplitThreads>(m, Max(), red);
  // a thread without a finite logit has st = s1 = 0, or NaN
  const float f = m == -INFINITY ? 1.f : exp2_((m - all) * kt), f1 = m == -INFINITY ? 1.f : exp2_((m - all) * kLog2e);
  st = row_reduce<kSplitThreads>(st * f, Sum(), red);
  s1 = row_reduce<kSplitThreads>(s1 * f1, Sum(), red);
  if (threadIdx.x == 0) {
    float* o = a.stats + 3 * static_cast<int64_t>(blockIdx.x);
    o[0] = all;
    o[1] = st;
    o[2] = s1;
  }
}

template <typename T>
__global__ __launch_bounds__(kSplitThreads) void k_distill_grad(DistillArgs a) {
  constexpr int E = Chunk<T>::N;
  extern __shared__ uint32_t lds[];
  __shared__ float red[16];
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < a.clear_n;
       i += static_cast<int64_t>(gridDim.x) * blockDim.x)
    a.clear[i] = 0;
  const int t = threadIdx.x;
  int32_t* ids = reinterpret_cast<int32_t*>(lds);
  float* ps = reinterpret_cast<float*>(lds + a.k);
  const int64_t row = blockIdx.x / a.parts;
  const int part = static_cast<int>(blockIdx.x % a.parts);
  const T* z = static_cast<const T*>(a.logits) + row * a.classes;
  const float kt = kLog2e / a.temperature;
  const float* stats = a.stats + 3 * row * a.parts;
  float m = -INFINITY;
  for (int i = 0; i < a.parts; ++i) m = fmaxf(m, stats[3 * i]);
  m = m == -INFINITY ? 0.f : m;
  float st = 0.f, s1 = 0.f;
  for (int i = 0; i < a.parts; ++i) {
    const float mi = stats[3 * i];
    st += stats[3 * i + 1] * (mi == -INFINITY ? 1.f : exp2_((mi - m) * kt));
    s1 += stats[3 * i + 2] * (mi == -INFINITY ? 1.f : exp2_((mi - m) * kLog2e));
  }
  float loss;
  const RowTerms r = row_terms<T, kSplitThreads>(a, row, true, z, m, st, s1, t, ids, ps, red, loss);
  if (part == 0 && t == 0) a.loss_rows[row] = loss;
  if (!a.grad) return;
  T* grad = static_cast<T*>(a.grad) + row * a.ld_grad;
  int64_t lo, hi;
  part_range(a.classes, a.parts, part, lo, hi);
  for (int64_t c = lo + t * E; c < hi; c += kSplitThreads * E) {
    float v[E], g[E];
    const bool whole = c + E <= hi;
    if (whole) {
      Chunk<T>::load(z + c, v);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = c + e < hi ? load_logit(z + c + e) : -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float d = v[e] - m;
      g[e] = r.ft == 0.f ? 0.f : r.ft * exp2_(d * r.kt);
      if (r.label >= 0) g[e] += r.f1 * exp2_(d * r.k1) - (c + e == r.label ? r.fy : 0.f);
    }
    if (whole) {
      Chunk<T>::store(grad + c, g);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (c + e < hi) Chunk<T>::store1(grad + c + e, g[e]);
    }
  }
  if (part == 0)
    for (int64_t c = a.classes + t; c < a.ld_grad; c += kSplitThreads) Chunk<T>::store1(grad + c, 0.f);
  __syncthreads();
  correct_entries<T, kSplitThreads>(a, r, z, grad, t, ids, ps, lo, hi);
}

__global__ __launch_bounds__(1024) void k_loss_mean(const float* rows, int64_t n, float* loss) {
  __shared__ float red[16];
  float s = 0.f;
  for (int64_t i = threadIdx.x; i < n; i += 1024) s += rows[i];
  s = row_reduce<1024>(s, Sum(), red);
  if (threadIdx.x == 0) *loss = s / static_cast<float>(n);
}

template <typename T, int TH, int V>
void held(const DistillArgs& a, hipStream_t s) {
  constexpr int ROWS = TH < 256 ? 256 / TH : 1;
  hipLaunchKernelGGL((k_distill_held<T, TH, V>), dim3(static_cast<unsigned>((a.rows + ROWS - 1) / ROWS)),
                     dim3(TH < 256 ? 256 : TH), 8 * static_cast<size_t>(a.k) * ROWS, s, a);
}

template <typename T>
void dispatch(const DistillArgs& a, hipStream_t s) {
  if (a.stats) {
    const dim3 grid(static_cast<unsigned>(a.rows * a.parts));
    hipLaunchKernelGGL((k_distill_stats<T>), grid, dim3(kSplitThreads), 0, s, a);
    hipLaunchKernelGGL((k_distill_grad<T>), grid, dim3(kSplitThreads), 8 * static_cast<size_t>(a.k), s, a);
  } else if (a.classes <= 512) {
    held<T, 64, 8>(a, s);
  } else if (a.classes <= 1024) {
    held<T, 64, 16>(a, s);
  } else if (a.classes <= 4096) {
    held<T, 256, 16>(a, s);
  } else if (a.classes <= 8192) {
    held<T, 256, 32>(a, s);
  } else {
    held<T, 1024, 32>(a, s);
  }
}

}  // namespace

int distill_parts(int64_t rows, int64_t classes) {
  if (classes > kDistillHeld || (classes > 4096 && rows < 64)) {
    int64_t parts = (2048 + rows - 1) / rows;
    const int64_t most = (classes + 2047) / 2048;
    parts = parts < most ? parts : most;
    return static_cast<int>(parts < 1 ? 1 : parts);
  }
  return 0;
}

hipError_t launch_distill(const DistillArgs& a, int bf16, hipStream_t s) {
  if (bf16) dispatch<uint16_t>(a, s);
  else dispatch<float>(a, s);
  return hipGetLastError();
}

hipError_t launch_loss_mean(const float* loss_rows, int64_t rows, float* loss, hipStream_t s) {
  hipLaunchKernelGGL(k_loss_mean, dim3(1), dim3(1024), 0, s, loss_rows, rows, loss);
  return hipGetLastError();
}

}  // namespace gmb
