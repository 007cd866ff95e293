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
//   k_distill_held   part of a wave (up to 256 pieces of 16 bytes) or a
//                    workgroup holds the row in registers: one read, one write
//                    of the logits' size
//   k_distill_stats, k_distill_grad
//                    rows too long for that, and few rows: workgroups share a
//                    row, each with a range of classes; the first kernel
//                    leaves their maxima and sums, the second joins them
//   k_loss_mean      the mean over the rows, in 64 bits and a fixed order
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

// 16 bytes of logits.
template <typename T>
struct Chunk;
template <>
struct Chunk<float> {
  static constexpr int N = 4;
  static constexpr uint32_t kMasked = 0xFF800000u;   // -inf, in each of a word's values
  static __device__ __forceinline__ void unpack(const uint4& x, float (&v)[4]) {
    v[0] = __uint_as_float(x.x);
    v[1] = __uint_as_float(x.y);
    v[2] = __uint_as_float(x.z);
    v[3] = __uint_as_float(x.w);
  }
  static __device__ __forceinline__ void store1(float* p, float v) { *p = v; }
};
template <>
struct Chunk<uint16_t> {
  static constexpr int N = 8;
  static constexpr uint32_t kMasked = 0xFF80FF80u;
  static __device__ __forceinline__ void unpack(const uint4& x, float (&v)[8]) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ void store1(uint16_t* p, float v) {
    *p = static_cast<uint16_t>(mx_bf16x2_bits(v, 0.f));
  }
};

template <typename T>
__device__ __forceinline__ uint4 masked_chunk() {
  constexpr uint32_t m = Chunk<T>::kMasked;
  return make_uint4(m, m, m, m);
}
// The chunk of classes c .. c + N - 1 (c < end), -inf at `end` and past it; its
// values are asked for together (the last one for those past it).
template <typename T>
__device__ __forceinline__ uint4 load_tail(const T* z, int64_t c, int64_t end) {
  T v[Chunk<T>::N];
#pragma unroll
  for (int i = 0; i < Chunk<T>::N; ++i) v[i] = z[c + i < end ? c + i : end - 1];
  uint4 x = masked_chunk<T>();
  T* e = reinterpret_cast<T*>(&x);
#pragma unroll
  for (int i = 0; i < Chunk<T>::N; ++i) e[i] = c + i < end ? v[i] : e[i];
  return x;
}
template <typename T>
__device__ __forceinline__ uint4 load_chunk(const T* z, int64_t c, int64_t end) {
  if (c + Chunk<T>::N > end) return load_tail(z, c, end);
  uint4 x;
  mx_get<16>(&x, z + c);
  return x;
}
template <bool STREAM, typename T>
__device__ __forceinline__ void store_chunk(T* grad, int64_t c, int64_t end, const float (&g)[Chunk<T>::N]) {
  const int64_t left = end - c;
  mx_store<STREAM>(grad + c, g, left < Chunk<T>::N ? static_cast<int>(left) : Chunk<T>::N);
}

// Reductions over the TH threads of a row (a part of a wave, a wave, or the
// workgroup).
struct Max {
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Sum {
  template <typename V>
  __device__ __forceinline__ V operator()(V a, V b) const {
    return a + b;
  }
};
template <int TH, typename V, typename Op>
__device__ __forceinline__ V row_reduce(V x, Op op, V* red) {
#pragma unroll
  for (int o = (TH < 64 ? TH : 64) / 2; o > 0; o >>= 1) x = op(x, __shfl_xor(x, o, 64));
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

// How exp(z - m) follows from u = exp((z - m) / T): it is u^T for T = 1, 2
// and 4 (POW), one exponential a class and pass instead of two; else (POW 0)
// it takes its own.  (Rows of T = 1, 2, 4 with POW and without: 4,099 x 32,768
// bf16 108 / 117 us, 112 / 116, 112 / 116; 2,000 x 30,000 fp32 98.9 / 102, 99.2 /
// 102, 100 / 102; 30,000 x 200 bf16 19.5 / 21.6, 19.9 / 21.7, 20.2 / 21.6.)
template <int POW>
__device__ __forceinline__ float hard_exp(float u, float d) {
  if constexpr (POW == 1) return u;
  if constexpr (POW == 2) return u * u;
  if constexpr (POW == 4) return (u * u) * (u * u);
  return exp2_(d * kLog2e);
}

// What a thread asks for before it has the row's statistics: its first
// teacher entry and the label, then their logits.
struct Early {
  int32_t id;      // -1: none
  float t, z;      // the entry's logit, and the student's at its class
  int32_t label;   // -1: none
  float zl;
};

__device__ __forceinline__ Early early_entry(const DistillArgs& a, int64_t row, bool live, int t) {
  Early e{-1, -INFINITY, 0.f, -1, 0.f};
  if (live && a.alpha > 0.f && t < a.k) {
    e.id = a.top_ids[row * a.k + t];
    e.t = a.top[row * a.k + t];
  }
  if (live && a.labels && a.alpha < 1.f) e.label = a.labels[row];
  return e;
}
template <typename T>
__device__ __forceinline__ void early_logits(const DistillArgs& a, const T* z, Early& e) {
  if (e.id < 0 || e.id >= a.classes || e.t == -INFINITY) {
    e.id = -1;
    e.t = -INFINITY;
  }
  if (e.label >= a.classes) e.label = -1;
  // (both at once, of some class if there is none)
  const T zi = z[e.id < 0 ? 0 : e.id], zl = z[e.label < 0 ? 0 : e.label];
  e.z = load_logit(&zi);
  e.zl = load_logit(&zl);
}

// What a row's gradient and loss are made of.
struct RowTerms {
  float m;          // the largest logit (0 where all are -inf)
  float kt;         // log2(e) / T
  float ft, f1;     // factors of exp((z - m) / T) and exp(z - m) in the gradient
  float fp;         // a teacher probability's share of the gradient: alpha T / n
  float fy;         // the label's: (1 - alpha) / n
  int label;        // -1: none
  bool none;        // no term at all: no gradient
};

// A row's entries in LDS: whole fours of them, 8 bytes each.  With many entries
// also two sets of bits, 16 bits an entry: a class's bit is in `seen` if an entry
// names it and in `twice` if two do, so that most entries are known to be alone
// without a look at the others.  A class's bit is its number where the sets have
// as many bits as there are classes; else classes share bits, and those whose
// bit is taken twice are looked for.  (T = 1.5, 37,472 rows of 357 bf16, 214
// entries: by comparing all 203 us, 118 so; 20,000 x 1,000, 64 entries: 42.0 and
// 36.0; 60,000 x 500, 30 entries: 50.7 and 46.8; with 8 entries comparing is two
// reads.)
constexpr int kFewEntries = 8;
__host__ __device__ inline int entry_room(int k) { return (k + 3) / 4 * 4; }
__host__ __device__ inline int entry_bytes(int k) { return entry_room(k) * (k > kFewEntries ? 12 : 8); }

struct Entries {
  int32_t* ids;
  float* ps;
  uint32_t *seen, *twice;   // room / 2 words each
  int room;
  bool many, exact;
  __device__ __forceinline__ Entries(uint32_t* lds, const DistillArgs& a, int row, int rows) {
    room = entry_room(a.k);
    many = a.k > kFewEntries;
    exact = a.classes <= 16 * room;
    ids = reinterpret_cast<int32_t*>(lds) + row * room;
    ps = reinterpret_cast<float*>(lds + rows * room) + row * room;
    seen = lds + 2 * rows * room + row * room;
    twice = seen + room / 2;
  }
  // By the row's threads; then a barrier.
  template <int TH>
  __device__ __forceinline__ void clear(int t) {
    if (many)
      for (int j = t; j < room; j += TH) seen[j] = 0;
  }
  __device__ __forceinline__ int place(int32_t id) const {
    if (exact) return id;
    return static_cast<int>(__umulhi(static_cast<uint32_t>(id) * 0x9E3779B1u, static_cast<uint32_t>(16 * room)));
  }
  __device__ __forceinline__ void put(int32_t id) {
    const int at = place(id);
    const uint32_t bit = 1u << (at & 31);
    if (atomicOr(&seen[at >> 5], bit) & bit) atomicOr(&twice[at >> 5], bit);
  }
  __device__ __forceinline__ int count(int32_t id) const {
    int same = 0;
    for (int i = 0; i < room; i += 4) {
      const int4 v = *reinterpret_cast<const int4*>(ids + i);
      same += (v.x == id) + (v.y == id) + (v.z == id) + (v.w == id);
    }
    return same;
  }
  // Whether an entry names class id.
  __device__ __forceinline__ bool named(int32_t id) const {
    if (many) {
      const int at = place(id);
      const bool in = seen[at >> 5] >> (at & 31) & 1;
      if (exact || !in) return in;
    }
    return count(id) > 0;
  }
  // What the entries of entry j's class add up to, in their order.
  __device__ __forceinline__ float share(int32_t id, int j) const {
    if (many) {
      const int at = place(id);
      if (!(twice[at >> 5] >> (at & 31) & 1)) return ps[j];
    }
    if (count(id) == 1) return ps[j];
    float p = 0.f;
    for (int i = 0; i < room; ++i) p += ids[i] == id ? ps[i] : 0.f;
    return p;
  }
};

// The teacher's entries of a row in LDS (classes in `ids`, -1 for an invalid
// one and past the last; probabilities in `ps`), then the loss and the gradient's factors; m,
// st and s1 are the row's statistics.  Every thread of the row calls it.
template <typename T, int TH>
__device__ __forceinline__ RowTerms row_terms(const DistillArgs& a, int64_t row, bool live, const T* z, float m,
                                              float st, float s1, const Early& first, int t, Entries& in, float* red,
                                              float& loss) {
  RowTerms r;
  const float inv_t = 1.f / a.temperature;
  const float inv_n = 1.f / static_cast<float>(a.rows);
  r.m = m;
  r.kt = kLog2e * inv_t;
  const bool some = live && !(st == 0.f);   // not: every logit is -inf
  // the teacher
  float mt = -INFINITY;
  int32_t* ids = in.ids;
  float* ps = in.ps;
  for (int j = t; j < in.room; j += TH) {
    int32_t id = -1;
    float v = -INFINITY;
    if (j == t) {
      id = some ? first.id : -1;
      v = some ? first.t : -INFINITY;
    } else if (j < a.k && some && a.alpha > 0.f) {
      id = a.top_ids[row * a.k + j];
      v = a.top[row * a.k + j];
      if (id < 0 || id >= a.classes || v == -INFINITY) {
        id = -1;
        v = -INFINITY;
      }
    }
    ids[j] = id;
    ps[j] = v;
    if (in.many && id >= 0) in.put(id);
    mt = fmaxf(mt, v);
  }
  mt = row_reduce<TH>(mt, Max(), red);
  mt = mt == -INFINITY ? 0.f : mt;
  float sum = 0.f;
  // (over T after the difference: the type's lowest value over T < 1 is -inf)
  for (int j = t; j < a.k; j += TH) sum += exp2_((ps[j] - mt) * r.kt);
  sum = row_reduce<TH>(sum, Sum(), red);
  const bool any = !(sum == 0.f);
  const float log_sum = logf(sum), log_st = logf(st), inv_sum = any ? 1.f / sum : 0.f;
  float kl = 0.f;
  if (any) {
    for (int j = t; j < a.k; j += TH) {
      const int32_t id = ids[j];
      const float u = ps[j] - mt;
      const float p = exp2_(u * r.kt) * inv_sum;
      ps[j] = p;
      if (id >= 0 && !(p == 0.f)) {
        const float zj = j == t ? first.z : load_logit(z + id);
        kl += p * ((u * inv_t - log_sum) - ((zj - m) * inv_t - log_st));
      }
    }
  }
  kl = row_reduce<TH>(kl, Sum(), red);
  r.ft = any ? a.alpha * a.temperature * inv_n / st : 0.f;
  r.fp = a.alpha * a.temperature * inv_n;
  r.label = some ? first.label : -1;
  r.fy = (1.f - a.alpha) * inv_n;
  r.f1 = r.label >= 0 ? r.fy / s1 : 0.f;
  r.none = !any && r.label < 0;
  loss = any ? a.alpha * a.temperature * a.temperature * kl : 0.f;
  if (r.label >= 0) loss += (1.f - a.alpha) * (logf(s1) - (first.zl - m));
  return r;
}

// The gradient of one chunk, what the teacher and the label take off left
// out (correct_entries).
template <int POW, typename T>
__device__ __forceinline__ void chunk_gradient(const RowTerms& r, const uint4& q, float (&g)[Chunk<T>::N]) {
  Chunk<T>::unpack(q, g);
#pragma unroll
  for (int e = 0; e < Chunk<T>::N; ++e) {
    const float d = g[e] - r.m, u = exp2_(d * r.kt);
    g[e] = r.ft * u + r.f1 * hard_exp<POW>(u, d);
  }
}

// The classes in [lo, hi) that the teacher's entries or the label name: the
// whole gradient again, less their shares.  Entries of one class add up in the
// entries' order, and all that name a class write the same value; the label's
// class is its entries' to write, if it has any.
template <typename T, int TH>
__device__ __forceinline__ void correct_entries(const DistillArgs& a, const RowTerms& r, const T* z, T* grad,
                                                const Early& first, int t, const Entries& in, int64_t lo, int64_t hi) {
  if (r.none) return;
  auto write = [&](int32_t id, float p, float zi) {
    const float d = zi - r.m;
    Chunk<T>::store1(grad + id, r.ft * exp2_(d * r.kt) - r.fp * p + r.f1 * exp2_(d * kLog2e) -
                                    (id == r.label ? r.fy : 0.f));
  };
  for (int j = t; j < a.k; j += TH) {
    const int32_t id = in.ids[j];
    if (id >= lo && id < hi) write(id, in.share(id, j), j == t ? first.z : load_logit(z + id));
  }
  if (t == TH - 1 && r.label >= lo && r.label < hi && !in.named(r.label)) write(r.label, 0.f, first.zl);
}

// Makes loaded chunks opaque, so that what one pass computed of them (their
// values, differences, exponentials) is not kept in registers for the next.
template <int K>
__device__ __forceinline__ void forget(uint4 (&q)[K]) {
#pragma unroll
  for (int k = 0; k < K; ++k) asm volatile("" : "+v"(q[k].x), "+v"(q[k].y), "+v"(q[k].z), "+v"(q[k].w));
}

// TH threads hold a row of up to TH * K chunks as they were loaded (the
// values twice over would halve the rows that a CU has in flight); WAVES: the
// waves a SIMD is to hold.
template <typename T, int TH, int K, int POW, int WAVES, bool STREAM>
__global__ __launch_bounds__(TH < 256 ? 256 : TH) __attribute__((amdgpu_waves_per_eu(WAVES)))
void k_distill_held(DistillArgs a) {
  constexpr int E = Chunk<T>::N;
  constexpr int ROWS = TH < 256 ? 256 / TH : 1;
  extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
  __shared__ float red[16];
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < a.clear_n;
       i += static_cast<int64_t>(gridDim.x) * blockDim.x)
    a.clear[i] = 0;
  const int sub = threadIdx.x / TH, t = threadIdx.x % TH;
  Entries in(lds, a, sub, ROWS);
  in.clear<TH>(t);
  __syncthreads();
  int64_t row = a.row0 + static_cast<int64_t>(blockIdx.x) * ROWS + sub;
  const bool live = row < a.rows;
  if (!live) row = a.rows - 1;
  const T* z = static_cast<const T*>(a.logits) + row * a.classes;
  // the row's loads, its entries' and its last chunk's are on the way together
  // (a fourteenth less time than each waited for by itself, 4,099 x 32,768 bf16)
  uint4 q[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = (k * TH + t) * E;
    q[k] = masked_chunk<T>();
    if (c + E <= a.classes) {
      if constexpr (STREAM) mx_get_once<16>(&q[k], z + c);
      else mx_get<16>(&q[k], z + c);
    }
  }
  Early first = early_entry(a, row, live, t);
  // the chunk that the row ends in, if it is not whole, by the thread whose it is
  const int whole = a.classes / E;
  if (whole * E < a.classes && whole % TH == t) {
    const uint4 tail = load_tail(z, whole * E, a.classes);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const bool here = k == whole / TH;
      q[k].x = here ? tail.x : q[k].x;
      q[k].y = here ? tail.y : q[k].y;
      q[k].z = here ? tail.z : q[k].z;
      q[k].w = here ? tail.w : q[k].w;
    }
  }
  early_logits(a, z, first);
  float m = -INFINITY;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    float v[E];
    Chunk<T>::unpack(q[k], v);
#pragma unroll
    for (int e = 0; e < E; ++e) m = fmaxf(m, v[e]);
  }
  m = row_reduce<TH>(m, Max(), red);
  m = m == -INFINITY ? 0.f : m;
  forget(q);
  const float kt = kLog2e / a.temperature;
  const bool hard = a.labels && a.alpha < 1.f;
  float st = 0.f, s1 = 0.f;
  if (hard) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float v[E];
      Chunk<T>::unpack(q[k], v);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float d = v[e] - m, u = exp2_(d * kt);
        st += u;
        s1 += hard_exp<POW>(u, d);
      }
      __builtin_amdgcn_sched_barrier(0);   // one chunk's values at a time
    }
  } else {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float v[E];
      Chunk<T>::unpack(q[k], v);
#pragma unroll
      for (int e = 0; e < E; ++e) st += exp2_((v[e] - m) * kt);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  st = row_reduce<TH>(st, Sum(), red);
  if (hard) s1 = row_reduce<TH>(s1, Sum(), red);
  float loss;
  const RowTerms r = row_terms<T, TH>(a, row, live, z, m, st, s1, first, t, in, red, loss);
  if (live && t == 0) a.loss_rows[row] = loss;
  if (!a.grad) return;
  T* grad = static_cast<T*>(a.grad) + row * a.ld_grad;
  forget(q);
  if (live) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * TH + t) * E;
      if (c >= a.classes) break;
      float g[E] = {};
      if (!r.none) chunk_gradient<POW, T>(r, q[k], g);   // (0 whatever the logits are)
      store_chunk<STREAM>(grad, c, a.classes, g);
      __builtin_amdgcn_sched_barrier(0);
    }
    for (int64_t c = a.classes + t; c < a.ld_grad; c += TH) Chunk<T>::store1(grad + c, 0.f);
  }
  __syncthreads();   // the entries' classes are written again
  if (live) correct_entries<T, TH>(a, r, z, grad, first, t, in, 0, a.classes);
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
    Chunk<T>::unpack(load_chunk(z, c, hi), v);
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
  extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
  __shared__ float red[16];
  const int t = threadIdx.x;
  Entries in(lds, a, 0, 1);
  in.clear<kSplitThreads>(t);   // (the reductions below are barriers)
  const int64_t row = blockIdx.x / a.parts;
  const int part = static_cast<int>(blockIdx.x % a.parts);
  const T* z = static_cast<const T*>(a.logits) + row * a.classes;
  Early first = early_entry(a, row, true, t);
  early_logits(a, z, first);
  const float kt = kLog2e / a.temperature;
  // the parts' statistics, each thread some of them (a row has at most as many parts as threads)
  const float* stats = a.stats + 3 * row * a.parts;
  const bool has = t < a.parts;
  const float mi = has ? stats[3 * t] : -INFINITY;
  float m = row_reduce<kSplitThreads>(mi, Max(), red);
  m = m == -INFINITY ? 0.f : m;
  const float st = row_reduce<kSplitThreads>(
      has ? stats[3 * t + 1] * (mi == -INFINITY ? 1.f : exp2_((mi - m) * kt)) : 0.f, Sum(), red);
  const float s1 = row_reduce<kSplitThreads>(
      has ? stats[3 * t + 2] * (mi == -INFINITY ? 1.f : exp2_((mi - m) * kLog2e)) : 0.f, Sum(), red);
  float loss;
  const RowTerms r = row_terms<T, kSplitThreads>(a, row, true, z, m, st, s1, first, t, in, red, loss);
  if (part == 0 && t == 0) a.loss_rows[row] = loss;
  if (!a.grad) return;
  T* grad = static_cast<T*>(a.grad) + row * a.ld_grad;
  int64_t lo, hi;
  part_range(a.classes, a.parts, part, lo, hi);
  for (int64_t c = lo + t * E; c < hi; c += kSplitThreads * E) {
    float g[E] = {};
    if (!r.none) chunk_gradient<0, T>(r, load_chunk(z, c, hi), g);
    store_chunk<false>(grad, c, hi, g);
  }
  __syncthreads();
  correct_entries<T, kSplitThreads>(a, r, z, grad, first, t, in, lo, hi);
}

// 64 bits: a chain is n / 8192 terms long, and terms alike are all rounded the
// same way (2^26 rows of one loss: fp32 chains of 2^14 terms were off by 4.9e-5 of
// it).
__global__ __launch_bounds__(1024) void k_loss_mean(const float* rows, int64_t n, float* loss) {
  constexpr int U = 8;
  __shared__ double red[16];
  double s[U] = {};
  for (int64_t i = threadIdx.x; i < n; i += 1024 * U) {
    float v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = rows[i + 1024 * u < n ? i + 1024 * u : i];
#pragma unroll
    for (int u = 0; u < U; ++u) s[u] += i + 1024 * u < n ? v[u] : 0.f;
  }
#pragma unroll
  for (int h = U / 2; h > 0; h /= 2)
#pragma unroll
    for (int u = 0; u < h; ++u) s[u] += s[u + h];
  const double all = row_reduce<1024>(s[0], Sum(), red);
  if (threadIdx.x == 0) *loss = static_cast<float>(all / static_cast<double>(n));
}

template <typename T, int TH, int K, int WAVES, bool STREAM = false>
void held(const DistillArgs& args, hipStream_t s) {
  constexpr int ROWS = TH < 256 ? 256 / TH : 1;
  constexpr int64_t kRows = kLaunchThreads / TH;   // of a launch
  DistillArgs a = args;
  const size_t lds = static_cast<size_t>(entry_bytes(a.k)) * ROWS;
  const float t = a.temperature;
  for (a.row0 = 0; a.row0 < a.rows; a.row0 += kRows) {
    const int64_t rows = a.rows - a.row0 < kRows ? a.rows - a.row0 : kRows;
    const dim3 grid(static_cast<unsigned>((rows + ROWS - 1) / ROWS)), block(TH < 256 ? 256 : TH);
    if (t == 1.f) hipLaunchKernelGGL((k_distill_held<T, TH, K, 1, WAVES, STREAM>), grid, block, lds, s, a);
    else if (t == 2.f) hipLaunchKernelGGL((k_distill_held<T, TH, K, 2, WAVES, STREAM>), grid, block, lds, s, a);
    else if (t == 4.f) hipLaunchKernelGGL((k_distill_held<T, TH, K, 4, WAVES, STREAM>), grid, block, lds, s, a);
    else hipLaunchKernelGGL((k_distill_held<T, TH, K, 0, WAVES, STREAM>), grid, block, lds, s, a);
    a.clear_n = 0;
  }
}

// Threads of a row.  Short rows: as few as hold them, so that a wave has several
// rows and shares their reductions (calls, T = 1.5, 8 entries: 30,000 x 200 bf16
// in 64 threads 43.4 us, 32 36.8, 16 22.2; 60,000 x 47 fp32 in 64 61.1, 32 43.4, 16
// 25.0, 8 20.0; 8,000 x 601 fp32 in 64 18.5, 32 16.7); but their rows' entries are
// to fit 48 KB of LDS.  Longer rows: 256 or 512, and of the waves of a SIMD the
// most whose registers hold their chunks without spilling (one register at 512 x
// 8): a row waits for its loads and its reductions, and another's exponentials
// fill the time.  4,099 x 32,768 bf16, 64 entries, 512 threads: 125 us at five (two
// workgroups a CU), 117 at six (three), 149 at eight (27 registers spilled); 2,000
// x 30,000 fp32: 126 us in 1,024 threads of 8 chunks, 102 in 512 of 16.
//   Long rows with a large gradient: logits and gradient past the caches (plain
// 121 and streaming 117 us, 105 and 102; 16,000 x 4,000 fp32, 256 MB, 8 entries
// 102 and 93, but 64 entries 107 and 119, as corrections come back to lines that
// have left; 8,000 x 1,000, 32 MB, no difference).
template <typename T, bool STREAM>
void long_rows(const DistillArgs& a, hipStream_t s) {
  constexpr int E = Chunk<T>::N;
  const int chunks = (a.classes + E - 1) / E;
  if (chunks <= 1024) {
    held<T, 256, 4, 8, STREAM>(a, s);
  } else if (chunks <= 2048) {
    held<T, 256, 8, 5, STREAM>(a, s);
  } else if (chunks <= 4096) {
    held<T, 512, 8, 6, STREAM>(a, s);
  } else if constexpr (E == 4) {
    held<T, 512, 16, 4, STREAM>(a, s);
  }
}

template <typename T>
void dispatch(const DistillArgs& a, hipStream_t s) {
  constexpr int E = Chunk<T>::N;
  const int chunks = (a.classes + E - 1) / E;
  if (a.stats) {
    const dim3 grid(static_cast<unsigned>(a.rows * a.parts));
    hipLaunchKernelGGL((k_distill_stats<T>), grid, dim3(kSplitThreads), 0, s, a);
    hipLaunchKernelGGL((k_distill_grad<T>), grid, dim3(kSplitThreads), entry_bytes(a.k), s, a);
  } else if (chunks <= 16 && a.k <= 128) {
    held<T, 8, 2, 4>(a, s);
  } else if (chunks <= 64 && a.k <= 256) {
    held<T, 16, 4, 4>(a, s);
  } else if (chunks <= 256 && a.k <= 512) {
    held<T, 32, 8, 5>(a, s);
  } else if (chunks <= 256) {
    held<T, 64, 4, 8>(a, s);
  } else if (a.rows * a.classes * static_cast<int64_t>(sizeof(T)) >= 4 * kStreamBytes) {
    long_rows<T, true>(a, s);
  } else {
    long_rows<T, false>(a, s);
  }
}

}  // namespace

int distill_parts(int64_t rows, int64_t classes) {
  if (classes > kDistillHeld || (classes > 4096 && rows < 64)) {
    int64_t parts = (2048 + rows - 1) / rows;
    const int64_t most = (classes + 2047) / 2048;
    parts = parts < most ? parts : most;
    parts = parts < kSplitThreads ? parts : kSplitThreads;
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
