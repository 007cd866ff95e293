// The microscaled vertex store on gfx950: rows written into it, read back
// from it, and averaged straight out of it (mx.hpp has the format).
//
//   k_mx_write       rows x -> records: a lane takes 16 bytes of a row, four
//                    (bf16) or eight (fp32) lanes a block; the block's largest
//                    magnitude in two or three lane exchanges
//   k_mx_write_cols  the same for rows that lie across memory (a weight
//                    matrix read by its columns): a lane takes a whole block,
//                    neighbouring lanes neighbouring rows
//   k_mx_claim       the last of several rows written to one vertex wins
//   k_mx_read        records -> rows
//   k_mx_mean        m_v = (1/k_v) sum_e value(table[ids[e]]), fp32 sums: a
//                    lane takes one block of a destination, so a neighbour is
//                    one 16-byte (4 bits) or two (8 bits) reads and a scale
#include <type_traits>

#include "edge_steps.hpp"
#include "mx.hpp"
#include "mx_kernels.hpp"

namespace gmb {

namespace {

constexpr int kMaxGrid = 1 << 16;

__device__ __forceinline__ int64_t row_count(const int32_t* n_dev, int64_t n_cap) {
  if (!n_dev) return n_cap;
  const int64_t m = load_size(n_dev);
  return m < 0 ? 0 : (m < n_cap ? m : n_cap);
}

// 16 bytes of a row's values (4 fp32, 8 bf16), zeros from `left` on; read
// once, so past the caches (350,000 rows of 128 bf16: 39.4 us, 30.7 so).
__device__ __forceinline__ void load_values(const float* p, int left, float (&v)[4]) {
  if (left >= 4) {
    mx_get_once<16>(v, p);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < left ? p[i] : 0.f;
  }
}
__device__ __forceinline__ void load_values(const uint16_t* p, int left, float (&v)[8]) {
  if (left >= 8) {
    uint32_t w[4];
    mx_get_once<16>(w, p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    if (left > 0) {
      // (together: one by one each is widened, and waited for, before the next;
      // 346,000 rows of 100 to 8 bits 55 us, so 43)
      uint16_t u[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = p[i < left ? i : 0];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < left ? bf16_to_f32(u[i]) : 0.f;
    }
  }
}
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const uint16_t* p) { return bf16_to_f32(*p); }

// Where row `row` of a write goes: the record of its vertex `id`, or nothing
// (an id outside the table, or a row that a later one of the same vertex
// replaces).
__device__ __forceinline__ uint8_t* write_to(const MxWriteArgs& a, int64_t row, int32_t id, bool& bad) {
  if (!a.ids) return a.table + row * a.table_stride;
  if (!valid_vertex(id, a.table_rows)) {
    bad = true;
    return nullptr;
  }
  if (a.slots && a.slots[id] != kEdgeTag - 1 - static_cast<uint32_t>(row)) return nullptr;
  return a.table + id * a.table_stride;
}

// A lane has 16 bytes of a row (E values), 32 / E lanes a block; a row's
// values and its id are asked for together.  TAIL: the scales and the
// zeros after them are one 16-byte piece (at most 16 blocks, all of them in
// one pass of the group), which the group's first lanes store at once.
template <typename T, int BITS, int G, bool TAIL>
__global__ __launch_bounds__(256) void k_mx_write(MxWriteArgs a) {
  constexpr int E = 16 / sizeof(T), LB = 32 / E;
  constexpr int kCode = 4 * BITS;   // element bytes of a block
  const int lane = threadIdx.x & (G - 1);
  const int64_t n = row_count(a.n_dev, a.n_cap);
  const T* x = static_cast<const T*>(a.x);
  bool bad = false;
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * (256 / G) + threadIdx.x / G; row < n;
       row += static_cast<int64_t>(gridDim.x) * (256 / G)) {
    uint8_t* rec = nullptr;
    const int32_t id = a.ids ? a.ids[row] : 0;
    for (int b0 = 0; b0 < a.blocks; b0 += G / LB) {
      const int b = b0 + lane / LB, at = (b0 * LB + lane) * E;
      float v[E];
      load_values(x + row * a.row_stride + (at < a.dim ? at : 0), a.dim - at, v);
      if (b0 == 0) rec = write_to(a, row, id, bad);   // the group's lanes agree
      const uint32_t code = mx_scale_code<BITS>(mx_lanes_max<LB>(mx_top(v)));   // (0 past the last block)
      uint32_t w[(E * BITS + 31) / 32];
      mx_pack<BITS, E>(v, code, w);
      if (b < a.blocks && rec) __builtin_memcpy(rec + at * BITS / 8, w, E * BITS / 8);
      if constexpr (TAIL) {
        // lane i of the first four has the scales of blocks 4 i .. 4 i + 3
        uint32_t word = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int from = LB * (4 * lane + i);
          const uint32_t c = __shfl(code, from < G ? from : 0, G);
          word |= (from < G ? c : 0u) << (8 * i);
        }
        if (lane < 4 && rec) __builtin_memcpy(rec + a.blocks * kCode + 4 * lane, &word, 4);
      } else if (lane % LB == 0 && b < a.blocks && rec) {
        rec[a.blocks * kCode + b] = static_cast<uint8_t>(code);
      }
    }
    if constexpr (!TAIL)
      if (rec)
        for (int i = a.blocks * (kCode + 1) + lane; i < a.record; i += G) rec[i] = 0;
  }
  if (bad) raise_status(a.status, GMB_STATUS_ERANGE);
}

template <typename T, int BITS>
__global__ __launch_bounds__(256) void k_mx_write_cols(MxWriteArgs a) {
  constexpr int kCode = 4 * BITS;
  const int64_t n = row_count(a.n_dev, a.n_cap);
  const T* x = static_cast<const T*>(a.x);
  const int b = blockIdx.y;
  bool bad = false;
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * 64 + (threadIdx.x & 63); row < n;
       row += static_cast<int64_t>(gridDim.x) * 64) {
    uint8_t* rec = write_to(a, row, a.ids ? a.ids[row] : 0, bad);
    if (!rec) continue;
    const T* xr = x + row * a.row_stride;
    for (int blk = b * 4 + (threadIdx.x >> 6); blk < a.blocks; blk += 4 * gridDim.y) {
      float v[kMxBlock];
#pragma unroll
      for (int i = 0; i < kMxBlock; ++i) {
        const int c = blk * kMxBlock + i;
        v[i] = c < a.dim ? load1(xr + c * a.col_stride) : 0.f;
      }
      const uint32_t code = mx_scale_code<BITS>(mx_top(v));
      uint32_t w[BITS];
      mx_pack<BITS, kMxBlock>(v, code, w);
      __builtin_memcpy(rec + blk * kCode, w, kCode);
      rec[a.blocks * kCode + blk] = static_cast<uint8_t>(code);
      if (blk == 0)
        for (int i = a.blocks * (kCode + 1); i < a.record; ++i) rec[i] = 0;
    }
  }
  if (bad) raise_status(a.status, GMB_STATUS_ERANGE);
}

// The vertex's slot takes the smallest of (2^31 - 1 - position) over the
// rows written to it: the last row.  release: every slot empty again.
__global__ __launch_bounds__(256) void k_mx_claim(const int32_t* ids, const int32_t* n_dev, int64_t n_cap,
                                                  int64_t rows, uint32_t* slots, int release) {
  const int64_t n = row_count(n_dev, n_cap);
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n;
       i += static_cast<int64_t>(gridDim.x) * 256) {
    const int32_t id = ids[i];
    if (!valid_vertex(id, rows)) continue;
    if (release)
      slots[id] = kEmpty;
    else
      atomicMin(&slots[id], kEdgeTag - 1 - static_cast<uint32_t>(i));
  }
}

// A lane writes 16 bytes of a row (E values), so that a group's stores are one
// contiguous piece (346,000 rows of 100 fp32, plain stores: 55 us, 69 where four
// lanes' 64 bytes lay 128 apart).  U rows of a group in flight, their ids asked
// for together (plain stores, one by one 47.7 us, so 43.0; U = 2 47.5, 8 45.1;
// streaming stores, U = 2 31.7, 4 33.2, 8 33.9); every load unconditional from a
// clamped address (row 0 for a group without a row or with an id outside the
// table).
template <typename T, int BITS, int G, int U, bool STREAM>
__global__ __launch_bounds__(256) void k_mx_read(MxReadArgs a) {
  constexpr int E = 16 / sizeof(T), kBytes = E * BITS / 8;
  const int lane = threadIdx.x & (G - 1);
  const int64_t n = row_count(a.n_dev, a.n_cap);
  const int64_t stride = static_cast<int64_t>(gridDim.x) * (256 / G);
  const int chunks = (a.dim + E - 1) / E, scales = a.blocks * 4 * BITS;
  T* out = static_cast<T*>(a.out);
  bool bad = false;
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * (256 / G) + threadIdx.x / G; row < n; row += stride * U) {
    int64_t id[U];
    bool in[U];
    if (a.ids) {
#pragma unroll
      for (int u = 0; u < U; ++u) id[u] = a.ids[row + u * stride < n ? row + u * stride : row];
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) id[u] = row + u * stride;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool here = row + u * stride < n, ok = id[u] >= 0 && id[u] < a.table_rows;
      bad |= here & !ok;
      in[u] = here & ok;
      id[u] = in[u] ? id[u] : 0;
    }
    for (int c = lane; c < chunks; c += G) {
      uint32_t w[U][(E * BITS + 31) / 32];
      uint32_t code[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint8_t* rec = a.table + id[u] * a.table_stride;
        if constexpr (kBytes == 2) w[u][0] = 0;
        __builtin_memcpy(w[u], rec + c * kBytes, kBytes);
        code[u] = rec[scales + c / (32 / E)];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t r = row + u * stride;
        float v[E];
        mx_unpack<BITS, E>(w[u], code[u], v);
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = in[u] ? v[i] : 0.f;
        if (r < n) mx_store<STREAM>(out + r * a.dim + c * E, v, a.dim - c * E);
      }
    }
  }
  if (bad) raise_status(a.status, GMB_STATUS_ERANGE);
}

// OUT: 0 fp32 rows, 1 bf16 rows, 2 records of 4 bits (of a 4-bit table).  A lane has E elements
// of a destination (16 bytes of its row), G lanes a destination; U neighbours
// in flight.  An id outside the table is read as row 0 (k_mean's rule); a
// model's forward (records) also reports it, by the largest id that it met, a
// negative one being larger than every row's.
template <int BITS, int OUT, int G, int U, bool STREAM>
__global__ __launch_bounds__(256) void k_mx_mean(MxMeanArgs a) {
  constexpr int E = OUT == 0 ? 4 : 8, LB = 32 / E, kBytes = E * BITS / 8, kWords = (E * BITS + 31) / 32;
  const int64_t row = a.row0 + (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) / G;
  const int lane = threadIdx.x & (G - 1);
  const int64_t rc = row < a.n_cap ? row : a.n_cap - 1;
  const int32_t beg = a.indptr[rc], end = a.indptr[rc + 1];
  if (row >= row_count(a.n_dev, a.n_cap)) return;
  const int32_t k = end - beg;
  const int chunks = OUT == 2 ? a.blocks * LB : (a.dim + E - 1) / E, scales = a.blocks * 4 * BITS;
  uint32_t largest = 0;
  for (int c = lane; c < chunks; c += G) {
    float acc[E];
#pragma unroll
    for (int i = 0; i < E; ++i) acc[i] = 0.f;
    edge_steps<U>(beg, end, [&](int32_t e, int32_t n, auto&& at) {
      int64_t id[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int32_t i = a.ids[at(u)];
        if constexpr (OUT == 2) largest = static_cast<uint32_t>(i) > largest ? static_cast<uint32_t>(i) : largest;
        id[u] = valid_vertex(i, a.table_rows) ? i : 0;
      }
      uint32_t w[U][kWords];
      uint32_t code[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint8_t* rec = a.table + id[u] * a.table_stride;
        if constexpr (kBytes == 2) w[u][0] = 0;
        __builtin_memcpy(w[u], rec + c * kBytes, kBytes);
        code[u] = rec[scales + c / LB];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        // a slot past the row's end: zeros at scale 1 (adding +0 changes
        // nothing)
        const bool in = u < n - e;
#pragma unroll
        for (int j = 0; j < kWords; ++j) w[u][j] = in ? w[u][j] : 0u;
        float v[E];
        mx_unpack<BITS, E>(w[u], in ? code[u] : 127u, v);
#pragma unroll
        for (int i = 0; i < E; ++i) acc[i] += v[i];
      }
    });
    if (k > 0) {
      const float kf = static_cast<float>(k);
#pragma unroll
      for (int i = 0; i < E; ++i) acc[i] = acc[i] / kf;
    }
    if constexpr (OUT == 2) {
      const uint32_t code = mx_scale_code<4>(mx_lanes_max<LB>(mx_top(acc)));
      uint8_t* rec = static_cast<uint8_t*>(a.out) + row * a.out_stride;
      uint32_t w[1];
      mx_pack<4, E>(acc, code, w);
      __builtin_memcpy(rec + c * 4, w, 4);
      if (c % LB == 0) rec[a.blocks * 16 + c / LB] = static_cast<uint8_t>(code);
    } else {
      using O = std::conditional_t<OUT == 0, float, uint16_t>;
      mx_store<STREAM>(static_cast<O*>(a.out) + row * a.dim + c * E, acc, a.dim - c * E);
    }
  }
  if constexpr (OUT == 2) {
    uint8_t* rec = static_cast<uint8_t*>(a.out) + row * a.out_stride;
    for (int i = a.blocks * 17 + lane; i < a.out_record; i += G) rec[i] = 0;
    if (largest >= a.table_rows) raise_status(a.status, GMB_STATUS_ERANGE);
  }
}

unsigned grid_for(int64_t rows, int64_t per_block) {
  int64_t g = (rows + per_block - 1) / per_block;
  g = g < 1 ? 1 : (g > kMaxGrid ? kMaxGrid : g);
  return static_cast<unsigned>(g);
}

// lanes of a row: a power of two that holds `units`, lo .. 64
int lanes_for(int units, int lo) {
  int g = lo;
  while (g < 64 && g < units) g *= 2;
  return g;
}

template <typename T, int BITS>
void write_dispatch(const MxWriteArgs& a, hipStream_t s) {
  if (a.col_stride != 1) {
    const unsigned gy = static_cast<unsigned>(a.blocks < 4 * 64 ? (a.blocks + 3) / 4 : 64);
    hipLaunchKernelGGL((k_mx_write_cols<T, BITS>), dim3(grid_for(a.n_cap, 64), gy), dim3(256), 0, s, a);
    return;
  }
#define GMB_MX_WRITE(GG, TAIL) \
  hipLaunchKernelGGL((k_mx_write<T, BITS, GG, TAIL>), dim3(grid_for(a.n_cap, 256 / GG)), dim3(256), 0, s, a)
  constexpr int LB = 2 * static_cast<int>(sizeof(T));   // lanes of a block
  switch (lanes_for(LB * a.blocks, LB)) {
    case 4: GMB_MX_WRITE(LB, true); break;
    case 8: GMB_MX_WRITE(8, true); break;
    case 16: GMB_MX_WRITE(16, true); break;
    case 32: GMB_MX_WRITE(32, true); break;
    default:
      if (LB * a.blocks <= 64) GMB_MX_WRITE(64, true);
      else GMB_MX_WRITE(64, false);
      break;
  }
#undef GMB_MX_WRITE
}

template <typename T, int BITS, bool STREAM>
void read_rows(const MxReadArgs& a, hipStream_t s) {
  constexpr int U = 4, E = 16 / static_cast<int>(sizeof(T));
#define GMB_MX_READ(GG) \
  hipLaunchKernelGGL((k_mx_read<T, BITS, GG, U, STREAM>), dim3(grid_for(a.n_cap, (256 / GG) * U)), dim3(256), 0, s, a)
  switch (lanes_for((a.dim + E - 1) / E, 2)) {
    case 2: GMB_MX_READ(2); break;
    case 4: GMB_MX_READ(4); break;
    case 8: GMB_MX_READ(8); break;
    case 16: GMB_MX_READ(16); break;
    case 32: GMB_MX_READ(32); break;
    default: GMB_MX_READ(64); break;
  }
#undef GMB_MX_READ
}

template <typename T, int BITS>
void read_dispatch(const MxReadArgs& a, hipStream_t s) {
  if (a.n_cap * a.dim * static_cast<int64_t>(sizeof(T)) >= kStreamBytes) read_rows<T, BITS, true>(a, s);
  else read_rows<T, BITS, false>(a, s);
}

template <int BITS, int OUT, bool STREAM>
void mean_rows(const MxMeanArgs& args, hipStream_t s) {
  constexpr int U = 8, E = OUT == 0 ? 4 : 8;
  MxMeanArgs a = args;
  const int g = lanes_for(OUT == 2 ? a.blocks * 4 : (a.dim + E - 1) / E, 4);
  for (a.row0 = 0; a.row0 < a.n_cap; a.row0 += kLaunchThreads / g) {
    const int64_t rows = a.n_cap - a.row0 < kLaunchThreads / g ? a.n_cap - a.row0 : kLaunchThreads / g;
    const dim3 grid(static_cast<unsigned>((rows * g + 255) / 256));
#define GMB_MX_MEAN(GG) hipLaunchKernelGGL((k_mx_mean<BITS, OUT, GG, U, STREAM>), grid, dim3(256), 0, s, a)
    switch (g) {
      case 4: GMB_MX_MEAN(4); break;
      case 8: GMB_MX_MEAN(8); break;
      case 16: GMB_MX_MEAN(16); break;
      case 32: GMB_MX_MEAN(32); break;
      default: GMB_MX_MEAN(64); break;
    }
  }
#undef GMB_MX_MEAN
}

template <int BITS, int OUT>
void mean_dispatch(const MxMeanArgs& a, hipStream_t s) {
  if constexpr (OUT != kMxOutRecords) {   // (records are the next layer's input)
    if (a.n_cap * a.dim * (OUT == kMxOutBf16 ? 2 : 4) >= kStreamBytes) return mean_rows<BITS, OUT, true>(a, s);
  }
  mean_rows<BITS, OUT, false>(a, s);
}

}  // namespace

hipError_t launch_mx_write(const MxWriteArgs& args, int bf16, int bits, uint32_t* slots, hipStream_t s) {
  MxWriteArgs a = args;
  a.slots = a.ids ? slots : nullptr;
  if (a.slots)
    hipLaunchKernelGGL(k_mx_claim, dim3(grid_for(a.n_cap, 256)), dim3(256), 0, s, a.ids, a.n_dev, a.n_cap,
                       a.table_rows, slots, 0);
  if (bits == 4) {
    if (bf16) write_dispatch<uint16_t, 4>(a, s);
    else write_dispatch<float, 4>(a, s);
  } else {
    if (bf16) write_dispatch<uint16_t, 8>(a, s);
    else write_dispatch<float, 8>(a, s);
  }
  if (a.slots)
    hipLaunchKernelGGL(k_mx_claim, dim3(grid_for(a.n_cap, 256)), dim3(256), 0, s, a.ids, a.n_dev, a.n_cap,
                       a.table_rows, slots, 1);
  return hipGetLastError();
}

hipError_t launch_mx_read(const MxReadArgs& a, int bf16, int bits, hipStream_t s) {
  if (bits == 4) {
    if (bf16) read_dispatch<uint16_t, 4>(a, s);
    else read_dispatch<float, 4>(a, s);
  } else {
    if (bf16) read_dispatch<uint16_t, 8>(a, s);
    else read_dispatch<float, 8>(a, s);
  }
  return hipGetLastError();
}

hipError_t launch_mx_mean(const MxMeanArgs& a, int bf16, int bits, hipStream_t s) {
  if (bits == 4) {
    if (bf16) mean_dispatch<4, kMxOutBf16>(a, s);
    else mean_dispatch<4, kMxOutF32>(a, s);
  } else {
    if (bf16) mean_dispatch<8, kMxOutBf16>(a, s);
    else mean_dispatch<8, kMxOutF32>(a, s);
  }
  return hipGetLastError();
}

hipError_t launch_mx_mean_records(const MxMeanArgs& a, hipStream_t s) {
  mean_dispatch<4, kMxOutRecords>(a, s);
  return hipGetLastError();
}

}  // namespace gmb
