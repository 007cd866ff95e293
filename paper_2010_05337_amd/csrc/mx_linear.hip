// The product of microscaled 4-bit rows and weights on gfx950:
// out = act(A W^T [+ A2 W2^T] + b) with v_mfma_scale_f32_16x16x128_f8f6f4,
// which takes 16 rows of 128 elements of each side, a scale for every 32
// elements of a row, and sums in fp32.  Lane l = 16 g + r of a wave supplies
// row r of its side, the 32 elements (16 bytes) of one of the four blocks and
// that block's scale byte; which blocks of the sum make up a step is free as
// long as both sides agree.  Accumulator register e of lane (g, r) is row
// 4 g + e of A and row r of W.  W's rows are dealt to the tiles of a wave so
// that a lane's CT column tiles are CT neighbouring columns: it stores them at
// once, and the lanes of a row store one contiguous piece.
//
//   k_mx_linear_rows      few rows: the waves of a workgroup split the sum
//   k_mx_linear_resident  short sums, many rows: the weights' whole records
//                         stay in LDS while the workgroup goes over row tiles
//   k_mx_linear_tiles     the rest: tiles of both sides in stages through LDS
//
// Loads: the vector memory unit takes neighbouring lanes' pieces of one
// 64-byte segment together, and a lane alone otherwise.  An operand read
// straight into its lanes (neighbouring lanes, different rows) is 64 accesses
// a kilobyte; the LDS kernels therefore load four neighbouring lanes a row (16
// accesses) and take the operands' order when they read LDS.  (8192 x 4096 x
// 4096, LDS filled in operand order: 125 us.)
#include "kernels.hpp"
#include "mx.hpp"
#include "mx_kernels.hpp"

namespace gmb {

namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx8 __attribute__((ext_vector_type(8)));

// Byte SEL of as and ws is the scale.  The 4-bit format (4) reads the first
// four words of an operand.
template <int SEL = 0>
__device__ __forceinline__ floatx4 mfma_mx4(const intx4& a, uint32_t as, const intx4& w, uint32_t ws, floatx4 c) {
  const intx8 a8 = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, w8 = {w[0], w[1], w[2], w[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, w8, c, 4, 4, SEL, static_cast<int>(as), SEL,
                                                          static_cast<int>(ws));
}

// What rows without a record, and blocks past a row's last, are loaded from.
__device__ __align__(16) const uint32_t kZeros[4] = {0, 0, 0, 0};

// 16 bytes a lane from global memory to LDS, at l + 16 lane.
__device__ __forceinline__ void load_lds(const void* g, void* l) {
  typedef const __attribute__((address_space(1))) void* gp;
  typedef __attribute__((address_space(3))) void* lp;
  __builtin_amdgcn_global_load_lds((gp)g, (lp)l, 16, 0, 0);
}

__device__ __forceinline__ int64_t count_rows(const MxLinearArgs& p) {
  if (!p.n_dev) return p.n_cap;
  const int64_t m = load_size(p.n_dev);
  return m < 0 ? 0 : (m < p.n_cap ? m : p.n_cap);
}

// The record of id v, or NULL for one outside the table, which is reported.
__device__ __forceinline__ const uint8_t* id_record(const MxLinearArgs& p, const MxPair& m, int32_t v) {
  if (valid_vertex(v, m.a_rows)) return m.a + v * m.a_stride;
  raise_status(p.status, GMB_STATUS_ERANGE);
  return nullptr;
}
// Row `row` (< n) of a pair's A.
__device__ __forceinline__ const uint8_t* a_record(const MxLinearArgs& p, const MxPair& m, int64_t row) {
  return m.ids ? id_record(p, m, m.ids[row]) : m.a + row * m.a_stride;
}
// Output column c's weights (the last column's past it: never stored).
__device__ __forceinline__ const uint8_t* w_record(const MxLinearArgs& p, const MxPair& m, int c) {
  return m.w + static_cast<int64_t>(c < p.d_out ? c : p.d_out - 1) * m.w_stride;
}

// Beside the form of the results (kMxOut...): stored past the caches.
constexpr int kStreamed = 4;

// CT neighbouring values of a row, from column c on.
template <int OUT, int CT>
__device__ __forceinline__ void store_values(const MxLinearArgs& p, int64_t row, int c, const float (&z)[CT]) {
  const int left = p.d_out - c;
  if constexpr ((OUT & 3) == kMxOutF32) {
    float* o = static_cast<float*>(p.out) + row * p.d_out + c;
    if (left >= CT) {
      mx_put<4 * CT, (OUT & kStreamed) != 0>(o, z);
    } else {
#pragma unroll
      for (int j = 0; j < CT; ++j)
        if (j < left) o[j] = z[j];
    }
  } else {
    uint16_t* o = static_cast<uint16_t*>(p.out) + row * p.d_out + c;
    uint32_t w[CT / 2];
#pragma unroll
    for (int j = 0; j < CT / 2; ++j) w[j] = mx_bf16x2_bits(z[2 * j], z[2 * j + 1]);
    if (left >= CT) {
      mx_put<2 * CT, (OUT & kStreamed) != 0>(o, w);
    } else {
#pragma unroll
      for (int j = 0; j < CT; ++j)
        if (j < left) o[j] = static_cast<uint16_t>(w[j / 2] >> (16 * (j & 1)));
    }
  }
}

// CT values of a row as elements of its output record: 32 / CT lanes hold a
// block.  Every lane takes part (its values are 0 past d_out).
template <int CT>
__device__ __forceinline__ void store_elements(const MxLinearArgs& p, bool in, int64_t row, int c,
                                               const float (&z)[CT]) {
  constexpr int LANES = 32 / CT;
  const int blocks = (p.d_out + 31) / 32;
  uint32_t top = mx_top(z);
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) {
    const uint32_t x = __shfl_xor(top, o, 64);
    top = x > top ? x : top;
  }
  const uint32_t code = mx_scale_code<4>(top);
  float v[4] = {};
#pragma unroll
  for (int j = 0; j < CT; ++j) v[j] = z[j];
  uint32_t w[1];
  mx_pack<4, 4>(v, code, w);
  const int blk = c / 32;
  if (!in || blk >= blocks) return;
  uint8_t* rec = static_cast<uint8_t*>(p.out) + row * p.out_stride;
  __builtin_memcpy(rec + c / 2, w, CT / 2);
  if (c % 32 == 0) rec[blocks * 16 + blk] = static_cast<uint8_t>(code);
  if (blk == blocks - 1)
    for (int b = blocks * 17 + (c % 32) / CT; b < p.out_record; b += LANES) rec[b] = 0;
}

// The bias of a lane's columns.
template <int CT>
__device__ __forceinline__ void load_bias(const MxLinearArgs& p, int c0, int lane, float (&bias)[CT]) {
  const int c = c0 + CT * (lane & 15);
#pragma unroll
  for (int j = 0; j < CT; ++j) bias[j] = p.bias && c + j < p.d_out ? p.bias[c + j] : 0.f;
}

// Bias, activation and store of a wave's tiles: rows r0 + 16 i + 4 g + e,
// columns c0 + CT r + j.
template <int RT, int CT, int OUT>
__device__ __forceinline__ void epilogue(const MxLinearArgs& p, int64_t n, int64_t r0, int c0, int lane,
                                         const float (&bias)[CT], const floatx4 (&acc)[RT][CT]) {
  const int c = c0 + CT * (lane & 15);
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t row = r0 + 16 * i + 4 * (lane >> 4) + e;
      float z[CT];
#pragma unroll
      for (int j = 0; j < CT; ++j) {
        z[j] = acc[i][j][e] + bias[j];
        if (p.relu) z[j] = z[j] > 0.f ? z[j] : 0.f;
        if (OUT == kMxOutRecords && c + j >= p.d_out) z[j] = 0.f;
      }
      if constexpr (OUT == kMxOutRecords)
        store_elements<CT>(p, row < n, row, c, z);
      else if (row < n && c < p.d_out)
        store_values<OUT, CT>(p, row, c, z);
    }
}

// ---- few rows -------------------------------------------------------------

// A workgroup of WK waves has 16 RT rows and 16 CT columns; wave k takes the
// units k, k + WK, ... of 16 blocks, of which lane group g has blocks 4 g ..
// 4 g + 3 (one scale word); the waves' sums meet in LDS in a fixed order.
template <int RT, int CT, int WK, int OUT>
__global__ __launch_bounds__(64 * WK) void k_mx_linear_rows(MxLinearArgs p) {
  const int lane = threadIdx.x & 63, wk = threadIdx.x >> 6, g = lane >> 4, r = lane & 15;
  const int64_t n = count_rows(p);
  const int64_t r0 = static_cast<int64_t>(blockIdx.x) * (16 * RT);
  if (r0 >= n) return;
  const int c0 = blockIdx.y * 16 * CT;
  floatx4 acc[RT][CT];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int j = 0; j < CT; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int units = (p.blocks + 15) / 16;
  for (int pr = 0; pr < p.pairs; ++pr) {
    const MxPair& m = p.pair[pr];
    const uint8_t* rec[RT + CT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int64_t row = r0 + 16 * i + r;
      rec[i] = a_record(p, m, row < n ? row : n - 1);
    }
#pragma unroll
    for (int j = 0; j < CT; ++j) rec[RT + j] = w_record(p, m, c0 + CT * r + j);
    for (int u = wk; u < units; u += WK) {
      const int b0 = 16 * u + 4 * g;
      intx4 q[RT + CT][4];
      uint32_t sc[RT + CT];
#pragma unroll
      for (int i = 0; i < RT + CT; ++i) {
        const uint8_t* some = reinterpret_cast<const uint8_t*>(kZeros);
        // (a record is padded to 16 bytes, so the scale word of a block in it
        // lies in it)
        const uint8_t* at = rec[i] && b0 < p.blocks ? rec[i] + p.blocks * 16 + b0 : some;
        __builtin_memcpy(&sc[i], at, 4);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          at = rec[i] && b0 + s < p.blocks ? rec[i] + (b0 + s) * 16 : some;
          __builtin_memcpy(&q[i][s], at, 16);
        }
      }
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < CT; ++j) {
          acc[i][j] = mfma_mx4<0>(q[i][0], sc[i], q[RT + j][0], sc[RT + j], acc[i][j]);
          acc[i][j] = mfma_mx4<1>(q[i][1], sc[i], q[RT + j][1], sc[RT + j], acc[i][j]);
          acc[i][j] = mfma_mx4<2>(q[i][2], sc[i], q[RT + j][2], sc[RT + j], acc[i][j]);
          acc[i][j] = mfma_mx4<3>(q[i][3], sc[i], q[RT + j][3], sc[RT + j], acc[i][j]);
        }
    }
  }
  if constexpr (WK > 1) {
    __shared__ floatx4 part[(WK - 1) * RT * CT * 64];
    if (wk > 0) {
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < CT; ++j) part[(((wk - 1) * RT + i) * CT + j) * 64 + lane] = acc[i][j];
    }
    __syncthreads();
    if (wk > 0) return;
#pragma unroll 1
    for (int k = 0; k < WK - 1; ++k)
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < CT; ++j) acc[i][j] += part[((k * RT + i) * CT + j) * 64 + lane];
  }
  float bias[CT];
  load_bias(p, c0, lane, bias);
  epilogue<RT, CT, OUT>(p, n, r0, c0, lane, bias, acc);
}

// ---- short sums, many rows ------------------------------------------------

// A workgroup of WR x WC waves has 64 WC columns, whose whole records lie in
// LDS from the start, and goes over tiles of 64 WR rows, whose records it
// brings tile by tile; workgroups of a CU hide each other's waits (45,000 rows,
// two pairs of 100 by 256: two a CU with 80 KB each 12.5 us, three 10.4).  With
// fp32 and bf16 results the registers (138) leave room for three, with records
// (177) for two.  In LDS a record is `slots` 16-byte pieces,
// an odd number: sixteen rows' reads of one block fall on different banks.  (The
// LDS serves half of such a sixteen with half of the next one's; pairs of blocks
// exchanged in rows 4 - 11 took those conflicts out, and 10.1 us for 9.7.)
constexpr int kResidentLds = 50 * 1024;

__host__ __device__ inline int resident_slots(int blocks) { return (((blocks * 17 + 15) / 16) | 1); }

// x / d for x < 2^16 and d >= 1 by one multiplication: m = floor((2^32 - 1) / d)
// + 1 is above 2^32 / d by at most 1, so x m is off by less than 2^16 of 2^32 a
// unit of the quotient, and a fraction of x / d is at most 1 - 1 / d.
__device__ __forceinline__ int quotient(int x, uint32_t m) {
  return static_cast<int>(__umulhi(static_cast<uint32_t>(x), m));
}

template <int WR, int WC, int OUT>
__global__ __launch_bounds__(64 * WR * WC, 2) void k_mx_linear_resident(MxLinearArgs p) {
  constexpr int WAVES = WR * WC, ROWS = 64 * WR, COLS = 64 * WC;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kResidentLds];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, r = lane & 15;
  const int wr = wave / WC, wc = wave % WC;
  const int64_t n = count_rows(p);
  const int tiles = static_cast<int>((n + ROWS - 1) / ROWS);
  const int c0 = blockIdx.y * COLS, cw = c0 + 64 * wc;
  const int slots = resident_slots(p.blocks), pieces = (p.blocks * 17 + 15) / 16;
  const uint32_t by_slots = 0xFFFFFFFFu / static_cast<uint32_t>(slots) + 1;   // (slots >= 3)
  const int a_side = ROWS * slots * 16, w_side = COLS * slots * 16;           // bytes of a pair's records
  uint8_t* lw = lds + p.pairs * a_side;
  int t = blockIdx.x;
  if (t >= tiles) return;
  // `count` records (record q of them at q * slots pieces), 64 pieces a load
  auto bring = [&](uint8_t* to, int count, auto&& record) {
    const int total = count * slots;
    for (int q0 = 64 * wave; q0 < total; q0 += 64 * WAVES) {
      const int q = q0 + lane, at = quotient(q, by_slots), piece = q - at * slots;
      if (q < total) {
        const uint8_t* rec = record(at);
        load_lds(rec && piece < pieces ? static_cast<const void*>(rec + piece * 16) : kZeros, to + q0 * 16);
      }
    }
  };
  auto bring_rows = [&](int tile) {
    const int64_t r0 = static_cast<int64_t>(tile) * ROWS;
    for (int pr = 0; pr < p.pairs; ++pr) {
      const MxPair& m = p.pair[pr];
      bring(lds + pr * a_side, ROWS,
            [&](int at) -> const uint8_t* { return r0 + at < n ? a_record(p, m, r0 + at) : nullptr; });
    }
  };
  float bias[4];
  load_bias(p, cw, lane, bias);
  for (int pr = 0; pr < p.pairs; ++pr) {
    const MxPair& m = p.pair[pr];
    bring(lw + pr * w_side, COLS, [&](int at) {
      // LDS order: 16-column tile j of 64 columns has columns 4 r + j
      return w_record(p, m, c0 + (at & ~63) + 4 * (at & 15) + ((at >> 4) & 3));
    });
  }
  bring_rows(t);
  const int steps = (p.blocks + 3) / 4;
  for (;;) {
    __syncthreads();            // the tile has arrived
    floatx4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int pr = 0; pr < p.pairs; ++pr) {
      const uint8_t* ra = lds + pr * a_side + (64 * wr + r) * slots * 16;
      const uint8_t* rw = lw + pr * w_side + (64 * wc + r) * slots * 16;
      for (int s = 0; s < steps; ++s) {
        const int b = 4 * s + g;
        const bool in = b < p.blocks;
        const int at = in ? b : 0;
        intx4 qa[4], qw[4];
        uint32_t sa[4], sw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint8_t* x = ra + i * 16 * slots * 16;
          qa[i] = *reinterpret_cast<const intx4*>(x + at * 16);
          sa[i] = x[p.blocks * 16 + at];
          const uint8_t* y = rw + i * 16 * slots * 16;
          qw[i] = *reinterpret_cast<const intx4*>(y + at * 16);
          sw[i] = y[p.blocks * 16 + at];
        }
        if (4 * s + 4 > p.blocks) {
          // a block past the last: zeros on one side, and no scale that is
          // not a number
#pragma unroll
          for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) qa[i][e] = in ? qa[i][e] : 0;
            sa[i] = in ? sa[i] : 127u;
            sw[i] = in ? sw[i] : 127u;
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j] = mfma_mx4<0>(qa[i], sa[i], qw[j], sw[j], acc[i][j]);
      }
    }
    const int64_t r0 = static_cast<int64_t>(t) * ROWS + 64 * wr;
    t += gridDim.x;
    if (t < tiles) {
      __syncthreads();          // the rows are read
      bring_rows(t);
    }
    if (cw < p.d_out) epilogue<4, 4, OUT>(p, n, r0, cw, lane, bias, acc);
    if (t >= tiles) break;
  }
}

// ---- tiles through LDS ----------------------------------------------------

// A workgroup of WM x WN waves has TM rows and TN columns, a wave TM / WM by
// TN / WN of them.  The sum goes in stages of eight blocks (256 elements); two
// stages are in LDS, one being read and one arriving straight from global
// memory.
//   Elements: 16 rows by four blocks are 1 KB, filled by one load, lane l
//   bringing row l / 4; piece (row, x) of them holds block x ^ swizzle(row).
//   The LDS serves lanes 0 - 3, 12 - 15 and 20 - 27 of a 32 at once, and then
//   the others (as timed): with neighbouring pieces exchanged in rows 8 - 15,
//   each such sixteen read 16 different pieces of 256 bytes (8,192 x 16,384 x
//   4,096: 278 us; with two lanes on each bank 284).
//   Scales: 16 bytes a row, for two stages, one lane a row.
// Step s of a stage takes block 2 g + s for lane group g: a lane's two scales
// are neighbours (one 16-bit read, the byte picked by the instruction).
__device__ __forceinline__ int tile_swizzle(int r) { return r >> 3; }

template <int TM, int TN, int WM, int WN, int OUT>
__global__ __launch_bounds__(64 * WM * WN, 2) void k_mx_linear_tiles(MxLinearArgs p, int gm, int gn) {
  constexpr int WAVES = WM * WN, T16 = (TM + TN) / 16, PER = T16 / WAVES;   // 16-row loads, of a wave
  constexpr int RT = TM / WM / 16, CT = TN / WN / 16;
  constexpr int SLOADS = ((TM + TN) / 64 + WAVES - 1) / WAVES;   // scale loads of a wave, 64 rows each
  static_assert(T16 % WAVES == 0 && CT == 4 && TM % 64 == 0 && TN % 64 == 0, "tile");
  constexpr int kStage = T16 * 2048, kScales = (TM + TN) * 16;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * (kStage + kScales)];
  const int64_t n = count_rows(p);
  // workgroup ids go round the eight XCDs: each takes a contiguous run of
  // tiles, eight row tiles wide, so that its L2 holds what they share
  const int tiles = gm * gn, per = (tiles + 7) / 8;
  const int id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= per || id >= tiles) return;
  const int band = id / (8 * gn), in_band = id - band * 8 * gn;
  const int height = gm - 8 * band < 8 ? gm - 8 * band : 8;
  const int64_t r0 = static_cast<int64_t>(8 * band + in_band % height) * TM;
  const int c0 = in_band / height * TN;
  if (r0 >= n) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wr = wave / WN, wc = wave % WN, g = lane >> 4, r = lane & 15;
  const int stages = (p.blocks + 7) / 8;
  floatx4 acc[RT][CT];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int j = 0; j < CT; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  for (int pr = 0; pr < p.pairs; ++pr) {
    const MxPair& m = p.pair[pr];
    // LDS row x: A's rows, then W's, dealt to a wave's column tiles.  The ids
    // are asked for together.
    int at[PER + SLOADS];
    int32_t id[PER + SLOADS];
#pragma unroll
    for (int i = 0; i < PER + SLOADS; ++i)
      at[i] = i < PER ? 16 * (PER * wave + i) + lane / 4 : 64 * (SLOADS * wave + i - PER) + lane;
    if (m.ids) {
#pragma unroll
      for (int i = 0; i < PER + SLOADS; ++i) id[i] = m.ids[at[i] < TM && r0 + at[i] < n ? r0 + at[i] : n - 1];
    }
    const uint8_t* from[PER + SLOADS];
#pragma unroll
    for (int i = 0; i < PER + SLOADS; ++i) {
      if (at[i] < TM) {
        const int64_t row = r0 + at[i] < n ? r0 + at[i] : n - 1;
        from[i] = m.ids ? id_record(p, m, id[i]) : m.a + row * m.a_stride;
      } else {
        const int c = at[i] - TM;
        from[i] = w_record(p, m, c0 + (c & ~63) + 4 * (c & 15) + ((c >> 4) & 3));
      }
    }
    const int x = (lane & 3) ^ tile_swizzle(lane / 4);
    auto fetch = [&](int k) {
      uint8_t* to = lds + (k & 1) * kStage + PER * wave * 2048;
#pragma unroll
      for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          const int b = 8 * k + 4 * f + x;
          load_lds(from[i] && b < p.blocks ? static_cast<const void*>(from[i] + b * 16) : kZeros,
                   to + (2 * i + f) * 1024);
        }
      // (16 scale bytes of blocks that there are lie in the padded record)
      if ((k & 1) == 0) {
#pragma unroll
        for (int i = 0; i < SLOADS; ++i) {
          const uint8_t* rec = from[PER + i];
          if (64 * (SLOADS * wave + i) < TM + TN)
            load_lds(rec ? static_cast<const void*>(rec + p.blocks * 16 + 8 * k) : kZeros,
                     lds + 2 * kStage + ((k >> 1) & 1) * kScales + (SLOADS * wave + i) * 1024);
        }
      }
    };
    __syncthreads();            // the last pair's reads
    fetch(0);
    __syncthreads();
    for (int k = 0; k < stages; ++k) {
      const uint8_t* la = lds + (k & 1) * kStage + RT * wr * 2048;
      const uint8_t* lw = lds + (k & 1) * kStage + (TM / 16 + CT * wc) * 2048;
      const uint8_t* ls = lds + 2 * kStage + ((k >> 1) & 1) * kScales + r * 16 + (k & 1) * 8 + 2 * g;
      if (k + 1 < stages) fetch(k + 1);
      uint32_t sa[RT], sw[CT];
#pragma unroll
      for (int i = 0; i < RT; ++i) sa[i] = *reinterpret_cast<const uint16_t*>(ls + (RT * wr + i) * 256);
#pragma unroll
      for (int j = 0; j < CT; ++j) sw[j] = *reinterpret_cast<const uint16_t*>(ls + (TM / 16 + CT * wc + j) * 256);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int at = (g >> 1) * 1024 + r * 64 + ((2 * (g & 1) + s) ^ tile_swizzle(r)) * 16;
        intx4 qa[RT], qw[CT];
#pragma unroll
        for (int j = 0; j < CT; ++j) qw[j] = *reinterpret_cast<const intx4*>(lw + j * 2048 + at);
#pragma unroll
        for (int i = 0; i < RT; ++i) qa[i] = *reinterpret_cast<const intx4*>(la + i * 2048 + at);
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int j = 0; j < CT; ++j)
            acc[i][j] = s == 0 ? mfma_mx4<0>(qa[i], sa[i], qw[j], sw[j], acc[i][j])
                               : mfma_mx4<1>(qa[i], sa[i], qw[j], sw[j], acc[i][j]);
      }
      __syncthreads();          // stage k is read, stage k + 1 has arrived
    }
  }
  const int cw = c0 + 16 * CT * wc;
  float bias[CT];
  load_bias(p, cw, lane, bias);
  if (cw < p.d_out) epilogue<RT, CT, OUT>(p, n, r0 + 16 * RT * wr, cw, lane, bias, acc);
}

// ---- dispatch -------------------------------------------------------------

template <int RT, int CT, int WK, int OUT>
void run_rows(const MxLinearArgs& p, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>((p.n_cap + 16 * RT - 1) / (16 * RT)),
                  static_cast<unsigned>((p.d_out + 16 * CT - 1) / (16 * CT)));
  hipLaunchKernelGGL((k_mx_linear_rows<RT, CT, WK, OUT>), grid, dim3(64 * WK), 0, s, p);
}

template <int TM, int TN, int WM, int WN, int OUT>
void run_tiles(const MxLinearArgs& p, hipStream_t s) {
  const int gm = static_cast<int>((p.n_cap + TM - 1) / TM), gn = (p.d_out + TN - 1) / TN;
  const int64_t tiles = static_cast<int64_t>(gm) * gn;
  hipLaunchKernelGGL((k_mx_linear_tiles<TM, TN, WM, WN, OUT>), dim3(static_cast<unsigned>((tiles + 7) / 8 * 8)),
                     dim3(64 * WM * WN), 0, s, p, gm, gn);
}

template <int WR, int WC, int OUT>
void run_resident(const MxLinearArgs& p, hipStream_t s) {
  const int64_t tiles = (p.n_cap + 64 * WR - 1) / (64 * WR);
  const unsigned gy = static_cast<unsigned>((p.d_out + 64 * WC - 1) / (64 * WC));
  const int64_t most = gy >= 768 ? 1 : 768 / gy;
  hipLaunchKernelGGL((k_mx_linear_resident<WR, WC, OUT>), dim3(static_cast<unsigned>(tiles < most ? tiles : most), gy),
                     dim3(64 * WR * WC), 0, s, p);
}

// Whether both sides' records fit LDS.
template <int WR, int WC>
bool resident_fits(const MxLinearArgs& p) {
  return p.blocks < 64 && 64 * (WC + WR) * p.pairs * resident_slots(p.blocks) * 16 <= kResidentLds;
}

// Which kernel, by the workgroups that its tiles give (us, bf16 results; calls
// below 7 us wait for the host, their figures are the kernel's own):
//   - up to two workgroups a CU of 16 rows by 32 columns: k_mx_linear_rows (64
//     x 4,096 x 1,024: 7.0, in 64 x 64 tiles 12.2; 300 x 1,024 x 256: 4.2 and
//     6.4; but 1,000 x 256 x 1,024, 2,016 workgroups: 9.7 and 7.1);
//   - resident weights where they fit and there are more tiles than CUs
//     (30,000 x 100 x 256: 8.2, tiles of 256, 128 and 64 11.3, 8.8 and 11.2;
//     200,000 x 256 x 256: 25.8, 38.6, 36.1, 46.4; 281 tiles of 18,000 x 100 x
//     256: 7.4, 10.3, 7.7, 9.0; 375 of 24,000 x 2 x 100 x 256: 9.6, 13.2, 10.0,
//     13.2; slower by 6% at most, 282 of 36,000 x 256 x 128: 8.2, 10.5, 7.9, 9.1,
//     422 of 27,000 x 256 x 256: 9.2, 11.1, 8.7, 10.7; but 250 of 16,000 x 256 x
//     256: 8.0, 10.2, 7.3, 7.0);
//   - else 256 x 256 tiles if there are three for every four CUs (8,192 x 4,096
//     x 4,096: 85, in 128 x 128 100, in 64 x 64 141; but 8,000 x 1,024 x 1,024,
//     128 of them: 18.2, 14.1, 17.9);
//   - 128 x 128 if there are three for two CUs (2,000 x 4,096 x 4,096: 29.0,
//     in 64 x 64 45.7; but 1,000 x 256 x 4,096, 256 of them: 7.6 and 7.0);
//   - 64 x 64.
template <int OUT>
void dispatch(const MxLinearArgs& p, hipStream_t s) {
  auto tiles = [&](int tm, int tn) { return ((p.n_cap + tm - 1) / tm) * ((p.d_out + tn - 1) / tn); };
  if constexpr ((OUT & kStreamed) == 0) {   // (1 MB of results at most)
    if (tiles(16, 32) <= 2 * kComputeUnits) return run_rows<1, 2, 8, OUT>(p, s);
  }
  if (p.d_out > 128 && resident_fits<1, 4>(p) && tiles(64, 256) > kComputeUnits) {
    run_resident<1, 4, OUT>(p, s);
  } else if (p.d_out > 64 && p.d_out <= 128 && resident_fits<2, 2>(p) && tiles(128, 128) > kComputeUnits) {
    run_resident<2, 2, OUT>(p, s);
  } else if (p.d_out <= 64 && resident_fits<4, 1>(p) && tiles(256, 64) > kComputeUnits) {
    run_resident<4, 1, OUT>(p, s);
  } else if (p.d_out > 128 && tiles(256, 256) >= kComputeUnits * 3 / 4) {
    run_tiles<256, 256, 2, 4, OUT>(p, s);
  } else if (p.d_out > 64 && tiles(128, 128) >= kComputeUnits * 3 / 2) {
    run_tiles<128, 128, 2, 2, OUT>(p, s);
  } else {
    run_tiles<64, 64, 2, 1, OUT>(p, s);
  }
}

}  // namespace

hipError_t launch_mx_linear(const MxLinearArgs& p, int out, hipStream_t s) {
  // past the caches if large and written by whole 64-byte pieces: rows of such,
  // or rows that a wave has whole (59,048 x 2 x 32 x 2,304 bf16: 59.1 us, plain
  // 65.2; x 2,272 70.8, 70.4; 300,000 x 2 x 100 x 47 fp32 25.2, 30.9; but 2,273 170
  // and 104, 200,000 x 256 x 240 bf16 39.1 and 33.4, 100,000 x 100 x 100 fp32 16.6
  // and 12.5)
  const int64_t row = p.d_out * (out == kMxOutBf16 ? 2 : 4);
  const bool stream = p.n_cap * row >= kStreamBytes && (row % 64 == 0 || p.d_out <= 64);
  if (out == kMxOutRecords) dispatch<kMxOutRecords>(p, s);
  else if (out == kMxOutBf16) stream ? dispatch<kMxOutBf16 | kStreamed>(p, s) : dispatch<kMxOutBf16>(p, s);
  else stream ? dispatch<kMxOutF32 | kStreamed>(p, s) : dispatch<kMxOutF32>(p, s);
  return hipGetLastError();
}

}  // namespace gmb
