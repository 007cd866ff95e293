// The product of microscaled 4-bit rows and weights on gfx950:
// out = act(A W^T [+ A2 W2^T] + b) with v_mfma_scale_f32_16x16x128_f8f6f4,
// which takes 16 x 128 elements of each side with a scale for every 32 of a
// row and sums in fp32.  A row's record is what a lane wants as it is: lane l
// of a wave supplies row l % 16 and the 32 elements of block 4 s + l / 16 of
// step s, 16 bytes and a scale byte.  The weights are the instruction's first
// operand, so that a lane holds four neighbouring output columns of one row.
#include "mx.hpp"
#include "mx_kernels.hpp"

namespace gmb {

namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx8 __attribute__((ext_vector_type(8)));

// Byte SEL of ws and as is the scale.  The 4-bit format (4) reads the first
// four words of an operand.
template <int SEL = 0>
__device__ __forceinline__ floatx4 mfma_mx4(const intx4& w, uint32_t ws, const intx4& a, uint32_t as, floatx4 c) {
  const intx8 w8 = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, a8 = {a[0], a[1], a[2], a[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w8, a8, c, 4, 4, SEL, static_cast<int>(ws), SEL,
                                                          static_cast<int>(as));
}

// One row's block for a lane: its elements and its scale, zeros at scale 1
// past the row's last block.
__device__ __forceinline__ void load_block(const uint8_t* rec, int blk, int blocks, intx4& q, uint32_t& sc) {
  const bool in = blk < blocks;
  const int b = in ? blk : 0;
  __builtin_memcpy(&q, rec + b * 16, 16);
  sc = rec[blocks * 16 + b];
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = in ? q[i] : 0;
  sc = in ? sc : 127u;
}

// Bias, activation and the store of one lane's four columns c .. c + 3 of
// `row`, fp32 or bf16.
template <int OUT>
__device__ __forceinline__ void store4(const MxLinearArgs& p, int64_t row, int c, const float (&z)[4]) {
  if constexpr (OUT == kMxOutF32) {
    float* o = static_cast<float*>(p.out) + row * p.d_out + c;
    if (c + 4 <= p.d_out) {
      const float4 v = make_float4(z[0], z[1], z[2], z[3]);
      __builtin_memcpy(o, &v, 16);
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (c + r < p.d_out) o[r] = z[r];
    }
  } else {
    uint16_t* o = static_cast<uint16_t*>(p.out) + row * p.d_out + c;
    const uint2 v = make_uint2(mx_bf16x2_bits(z[0], z[1]), mx_bf16x2_bits(z[2], z[3]));
    if (c + 4 <= p.d_out) {
      __builtin_memcpy(o, &v, 8);
    } else {
      const uint32_t w[2] = {v.x, v.y};
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (c + r < p.d_out) o[r] = static_cast<uint16_t>(w[r / 2] >> (16 * (r & 1)));
    }
  }
}

__device__ __forceinline__ void finish4(const MxLinearArgs& p, int c, const floatx4& acc, float (&z)[4]) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    z[r] = acc[r] + (p.bias && c + r < p.d_out ? p.bias[c + r] : 0.f);
    if (p.relu) z[r] = z[r] > 0.f ? z[r] : 0.f;
  }
}

// The epilogue of a wave's RT x CT tiles: rows r0 + 16 i + l % 16, columns
// c0 + 16 j + 4 (l / 16) .. + 3.
template <int RT, int CT, int OUT>
__device__ __forceinline__ void epilogue(const MxLinearArgs& p, int64_t n, int64_t r0, int c0, int lane,
                                         const floatx4 (&acc)[RT][CT]) {
  const int g = lane >> 4;
  if constexpr (OUT != kMxOutRecords) {
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int64_t row = r0 + 16 * i + (lane & 15);
#pragma unroll
      for (int j = 0; j < CT; ++j) {
        const int c = c0 + 16 * j + 4 * g;
        if (row >= n || c >= p.d_out) continue;
        float z[4];
        finish4(p, c, acc[i][j], z);
        store4<OUT>(p, row, c, z);
      }
    }
  } else {
    // a record's block is two column tiles: eight values a lane, four lanes
    const int blocks = (p.d_out + 31) / 32;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int64_t row = r0 + 16 * i + (lane & 15);
#pragma unroll
      for (int j = 0; j < CT; j += 2) {
        float v[8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int c = c0 + 16 * (j + t) + 4 * g;
          float z[4];
          finish4(p, c, acc[i][j + t], z);
#pragma unroll
          for (int r = 0; r < 4; ++r) v[4 * t + r] = c + r < p.d_out ? z[r] : 0.f;
        }
        uint32_t top = 0;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const uint32_t m = __float_as_uint(v[r]) & 0x7FFFFFFFu;
          top = m > top ? m : top;
        }
        uint32_t o = __shfl_xor(top, 16, 64);
        top = o > top ? o : top;
        o = __shfl_xor(top, 32, 64);
        top = o > top ? o : top;
        const uint32_t code = mx_scale_code<4>(top);
        uint32_t w[1];
        mx_pack8<4>(v, code, w);
        const int blk = (c0 + 16 * j) / 32;
        if (row < n && blk < blocks) {
          uint8_t* rec = static_cast<uint8_t*>(p.out) + row * p.out_stride;
          const uint16_t lo = static_cast<uint16_t>(w[0]), hi = static_cast<uint16_t>(w[0] >> 16);
          __builtin_memcpy(rec + blk * 16 + 2 * g, &lo, 2);
          __builtin_memcpy(rec + blk * 16 + 8 + 2 * g, &hi, 2);
          if (g == 0) rec[blocks * 16 + blk] = static_cast<uint8_t>(code);
          if (blk == blocks - 1)
            for (int b = blocks * 17 + g; b < p.out_record; b += 4) rec[b] = 0;
        }
      }
    }
  }
}

// A workgroup of WC x WK waves: wave (wc, wk) has the 16 RT rows of the
// workgroup, columns [16 CT (WC y + wc), + 16 CT), and the steps wk, wk + WK,
// ... of the sum; the WK sums meet in LDS in a fixed order.
template <int RT, int CT, int WC, int WK, int OUT>
__global__ __launch_bounds__(64 * WC * WK) void k_mx_linear(MxLinearArgs p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wc = wave % WC, wk = wave / WC;
  int64_t n = p.n_cap;
  if (p.n_dev) {
    const int64_t m = load_size(p.n_dev);
    n = m < 0 ? 0 : (m < n ? m : n);
  }
  const int64_t r0 = static_cast<int64_t>(blockIdx.x) * (16 * RT);
  if (r0 >= n) return;
  const int c0 = (blockIdx.y * WC + wc) * 16 * CT;
  const int g = lane >> 4;
  const int steps = (p.blocks + 3) / 4;
  floatx4 acc[RT][CT];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int j = 0; j < CT; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  for (int pr = 0; pr < p.pairs; ++pr) {
    const MxPair& m = p.pair[pr];
    const uint8_t* ra[RT];
    bool ok[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int64_t row = r0 + 16 * i + (lane & 15);
      const int64_t rc = row < n ? row : n - 1;
      int64_t at = rc;
      ok[i] = true;
      if (m.ids) {
        const int32_t id = m.ids[rc];
        ok[i] = valid_vertex(id, m.a_rows);
        if (!ok[i] && wave == 0 && blockIdx.y == 0) raise_status(p.status, GMB_STATUS_ERANGE);
        at = ok[i] ? id : 0;
      }
      ra[i] = m.a + at * m.a_stride;
    }
    const uint8_t* rw[CT];
#pragma unroll
    for (int j = 0; j < CT; ++j) {
      const int c = c0 + 16 * j + (lane & 15);
      rw[j] = m.w + static_cast<int64_t>(c < p.d_out ? c : p.d_out - 1) * m.w_stride;
    }
    for (int s = wk; s < steps; s += WK) {
      intx4 qa[RT], qw[CT];
      uint32_t sa[RT], sw[CT];
#pragma unroll
      for (int i = 0; i < RT; ++i) load_block(ra[i], 4 * s + g, p.blocks, qa[i], sa[i]);
#pragma unroll
      for (int j = 0; j < CT; ++j) load_block(rw[j], 4 * s + g, p.blocks, qw[j], sw[j]);
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < CT; ++j) acc[i][j] = mfma_mx4(qw[j], sw[j], qa[i], sa[i], acc[i][j]);
    }
    // a row whose id is outside the table counts as zeros (only the first
    // pair has ids, so what is summed so far is that row's)
    if (m.ids) {
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < CT; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[i][j][r] = ok[i] ? acc[i][j][r] : 0.f;
    }
  }
  if constexpr (WK > 1) {
    __shared__ floatx4 part[(WK - 1) * WC * RT * CT * 64];
    if (wk > 0) {
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < CT; ++j)
          part[((((wk - 1) * WC + wc) * RT + i) * CT + j) * 64 + lane] = acc[i][j];
    }
    __syncthreads();
    if (wk > 0) return;
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int j = 0; j < CT; ++j)
        for (int k = 0; k < WK - 1; ++k) acc[i][j] += part[(((k * WC + wc) * RT + i) * CT + j) * 64 + lane];
  }
  if (c0 < p.d_out) epilogue<RT, CT, OUT>(p, n, r0, c0, lane, acc);
}

// ---- products that the matrix cores bound ---------------------------------

// A workgroup of eight waves has 256 rows and 256 columns; wave (wr, wc) of
// 2 x 4 has 128 rows and 64 columns of them.  The sum goes in stages of eight
// blocks (256 elements); two stages are in LDS, one being read and one
// arriving (global_load_lds: no registers in between).
//   LDS, elements: a fragment is 16 rows by 4 blocks in the order that one
//   load instruction leaves it, slot 16 g' + r for block 4 f + g' of row r;
//   fragments (16-row tile t, half f) at 1 KB each, 32 a side and stage.
//   Scales: 8 bytes a row and stage.
// Step s of a stage takes block 2 g + s for lane group g, so that a lane's two
// scales are neighbours (one 16-bit read, the byte picked by the
// instruction's selector).  Blocks past the row's end and rows without a
// record load zeros from kZeros.
constexpr int kBigTile = 256;
constexpr int kBigSide = 32 * 1024;               // element bytes of a side and stage
constexpr int kBigScales = kBigTile * 8;
constexpr int kBigStage = 2 * (kBigSide + kBigScales);

__device__ __align__(16) const uint32_t kZeros[4] = {0, 0, 0, 0};

__device__ __forceinline__ void load_lds(const void* g, void* l, int bytes) {
  typedef const __attribute__((address_space(1))) void* gp;
  typedef __attribute__((address_space(3))) void* lp;
  if (bytes == 16)
    __builtin_amdgcn_global_load_lds((gp)g, (lp)l, 16, 0, 0);
  else
    __builtin_amdgcn_global_load_lds((gp)g, (lp)l, 4, 0, 0);
}

struct BigRows {
  const uint8_t* rec[4];    // the lane's row of four of the wave's 16-row tiles (NULL: none)
  const uint8_t* scales[2]; // the lane's row of two of the wave's scale loads
};

// Loads stage k of one side: wave `w` of eight brings tiles 4 (w % 4) ..
// + 3 of side w / 4, and the scales of rows 64 (w % 4) .. + 63.
__device__ __forceinline__ void big_load(const BigRows& r, int k, int blocks, uint8_t* elems, uint8_t* scales, int tile0,
                                         int row0, int lane) {
  const int g = lane >> 4;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int f = 0; f < 2; ++f) {
      const int b = 8 * k + 4 * f + g;
      const void* at = r.rec[i] && b < blocks ? static_cast<const void*>(r.rec[i] + b * 16) : kZeros;
      load_lds(at, elems + ((tile0 + i) * 2 + f) * 1024, 16);
    }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int b = 8 * k + 4 * (lane & 1);
    const int last = (blocks - 1) & ~3;           // (scales of no block belong to zeros)
    const void* at = r.scales[i] ? static_cast<const void*>(r.scales[i] + (b < blocks ? b : last)) : kZeros;
    load_lds(at, scales + (row0 + 32 * i) * 8, 4);
  }
}

template <int OUT>
__global__ __launch_bounds__(512, 2) void k_mx_linear_big(MxLinearArgs p, int gm, int gn) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * kBigStage];
  int64_t n = p.n_cap;
  if (p.n_dev) {
    const int64_t m = load_size(p.n_dev);
    n = m < 0 ? 0 : (m < n ? m : n);
  }
  // workgroup ids go round the eight XCDs: each takes a contiguous run of
  // tiles, eight row tiles wide, so that its L2 holds what they share
  const int tiles = gm * gn, per = (tiles + 7) / 8;
  const int id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if (id >= tiles) return;
  const int band = id / (8 * gn), in_band = id - band * 8 * gn;
  const int height = gm - 8 * band < 8 ? gm - 8 * band : 8;
  const int64_t r0 = static_cast<int64_t>(8 * band + in_band % height) * kBigTile;
  const int c0 = in_band / height * kBigTile;
  if (r0 >= n) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wr = wave >> 2, wc = wave & 3, g = lane >> 4;
  const int side = wave >> 2, quarter = wave & 3;
  const int stages = (p.blocks + 7) / 8;
  floatx4 acc[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  for (int pr = 0; pr < p.pairs; ++pr) {
    const MxPair& m = p.pair[pr];
    BigRows rows;
    auto record = [&](int r) -> const uint8_t* {   // row r of the tile on this wave's side
      if (side == 0) {
        const int64_t row = r0 + r < n ? r0 + r : n - 1;
        if (!m.ids) return m.a + row * m.a_stride;
        const int32_t v = m.ids[row];
        if (valid_vertex(v, m.a_rows)) return m.a + v * m.a_stride;
        raise_status(p.status, GMB_STATUS_ERANGE);
        return nullptr;
      }
      const int c = c0 + r < p.d_out ? c0 + r : p.d_out - 1;
      return m.w + static_cast<int64_t>(c) * m.w_stride;
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) rows.rec[i] = record(64 * quarter + 16 * i + (lane & 15));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint8_t* q = record(64 * quarter + 32 * i + lane / 2);
      rows.scales[i] = q ? q + p.blocks * 16 : nullptr;
    }
    auto fetch = [&](int k, int buf) {
      uint8_t* base = lds + buf * kBigStage + side * (kBigSide + kBigScales);
      big_load(rows, k, p.blocks, base, base + kBigSide, 4 * quarter, 64 * quarter, lane);
    };
    __syncthreads();            // the last pair's reads
    fetch(0, 0);
    __syncthreads();
    for (int k = 0; k < stages; ++k) {
      const uint8_t* la = lds + (k & 1) * kBigStage;
      const uint8_t* lw = la + kBigSide + kBigScales;
      if (k + 1 < stages) fetch(k + 1, (k + 1) & 1);
      uint32_t sa[8], sw[4];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        sa[i] = *reinterpret_cast<const uint16_t*>(la + kBigSide + (wr * 128 + 16 * i + (lane & 15)) * 8 + 2 * g);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        sw[j] = *reinterpret_cast<const uint16_t*>(lw + kBigSide + (wc * 64 + 16 * j + (lane & 15)) * 8 + 2 * g);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int at = (g >> 1) * 1024 + (2 * (g & 1) + s) * 256 + (lane & 15) * 16;
        intx4 qa[8], qw[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) qw[j] = *reinterpret_cast<const intx4*>(lw + (wc * 4 + j) * 2048 + at);
#pragma unroll
        for (int i = 0; i < 8; ++i) qa[i] = *reinterpret_cast<const intx4*>(la + (wr * 8 + i) * 2048 + at);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[i][j] = s == 0 ? mfma_mx4<0>(qw[j], sw[j], qa[i], sa[i], acc[i][j])
                               : mfma_mx4<1>(qw[j], sw[j], qa[i], sa[i], acc[i][j]);
      }
      __syncthreads();          // stage k is read, stage k + 1 has arrived
    }
  }
  const int cw = c0 + 64 * wc;
  if (cw < p.d_out) epilogue<8, 4, OUT>(p, n, r0 + 128 * wr, cw, lane, acc);
}

template <int RT, int CT, int WC, int WK, int OUT>
void run(const MxLinearArgs& p, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>((p.n_cap + 16 * RT - 1) / (16 * RT)),
                  static_cast<unsigned>((p.d_out + 16 * CT * WC - 1) / (16 * CT * WC)));
  hipLaunchKernelGGL((k_mx_linear<RT, CT, WC, WK, OUT>), grid, dim3(64 * WC * WK), 0, s, p);
}

template <int OUT>
void dispatch(const MxLinearArgs& p, hipStream_t s) {
  const int64_t tiles = ((p.n_cap + 63) / 64) * ((p.d_out + 63) / 64);
  const int64_t big = ((p.n_cap + kBigTile - 1) / kBigTile) * ((p.d_out + kBigTile - 1) / kBigTile);
  if (big >= 128 && p.blocks >= 16 && p.d_out > 128) {
    const int gm = static_cast<int>((p.n_cap + kBigTile - 1) / kBigTile), gn = (p.d_out + kBigTile - 1) / kBigTile;
    hipLaunchKernelGGL((k_mx_linear_big<OUT>), dim3((gm * gn + 7) / 8 * 8), dim3(512), 0, s, p, gm, gn);
  } else if (tiles >= 1024) {
    if (p.d_out > 128) run<4, 4, 4, 1, OUT>(p, s);
    else if (p.d_out > 64) run<4, 4, 2, 1, OUT>(p, s);
    else run<4, 4, 1, 1, OUT>(p, s);
  } else if (p.n_cap > 16) {
    run<4, 2, 1, 8, OUT>(p, s);
  } else {
    run<1, 2, 1, 8, OUT>(p, s);
  }
}

}  // namespace

hipError_t launch_mx_linear(const MxLinearArgs& p, int out, hipStream_t s) {
  if (out == kMxOutRecords) dispatch<kMxOutRecords>(p, s);
  else if (out == kMxOutBf16) dispatch<kMxOutBf16>(p, s);
  else dispatch<kMxOutF32>(p, s);
  return hipGetLastError();
}

}  // namespace gmb
