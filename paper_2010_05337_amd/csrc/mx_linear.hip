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

__device__ __forceinline__ floatx4 mfma_mx4(const intx4& w, uint32_t ws, const intx4& a, uint32_t as, floatx4 c) {
  // the 4-bit format (4) reads the first four words of an operand
  const intx8 w8 = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, a8 = {a[0], a[1], a[2], a[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w8, a8, c, 4, 4, 0, static_cast<int>(ws), 0,
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

template <int RT, int CT, int WC, int WK, int OUT>
void run(const MxLinearArgs& p, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>((p.n_cap + 16 * RT - 1) / (16 * RT)),
                  static_cast<unsigned>((p.d_out + 16 * CT * WC - 1) / (16 * CT * WC)));
  hipLaunchKernelGGL((k_mx_linear<RT, CT, WC, WK, OUT>), grid, dim3(64 * WC * WK), 0, s, p);
}

template <int OUT>
void dispatch(const MxLinearArgs& p, hipStream_t s) {
  const int64_t tiles = ((p.n_cap + 63) / 64) * ((p.d_out + 63) / 64);
  if (tiles >= 1024) {
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
