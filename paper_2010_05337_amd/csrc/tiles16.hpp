// Tiles of a product of 16-bit operands on gfx950: acc[m][n] = sum over k of
// A(m, k) B(n, k) with v_mfma_f32_16x16x32, both sides brought through LDS
// straight from memory, stage by stage.
//
// An operand lies in memory in one of two ways and is read from LDS to match:
//   kByRow   rows of A (or B), each contiguous along k: a lane takes the eight
//            k of its row at once
//   kByK     rows of k, each contiguous along m (or n): ds_read_b64_tr_b16
//            hands a lane four k of its column
// so none is ever transposed in memory.
//
// kBf16: elements are bf16, a stage is 64 of k.  kSplit: a value v is two fp16,
// hi = v rounded and lo = v - hi rounded, with v scaled by a power of two so
// that the largest is in [2^14, 2^15): what is lost is below 2^-22 |v| + 2^-25.
// Rows hold 32 hi, 32 lo, 32 hi, ... (a 128-byte piece has both parts of 32
// values), a stage is 32 of k, and a product is hi hi + hi lo + lo hi: three
// instructions where cutting into three bf16 takes six, both at fp32's error.
#pragma once

#include "common.hpp"

namespace gmb {

typedef float t16_f32x4 __attribute__((ext_vector_type(4)));
typedef short t16_i16x4 __attribute__((ext_vector_type(4)));
typedef short t16_i16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 t16_bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 t16_f16x8 __attribute__((ext_vector_type(8)));

enum T16Type { kBf16, kSplit };
enum T16Form { kByRow, kByK };

// One side of a product.  kByRow: `rows` rows of `ld` 16-bit elements, the
// tile's first row `first`; kByK: `rows` rows of k, `cols` values wide (a
// multiple of 64), the tile's first column `first`.  Rows and columns past the
// end are read as some that there are: of rows and columns nothing is stored,
// of k one of the two sides must hold zeros.
struct T16Side {
  const uint16_t* data;
  int64_t ld;
  int64_t rows;
  int cols;
  int64_t first;
};

// A stage of KS 16-bit elements of either side's rows.
template <int TM, int TN, int KS>
constexpr int t16_stage_bytes() { return (TM + TN) * KS * 2; }

// 16 bytes a lane from global memory to LDS, at l + 16 lane.
__device__ __forceinline__ void t16_load_lds(const void* g, void* l) {
  typedef const __attribute__((address_space(1))) void* gp;
  typedef __attribute__((address_space(3))) void* lp;
  __builtin_amdgcn_global_load_lds((gp)g, (lp)l, 16, 0, 0);
}

// Waits until at most N of this wave's loads are still on their way, and for the
// workgroup.  (Loads and stores end in the order they were issued.)
template <int N>
__device__ __forceinline__ void t16_wait() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N < 63 ? N : 63) : "memory");
}

// What brings a side's tile of T rows (or columns) into LDS.  LDS holds T x KS
// elements a stage (KS 64, or for bf16 32): kByRow T rows of KS / 8 16-byte
// pieces, piece q at q ^ t16_spread(row); kByK KS rows of T columns (kSplit: the
// hi parts of 32 of k, then the lo parts), pairs of pieces exchanged by t16_turn.
// Both spread the rows that are read together over the banks.
//
// An address is a part that the whole wave has (scalar registers) and a lane's
// offset of 32 bits, the same for every tile and stage but those at the end
// (64-bit addresses of eight loads took 16 registers more, which spilled): a
// side's rows are at most 2^31 / 256 bytes apart.
//
// DEAL (kByRow): LDS row 16 i + 4 g + e holds the tile's row 32 (i / 2) + 8 g + 4
// (i % 2) + e, so that the registers of a lane's two neighbouring 16-row tiles
// are eight rows in order.
constexpr int64_t kT16MostBytes = (int64_t{1} << 31) / 256;
__device__ __forceinline__ int t16_turn(int krow) { return (krow & 3) | ((krow >> 3) & 1) << 2; }

template <int KS>
__device__ __forceinline__ int t16_spread(int row) { return KS == 64 ? (row >> 1) & 7 : (row >> 2) & 3; }

template <T16Type TYPE, T16Form FORM, int T, int WAVES, int KS, bool DEAL = false>
struct T16Loader {
  static constexpr int PIECES = KS / 8;     // of a row
  static constexpr int LOADS = T * PIECES / (64 * WAVES);
  static_assert(LOADS * 64 * WAVES == T * PIECES, "a stage is whole loads");
  static_assert(KS == 64 || (KS == 32 && TYPE == kBf16), "a stage has whole products");
  static constexpr int KROWS = TYPE == kSplit ? 32 : KS;
  static constexpr int P = T / 8;           // pieces of a row of k
  const char* base;                         // the tile's first row, or its first row of k
  uint32_t off[LOADS];
  uint32_t ld_bytes;
  int64_t rows;                             // kByRow: from the tile's first on; kByK: of k
  int wave, lane;

  // Load i's row (kByRow) or row of k in a stage, and the offset in it.
  __device__ __forceinline__ int row_of(int i) const {
    const int q = (i * WAVES + wave) * 64 + lane;
    if constexpr (FORM == kByRow) {
      const int row = q / PIECES;
      return DEAL ? (row & ~31) + (row & 12) * 2 + ((row >> 4) & 1) * 4 + (row & 3) : row;
    } else {
      const int row = q / P;
      return TYPE == kSplit ? row & 31 : row;
    }
  }
  __device__ __forceinline__ uint32_t in_row(int i, const T16Side& s) const {
    const int q = (i * WAVES + wave) * 64 + lane;
    if constexpr (FORM == kByRow) {
      return ((q % PIECES) ^ t16_spread<KS>(q / PIECES)) * 16;
    } else {
      const int row = q / P, slot = q % P;
      const int chunk = (slot >> 1) ^ (t16_turn(row) & (P / 2 - 1));
      int64_t col = s.first + (chunk * 2 + (slot & 1)) * 8;
      if (col >= s.cols) col = 0;
      return static_cast<uint32_t>(TYPE == kSplit ? (col / 32) * 128 + (row >> 5) * 64 + (col % 32) * 2 : col * 2);
    }
  }
  __device__ __forceinline__ void init(const T16Side& s, int wave_, int lane_) {
    wave = wave_;
    lane = lane_;
    ld_bytes = static_cast<uint32_t>(s.ld * 2);
    rows = FORM == kByRow ? s.rows - s.first : s.rows;
    base = reinterpret_cast<const char*>(s.data) + (FORM == kByRow ? s.first * s.ld * 2 : 0);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) off[i] = row_of(i) * ld_bytes + in_row(i, s);
    if (FORM == kByRow && rows < T) clamp();
  }
  // kByRow: rows past the end
  __device__ __forceinline__ void clamp() {
    const int last = rows < 1 ? 0 : static_cast<int>(rows) - 1;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int row = row_of(i);
      if (row > last) off[i] -= (row - last) * ld_bytes;
    }
  }
  // kByRow: the next T rows (only forwards; past the end nothing may be fetched)
  __device__ __forceinline__ void advance() {
    base += static_cast<int64_t>(T) * ld_bytes;
    rows -= T;
    if (rows < T && rows > 0) clamp();
  }
  // stage k into the side's half of an LDS stage
  __device__ __forceinline__ void fetch(int64_t k, char* lds) const {
    const char* from = base + k * (FORM == kByRow ? KS * 2 : static_cast<int64_t>(KROWS) * ld_bytes);
    if (FORM == kByK && (k + 1) * KROWS > rows) {
      const int last = static_cast<int>(rows - 1 - k * KROWS);    // (of this stage: 0 at least)
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int row = row_of(i);
        t16_load_lds(from + (row > last ? off[i] - (row - last) * ld_bytes : off[i]), lds + (i * WAVES + wave) * 1024);
      }
    } else {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) t16_load_lds(from + off[i], lds + (i * WAVES + wave) * 1024);
    }
  }
};

// The operand of 16 rows (or columns) from `at` on in an LDS stage, for the
// stage's s-th 32 (kSplit: s = 0 the hi parts, 1 the lo parts).
template <T16Form FORM, int T, int KS>
__device__ __forceinline__ t16_i16x8 t16_operand(const char* lds, int at, int s, int lane) {
  const int r = lane & 15, g = lane >> 4;
  if constexpr (FORM == kByRow) {
    return *reinterpret_cast<const t16_i16x8*>(lds + (at + r) * (KS * 2) + ((4 * s + g) ^ t16_spread<KS>(r)) * 16);
  } else {
    typedef __attribute__((address_space(3))) t16_i16x4* lp;
    const int chunk = (at / 16) ^ (((r >> 2) | (g & 1) << 2) & (T / 16 - 1));
    const char* p = lds + (32 * s + 8 * g + (r >> 2)) * (2 * T) + chunk * 32 + (r & 3) * 8;
    const t16_i16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)p);
    const t16_i16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(p + 4 * (2 * T)));
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  }
}

template <T16Type TYPE>
__device__ __forceinline__ t16_f32x4 t16_mfma(t16_i16x8 a, t16_i16x8 b, t16_f32x4 c) {
  if constexpr (TYPE == kBf16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(t16_bf16x8, a), __builtin_bit_cast(t16_bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(t16_f16x8, a), __builtin_bit_cast(t16_f16x8, b), c, 0, 0, 0);
}

// A workgroup of WM x WN waves, a wave RT x CT tiles of 16 x 16: its rows of A
// from 16 RT wm on, of B from 16 CT wn on.  Register e of lane (g, r) of
// acc[i][j] is row 16 i + 4 g + e of A (with DEAL, of LDS), row 16 j + r of B.
// LDS holds NST stages: NST - 1 are on their way or waiting while one is used.
template <T16Type TYPE, T16Form FA, T16Form FB, int TM, int TN, int WM, int WN, int NST, int KS, bool DEAL = false>
struct T16Tile {
  static constexpr int WAVES = WM * WN, RT = TM / (16 * WM), CT = TN / (16 * WN), STAGES = NST;
  static constexpr int kStage = t16_stage_bytes<TM, TN, KS>();
  static constexpr int K = TYPE == kSplit ? KS / 2 : KS;      // values of a stage
  using LoadA = T16Loader<TYPE, FA, TM, WAVES, KS, DEAL>;
  using LoadB = T16Loader<TYPE, FB, TN, WAVES, KS>;
  static constexpr int LOADS = LoadA::LOADS + LoadB::LOADS;

  static __device__ __forceinline__ void clear(t16_f32x4 (&acc)[RT][CT]) {
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int j = 0; j < CT; ++j) acc[i][j] = t16_f32x4{0.f, 0.f, 0.f, 0.f};
  }

  static __device__ __forceinline__ void fetch(const LoadA& la, const LoadB& lb, int64_t k, char* to) {
    la.fetch(k, to);
    lb.fetch(k, to + TM * KS * 2);
  }

  // The oldest stage has arrived, for every wave, and the one before it is read:
  // `full`: NST - 1 stages were asked for since that one.
  static __device__ __forceinline__ void wait(bool full) {
    if (NST > 2 && full) t16_wait<(NST - 2) * LOADS>();
    else t16_wait<0>();
  }

  // acc += the stages first .. last - 1 of k; lds: NST stages.  Every wave of the
  // workgroup calls it with the same stages.
  static __device__ __forceinline__ void run(const T16Side& a, const T16Side& b, int64_t first, int64_t last, char* lds,
                                             t16_f32x4 (&acc)[RT][CT]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    LoadA la;
    LoadB lb;
    la.init(a, wave, lane);
    lb.init(b, wave, lane);
#pragma unroll
    for (int s = 0; s < NST - 1; ++s)
      if (first + s < last) fetch(la, lb, first + s, lds + s * kStage);
    int at = 0;
    for (int64_t k = first; k < last; ++k) {
      wait(k + NST - 2 < last);
      const int to = at == 0 ? NST - 1 : at - 1;
      step(la, lb, k + NST - 1, k + NST - 1 < last, lds + at * kStage, lds + to * kStage, wave, lane, acc);
      at = at == NST - 1 ? 0 : at + 1;
    }
    __syncthreads();
  }

  // acc += the stage that lies at `now`, while (with `more`) stage k comes to
  // `next`.  (The two are apart, and said to be: else the compiler lets the
  // transposing reads of `now` wait for the loads into `next`.)
  static __device__ __forceinline__ void step(const LoadA& la, const LoadB& lb, int64_t k, bool more,
                                              const char* __restrict__ now, char* __restrict__ next, int wave, int lane,
                                              t16_f32x4 (&acc)[RT][CT]) {
    const int wm = wave / WN, wn = wave % WN;
    if (more) fetch(la, lb, k, next);
    const char* now_b = now + TM * KS * 2;
    if constexpr (TYPE == kBf16) {
      // (unrolled, the operands of both halves would be held at once: with large
      // tiles that spills)
#pragma unroll RT * CT >= 32 ? 1 : 2
      for (int s = 0; s < KS / 32; ++s) {
        t16_i16x8 qa[RT], qb[CT];
#pragma unroll
        for (int j = 0; j < CT; ++j) qb[j] = t16_operand<FB, TN, KS>(now_b, 16 * (CT * wn + j), s, lane);
#pragma unroll
        for (int i = 0; i < RT; ++i) qa[i] = t16_operand<FA, TM, KS>(now, 16 * (RT * wm + i), s, lane);
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int j = 0; j < CT; ++j) acc[i][j] = t16_mfma<TYPE>(qa[i], qb[j], acc[i][j]);
      }
    } else {
      t16_i16x8 bh[CT], bl[CT];
#pragma unroll
      for (int j = 0; j < CT; ++j) {
        bh[j] = t16_operand<FB, TN, KS>(now_b, 16 * (CT * wn + j), 0, lane);
        bl[j] = t16_operand<FB, TN, KS>(now_b, 16 * (CT * wn + j), 1, lane);
      }
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const t16_i16x8 ah = t16_operand<FA, TM, KS>(now, 16 * (RT * wm + i), 0, lane);
        const t16_i16x8 al = t16_operand<FA, TM, KS>(now, 16 * (RT * wm + i), 1, lane);
#pragma unroll
        for (int j = 0; j < CT; ++j) acc[i][j] = t16_mfma<TYPE>(al, bh[j], acc[i][j]);
#pragma unroll
        for (int j = 0; j < CT; ++j) acc[i][j] = t16_mfma<TYPE>(ah, bl[j], acc[i][j]);
#pragma unroll
        for (int j = 0; j < CT; ++j) acc[i][j] = t16_mfma<TYPE>(ah, bh[j], acc[i][j]);
      }
    }
  }
};

}  // namespace gmb
