// Products of row-major operands, out[m][n] = sum_k x[m][k] w[n][k], for the operators (ops_gemm.hip): 16-bit numbers with
// fp32 sums, or 8-bit integers with 32-bit sums.  Both operands are read as they lie in the caller's memory (rows at any pitch
// that keeps them on 16 bytes; others are copied first): nothing is laid out ahead, so weights that change every training step
// cost nothing extra.
//
// All element types share one geometry, counted in bytes of k: a matrix instruction takes 16 bytes a lane of each operand
// (8 numbers of 16 bits, 16 integers of 8), 32 bytes of k for 32 rows, and runs for as many cycles with either.
//
// A result's bits do not depend on the tile: all tiles add 32 or 64 bytes of k at a time from its start on, what is left of k over whole
// stages first, and the instructions of either shape add up what they take in the same order (as their results say, which the tests
// compare).  The kernel for few rows adds in another order.
//
// The channels' fragment goes in as the instruction's first operand, the rows' as its second: a lane then holds four
// neighbouring channels of one row in four neighbouring registers, which is what the epilogues store.
//
// Gated products (GATED): the tile's channels are groups of 32 of one weight matrix and the same 32 of the other, in turn, so
// that a wavefront's registers hold both factors of an output element, and the activation and the product are formed there.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "gemm_bf16.h"

namespace asd {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v4f_b __attribute__((ext_vector_type(4)));

// Matrix instructions and sums by element type.
struct ElemBf16 {
  typedef v16f_b Acc32;
  typedef v4f_b Acc16;
  typedef float Sum;
  static constexpr int kBytes = 2;
  static __device__ __forceinline__ Acc32 mma32(v4i_b a, v4i_b b, Acc32 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ Acc16 mma16(v4i_b a, v4i_b b, Acc16 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
  }
};
struct ElemF16 {
  typedef v16f_b Acc32;
  typedef v4f_b Acc16;
  typedef float Sum;
  static constexpr int kBytes = 2;
  static __device__ __forceinline__ Acc32 mma32(v4i_b a, v4i_b b, Acc32 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ Acc16 mma16(v4i_b a, v4i_b b, Acc16 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
  }
};
struct ElemI8 {
  typedef v16i_b Acc32;
  typedef v4i_b Acc16;
  typedef int Sum;
  static constexpr int kBytes = 1;
  static __device__ __forceinline__ Acc32 mma32(v4i_b a, v4i_b b, Acc32 c) { return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ Acc16 mma16(v4i_b a, v4i_b b, Acc16 c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
};

// Rows of x and of one or two weight matrices (w1 NULL: one); pitches and kb, the bytes of a row, are multiples of 16, and so are
// the pointers.
struct RowsProduct {
  const uint8_t* x;
  const uint8_t* w0;
  const uint8_t* w1;
  int64_t x_pitch, w_pitch0, w_pitch1;   // bytes between rows
  int M, N;                              // rows; channels (of one weight matrix)
  int64_t kb;
  const int32_t* rows_used;              // DEV or NULL: rows to work on where the host knows a bound, M, only
  // Epilogues with kWrap: k runs over sums of several products one behind the other.  From these bytes of k on (multiples of 128, and
  // so is kb) an operand's row is read again from its start.
  uint32_t x_wrap = ~0u, w_wrap = ~0u;
};
template <class Epi>
__device__ __forceinline__ uint32_t wrapped(uint32_t k, uint32_t at) {
  return Epi::kWrap && k >= at ? k - at : k;
}

// BM x BN workgroup tile (BN counts both matrices' channels in a gated product), WGM x WGN wavefronts, BKB bytes of k per stage.
template <int BM_, int BN_, int WGM_, int WGN_, int BKB_, int STAGES_>
struct RowsCfg {
  static constexpr int BM = BM_, BN = BN_, WGM = WGM_, WGN = WGN_, BKB = BKB_, STAGES = STAGES_;
  static constexpr int NW = WGM * WGN, THREADS = 64 * NW;
  static constexpr int WM = BM / WGM, WN = BN / WGN, MI = WM / 32, NJ = WN / 32;
  static constexpr int RPL = 1024 / BKB;                              // rows a wavefront's load of 1 KB covers
  static constexpr int X_LOADS = BM / RPL / NW, W_LOADS = BN / RPL / NW, LPS = X_LOADS + W_LOADS;
  static constexpr int STAGE_BYTES = (BM + BN) * BKB, NG = BKB / 32;  // groups of 32 bytes of k per stage
  static constexpr int PIPE_BYTES = STAGES * STAGE_BYTES;
  static_assert(WM % 32 == 0 && WN % 32 == 0 && STAGES >= 2 && (BKB == 64 || BKB == 128), "tile shape");
  static_assert(BM % (RPL * NW) == 0 && BN % (RPL * NW) == 0, "loads must divide evenly among the wavefronts");
  static_assert(PIPE_BYTES <= 160 * 1024 && LPS * (STAGES - 1) <= 63, "LDS of a CU, vmcnt range");
};

// Wait until at most `stages` * LPS of this wavefront's loads are outstanding.
template <int LPS, int MAX>
__device__ __forceinline__ void wait_rows_stages(int stages) {
  if constexpr (MAX == 0) {
    wait_vmcnt<0>();
  } else {
    if (stages >= MAX) wait_vmcnt<LPS * MAX>();
    else wait_rows_stages<LPS, MAX - 1>(stages);
  }
}

// As load_to_lds, with a scalar part of the offset.
__device__ __forceinline__ void load_rows_to_lds(__amdgpu_buffer_rsrc_t from, uint32_t off, uint32_t k, void* dst) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_ptr_t)dst, 16, (int)off, (int)k, 0, 0);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const void* base) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, -1, 0x00027000);
}

// Tile of a workgroup.  Workgroups go to the XCDs in turn; each XCD takes a run of consecutive tiles, which go down kGroupRows
// row tiles before they go right, so that the 32 tiles an XCD works on at a time share operands in its L2.
constexpr int kGroupRows = 8;
__device__ __forceinline__ bool rows_tile(int tiles_m, int tiles_n, int* tm, int* tn) {
  const int total = tiles_m * tiles_n, per_xcd = (total + 7) / 8;
  const int lin = blockIdx.x, xcd = lin & 7, at = lin >> 3;
  const int full = total - 8 * (per_xcd - 1);          // XCDs with per_xcd tiles; the others have one less
  const int id = xcd < full ? xcd * per_xcd + at : full * per_xcd + (xcd - full) * (per_xcd - 1) + at;
  if (at >= (xcd < full ? per_xcd : per_xcd - 1)) return false;
  const int group = id / (kGroupRows * tiles_n), rest = id - group * kGroupRows * tiles_n;
  const int high = min(kGroupRows, tiles_m - group * kGroupRows);
  *tm = group * kGroupRows + rest % high;
  *tn = rest / high;
  return true;
}

// LDS of a wavefront's transposed results, and of a kernel.
template <class Cfg>
constexpr int rows_turned() {   // rows that are turned at a time
  return Cfg::WM < 64 ? Cfg::WM : 64;
}
template <class Cfg, class Epi>
constexpr int rows_turned_bytes() {
  return Epi::kTurned ? Epi::kOutputs * (Cfg::WN / 2) * rows_turned<Cfg>() * 2 : 0;
}
template <class Cfg, class Epi, int B>
constexpr int rows_lds_bytes() {
  const int parked = Cfg::NW * (B * Epi::kOutputs * (Cfg::WN / (Epi::kGated ? 2 : 1)) * (int)sizeof(typename Epi::Out) + rows_turned_bytes<Cfg, Epi>());
  return parked > Cfg::PIPE_BYTES ? parked : Cfg::PIPE_BYTES;
}

// Epilogue.  acc[j][i]: blocks of B x B results (B = 32 or 16 by the matrix instruction), channels by rows; a lane holds, of its
// row of a block, four channels at 4 (lane / B), and with B = 32 those 8, 16 and 24 further on.  The results go through LDS, in
// the output's type, 64 columns a wavefront or 32 where two factors become one, so that rows leave in whole runs; LDS slots of 16
// bytes are permuted by the row for the banks.
template <class E, class Cfg, class Epi, class Acc, int NB, int MB>
__device__ __forceinline__ void rows_epilogue(const Epi& epi, Acc (&acc)[NB][MB], uint8_t* lds, int m0, int n0, int M) {
  constexpr bool GATED = Epi::kGated;
  constexpr int NW = Cfg::NW, B = Cfg::WN / NB;
  constexpr int RUNS = B == 32 ? 4 : 1;                     // a lane's runs of four channels in a block
  lds_handover();
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / Cfg::WGN, wn = wave % Cfg::WGN;
  const int lrow = lane % B, part = lane / B;
  typedef typename Epi::Out Out;
  constexpr int COLS = Cfg::WN / (GATED ? 2 : 1), OB = (int)sizeof(Out), OUTS = Epi::kOutputs;
  constexpr int ROWB = OUTS * COLS * OB, SL = ROWB / 16;    // bytes and slots of a parked row: one output after the other
  static_assert(rows_lds_bytes<Cfg, Epi, B>() <= 160 * 1024, "LDS of a CU");
  static_assert(SL >= 2 && SL <= 64 && (SL & (SL - 1)) == 0, "slots of a parked row");
  constexpr int FACTOR = GATED ? 32 / B : 0;                // blocks from a gate's to the matching up's
  uint8_t* park = lds + wave * (B * ROWB);
  // the transposed copy, in 16-bit numbers: the wavefront's columns, TURN rows each, behind the parked rows of all wavefronts; chunks of
  // eight rows are permuted by the column for the banks
  constexpr int TURN = rows_turned<Cfg>(), CH = TURN / 8;
  static_assert(!Epi::kTurned || (OB == 2 && TURN % B == 0 && CH >= 4), "16-bit numbers, whole blocks");
  uint8_t* turned = lds + NW * (B * ROWB) + wave * rows_turned_bytes<Cfg, Epi>();
  auto turned_key = [](int col) { return (col >> 2) * 2 & (CH - 1); };
  const int col0 = n0 + wn * COLS;                          // channel of the wavefront's first column
  auto column = [&](int j, int q) { return (GATED ? j * B / 64 * 32 + j * B % 32 : j * B) + (B == 32 ? 8 * q : 0) + 4 * part; };
  // what belongs to columns is the same for all rows: loaded once
  typename Epi::Cols cc[NB][RUNS];
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int q = 0; q < RUNS; ++q)
      if (!(GATED && (j * B / 32) % 2)) cc[j][q] = epi.cols(col0 + column(j, q));
  // what a result takes besides (dh, in a gradient) is fetched a block of rows ahead
  typename Epi::Extra extra[2][NB][RUNS];
  auto fetch = [&](int i) {
    const int m = min(m0 + wm * Cfg::WM + i * B + lrow, M - 1);
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int q = 0; q < RUNS; ++q)
        if (!(GATED && (j * B / 32) % 2)) extra[i & 1][j][q] = epi.extra(m, col0 + column(j, q));
  };
  fetch(0);
#pragma unroll
  for (int i = 0; i < MB; ++i) {
    const int mrow = m0 + wm * Cfg::WM + i * B;
    bool over = mrow >= M;
    if constexpr (Epi::kTurned) over = mrow >= epi.turned_rows(M);
    if (over) break;
    if (i + 1 < MB) fetch(i + 1);
    const int m = min(mrow + lrow, M - 1);
    const auto rc = epi.row(m);
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      if (GATED && (j * B / 32) % 2) continue;
#pragma unroll
      for (int q = 0; q < RUNS; ++q) {
        const int c = column(j, q);
        typename E::Sum a[4], b[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          a[r] = acc[j][i][4 * q + r];
          b[r] = acc[j + FACTOR][i][4 * q + r];
        }
        Out v[OUTS][4];
        epi.values(rc, cc[j][q], extra[i & 1][j][q], col0 + c, a, b, v);
#pragma unroll
        for (int o = 0; o < OUTS; ++o) {
          const int byte = (o * COLS + c) * OB, sl = (byte >> 4) ^ (lrow & (SL - 1));
          if constexpr (Epi::kTurned) {
            if (epi.turned) {
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const int col = o * COLS + c + r, at = i * B % TURN + lrow;
                *reinterpret_cast<Out*>(turned + col * (TURN * 2) + (((at >> 3) ^ turned_key(col)) * 16) + (at & 7) * 2) =
                    mrow + lrow < M ? v[o][r] : (Out)0.f;
              }
            }
          }
          if constexpr (OB == 2) *reinterpret_cast<uint2*>(park + lrow * ROWB + sl * 16 + (byte & 15)) = *reinterpret_cast<const uint2*>(v[o]);
          else *reinterpret_cast<uint4*>(park + lrow * ROWB + sl * 16) = *reinterpret_cast<const uint4*>(v[o]);
        }
      }
    }
    // (the region is this wavefront's own, whose LDS operations complete in order)
    if (!epi.wide) {   // rows at no multiple of 16 bytes: number by number, neighbours by neighbouring lanes
#pragma unroll 4
      for (int e = lane; e < B * COLS; e += 64) {
        const int r = e / COLS, byte = e % COLS * OB;
        const Out v = *reinterpret_cast<const Out*>(park + r * ROWB + (((byte >> 4) ^ (r & (SL - 1))) * 16) + (byte & 15));
        if (mrow + r < M) epi.store1(mrow + r, col0 + e % COLS, v);
      }
      continue;
    }
    constexpr int RPI = 64 / SL < B ? 64 / SL : B;        // rows a pass of the wavefront covers
#pragma unroll
    for (int r0 = 0; r0 < B; r0 += RPI) {
      const int r = r0 + lane / SL, sl = lane % SL;
      const uint4 v = *reinterpret_cast<const uint4*>(park + r * ROWB + ((sl ^ (r & (SL - 1))) * 16));
      if (lane < RPI * SL && mrow + r < M) epi.store(sl / (SL / OUTS), mrow + r, col0 + sl % (SL / OUTS) * (16 / OB), v);
    }
    if constexpr (Epi::kTurned) {   // (rows end, for the transposed copy, at a multiple of 64: no block is left over)
      if (epi.turned && (i + 1) * B % TURN == 0)
#pragma unroll 4
        for (int e = lane; e < OUTS * COLS * CH; e += 64) {
          const int col = e / CH, ch = e % CH;
          const uint4 v = *reinterpret_cast<const uint4*>(turned + col * (TURN * 2) + ((ch ^ turned_key(col)) * 16));
          epi.store_turned(col / COLS, mrow + B - TURN + ch * 8, col0 + col % COLS, v);
        }
    }
  }
}

// The share of k of a launch that splits it (gridDim.y workgroups a tile): whole stages, the last one takes what is left.  Returned:
// what is to be added to k, where operands wrap; the operands start there otherwise.
template <bool WRAP>
__device__ __forceinline__ uint32_t take_share(RowsProduct& p) {
  const int64_t share = (p.kb + 128 * (int64_t)gridDim.y - 1) / (128 * (int64_t)gridDim.y) * 128, from = min(share * blockIdx.y, p.kb);
  p.kb = min(share, p.kb - from);
  if (WRAP) return (uint32_t)from;
  p.x += from;
  p.w0 += from;
  return 0;
}

template <class E, class Cfg, class Epi>
__global__ __launch_bounds__(Cfg::THREADS) void gemm_rows_kernel(RowsProduct p, int tiles_m, int tiles_n, Epi epi) {
  constexpr bool GATED = Epi::kGated;
  uint32_t k_base = 0;
  if constexpr (Epi::kSplit) {
    k_base = take_share<Epi::kWrap>(p);
    epi.out += blockIdx.y * epi.part_stride;
  }
  constexpr int BM = Cfg::BM, BN = Cfg::BN, MI = Cfg::MI, NJ = Cfg::NJ, BKB = Cfg::BKB, STAGES = Cfg::STAGES, NG = Cfg::NG;
  constexpr int X_LOADS = Cfg::X_LOADS, W_LOADS = Cfg::W_LOADS, LPS = Cfg::LPS, NW = Cfg::NW, RPL = Cfg::RPL;
  constexpr int CPR = BKB / 16;                       // chunks of 16 bytes per row of a stage
  static_assert(!GATED || NJ % 2 == 0, "both factors in one wavefront");
  extern __shared__ __attribute__((aligned(16))) uint8_t rows_lds[];

  int tm, tn;
  if (!rows_tile(tiles_m, tiles_n, &tm, &tn)) return;
  const int M = p.rows_used ? min(max(*p.rows_used, 0), p.M) : p.M;
  const int m0 = tm * BM, n0 = tn * (GATED ? BN / 2 : BN);
  if (m0 >= M) return;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / Cfg::WGN, wn = wave % Cfg::WGN;
  const int l32 = lane & 31, half = lane >> 5;

  // LDS: a stage holds the tile's rows of x, then of the weights, BKB bytes each.  Chunk c of row r lies in slot
  // c ^ key(r), so that the 32 rows of a fragment read spread over all banks; the permutation is applied on the global side of
  // the loads, inside a row's own BKB bytes.
  constexpr int KEY_SHIFT = BKB == 128 ? 1 : 2;
  auto key_of = [](int row) { return (row >> KEY_SHIFT) & (CPR - 1); };
  const __amdgpu_buffer_rsrc_t xr = rows_rsrc(p.x + (int64_t)m0 * p.x_pitch);
  const __amdgpu_buffer_rsrc_t w0r = rows_rsrc(p.w0 + (int64_t)n0 * p.w_pitch0);
  const __amdgpu_buffer_rsrc_t w1r = rows_rsrc(GATED ? p.w1 + (int64_t)n0 * p.w_pitch1 : p.w0);
  uint32_t x_off[X_LOADS], w_off[W_LOADS];
  const int sub_row = lane / CPR, slot = lane % CPR;
#pragma unroll
  for (int i = 0; i < X_LOADS; ++i) {                 // (rows past the last repeat it; their results are not stored)
    const int row = (wave + NW * i) * RPL + sub_row;
    x_off[i] = (uint32_t)((int64_t)min(row, M - 1 - m0) * p.x_pitch) + (uint32_t)((slot ^ key_of(row)) * 16);
  }
#pragma unroll
  for (int i = 0; i < W_LOADS; ++i) {
    const int row = (wave + NW * i) * RPL + sub_row;
    const int ch = GATED ? (row >> 6) * 32 + (row & 31) : row;
    const int64_t pitch = GATED && ((row >> 5) & 1) ? p.w_pitch1 : p.w_pitch0;
    w_off[i] = (uint32_t)((int64_t)min(ch, p.N - 1 - n0) * pitch) + (uint32_t)((slot ^ key_of(row)) * 16);
  }
  auto second = [&](int i) { return GATED && (((wave + NW * i) * RPL >> 5) & 1); };   // the wavefront's load i is of w1

  // k runs over whole stages; what is left of it over BKB comes first, through registers and filled with zeros.
  const int rest = Epi::kWrap ? 0 : (int)(p.kb % BKB), nk = (int)(p.kb / BKB) + (rest ? 1 : 0);
  const uint32_t k_first = rest ? (uint32_t)rest : 0u;   // the first stage that is loaded directly starts here: stage s at
  auto k_of = [&](int s) { return k_base + (uint32_t)(rest ? (s - 1) * BKB + (int)k_first : s * BKB); };
  auto issue = [&](int s, uint8_t* sb, int first, int count) {
    const uint32_t k = k_of(s), kx = wrapped<Epi>(k, p.x_wrap), kw = wrapped<Epi>(k, p.w_wrap);
#pragma unroll
    for (int q = 0; q < LPS; ++q) {
      if (q < first || q >= first + count) continue;
      if (q < X_LOADS) load_rows_to_lds(xr, x_off[q], kx, sb + (wave + NW * q) * 1024);
      else load_rows_to_lds(second(q - X_LOADS) ? w1r : w0r, w_off[q - X_LOADS], kw, sb + BM * BKB + (wave + NW * (q - X_LOADS)) * 1024);
    }
  };

  typename E::Acc32 acc[NJ][MI];
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[j][i][r] = 0;

  uint4 part[LPS];   // the partial stage, on its way (it is parked when the loads behind it are)
  if (rest) {
#pragma unroll
    for (int q = 0; q < LPS; ++q) {
      const int b = q < X_LOADS ? wave + NW * q : wave + NW * (q - X_LOADS);
      const int at = (slot ^ key_of(b * RPL + sub_row)) * 16;
      const uint8_t* base = q < X_LOADS ? p.x + (int64_t)m0 * p.x_pitch
                            : second(q - X_LOADS) ? p.w1 + (int64_t)n0 * p.w_pitch1 : p.w0 + (int64_t)n0 * p.w_pitch0;
      part[q] = make_uint4(0u, 0u, 0u, 0u);
      if (at < rest) part[q] = *reinterpret_cast<const uint4*>(base + (q < X_LOADS ? x_off[q < X_LOADS ? q : 0] : w_off[q < X_LOADS ? 0 : q - X_LOADS]));
    }
  } else if (nk > 0) {
    issue(0, rows_lds, 0, LPS);
  }
#pragma unroll
  for (int s = 1; s < STAGES - 1; ++s)
    if (s < nk) issue(s, rows_lds + s * Cfg::STAGE_BYTES, 0, LPS);
  if (rest) {
#pragma unroll
    for (int q = 0; q < LPS; ++q)
      *reinterpret_cast<uint4*>(rows_lds + (q < X_LOADS ? (wave + NW * q) * 1024 : BM * BKB + (wave + NW * (q - X_LOADS)) * 1024) + lane * 16) = part[q];
  }

  v4i_b xf[2][MI], wf[2][NJ];
  const int x_row = (wm * Cfg::WM + l32) * BKB, w_row = BM * BKB + (wn * Cfg::WN + l32) * BKB;
  int cp[NG];
#pragma unroll
  for (int g = 0; g < NG; ++g) cp[g] = ((2 * g + half) ^ key_of(l32)) * 16;   // (tile offsets are multiples of 32: same keys)
  auto read_frags = [&](const uint8_t* sb, int g, int buf) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) wf[buf][j] = *reinterpret_cast<const v4i_b*>(sb + w_row + j * 32 * BKB + cp[g]);
#pragma unroll
    for (int i = 0; i < MI; ++i) xf[buf][i] = *reinterpret_cast<const v4i_b*>(sb + x_row + i * 32 * BKB + cp[g]);
  };
  constexpr int G = MI * NJ;
  auto mma = [&](int buf, int first, int count) {
#pragma unroll
    for (int q = 0; q < G; ++q)
      if (q >= first && q < first + count) acc[q % NJ][q / NJ] = E::mma32(wf[buf][q % NJ], xf[buf][q / NJ], acc[q % NJ][q / NJ]);
  };

  // ---- pipeline: everything that is not a matrix instruction runs in the shadow of one (as in gemm_bf16_slab.h).  Each group's
  // instructions have the next group's fragment reads and a share of the loads of stage kt + STAGES - 1 slotted in; half-way
  // through a stage's last group the wavefront waits for its loads of the next stage, meets the others and reads on there.
  constexpr int H1 = (G + 1) / 2, H2 = G - H1, RD = MI + NJ, SLOTS = (RD + 1) / 2, RLAST = RD - 2 * (SLOTS - 1);
  constexpr int REM = G > SLOTS ? G - SLOTS : 0;
  constexpr int LPG = (LPS + NG - 1) / NG;
  if (nk > 0) {
    wait_rows_stages<LPS, STAGES - 2>(nk - 1);
    lds_handover();
    read_frags(rows_lds, 0, 0);
  }
  int cur = 0, nst = STAGES - 1;
  auto step = [&](int kt, auto steady_c) {
    constexpr bool steady = decltype(steady_c)::value;
    const uint8_t* sb = rows_lds + cur * Cfg::STAGE_BYTES;
    uint8_t* nb = rows_lds + nst * Cfg::STAGE_BYTES;
    const int nxt = kt + STAGES - 1;
    nst = cur;
    cur = cur + 1 == STAGES ? 0 : cur + 1;
#pragma unroll
    for (int g = 0; g < NG - 1; ++g) {
      read_frags(sb, g + 1, (g + 1) & 1);
      if constexpr (steady) issue(nxt, nb, g * LPG, LPG);
      mma(g & 1, 0, G);
      sched_pairs<0x100, (SLOTS - 1 < G ? SLOTS - 1 : G), 2>();
      if constexpr (SLOTS <= G) sched_pairs<0x100, 1, RLAST>();
      sched_pairs<0x010, (LPG < REM ? LPG : REM), 1>();
      sched_mfma<REM - (LPG < REM ? LPG : REM)>();
    }
    if constexpr (steady) issue(nxt, nb, (NG - 1) * LPG, LPG);
    mma((NG - 1) & 1, 0, H1);
    sched_pairs<0x010, (LPG < H1 ? LPG : H1), 1>();
    sched_mfma<H1 - (LPG < H1 ? LPG : H1)>();
    if (steady || kt + 1 < nk) {
      if constexpr (steady) wait_vmcnt<LPS * (STAGES - 2)>();
      else wait_rows_stages<LPS, STAGES - 2>(nk - 2 - kt);
      lds_handover();
      read_frags(rows_lds + cur * Cfg::STAGE_BYTES, 0, 0);
    }
    mma((NG - 1) & 1, H1, H2);
    sched_pairs<0x100, (SLOTS - 1 < H2 ? SLOTS - 1 : H2), 2>();
  };
  static_assert(NG % 2 == 0, "a stage's first group is in the first buffer");
  int kt = 0;
  for (; kt + STAGES - 1 < nk; ++kt) step(kt, std::true_type());
  for (; kt < nk; ++kt) step(kt, std::false_type());

  rows_epilogue<E, Cfg>(epi, acc, rows_lds, m0, n0, M);
}

// ---- the large tile ----------------------------------------------------------------------------------------------------
// 256 x 256 by eight wavefronts of 128 x 64, 128 bytes of k per stage, two stages (128 KB).  What bounds it is how fast a CU
// pulls its operands: alone, the loads of 4096 such tiles run at 13.6 TB/s in rows of 64 bytes and at 19.0 in rows of 128, the
// matrix cores ask for 14 at 1.9 GHz, and with all of a stage's loads waited for at its end (the pipeline above) 11.9 arrive.
// So a stage is handed over in halves: the x rows a wavefront multiplies first (X0, half of its rows) with the channels it
// multiplies first (W0), and the rest (X1, W1).  A stage takes two steps of 16 matrix instructions a wavefront,
//   A: X0 W0, X0 W1     reads W1, X1 of this stage       fetches X0, W0 of the stage after the next
//   B: X1 W0, X1 W1     reads X0, W0 of the next stage   fetches W1, X1 of the stage after the next
// each half being refilled right after the step that has read it into registers: three steps of loads (96 KB) are always in
// flight, and every step's operands are in registers when it starts.  One barrier a step.
//
// 16 x 16 instructions: of the same rate as the 32 x 32 ones of the other tiles, they read and write their sums half as often per
// product, and this kernel is where the chip's power is the limit (1.5 GHz on random operands, 2.4 on zeros): 8192 x 32768 x 4096
// in bf16 1703 us for 1800, and 1885 with the pipeline above.  (A workgroup that takes one tile after the other, the next one's
// first stages under the results of the last, saves 2 us of a tile's 10 of fill and drain and loses 0.07 of each of its stages' 1.13: 7.09
// ms for 7.00 of a training step, dg and du being one number each.)
typedef RowsCfg<256, 256, 2, 4, 128, 2> Rows256;

template <class E, class Epi>
__global__ __launch_bounds__(512) void gemm_rows_big_kernel(RowsProduct p, int tiles_m, int tiles_n, Epi epi) {
  typedef Rows256 Cfg;
  constexpr bool GATED = Epi::kGated;
  uint32_t k_base = 0;
  if constexpr (Epi::kSplit) {
    k_base = take_share<Epi::kWrap>(p);
    epi.out += blockIdx.y * epi.part_stride;
  }
  constexpr int BM = 256, BKB = 128;
  extern __shared__ __attribute__((aligned(16))) uint8_t rows_lds[];

  int tm, tn;
  if (!rows_tile(tiles_m, tiles_n, &tm, &tn)) return;
  const int M = p.rows_used ? min(max(*p.rows_used, 0), p.M) : p.M;
  const int m0 = tm * BM, n0 = tn * (GATED ? 128 : 256);
  if (m0 >= M) return;

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 2, wn = wave & 3, l16 = lane & 15, quarter = lane >> 4;

  // A wavefront's loads of a half: 8 rows each, of x rows h * 64 + q * 128 + 8 wave .. (q = 0, 1), and of channel rows
  // h * 32 + 64 (2 q + wave / 4) + 8 (wave % 4) ..  Slots of a row's eight chunks are permuted as above.
  const __amdgpu_buffer_rsrc_t xr = rows_rsrc(p.x + (int64_t)m0 * p.x_pitch);
  const __amdgpu_buffer_rsrc_t w0r = rows_rsrc(p.w0 + (int64_t)n0 * p.w_pitch0);
  const __amdgpu_buffer_rsrc_t w1r = rows_rsrc(GATED ? p.w1 + (int64_t)n0 * p.w_pitch1 : p.w0 + (int64_t)n0 * p.w_pitch0);
  const int sub = lane >> 3, slot = lane & 7;
  uint32_t x_off[2][2], w_off[2][2];
  int x_blk[2][2], w_blk[2][2];                       // LDS, in kilobytes
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      x_blk[h][q] = h * 8 + q * 16 + wave;
      w_blk[h][q] = BM / 8 + h * 4 + 8 * (2 * q + (wave >> 2)) + (wave & 3);
      const int xrow = x_blk[h][q] * 8 + sub, wrow = (w_blk[h][q] - BM / 8) * 8 + sub;
      const int chunk = (slot ^ ((xrow >> 1) & 7)) * 16, wchunk = (slot ^ ((wrow >> 1) & 7)) * 16;
      x_off[h][q] = (uint32_t)((int64_t)min(xrow, M - 1 - m0) * p.x_pitch) + chunk;
      const int ch = GATED ? (wrow >> 6) * 32 + (wrow & 31) : wrow;
      w_off[h][q] = (uint32_t)((int64_t)min(ch, p.N - 1 - n0) * (GATED && h ? p.w_pitch1 : p.w_pitch0)) + wchunk;
    }
  const int rest = Epi::kWrap ? 0 : (int)(p.kb % BKB), nk = (int)(p.kb / BKB) + (rest ? 1 : 0);
  auto k_of = [&](int s) { return k_base + (uint32_t)(rest ? (s - 1) * BKB + rest : s * BKB); };
  auto issue = [&](int s, int h) {
    const uint32_t k = k_of(s), kx = wrapped<Epi>(k, p.x_wrap), kw = wrapped<Epi>(k, p.w_wrap);
    uint8_t* sb = rows_lds + (s & 1) * Cfg::STAGE_BYTES;
#pragma unroll
    for (int q = 0; q < 2; ++q) load_rows_to_lds(xr, x_off[h][q], kx, sb + x_blk[h][q] * 1024);
#pragma unroll
    for (int q = 0; q < 2; ++q) load_rows_to_lds(h ? w1r : w0r, w_off[h][q], kw, sb + w_blk[h][q] * 1024);
  };

  typename E::Acc16 acc[4][8];
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[j][i][r] = 0;

  // fragments: x[h][i][g]: rows h * 64 + i * 16 .., w[h][j][g]: channels h * 32 + j * 16 ..; g: 64 bytes of k
  v4i_b x[2][4][2], w[2][2][2];
  int cp[2];
#pragma unroll
  for (int g = 0; g < 2; ++g) cp[g] = ((4 * g + quarter) ^ ((l16 >> 1) & 7)) * 16;
  const int x_row = (wm * 128 + l16) * BKB, w_row = (BM + wn * 64 + l16) * BKB;
  auto read_x = [&](int s, int h) {
    const uint8_t* sb = rows_lds + (s & 1) * Cfg::STAGE_BYTES + x_row + h * 64 * BKB;
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[h][i][g] = *reinterpret_cast<const v4i_b*>(sb + i * 16 * BKB + cp[g]);
  };
  auto read_w = [&](int s, int h) {
    const uint8_t* sb = rows_lds + (s & 1) * Cfg::STAGE_BYTES + w_row + h * 32 * BKB;
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int j = 0; j < 2; ++j) w[h][j][g] = *reinterpret_cast<const v4i_b*>(sb + j * 16 * BKB + cp[g]);
  };
  auto mma = [&](int hx, int hw) {
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[2 * hw + j][4 * hx + i] = E::mma16(w[hw][j][g], x[hx][i][g], acc[2 * hw + j][4 * hx + i]);
  };

  // the first stage, through registers if it is what is left of k over whole stages (zeros behind it), and the second
  uint4 part[2][2][2];   // (parked when the loads behind it are on their way)
  if (rest) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int xk = (slot ^ (((x_blk[h][q] * 8 + sub) >> 1) & 7)) * 16, wk = (slot ^ (((w_blk[h][q] * 8 + sub) >> 1) & 7)) * 16;
        part[h][q][0] = part[h][q][1] = make_uint4(0u, 0u, 0u, 0u);
        if (xk < rest) part[h][q][0] = *reinterpret_cast<const uint4*>(p.x + (int64_t)m0 * p.x_pitch + x_off[h][q]);
        if (wk < rest)
          part[h][q][1] = *reinterpret_cast<const uint4*>((GATED && h ? p.w1 + (int64_t)n0 * p.w_pitch1 : p.w0 + (int64_t)n0 * p.w_pitch0) + w_off[h][q]);
      }
  } else if (nk > 0) {   // (a share of k may be empty)
    issue(0, 0);
    issue(0, 1);
  }
  if (nk > 1) {
    issue(1, 0);
    issue(1, 1);
  }
  if (rest) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        *reinterpret_cast<uint4*>(rows_lds + x_blk[h][q] * 1024 + lane * 16) = part[h][q][0];
        *reinterpret_cast<uint4*>(rows_lds + w_blk[h][q] * 1024 + lane * 16) = part[h][q][1];
      }
  }
  if (nk > 1) wait_vmcnt<8>();
  else wait_vmcnt<0>();
  lds_handover();
  read_x(0, 0);
  read_w(0, 0);
  lds_handover();
  // steady: stages s + 1 and s + 2 exist.  The loads outstanding behind the half a wait is for are those of two steps.
  auto stage = [&](int s, auto steady_c) {
    constexpr bool steady = decltype(steady_c)::value;
    if constexpr (steady) issue(s + 2, 0);
    read_w(s, 1);
    mma(0, 0);
    read_x(s, 1);
    mma(0, 1);
    sched_pairs<0x100, 4, 1>();
    sched_pairs<0x010, 4, 1>();
    sched_mfma<8>();
    sched_pairs<0x100, 8, 1>();
    sched_mfma<8>();
    if constexpr (steady) wait_vmcnt<8>();
    else wait_vmcnt<4>();
    lds_handover();
    if constexpr (steady) issue(s + 2, 1);
    if (steady || s + 1 < nk) read_x(s + 1, 0);
    mma(1, 0);
    if (steady || s + 1 < nk) read_w(s + 1, 0);
    mma(1, 1);
    sched_pairs<0x010, 4, 1>();
    sched_pairs<0x100, 8, 1>();
    sched_mfma<4>();
    sched_pairs<0x100, 4, 1>();
    sched_mfma<12>();
    if constexpr (steady) wait_vmcnt<8>();
    else wait_vmcnt<0>();
    lds_handover();
  };
  int s = 0;
  for (; s + 2 < nk; ++s) stage(s, std::true_type());
  for (; s < nk; ++s) stage(s, std::false_type());
  rows_epilogue<E, Cfg>(epi, acc, rows_lds, m0, n0, M);
}

// ---- few rows ----------------------------------------------------------------------------------------------------------
// Up to 64 rows: a stream of the weights.  A workgroup of eight wavefronts owns 16 channels (of each matrix) and all rows; the
// wavefronts take 128 bytes of k in turn, straight from memory into the matrix instructions' operands (an instruction takes
// 64 bytes of 16 rows), DEPTH such pieces in flight, and the eight partial sums meet in LDS.  Sums are added in the order of
// the wavefronts: the same bits every time, and for any number of rows.  Plain loads: marked as not to be kept, the weights of a
// network that the Infinity Cache holds came from memory every time (67 MB of 8-bit gated weights, one row, 15.5 -> 13.0 us).
constexpr int kFewGrid = 65536;
template <class E, int MT, class Epi>
__global__ __launch_bounds__(512) void gemm_few_rows_kernel(RowsProduct p, Epi epi) {
  constexpr bool GATED = Epi::kGated;
  constexpr int WT = GATED ? 2 : 1, NWAVES = 8, DEPTH = MT == 1 ? 4 : 2;
  const int M = p.rows_used ? min(max(*p.rows_used, 0), p.M) : p.M;
  // (channels over two dimensions of the grid, 2^28 of them being more than 2^32 threads, in rows of kFewGrid workgroups: gridDim.x
  // is a load from memory)
  const int m0 = blockIdx.z * (16 * MT), n0 = (int)(blockIdx.y * kFewGrid + blockIdx.x) * 16;
  if (m0 >= M || n0 >= epi.columns()) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, quarter = lane >> 4;
  const uint8_t* wrow[WT];
  wrow[0] = p.w0 + (int64_t)min(n0 + l16, p.N - 1) * p.w_pitch0;
  if constexpr (GATED) wrow[1] = p.w1 + (int64_t)min(n0 + l16, p.N - 1) * p.w_pitch1;
  // (lanes of rows that are not there load nothing: with one row, a sixteenth of the requests)
  const uint8_t* xrow[MT];
  bool there[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    there[i] = m0 + i * 16 + l16 < M;
    xrow[i] = p.x + (int64_t)min(m0 + i * 16 + l16, M - 1) * p.x_pitch;
  }
  typename E::Acc16 acc[WT][MT];
#pragma unroll
  for (int t = 0; t < WT; ++t)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[t][i][r] = 0;
  const v4i_b zero = {0, 0, 0, 0};
  for (int64_t k0 = (int64_t)wave * 128; k0 < p.kb; k0 += (int64_t)NWAVES * 128 * DEPTH) {
    v4i_b wf[DEPTH][2][WT], xf[DEPTH][2][MT];
#pragma unroll
    for (int s = 0; s < DEPTH; ++s)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t k = k0 + (int64_t)s * NWAVES * 128 + h * 64 + quarter * 16;
        const bool in = k < p.kb;
        const int64_t kx = Epi::kWrap && k >= p.x_wrap ? k - p.x_wrap : k, kw = Epi::kWrap && k >= p.w_wrap ? k - p.w_wrap : k;
#pragma unroll
        for (int t = 0; t < WT; ++t) wf[s][h][t] = in ? *reinterpret_cast<const v4i_b*>(wrow[t] + kw) : zero;
#pragma unroll
        for (int i = 0; i < MT; ++i) xf[s][h][i] = in && there[i] ? *reinterpret_cast<const v4i_b*>(xrow[i] + kx) : zero;
      }
#pragma unroll
    for (int s = 0; s < DEPTH; ++s)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < WT; ++t)
#pragma unroll
          for (int i = 0; i < MT; ++i) acc[t][i] = E::mma16(wf[s][h][t], xf[s][h][i], acc[t][i]);
  }
  // lane: row l16, channels 4 quarter .. + 3
  __shared__ __attribute__((aligned(16))) typename E::Sum part[NWAVES][WT][MT][16][16];
#pragma unroll
  for (int t = 0; t < WT; ++t)
#pragma unroll
    for (int i = 0; i < MT; ++i) *reinterpret_cast<typename E::Acc16*>(&part[wave][t][i][l16][4 * quarter]) = acc[t][i];
  __syncthreads();
  for (int e = tid; e < MT * 256; e += 512) {
    const int i = e >> 8, row = (e >> 4) & 15, c = e & 15, m = m0 + i * 16 + row, n = n0 + c;
    if (m >= M || n >= epi.columns()) continue;
    typename E::Sum a = part[0][0][i][row][c], b = part[0][WT - 1][i][row][c];
#pragma unroll
    for (int w = 1; w < NWAVES; ++w) {
      a += part[w][0][i][row][c];
      if constexpr (GATED) b += part[w][1][i][row][c];
    }
    epi.one(m, n, a, b);
  }
}

}  // namespace asd
