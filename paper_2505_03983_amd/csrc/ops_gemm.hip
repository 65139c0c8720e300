// The operators that are products: 8-bit linear layer, gated unit and its gradient.  The kernels are in gemm_rows.h; here are
// their epilogues, the choice of tile, and the passes that bring operands into a form the kernels read (copies of rows that
// start at no multiple of 16 bytes; the gradient's transposed operands).
#include <math.h>

#include <atomic>
#include <initializer_list>

#include "gemm_rows.h"
#include "ops.h"

namespace asd {

// ---- epilogues -----------------------------------------------------------------------------------------------------------
// A run of 16 bytes of results, columns n .. of a row of n_cols that starts on 16 bytes.
template <class T>
__device__ __forceinline__ void store_cols(T* row, int n, int n_cols, uint4 v) {
  constexpr int CNT = 16 / (int)sizeof(T);
  if (n + CNT <= n_cols) {
    *reinterpret_cast<uint4*>(row + n) = v;
    return;
  }
  T e[CNT];
  *reinterpret_cast<uint4*>(e) = v;
#pragma unroll
  for (int k = 0; k < CNT; ++k)
    if (n + k < n_cols) row[n + k] = e[k];
}

// out = sum (a gradient's product); rows from `second` on go to the other output (dw_gate, dw_up as one product)
template <class T, bool WRAP = false>
struct SumEpi {
  T* out;
  T* out2;
  int64_t ld, ld2;
  int N, first_rows, second;   // rows 0 .. first_rows - 1 and second .. second + first_rows - 1 are stored
  bool wide;
  __host__ __device__ __forceinline__ int columns() const { return N; }
  typedef T Out;
  static constexpr bool kGated = false, kSplit = false, kTurned = false, kWrap = WRAP;
  static constexpr int kOutputs = 1;
  struct Row {};
  __device__ __forceinline__ Row row(int) const { return Row{}; }
  struct Cols {};
  __device__ __forceinline__ Cols cols(int) const { return Cols{}; }
  struct Extra {};
  __device__ __forceinline__ Extra extra(int, int) const { return Extra{}; }
  __device__ __forceinline__ void values(Row, Cols, Extra, int, const float* a, const float*, T (&v)[1][4]) const {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[0][r] = (T)a[r];
  }
  __device__ __forceinline__ void store(int, int m, int n, uint4 v) const {
    if (m < first_rows) store_cols(out + m * ld, n, N, v);
    else if (m >= second && m < second + first_rows) store_cols(out2 + (m - second) * ld2, n, N, v);
  }
  __device__ __forceinline__ void store1(int m, int n, T v) const {
    if (n >= N) return;
    if (m < first_rows) out[m * ld + n] = v;
    else if (m >= second && m < second + first_rows) out2[(m - second) * ld2 + n] = v;
  }
  __device__ __forceinline__ void one(int m, int n, float a, float) const {
    if (m < first_rows) out[m * ld + n] = (T)a;
    else if (m >= second && m < second + first_rows) out2[(m - second) * ld2 + n] = (T)a;
  }
};

// Partial sums of a launch that splits k: part [split][rows][N] (S: float or int), added up in order by finish_kernel.
template <class S, bool WRAP>
struct PartEpi {
  S* out;
  int64_t part_stride;
  int N;
  bool wide;
  __host__ __device__ __forceinline__ int columns() const { return N; }
  typedef S Out;
  static constexpr bool kGated = false, kSplit = true, kTurned = false, kWrap = WRAP;
  static constexpr int kOutputs = 1;
  struct Row {};
  __device__ __forceinline__ Row row(int) const { return Row{}; }
  struct Cols {};
  __device__ __forceinline__ Cols cols(int) const { return Cols{}; }
  struct Extra {};
  __device__ __forceinline__ Extra extra(int, int) const { return Extra{}; }
  __device__ __forceinline__ void values(Row, Cols, Extra, int, const S* a, const S*, S (&v)[1][4]) const {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[0][r] = a[r];
  }
  __device__ __forceinline__ void store(int, int m, int n, uint4 v) const { store_cols(out + (int64_t)m * N, n, N, v); }
  __device__ __forceinline__ void store1(int m, int n, S v) const {
    if (n < N) out[(int64_t)m * N + n] = v;
  }
};
template <class S, class Epi>
__global__ __launch_bounds__(256) void finish_kernel(const S* __restrict__ part, int64_t stride, int splits, int rows, const int32_t* rows_used, Epi epi) {
  const int N = epi.columns(), M = rows_used ? min(max(*rows_used, 0), rows) : rows;
  const int64_t at = workgroup() * 256 + threadIdx.x;
  const int64_t m = at / N;
  if (m >= M) return;
  S s = part[at];
  for (int z = 1; z < splits; ++z) s += part[z * stride + at];
  epi.one((int)m, (int)(at - m * N), s, s);
}

// A row's scale: s up.  A sum of 31 bits times a scale above 2^96 may leave fp32, where the channel's scale brings it back: such a scale
// goes in as 2^-32 of itself, and 2^32 at the end.
struct RowScale {
  float s, up;
};
__device__ __forceinline__ RowScale row_scale(float v) {
  return fabsf(v) > 0x1p96f ? RowScale{v * 0x1p-32f, 0x1p32f} : RowScale{v, 1.f};
}

// out = sum x_scale w_scale + bias
template <class T>
struct Scaled8Epi {
  T* out;
  int64_t ld;
  const float* x_scale;
  const float* w_scale;
  const float* bias;   // or NULL
  int N;
  bool wide;
  __host__ __device__ __forceinline__ int columns() const { return N; }
  typedef T Out;
  static constexpr bool kGated = false, kSplit = false, kTurned = false, kWrap = false;
  static constexpr int kOutputs = 1;
  struct Cols {
    float s[4], b[4];
  };
  struct Extra {};
  __device__ __forceinline__ Extra extra(int, int) const { return Extra{}; }
  __device__ __forceinline__ RowScale row(int m) const { return row_scale(x_scale[m]); }
  __device__ __forceinline__ Cols cols(int n) const {
    Cols c;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      c.s[r] = w_scale[min(n + r, N - 1)];
      c.b[r] = bias ? bias[min(n + r, N - 1)] : 0.f;
    }
    return c;
  }
  __device__ __forceinline__ void values(RowScale x, const Cols& c, Extra, int, const int* a, const int*, T (&v)[1][4]) const {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[0][r] = (T)fmaf((float)a[r] * x.s * c.s[r], x.up, c.b[r]);
  }
  __device__ __forceinline__ void store(int, int m, int n, uint4 v) const { store_cols(out + m * ld, n, N, v); }
  __device__ __forceinline__ void store1(int m, int n, T v) const {
    if (n < N) out[m * ld + n] = v;
  }
  __device__ __forceinline__ void one(int m, int n, int a, int) const {
    const RowScale x = row(m);
    out[m * ld + n] = (T)fmaf((float)a * x.s * w_scale[n], x.up, bias ? bias[n] : 0.f);
  }
};

// Activations and their derivatives, in fp32.  exp2 and the reciprocal are the hardware's (1 ulp each): about 1e-6 of the value,
// far inside a 16-bit result.  An exponential that overflows is infinity, and its reciprocal 0: the limits.
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z));
}
constexpr float kGeluC = 0.7978845608028654f, kGeluA = 0.044715f;   // sqrt(2 / pi)
__device__ __forceinline__ float act_value(int act, float z) {
  // 0.5 (1 + tanh s) = sigmoid(2 s)
  return z * sigmoid(act == ASD_ACT_SILU ? z : 2.f * kGeluC * fmaf(kGeluA * z * z, z, z));
}
__device__ __forceinline__ void act_both(int act, float z, float* value, float* slope) {
  const float on = sigmoid(act == ASD_ACT_SILU ? z : 2.f * kGeluC * fmaf(kGeluA * z * z, z, z));
  const float inner = act == ASD_ACT_SILU ? 1.f : 2.f * kGeluC * fmaf(3.f * kGeluA * z, z, 1.f);
  *value = z * on;
  // (on (1 - on) is 0 where the sigmoid is saturated, whatever inner grows to)
  const float bend = on * (1.f - on);
  *slope = bend > 0.f ? fmaf(z * inner, bend, on) : on;
}

template <class T>
struct GatedEpi {
  T* out;
  int64_t ld;
  int N, act;
  bool wide;
  __host__ __device__ __forceinline__ int columns() const { return N; }
  typedef T Out;
  static constexpr bool kGated = true, kSplit = false, kTurned = false, kWrap = false;
  static constexpr int kOutputs = 1;
  struct Row {};
  __device__ __forceinline__ Row row(int) const { return Row{}; }
  struct Cols {};
  __device__ __forceinline__ Cols cols(int) const { return Cols{}; }
  struct Extra {};
  __device__ __forceinline__ Extra extra(int, int) const { return Extra{}; }
  __device__ __forceinline__ void values(Row, Cols, Extra, int, const float* g, const float* u, T (&v)[1][4]) const {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[0][r] = (T)(act_value(act, g[r]) * u[r]);
  }
  __device__ __forceinline__ void store(int, int m, int n, uint4 v) const { store_cols(out + m * ld, n, N, v); }
  __device__ __forceinline__ void store1(int m, int n, T v) const {
    if (n < N) out[m * ld + n] = v;
  }
  __device__ __forceinline__ void one(int m, int n, float g, float u) const { out[m * ld + n] = (T)(act_value(act, g) * u); }
};

template <class T>
struct Gated8Epi {
  T* out;
  int64_t ld;
  const float* x_scale;
  const float* gate_scale;
  const float* up_scale;
  int N, act;
  bool wide;
  __host__ __device__ __forceinline__ int columns() const { return N; }
  typedef T Out;
  static constexpr bool kGated = true, kSplit = false, kTurned = false, kWrap = false;
  static constexpr int kOutputs = 1;
  struct Cols {
    float g[4], u[4];
  };
  struct Extra {};
  __device__ __forceinline__ Extra extra(int, int) const { return Extra{}; }
  __device__ __forceinline__ RowScale row(int m) const { return row_scale(x_scale[m]); }
  __device__ __forceinline__ Cols cols(int n) const {
    Cols c;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      c.g[r] = gate_scale[min(n + r, N - 1)];
      c.u[r] = up_scale[min(n + r, N - 1)];
    }
    return c;
  }
  __device__ __forceinline__ T value(RowScale x, float gs, float us, int g, int u) const {
    return (T)(act_value(act, (float)g * x.s * gs * x.up) * ((float)u * x.s * us * x.up));
  }
  __device__ __forceinline__ void values(RowScale x, const Cols& c, Extra, int, const int* g, const int* u, T (&v)[1][4]) const {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[0][r] = value(x, c.g[r], c.u[r], g[r], u[r]);
  }
  __device__ __forceinline__ void store(int, int m, int n, uint4 v) const { store_cols(out + m * ld, n, N, v); }
  __device__ __forceinline__ void store1(int m, int n, T v) const {
    if (n < N) out[m * ld + n] = v;
  }
  __device__ __forceinline__ void one(int m, int n, int g, int u) const { out[m * ld + n] = value(row(m), gate_scale[n], up_scale[n], g, u); }
};

// dg = dh u act'(g) and du = dh act(g), each as the sum of two bf16 numbers, what the products that follow take: dgu [rows][2][2 Np]
// holds the numbers next to dg, du, then what their rounding leaves, rounded; zeros in the columns N .. Np - 1 of every quarter.  (One
// number alone makes an error of the size of the results' own rounding: 1.41 of it together, and 1.8 over few numbers.  In fp16 dg and
// du may also leave the type: a gradient of 1e-5 lies among its last bits, and dh u above 65504, where the sums are well inside.)
// The tiles store them transposed, too, for the product that contracts over rows (as a pass of its own 230 us of 8192 x 2 * 16384
// numbers, and a launch).
template <class T>
struct GatedGradEpi {
  __bf16* dgu;
  int Np;
  const T* dh;
  int64_t ld_dh;
  int N, act;
  bool dh_wide;   // runs of four of dh lie on 8 bytes
  __bf16* turned;      // NULL, or the same transposed: [2 Np][2][Mp], zeros in the columns M .. Mp - 1 of either half
  int64_t Mp;
  __device__ __forceinline__ int turned_rows(int M) const { return turned ? (int)Mp : M; }
  __device__ __forceinline__ void store_turned(int which, int m, int n, uint4 v) const {
    if (n < Np && m < Mp) *reinterpret_cast<uint4*>(turned + (((int64_t)(which & 1) * Np + n) * 2 + (which >> 1)) * Mp + m) = v;
  }
  __host__ __device__ __forceinline__ int columns() const { return Np; }
  typedef __bf16 Out;
  static constexpr bool kGated = true, kSplit = false, kTurned = true, kWrap = false;
  static constexpr int kOutputs = 4;   // dg, du, and what is left of them
  struct Row {};
  __device__ __forceinline__ Row row(int) const { return Row{}; }
  struct Cols {};
  __device__ __forceinline__ Cols cols(int) const { return Cols{}; }
  struct Extra {
    T dh[4];
  };
  __device__ __forceinline__ Extra extra(int m, int n) const {
    Extra x;
    const T* at = dh + m * ld_dh + n;
    if (dh_wide && n + 4 <= N) {
      *reinterpret_cast<uint2*>(x.dh) = *reinterpret_cast<const uint2*>(at);
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) x.dh[r] = n + r < N ? at[r] : (T)0.f;
    }
    return x;
  }
  static __device__ __forceinline__ void split(float v, __bf16* hi, __bf16* lo) {
    *hi = (__bf16)v;
    const float left = v - (float)*hi;
    *lo = fabsf(left) < INFINITY ? (__bf16)left : (__bf16)0.f;   // (nothing is left of an infinity)
  }
  __device__ __forceinline__ void values(Row, Cols, const Extra& x, int n, const float* g, const float* u, __bf16 (&v)[4][4]) const {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float d = (float)x.dh[r];
      float value, slope;
      act_both(act, g[r], &value, &slope);
      split(n + r < N ? d * u[r] * slope : 0.f, &v[0][r], &v[2][r]);
      split(n + r < N ? d * value : 0.f, &v[1][r], &v[3][r]);
    }
  }
  static constexpr bool wide = true;
  __device__ __forceinline__ void store1(int, int, __bf16) const {}
  __device__ __forceinline__ void one(int m, int n, float g, float u) const {
    float dg = 0.f, du = 0.f;
    if (n < N) {
      const float d = (float)dh[m * ld_dh + n];
      float value, slope;
      act_both(act, g, &value, &slope);
      dg = d * u * slope;
      du = d * value;
    }
    __bf16* at = dgu + (int64_t)m * 4 * Np + n;
    split(dg, at, at + 2 * (int64_t)Np);
    split(du, at + Np, at + 3 * (int64_t)Np);
  }
  __device__ __forceinline__ void store(int which, int m, int n, uint4 v) const {
    if (n < Np) *reinterpret_cast<uint4*>(dgu + ((int64_t)m * 4 + which) * Np + n) = v;
  }
};

// ---- passes over operands --------------------------------------------------------------------------------------------------
// Rows of `bytes` bytes at any address and pitch, copied to rows on multiples of 128 bytes, zeros behind them.
struct RowsCopy {
  const uint8_t* src;
  uint8_t* dst;
  int64_t pitch, dst_pitch, bytes;
  int rows;
};
struct RowsCopies {
  RowsCopy c[3];
  int64_t first[3];   // its first workgroup
  int n;
};
// A row a wavefront, sixteen bytes of the copy a thread at a time.
constexpr int kCopyRows = 4;   // rows a workgroup
__global__ __launch_bounds__(64 * kCopyRows) void pack_rows_kernel(RowsCopies all) {
  int i = 0;
  while (i + 1 < all.n && workgroup() >= all.first[i + 1]) ++i;
  const RowsCopy& c = all.c[i];
  const int64_t row = (workgroup() - all.first[i]) * kCopyRows + (threadIdx.x >> 6);
  if (row >= c.rows) return;
  const uint8_t* src = c.src + row * c.pitch;
  uint8_t* dst = c.dst + row * c.dst_pitch;
  const int lane = threadIdx.x & 63, shift = (int)((uintptr_t)src & 3);
  // inside the row: five words around the sixteen bytes, all of this row; the first sixteen and the end byte by byte
  const int64_t inner = c.bytes < 36 ? 16 : (c.bytes - 20) / 16 * 16 + 16;
#pragma unroll 4
  for (int64_t k = 16 + lane * 16; k < inner; k += 1024) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(src + k - shift);
    uint32_t a[5], v[4];
#pragma unroll
    for (int j = 0; j < 5; ++j) a[j] = w[j];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __builtin_amdgcn_alignbyte(a[j + 1], a[j], shift);
    *reinterpret_cast<uint4*>(dst + k) = make_uint4(v[0], v[1], v[2], v[3]);
  }
  if (lane < 16) dst[lane] = lane < c.bytes ? src[lane] : (uint8_t)0;
  for (int64_t k = inner + lane; k < c.dst_pitch; k += 64) dst[k] = k < c.bytes ? src[k] : (uint8_t)0;
}

// dst [cols][dst_ld] = src [rows][cols] transposed, 16-bit elements, 64 x 64 a workgroup; columns rows .. of dst up to the next
// multiple of 64 are zero (dst_ld and dst are multiples of 16 bytes and hold them).  Up to six matrices a launch.  lo > 0: src is fp16,
// dst two bf16 numbers whose sum it is, the second `lo` elements behind the first (11 bits in 8 and what is left, 3).
struct Transpose16 {
  const uint16_t* src;
  uint16_t* dst;
  int64_t ld, dst_ld, lo;
  int rows, cols;
  bool wide;   // rows on 16 bytes
};
struct Transposes16 {
  Transpose16 t[6];
  int64_t first[6];   // its first workgroup
  int n;
};
__global__ __launch_bounds__(256) void transpose16_kernel(Transposes16 all) {
  int i = 0;
  while (i + 1 < all.n && workgroup() >= all.first[i + 1]) ++i;
  const uint16_t* src = all.t[i].src;
  uint16_t* dst = all.t[i].dst;
  const int64_t ld = all.t[i].ld, dst_ld = all.t[i].dst_ld, lo = all.t[i].lo;
  const int rows = all.t[i].rows, cols = all.t[i].cols;
  const bool wide = all.t[i].wide;
  const unsigned at = (unsigned)(workgroup() - all.first[i]), across = (unsigned)(cols + 63) / 64;
  if (at / across * 64 >= (unsigned)rows) return;   // (the grid's last row of workgroups)
  __shared__ uint16_t tile[64][72];   // (rows 144 bytes apart: columns of eight rows fall on different banks)
  const int r0 = (int)(at / across) * 64, c0 = (int)(at % across) * 64, t = threadIdx.x;
#pragma unroll
  for (int pass = 0; pass < 2; ++pass) {
    const int r = pass * 32 + (t >> 3), c = (t & 7) * 8;
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (r0 + r < rows) {
      const uint16_t* s = src + (int64_t)(r0 + r) * ld + c0 + c;
      if (wide && c0 + c + 8 <= cols) {
        v = *reinterpret_cast<const uint4*>(s);
      } else {
        uint32_t e[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (c0 + c + k < cols) e[k >> 1] |= (uint32_t)s[k] << (16 * (k & 1));
        v = make_uint4(e[0], e[1], e[2], e[3]);
      }
    }
    *reinterpret_cast<uint4*>(&tile[r][c]) = v;
  }
  __syncthreads();
#pragma unroll
  for (int pass = 0; pass < 2; ++pass) {
    const int c = pass * 32 + (t >> 3), r = (t & 7) * 8;
    if (c0 + c >= cols) continue;
    uint16_t* to = dst + (int64_t)(c0 + c) * dst_ld + r0 + r;
    uint32_t e[4] = {0u, 0u, 0u, 0u}, left[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      uint16_t v = tile[r + k][c];
      if (lo) {
        const float f = (float)__builtin_bit_cast(_Float16, v);
        const __bf16 hi = (__bf16)f;
        const float d = f - (float)hi;   // (nothing is left of an infinity or a NaN)
        v = __builtin_bit_cast(uint16_t, hi);
        left[k >> 1] |= (uint32_t)__builtin_bit_cast(uint16_t, fabsf(d) < INFINITY ? (__bf16)d : (__bf16)0.f) << (16 * (k & 1));
      }
      e[k >> 1] |= (uint32_t)v << (16 * (k & 1));
    }
    *reinterpret_cast<uint4*>(to) = make_uint4(e[0], e[1], e[2], e[3]);
    if (lo) *reinterpret_cast<uint4*>(to + lo) = make_uint4(left[0], left[1], left[2], left[3]);
  }
}

// ---- launches ----------------------------------------------------------------------------------------------------------------
typedef RowsCfg<128, 128, 2, 2, 128, 4> Rows128;
typedef RowsCfg<64, 128, 2, 2, 128, 5> Rows64;

template <class E, class Cfg, class Epi>
static hipError_t launch_rows(const RowsProduct& p, const Epi& e, hipStream_t st, int splits = 1) {
  constexpr bool BIG = std::is_same<Cfg, Rows256>::value;
  constexpr int LDS = rows_lds_bytes<Cfg, Epi, BIG ? 16 : 32>();
  void (*kern)(RowsProduct, int, int, Epi);
  if constexpr (BIG) kern = gemm_rows_big_kernel<E, Epi>;
  else kern = gemm_rows_kernel<E, Cfg, Epi>;
  static std::atomic<uint64_t> ready{0};   // devices whose limit of dynamic LDS has been raised for this kernel
  int dev = 0;
  hipError_t err = hipGetDevice(&dev);
  if (err != hipSuccess) return err;
  if (!(ready.load() >> (dev & 63) & 1)) {
    err = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    if (err != hipSuccess) return err;
    ready.fetch_or(1ull << (dev & 63));
  }
  const int tm = (int)ceil_div(p.M, Cfg::BM), tn = (int)ceil_div(p.N, Epi::kGated ? Cfg::BN / 2 : Cfg::BN);
  const int64_t grid = ceil_div((int64_t)tm * tn, 8) * 8;
  hipLaunchKernelGGL(kern, dim3((unsigned)grid, (unsigned)splits), dim3(Cfg::THREADS), LDS, st, p, tm, tn, e);
  return hipGetLastError();
}

// Which kernel: the least of the estimates below, in microseconds.  A tile takes f + k per 128 bytes of k, a workgroup has its CU
// to itself, and from the third round on the CUs no longer finish together.  Few rows: a workgroup of 16 channels pulls its rows of
// both operands at 32 KB a microsecond.  Fitted to 1 .. 4000 rows by 320 .. 11000 channels of 1024 .. 14848 numbers, 8-bit products and
// bf16 gated units (both matrices' channels count), operands from the Infinity Cache.
// Measured, few / 64 x 128 / 128 x 128 / 256 x 256: 8 bits, 4096 channels of 4096: 1 row 6.4 / 12.6 / 14.1 / -, 64 rows 13.4 / 12.7 /
// 14.8 / -, 1000 rows - / 29 / 24 / 48, 4000 rows - / 110 / 83 / 59; gated bf16, 4096 channels of 4096: 1 row 16 / 20 / 23 / -, 64 rows
// 30 / 21 / 24 / -, 400 rows - / 42 / 32 / 82, 2000 rows - / 177 / 129 / 108.  Of 140 such calls the rule misses the fastest kernel by
// more than a quarter in none, by more than a tenth in nine.
// Split k (pick_split), where the caller has room for the parts: 768 channels of 14848 in 8 bits, 64 rows 17.5 -> 12.9, 200 rows 33 ->
// 15.5; 4096 of 11008, 64 rows 28.6 -> 17.5.
struct RowsCost {
  int bm, bn;
  float f, k;
  float full;   // a tile takes this much longer where there are more tiles than CUs
};
constexpr RowsCost kRowsCost[3] = {{256, 256, 8.f, 1.14f, 1.15f}, {128, 128, 4.5f, 0.34f, 1.3f}, {64, 128, 4.5f, 0.27f, 1.1f}};
constexpr int kFewRows = 64;

// Kernel 0 .. 2: a tile; 3 .. 5: few rows, 16, 32 or 64 a workgroup.  splits: workgroups that share a tile's k.
static float kernel_us(int kernel, int M, int64_t n, int64_t kb, int splits = 1) {
  if (kernel >= 3) {   // a workgroup pulls its rows of both operands at 32 KB a microsecond, the chip at 4.8 MB
    const int rows = 16 << (kernel - 3);
    const float wgs = (float)(ceil_div(M, rows) * ceil_div(n, 16)), bytes = (float)kb * (float)(16 + std::min(M, rows));
    return 3.f + std::max(1.f, wgs / 256.f) * bytes / 32e3f;
  }
  const RowsCost& c = kRowsCost[kernel];
  const int64_t tiles = ceil_div(M, c.bm) * ceil_div(n, c.bn) * splits;
  float rounds = (float)ceil_div(tiles, 256);
  if (rounds > 2.f) rounds = 0.4f * rounds + 0.6f * (float)tiles / 256.f;
  const float t = rounds * (tiles > 256 ? c.full : 1.f) * (c.f + c.k * (float)ceil_div(kb, 128 * splits));
  // the parts are written, read again and added by a kernel of its own
  return splits == 1 ? t : t + 5.f + 8e-6f * (float)splits * (float)M * (float)n / 4.f;
}
static int best_tile(int M, int64_t n, int64_t kb) {
  int best = 0;
  for (int i = 1; i < 3; ++i)
    if (kernel_us(i, M, n, kb) < kernel_us(best, M, n, kb)) best = i;
  return best;
}
static int best_few(int M, int64_t n, int64_t kb) {
  int best = 3;
  for (int i = 4; i < 6; ++i)
    if (kernel_us(i, M, n, kb) < kernel_us(best, M, n, kb)) best = i;
  return best;
}
// likely: rows to expect of the M there may be.  They choose among the tiles, or among the forms of the kernel for few rows, which all
// give a row the same bits; which of the two it is goes by M alone.
static int pick_product(int M, int64_t n, int64_t kb, int likely) {
  const int tile = best_tile(M, n, kb), few = best_few(M, n, kb);
  return M <= kFewRows && kernel_us(few, M, n, kb) < kernel_us(tile, M, n, kb) ? best_few(likely, n, kb) : best_tile(likely, n, kb);
}
static int pick_product(int M, int64_t n, int64_t kb) { return pick_product(M, n, kb, M); }
int product_pick(int rows, int most, int64_t channels, int64_t kb) { return pick_product(most, channels, kb, rows); }
double product_us(int rows, int most, int64_t channels, int64_t kb) { return kernel_us(pick_product(most, channels, kb), rows, channels, kb); }

// How a product whose caller has room for partial sums splits k: few tiles and long sums.  {1, 0}: not at all.
struct Split {
  int splits, tile;
};
constexpr int kMaxSplits = 16;
static Split pick_split(int M, int64_t n, int64_t kb) {
  Split best{1, 0};
  float least = 0.9f * kernel_us(pick_product(M, n, kb), M, n, kb);   // (a second kernel for less is not worth its place)
  for (int tile = 0; tile < 3; ++tile)
    for (int s = 2; s <= kMaxSplits && kb >= (int64_t)s * 1024; ++s)
      if (const float t = kernel_us(tile, M, n, kb, s); t < least) {
        least = t;
        best = {s, tile};
      }
  return best;
}

template <class E, int MT, class Epi>
static hipError_t launch_few(const RowsProduct& p, const Epi& e, hipStream_t st) {
  const int64_t wgs = ceil_div(e.columns(), 16);
  const dim3 grid((unsigned)std::min<int64_t>(wgs, kFewGrid), (unsigned)ceil_div(wgs, kFewGrid), (unsigned)ceil_div(p.M, 16 * MT));
  hipLaunchKernelGGL((gemm_few_rows_kernel<E, MT, Epi>), grid, dim3(512), 0, st, p, e);
  return hipGetLastError();
}

// part: room for splits * M * N sums.
template <class E, class Epi>
static hipError_t launch_split(const RowsProduct& p, const Epi& e, Split sp, void* part, hipStream_t st) {
  typedef typename E::Sum S;
  const PartEpi<S, Epi::kWrap> pe{static_cast<S*>(part), (int64_t)p.M * p.N, p.N, (p.N & 3) == 0};
  hipError_t err = sp.tile == 0   ? launch_rows<E, Rows256>(p, pe, st, sp.splits)
                   : sp.tile == 1 ? launch_rows<E, Rows128>(p, pe, st, sp.splits)
                                  : launch_rows<E, Rows64>(p, pe, st, sp.splits);
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL((finish_kernel<S, Epi>), grid_of(ceil_div((int64_t)p.M * p.N, 256)), dim3(256), 0, st, pe.out, pe.part_stride, sp.splits,
                     p.M, p.rows_used, e);
  return hipGetLastError();
}

template <class E, class Epi>
static hipError_t launch_product(const RowsProduct& p, const Epi& e, hipStream_t st, int likely = 0) {
  const int pick = pick_product(p.M, Epi::kGated ? 2 * (int64_t)p.N : p.N, p.kb, likely > 0 ? std::min(likely, p.M) : p.M);
  if (pick == 3) return launch_few<E, 1>(p, e, st);
  if (pick == 4) return launch_few<E, 2>(p, e, st);
  if (pick == 5) return launch_few<E, 4>(p, e, st);
  if (pick == 0) return launch_rows<E, Rows256>(p, e, st);
  return pick == 1 ? launch_rows<E, Rows128>(p, e, st) : launch_rows<E, Rows64>(p, e, st);
}

constexpr int64_t kMaxPitch = (int64_t)4 << 20;   // bytes: a tile's offsets stay within 32 bits

// Part of a workspace, in order; bytes are rounded up to 256.
struct Carve {
  uint8_t* base;
  size_t used = 0;
  uint8_t* take(size_t bytes) {
    uint8_t* p = base ? base + used : nullptr;
    used += (bytes + 255) & ~(size_t)255;
    return p;
  }
};

// An operand as the kernels read it: itself, or a copy in the workspace.
struct Operand {
  const uint8_t* p;
  int64_t pitch;   // bytes
  bool copied;
  RowsCopy copy;
};
static Operand operand(const void* p, int rows, int64_t cols, int64_t ld, int bytes, Carve* ws) {
  const int64_t row = cols * bytes;
  const uint8_t* src = static_cast<const uint8_t*>(p);
  if (on16(p, rows > 1 ? ld : 0, bytes) && (row & 15) == 0 && (rows == 1 || ld * bytes <= kMaxPitch))
    return Operand{src, rows > 1 ? ld * bytes : row, false, RowsCopy{}};
  const int64_t pitch = ceil_div(row, 128) * 128;
  uint8_t* c = ws->take((size_t)pitch * rows);
  return Operand{c, pitch, true, RowsCopy{src, c, ld * bytes, pitch, row, rows}};
}
static hipError_t bring(std::initializer_list<const Operand*> operands, hipStream_t st) {
  RowsCopies all{};
  int64_t grid = 0;
  for (const Operand* o : operands) {
    if (!o->copied) continue;
    all.first[all.n] = grid;
    all.c[all.n++] = o->copy;
    grid += ceil_div(o->copy.rows, kCopyRows);
  }
  if (!all.n) return hipSuccess;
  hipLaunchKernelGGL(pack_rows_kernel, grid_of(grid), dim3(64 * kCopyRows), 0, st, all);
  return hipGetLastError();
}
// Bytes of k the kernels run over: copies have zeros behind their rows.
static int64_t k_bytes(int64_t row) { return ceil_div(row, 16) * 16; }

// ---- the 8-bit linear layer ----------------------------------------------------------------------------------------------------
struct Linear8Plan {
  Operand x, w;
  Split split;
  uint8_t* part;
  size_t bytes;
};
static Linear8Plan plan_linear8(const asd_linear8& p, void* ws, bool split) {
  Carve c{static_cast<uint8_t*>(ws)};
  Linear8Plan r;
  r.split = split ? pick_split(p.rows, p.channels, k_bytes(p.cols)) : Split{1, 0};
  r.part = r.split.splits > 1 ? c.take(sizeof(int) * (size_t)r.split.splits * p.rows * p.channels) : nullptr;
  r.x = operand(p.x, p.rows, p.cols, p.ld_x, 1, &c);
  r.w = operand(p.w, p.channels, p.cols, p.ld_w, 1, &c);
  r.bytes = c.used;
  return r;
}

template <class T>
static asd_status run_linear8(const asd_linear8& p, const Linear8Plan& o, hipStream_t st, int likely) {
  const RowsProduct g{o.x.p, o.w.p, nullptr, o.x.pitch, o.w.pitch, 0, p.rows, p.channels, k_bytes(p.cols), p.rows_used};
  const Scaled8Epi<T> e{static_cast<T*>(p.out), p.ld_out, p.x_scale, p.w_scale, p.bias, p.channels, on16(p.out, p.ld_out, sizeof(T))};
  if (o.split.splits > 1) ASD_HIP(launch_split<ElemI8>(g, e, o.split, o.part, st));
  else ASD_HIP(launch_product<ElemI8>(g, e, st, likely));
  return ASD_OK;
}

asd_status launch_linear8(const asd_linear8& p, hipStream_t st, bool split, int likely) {
  const Linear8Plan o = plan_linear8(p, p.workspace, split);
  ASD_HIP(bring({&o.x, &o.w}, st));
  return p.out_type == ASD_F32    ? run_linear8<float>(p, o, st, likely)
         : p.out_type == ASD_BF16 ? run_linear8<__bf16>(p, o, st, likely)
                                  : run_linear8<_Float16>(p, o, st, likely);
}

asd_status launch_linear_bf16(const void* x, const void* w, float* out, int rows, int cols, int channels, const int32_t* rows_used,
                              hipStream_t st, int likely) {
  const RowsProduct g{static_cast<const uint8_t*>(x), static_cast<const uint8_t*>(w), nullptr, 2 * (int64_t)cols, 2 * (int64_t)cols, 0, rows,
                      channels, 2 * (int64_t)cols, rows_used};
  const SumEpi<float> e{out, nullptr, channels, 0, channels, rows, rows, on16(out, channels, 4)};
  ASD_HIP(launch_product<ElemBf16>(g, e, st, likely));
  return ASD_OK;
}

// ---- the gated unit --------------------------------------------------------------------------------------------------------------
struct GatedPlan {
  Operand x, g, u;
  size_t bytes;
};
static GatedPlan plan_gated(const asd_gated& p, Carve* c) {
  const int e = type_bytes(p.type);
  GatedPlan r;
  r.x = operand(p.x, p.rows, p.cols, p.ld_x, e, c);
  r.g = operand(p.w_gate, p.channels, p.cols, p.ld_w_gate, e, c);
  r.u = operand(p.w_up, p.channels, p.cols, p.ld_w_up, e, c);
  r.bytes = c->used;
  return r;
}
static RowsProduct gated_product(const asd_gated& p, const GatedPlan& o) {
  return RowsProduct{o.x.p, o.g.p, o.u.p, o.x.pitch, o.g.pitch, o.u.pitch, p.rows, p.channels, k_bytes((int64_t)p.cols * type_bytes(p.type)), p.rows_used};
}

template <class E, class T>
static asd_status run_gated(const asd_gated& p, const GatedPlan& o, hipStream_t st, int likely) {
  const bool wide = on16(p.out, p.ld_out, sizeof(T));
  if constexpr (E::kBytes == 1) {
    const Gated8Epi<T> e{static_cast<T*>(p.out), p.ld_out, p.x_scale, p.gate_scale, p.up_scale, p.channels, p.act, wide};
    ASD_HIP(launch_product<E>(gated_product(p, o), e, st, likely));
  } else {
    const GatedEpi<T> e{static_cast<T*>(p.out), p.ld_out, p.channels, p.act, wide};
    ASD_HIP(launch_product<E>(gated_product(p, o), e, st, likely));
  }
  return ASD_OK;
}

asd_status launch_gated(const asd_gated& p, hipStream_t st, int likely) {
  Carve c{static_cast<uint8_t*>(p.workspace)};
  const GatedPlan o = plan_gated(p, &c);
  ASD_HIP(bring({&o.x, &o.g, &o.u}, st));
  if (p.type == ASD_I8) return p.out_type == ASD_BF16 ? run_gated<ElemI8, __bf16>(p, o, st, likely) : run_gated<ElemI8, _Float16>(p, o, st, likely);
  return p.type == ASD_BF16 ? run_gated<ElemBf16, __bf16>(p, o, st, likely) : run_gated<ElemF16, _Float16>(p, o, st, likely);
}

// Gradient.  g and u are computed again in the kernel that forms dg and du from them and dh; both products that follow contract
// over an index that is not the operands' rows' own (channels, rows), so their operands are transposed first, in passes that
// cost a few hundredths of the products at training sizes.  dg and du enter as the sum of two bf16 numbers: k runs over the products of
// the first ones and then of the second, against the same rows of the other operand; an fp16 operand is the sum of two as well, and
// the first ones run over its second in a third pass (what is left out is 2^-16 of a product).
struct GatedGradPlan {
  GatedPlan in;
  int Np;        // channels, padded to whole stages of k
  int64_t Mp;    // rows, likewise
  int terms;     // numbers an operand transposed consists of
  bool few;      // the kernel for few rows forms dg and du: nothing is stored transposed yet
  uint8_t *dgu, *dgu_t, *w_t, *x_t;
  Split dx, dw;
  uint8_t* part;   // partial sums of the one product, then of the other
  size_t bytes;
};
static GatedGradPlan plan_gated_grad(const asd_gated& p) {
  Carve c{static_cast<uint8_t*>(p.workspace)};
  GatedGradPlan r;
  r.in = plan_gated(p, &c);
  r.Np = (int)(ceil_div(p.channels, 64) * 64);
  r.Mp = ceil_div(p.rows, 64) * 64;
  r.few = pick_product(p.rows, 2 * (int64_t)p.channels, k_bytes((int64_t)p.cols * 2)) >= 3;
  r.terms = p.type == ASD_F16 ? 2 : 1;
  r.dgu = c.take((size_t)2 * p.rows * 4 * r.Np);
  r.w_t = p.dx ? c.take((size_t)2 * p.cols * r.terms * 2 * r.Np) : nullptr;
  r.dgu_t = p.dw_gate ? c.take((size_t)2 * 2 * r.Np * 2 * r.Mp) : nullptr;
  r.x_t = p.dw_gate ? c.take((size_t)2 * p.cols * r.terms * r.Mp) : nullptr;
  r.dx = p.dx ? pick_split(p.rows, p.cols, (r.terms + 1) * 4 * (int64_t)r.Np) : Split{1, 0};
  r.dw = p.dw_gate ? pick_split(2 * r.Np, p.cols, (r.terms + 1) * 2 * r.Mp) : Split{1, 0};
  const size_t dx_sums = r.dx.splits > 1 ? (size_t)r.dx.splits * p.rows * p.cols : 0,
               dw_sums = r.dw.splits > 1 ? (size_t)r.dw.splits * 2 * r.Np * p.cols : 0;
  r.part = c.take(sizeof(float) * std::max(dx_sums, dw_sums));
  r.bytes = c.used;
  return r;
}

static Transpose16 transposed(const void* src, int64_t ld, int rows, int cols, uint8_t* dst, int64_t dst_ld, int64_t lo) {
  return Transpose16{static_cast<const uint16_t*>(src), reinterpret_cast<uint16_t*>(dst), ld, dst_ld, lo, rows, cols, on16(src, ld, 2)};
}
static void add(Transposes16* all, int64_t* grid, const Transpose16& t) {
  all->first[all->n] = *grid;
  all->t[all->n++] = t;
  *grid += ceil_div(t.cols, 64) * ceil_div(t.rows, 64);
}

__global__ __launch_bounds__(256) void zero16_kernel(uint16_t* p, int64_t ld, int rows, int cols) {
  const int64_t at = workgroup() * 256 + threadIdx.x;
  if (at < (int64_t)rows * cols) p[at / cols * ld + at % cols] = 0;
}

template <class E, class T>
static asd_status run_gated_grad(const asd_gated& p, hipStream_t st) {
  const GatedGradPlan o = plan_gated_grad(p);
  ASD_HIP(bring({&o.in.x, &o.in.g, &o.in.u}, st));
  __bf16 *dgu = reinterpret_cast<__bf16*>(o.dgu), *dgu_t = reinterpret_cast<__bf16*>(o.dgu_t);
  const int Np2 = 2 * o.Np;
  const GatedGradEpi<T> e{dgu, o.Np, static_cast<const T*>(p.dh), p.ld_dh, p.channels, p.act,
                          ((uintptr_t)p.dh & 7) == 0 && (p.ld_dh & 3) == 0, o.few ? nullptr : dgu_t, o.Mp};
  ASD_HIP(launch_product<E>(gated_product(p, o.in), e, st));
  Transposes16 all{};   // (of copies, where there are any: their rows are on 16 bytes)
  int64_t grid = 0;
  const int64_t w_ld = (int64_t)o.terms * Np2, x_ld = o.terms * o.Mp, w_lo = o.terms > 1 ? Np2 : 0, x_lo = o.terms > 1 ? o.Mp : 0;
  if (p.dx) {
    add(&all, &grid, transposed(o.in.g.p, o.in.g.pitch / 2, p.channels, p.cols, o.w_t, w_ld, w_lo));
    add(&all, &grid, transposed(o.in.u.p, o.in.u.pitch / 2, p.channels, p.cols, o.w_t + 2 * (size_t)o.Np, w_ld, w_lo));
  }
  if (p.dw_gate) {
    add(&all, &grid, transposed(o.in.x.p, o.in.x.pitch / 2, p.rows, p.cols, o.x_t, x_ld, x_lo));
    for (int t = 0; o.few && t < 2; ++t)
      add(&all, &grid, transposed(dgu + t * Np2, 2 * (int64_t)Np2, p.rows, Np2, o.dgu_t + 2 * t * o.Mp, 2 * o.Mp, 0));
  }
  hipLaunchKernelGGL(transpose16_kernel, grid_of(grid), dim3(256), 0, st, all);
  ASD_HIP(hipGetLastError());
  // bytes of k of one product: 2 Np2, or 2 Mp
  const auto product = [&](const uint8_t* x, const uint8_t* w, int rows, int64_t kb) {
    RowsProduct g{x, w, nullptr, 2 * kb, o.terms * kb, 0, rows, p.cols, (o.terms + 1) * kb, nullptr};
    g.x_wrap = 2 * (uint32_t)kb;
    g.w_wrap = (uint32_t)kb;
    return g;
  };
  if (p.dx) {
    const RowsProduct g = product(o.dgu, o.w_t, p.rows, 2 * (int64_t)Np2);
    const SumEpi<T, true> s{static_cast<T*>(p.dx), nullptr, p.ld_dx, 0, p.cols, p.rows, p.rows, on16(p.dx, p.ld_dx, 2)};
    ASD_HIP(o.dx.splits > 1 ? launch_split<ElemBf16>(g, s, o.dx, o.part, st) : launch_product<ElemBf16>(g, s, st));
  }
  if (p.dw_gate) {
    const RowsProduct g = product(o.dgu_t, o.x_t, Np2, 2 * o.Mp);
    const SumEpi<T, true> s{static_cast<T*>(p.dw_gate), static_cast<T*>(p.dw_up), p.ld_dw_gate, p.ld_dw_up, p.cols, p.channels, o.Np,
                            on16(p.dw_gate, p.ld_dw_gate, 2) && on16(p.dw_up, p.ld_dw_up, 2)};
    ASD_HIP(o.dw.splits > 1 ? launch_split<ElemBf16>(g, s, o.dw, o.part, st) : launch_product<ElemBf16>(g, s, st));
  }
  return ASD_OK;
}

// ---- checks --------------------------------------------------------------------------------------------------------------------
constexpr int kMaxI8Cols = 131071;         // 2^14 times as many fits 31 bits
constexpr int kMaxCols = 1 << 20;

static asd_status check_sizes(int rows, int cols, int channels) {
  if (rows < 0 || cols < 1 || channels < 1)
    return fail(ASD_EINVAL, "rows must be >= 0, cols and channels >= 1 (got %d, %d, %d)", rows, cols, channels);
  if (rows > (1 << 28) || channels > (1 << 28)) return fail(ASD_EUNSUPPORTED, "rows and channels up to 2^28 (got %d, %d)", rows, channels);
  return ASD_OK;
}
static asd_status check_workspace(const void* ws, size_t have, size_t need) {
  if (need && (!ws || have < need || ((uintptr_t)ws & 15)))
    return fail(ASD_EINVAL, "workspace: %zu bytes at a multiple of 16 are needed", need);
  return ASD_OK;
}

static asd_status check_linear8_sizes(const asd_linear8* p) {
  if (!p) return fail(ASD_EINVAL, "arguments are NULL");
  ASD_TRY(check_sizes(p->rows, p->cols, p->channels));
  if (p->cols > kMaxI8Cols) return fail(ASD_EUNSUPPORTED, "cols > %d: a sum may leave 32 bits (got %d)", kMaxI8Cols, p->cols);
  return ASD_OK;
}
static asd_status check_linear8(const asd_linear8* p) {
  ASD_TRY(check_linear8_sizes(p));
  if (!float_type(p->out_type)) return fail(ASD_EINVAL, "unknown out_type %d", p->out_type);
  if (p->rows == 0) return ASD_OK;
  if (!p->x || !p->x_scale || !p->w || !p->w_scale || !p->out) return fail(ASD_EINVAL, "a pointer is NULL");
  const MatArg m[] = {{"out", p->out, p->rows, p->channels, p->ld_out, type_bytes(p->out_type), true},
                      {"workspace", p->workspace, p->workspace_bytes ? 1 : 0, (int64_t)p->workspace_bytes, (int64_t)p->workspace_bytes, 1, true},
                      {"x", p->x, p->rows, p->cols, p->ld_x, 1, false},
                      {"w", p->w, p->channels, p->cols, p->ld_w, 1, false},
                      {"x_scale", p->x_scale, 1, p->rows, p->rows, 4, false},
                      {"w_scale", p->w_scale, 1, p->channels, p->channels, 4, false},
                      {"bias", p->bias, 1, p->channels, p->channels, 4, false},
                      {"rows_used", p->rows_used, 1, 1, 1, 4, false}};
  ASD_TRY(check_mats(m, 8));
  return check_workspace(p->workspace, p->workspace_bytes, plan_linear8(*p, nullptr, true).bytes);
}

static asd_status check_gated_sizes(const asd_gated* p, bool backward) {
  if (!p) return fail(ASD_EINVAL, "arguments are NULL");
  ASD_TRY(check_sizes(p->rows, p->cols, p->channels));
  if (!half_type(p->type) && (backward || p->type != ASD_I8)) return fail(ASD_EINVAL, "type %d is not one of the unit's", p->type);
  if (!half_type(p->type) && p->cols > kMaxI8Cols) return fail(ASD_EUNSUPPORTED, "cols > %d: a sum may leave 32 bits (got %d)", kMaxI8Cols, p->cols);
  if (p->cols > kMaxCols) return fail(ASD_EUNSUPPORTED, "cols > %d (got %d)", kMaxCols, p->cols);
  if (backward && (p->rows > kMaxCols || p->channels > kMaxCols)) return fail(ASD_EUNSUPPORTED, "gradients: rows and channels up to %d", kMaxCols);
  return ASD_OK;
}
static asd_status check_gated(const asd_gated* p, bool backward) {
  ASD_TRY(check_gated_sizes(p, backward));
  if (p->act != ASD_ACT_SILU && p->act != ASD_ACT_GELU) return fail(ASD_EINVAL, "unknown activation %d", p->act);
  if (backward && p->rows_used) return fail(ASD_EINVAL, "gradients take no rows_used");
  if (backward && (p->dw_gate != nullptr) != (p->dw_up != nullptr)) return fail(ASD_EINVAL, "dw_gate and dw_up go together");
  if (!backward && (p->type == ASD_I8 ? !half_type(p->out_type) : p->out_type != p->type))
    return fail(ASD_EINVAL, "out_type %d does not go with type %d", p->out_type, p->type);
  if (p->rows == 0 && !backward) return ASD_OK;
  if (p->rows > 0) {
    if (!p->x || !p->w_gate || !p->w_up) return fail(ASD_EINVAL, "a pointer is NULL");
    if (!backward && !p->out) return fail(ASD_EINVAL, "out is NULL");
    if (backward && !p->dh) return fail(ASD_EINVAL, "dh is NULL");
    if (p->type == ASD_I8 && (!p->x_scale || !p->gate_scale || !p->up_scale)) return fail(ASD_EINVAL, "8-bit operands need their scales");
  }
  const int e = type_bytes(p->type), oe = backward ? e : type_bytes(p->out_type);
  const bool i8 = p->type == ASD_I8;
  const MatArg m[] = {{"out", backward ? nullptr : p->out, p->rows, p->channels, p->ld_out, oe, true},
                      {"dx", backward ? p->dx : nullptr, p->rows, p->cols, p->ld_dx, e, true},
                      {"dw_gate", backward ? p->dw_gate : nullptr, p->channels, p->cols, p->ld_dw_gate, e, true},
                      {"dw_up", backward ? p->dw_up : nullptr, p->channels, p->cols, p->ld_dw_up, e, true},
                      {"workspace", p->workspace, p->workspace_bytes ? 1 : 0, (int64_t)p->workspace_bytes, (int64_t)p->workspace_bytes, 1, true},
                      {"x", p->x, p->rows, p->cols, p->ld_x, e, false},
                      {"w_gate", p->w_gate, p->channels, p->cols, p->ld_w_gate, e, false},
                      {"w_up", p->w_up, p->channels, p->cols, p->ld_w_up, e, false},
                      {"dh", backward ? p->dh : nullptr, p->rows, p->channels, p->ld_dh, e, false},
                      {"x_scale", i8 ? p->x_scale : nullptr, 1, p->rows, p->rows, 4, false},
                      {"gate_scale", i8 ? p->gate_scale : nullptr, 1, p->channels, p->channels, 4, false},
                      {"up_scale", i8 ? p->up_scale : nullptr, 1, p->channels, p->channels, 4, false},
                      {"rows_used", p->rows_used, 1, 1, 1, 4, false}};
  ASD_TRY(check_mats(m, 13));
  if (p->rows == 0) return ASD_OK;
  asd_gated q = *p;
  q.workspace = nullptr;
  Carve c{nullptr};
  return check_workspace(p->workspace, p->workspace_bytes, backward ? plan_gated_grad(q).bytes : plan_gated(q, &c).bytes);
}

}  // namespace asd

using namespace asd;

extern "C" {

// (sizes that the call refuses need nothing: it says so itself, where an allocation for them would fail first)
size_t asd_linear_i8_workspace(const asd_linear8* p) {
  return check_linear8_sizes(p) != ASD_OK || p->rows == 0 ? 0 : plan_linear8(*p, nullptr, true).bytes;
}

asd_status asd_linear_i8(const asd_linear8* p, void* stream) {
  ASD_TRY(check_linear8(p));
  return p->rows ? launch_linear8(*p, (hipStream_t)stream, true) : ASD_OK;
}

size_t asd_gated_ff_workspace(const asd_gated* p) {
  if (check_gated_sizes(p, false) != ASD_OK || p->rows == 0) return 0;
  Carve c{nullptr};
  return plan_gated(*p, &c).bytes;
}

asd_status asd_gated_ff(const asd_gated* p, void* stream) {
  ASD_TRY(check_gated(p, false));
  return p->rows ? launch_gated(*p, (hipStream_t)stream) : ASD_OK;
}

size_t asd_gated_ff_backward_workspace(const asd_gated* p) {
  if (check_gated_sizes(p, true) != ASD_OK || p->rows == 0) return 0;
  asd_gated q = *p;
  q.workspace = nullptr;
  return plan_gated_grad(q).bytes;
}

asd_status asd_gated_ff_backward(const asd_gated* p, void* stream) {
  ASD_TRY(check_gated(p, true));
  const hipStream_t st = (hipStream_t)stream;
  if (p->rows == 0) {
    const int64_t n = (int64_t)p->channels * p->cols;
    if (p->dw_gate) {
      hipLaunchKernelGGL(zero16_kernel, grid_of(ceil_div(n, 256)), dim3(256), 0, st, static_cast<uint16_t*>(p->dw_gate), p->ld_dw_gate, p->channels, p->cols);
      hipLaunchKernelGGL(zero16_kernel, grid_of(ceil_div(n, 256)), dim3(256), 0, st, static_cast<uint16_t*>(p->dw_up), p->ld_dw_up, p->channels, p->cols);
      ASD_HIP(hipGetLastError());
    }
    return ASD_OK;
  }
  if (!p->dx && !p->dw_gate) return ASD_OK;
  return p->type == ASD_BF16 ? run_gated_grad<ElemBf16, __bf16>(*p, st) : run_gated_grad<ElemF16, _Float16>(*p, st);
}

}  // extern "C"
