// Root-mean-square norm of rows, with a residual added on the way in and 8-bit rows with scales on the way out; the row
// quantiser on its own; and the norm's gradient.
//
//   r = x + residual,  rstd = (mean r^2 + eps)^(-1/2),  y = r rstd gain
//   8 bits: v = r gain, q = nearest integer to 127 v / max |v|, scale = max |v| rstd / 127
// rstd cancels from q: the integers depend on v alone, and a tie is a tie in exact arithmetic (v = max |v| / 2 is 63.5 steps, a
// common case with 16-bit inputs).  So the squares' sum, v and its largest are kept in 64 bits; a quotient is formed in 32 and, next
// to a border, again in 64: a multiplication by the reciprocal with one step of correction (the remainder, exact in a fused
// multiply-add, times the reciprocal) is the correctly rounded one, exact where it has to be.  The kernels are bound by memory; the
// 64-bit arithmetic of the norm, some six instructions a number at half the fp32 rate, runs under the loads of other rows, nearly
// all of it.
//
// One pass: a row lies in the registers of a wavefront (up to 1024 numbers), a workgroup of four, or of sixteen; each thread holds
// runs of eight, loaded 16 bytes at a time, or single numbers a stride apart where rows are not whole runs on 16 bytes.
#include <math.h>

#include <type_traits>

#include "ops.h"

namespace asd {

constexpr int kRun = 8;   // numbers a thread loads at once

// Numbers a thread holds of a row, in the row's own type: its c-th run of eight (WIDE: rows of whole runs on multiples of 16
// bytes), or eight single ones, `threads` apart.
template <class T>
struct __attribute__((aligned(sizeof(T) == 1 ? 8 : 16))) Run {
  T v[kRun];
};
template <bool WIDE, class T>
__device__ __forceinline__ void fetch_run(const T* row, int cols, int threads, int t, int c, Run<T>& v) {
  if constexpr (WIDE) {
    const int first = (c * threads + t) * kRun;
    if (first < cols) v = *reinterpret_cast<const Run<T>*>(row + first);
    else v = Run<T>{};
  } else {
#pragma unroll
    for (int k = 0; k < kRun; ++k) {
      const int i = (c * kRun + k) * threads + t;
      v.v[k] = i < cols ? row[i] : (T)0.f;
    }
  }
}
template <bool WIDE, class T>
__device__ __forceinline__ void store_run(T* row, int cols, int threads, int t, int c, const Run<T>& v) {
  if constexpr (WIDE) {
    const int first = (c * threads + t) * kRun;
    if (first < cols) *reinterpret_cast<Run<T>*>(row + first) = v;
  } else {
#pragma unroll
    for (int k = 0; k < kRun; ++k) {
      const int i = (c * kRun + k) * threads + t;
      if (i < cols) row[i] = v.v[k];
    }
  }
}

// The same in two steps, a load that every thread makes and, where the run is used, zeros for those behind the row's end: a load behind
// a branch was waited for there, as soon as the compiler took its numbers apart in it.  (4096 x 16384 bf16, two runs a thread, 130 ->
// 117 us.  With four runs, which spill registers anyway, more would: 795 -> 934.)
template <bool WIDE, int RUNS, class T>
__device__ __forceinline__ void fetch_ahead(const T* row, int cols, int threads, int t, int c, Run<T>& v) {
  if constexpr (WIDE && RUNS < 4) v = *reinterpret_cast<const Run<T>*>(row + min((c * threads + t) * kRun, cols - kRun));
  else fetch_run<WIDE>(row, cols, threads, t, c, v);
}
template <bool WIDE, int RUNS, class T>
__device__ __forceinline__ void end_run(int cols, int threads, int t, int c, Run<T>& v) {
  if constexpr (WIDE && RUNS < 4) {
    const bool in = (c * threads + t) * kRun < cols;
    uint32_t w[sizeof(Run<T>) / 4];
    __builtin_memcpy(w, &v, sizeof(w));
#pragma unroll
    for (uint32_t& x : w) x = in ? x : 0u;
    __builtin_memcpy(&v, w, sizeof(w));
  }
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ double wave_max64(double v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v = fmax(v, __shfl_xor(v, d));
  return v;
}

// Sums (and the largest of `top`) over the THREADS threads of a row, in every one of them.  The parts of a workgroup's wavefronts
// are added in their order.
template <int THREADS>
__device__ __forceinline__ void row_total(double& a, double& b, double& top, double (*lds)[3]) {
  a = wave_sum64(a);
  b = wave_sum64(b);
  top = wave_max64(top);
  if constexpr (THREADS > 64) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();   // (the last row's parts have been read)
    if ((threadIdx.x & 63) == 0) {
      lds[wave][0] = a;
      lds[wave][1] = b;
      lds[wave][2] = top;
    }
    __syncthreads();
    a = b = top = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
      a += lds[w][0];
      b += lds[w][1];
      top = fmax(top, lds[w][2]);
    }
  }
}

// x, residual, sum and gain of type T; out of type O (int8_t: with scales).  THREADS threads a row, RUNS runs a thread.
template <class T, class O, int THREADS, int RUNS, bool NORM, bool WIDE>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void rms_norm_kernel(asd_norm p) {
  constexpr bool I8 = sizeof(O) == 1;
  constexpr int PER_WG = THREADS < 256 ? 256 / THREADS : 1;
  __shared__ double lds[THREADS / 64][3];
  const int rows = p.rows_used ? min(max(*p.rows_used, 0), p.rows) : p.rows;
  const int t = threadIdx.x % THREADS;
  const int64_t row = workgroup() * PER_WG + (PER_WG > 1 ? (int)threadIdx.x / THREADS : 0);
  if (row >= rows) return;   // (whole workgroups, or wavefronts that wait for nobody)
  const T* x = static_cast<const T*>(p.x) + row * p.ld_x;
  const T* res = NORM && p.residual ? static_cast<const T*>(p.residual) + row * p.ld_residual : nullptr;
  const T* gain = NORM ? static_cast<const T*>(p.gain) : nullptr;
  // (the quantiser's rows stay in their own type: half the registers, twice the rows in flight; 8192 x 16384 bf16 110 -> 88 us with the
  // quotients in fp32)
  Run<typename std::conditional<NORM, float, T>::type> r[RUNS];
  Run<T> g[RUNS];
  if constexpr (!NORM) {
#pragma unroll
    for (int c = 0; c < RUNS; ++c) fetch_run<WIDE>(x, p.cols, THREADS, t, c, r[c]);
  } else {
    Run<T> a[RUNS], b[RUNS];
#pragma unroll
    for (int c = 0; c < RUNS; ++c) fetch_run<WIDE>(x, p.cols, THREADS, t, c, a[c]);
    if (res)
#pragma unroll
      for (int c = 0; c < RUNS; ++c) fetch_run<WIDE>(res, p.cols, THREADS, t, c, b[c]);
#pragma unroll
    for (int c = 0; c < RUNS; ++c) {
      if (gain) fetch_run<WIDE>(gain, p.cols, THREADS, t, c, g[c]);
      else
#pragma unroll
        for (int k = 0; k < kRun; ++k) g[c].v[k] = (T)1.f;
    }
#pragma unroll
    for (int c = 0; c < RUNS; ++c)
#pragma unroll
      for (int k = 0; k < kRun; ++k) r[c].v[k] = res ? (float)a[c].v[k] + (float)b[c].v[k] : (float)a[c].v[k];
  }
  if (NORM && p.sum) {
    T* sum = static_cast<T*>(p.sum) + row * p.ld_sum;
#pragma unroll
    for (int c = 0; c < RUNS; ++c) {
      Run<T> v;
#pragma unroll
      for (int k = 0; k < kRun; ++k) v.v[k] = (T)r[c].v[k];
      store_run<WIDE>(sum, p.cols, THREADS, t, c, v);
    }
  }
  // odd: NaN as soon as one of the row's v is not a number below infinity
  double squares = 0.0, odd = 0.0, top = 0.0;
  float odd32 = 0.f, top32 = 0.f;
#pragma unroll
  for (int c = 0; c < RUNS; ++c)
#pragma unroll
    for (int k = 0; k < kRun; ++k) {
      const double d = (double)(float)r[c].v[k];
      if constexpr (NORM) squares = fma(d, d, squares);
      if constexpr (I8 && NORM) {
        const double v = d * (double)(float)g[c].v[k];
        odd = fma(v, 0.0, odd);
        top = fmax(top, fabs(v));
      }
      if constexpr (I8 && !NORM) {
        odd32 = fmaf((float)r[c].v[k], 0.f, odd32);
        top32 = fmaxf(top32, fabsf((float)r[c].v[k]));
      }
    }
  if constexpr (I8 && !NORM) {
    odd = (double)odd32;
    top = (double)top32;
  }
  row_total<THREADS>(squares, odd, top, lds);
  const double rstd = NORM ? 1.0 / sqrt(squares / (double)p.cols + p.eps) : 1.0;
  O* out = static_cast<O*>(p.out) + row * p.ld_out;
  if constexpr (I8) {
    const bool good = odd == 0.0 && (!NORM || squares < INFINITY);
    const double inv = 1.0 / top;
    if (t == 0) p.scale[row] = !good ? __uint_as_float(0x7fc00000u) : top > 0.0 ? (float)(top * rstd / 127.0) : 0.f;
    const bool some = good && top > 0.0;
    // (127 / top may leave fp32, and so may v: such rows, of numbers next to either end of fp32's range, are done exactly throughout)
    const bool plain = top > 1e-30 && top < 1e30;
    const float fast = (float)(127.0 * inv);
#pragma unroll
    for (int c = 0; c < RUNS; ++c) {
      // In fp32 first: the quotient is off by less than 127 times a few 2^-24, 1e-4 with room to spare, so an integer is wrong
      // only if the quotient seems that near to a border; a run that holds such a number (one in eighty) is done exactly.
      Run<int8_t> q;
      float nearest = 0.f;
#pragma unroll
      for (int k = 0; k < kRun; ++k) {
        const float z = (NORM ? (float)r[c].v[k] * (float)g[c].v[k] : (float)r[c].v[k]) * fast, n = rintf(z);
        nearest = fmaxf(nearest, fabsf(z - n));
        q.v[k] = (int8_t)(int)n;
      }
      if (!plain || nearest > 0.4999f) {
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
          const double d = (double)(float)r[c].v[k], a = 127.0 * (NORM ? d * (double)(float)g[c].v[k] : d);
          const double q0 = a * inv, q1 = fma(fma(-q0, top, a), inv, q0);
          q.v[k] = (int8_t)(int)rint(q1);
        }
      }
      if (!some) q = Run<int8_t>{};
      store_run<WIDE>(out, p.cols, THREADS, t, c, q);
    }
  } else {
#pragma unroll
    for (int c = 0; c < RUNS; ++c) {
      Run<O> v;
#pragma unroll
      for (int k = 0; k < kRun; ++k) v.v[k] = (O)((float)((double)(float)r[c].v[k] * rstd) * (float)g[c].v[k]);   // (rstd alone may leave fp32)
      store_run<WIDE>(out, p.cols, THREADS, t, c, v);
    }
  }
}

// Gradient.  A workgroup (or, for short rows, a wavefront) takes every n-th row, fetching the next one while it works, and adds
// dy n up by column as it goes; the columns' parts, one row of them for each, are added in their order by the second kernel.
// n is about 1 and dx may be anything, but r, 1 / |r| and gain dy r leave 32 bits where rows are large or small (1e38, or denormal
// numbers with eps = 0).  So a row's sums are in 64 bits, and where 1 / |r| is no number of 32, r is multiplied by a power of two before,
// and dx by the same one after.  (All of it in 64 bits: 8191 x 4104 bf16 69 us for 56.)
template <class T, int THREADS, int RUNS, bool WIDE>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void rms_norm_grad_kernel(asd_norm_grad p, float* parts) {
  constexpr int PER_WG = THREADS < 256 ? 256 / THREADS : 1;
  constexpr bool AHEAD = RUNS * (int)sizeof(T) <= (THREADS == 1024 ? 2 : 6);   // (where registers last)
  __shared__ double lds[2][THREADS / 64][2];
  const int t = threadIdx.x % THREADS, lane_row = PER_WG > 1 ? (int)threadIdx.x / THREADS : 0;
  const int part = (int)blockIdx.x * PER_WG + lane_row, n_parts = (int)gridDim.x * PER_WG;
  Run<T> g[RUNS], r[RUNS], dy[RUNS];
  Run<float> dg[RUNS];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int c = 0; c < RUNS; ++c) {
      fetch_ahead<WIDE, RUNS>(static_cast<const T*>(p.sum) + row * p.ld_sum, p.cols, THREADS, t, c, r[c]);
      fetch_ahead<WIDE, RUNS>(static_cast<const T*>(p.dy) + row * p.ld_dy, p.cols, THREADS, t, c, dy[c]);
    }
  };
  if (AHEAD && part < p.rows) fetch(part);
#pragma unroll
  for (int c = 0; c < RUNS; ++c) {
    if (p.gain) fetch_run<WIDE>(static_cast<const T*>(p.gain), p.cols, THREADS, t, c, g[c]);
#pragma unroll
    for (int k = 0; k < kRun; ++k) {
      if (!p.gain) g[c].v[k] = (T)1.f;
      dg[c].v[k] = 0.f;
    }
  }
  int turn = 0;
  for (int64_t row = part; row < p.rows; row += n_parts) {
    Run<T> rn[RUNS], dyn[RUNS], ds[RUNS];
    if (!AHEAD) fetch(row);
#pragma unroll
    for (int c = 0; c < RUNS; ++c) {
      rn[c] = r[c];
      dyn[c] = dy[c];
      end_run<WIDE, RUNS>(p.cols, THREADS, t, c, rn[c]);
      end_run<WIDE, RUNS>(p.cols, THREADS, t, c, dyn[c]);
    }
    if (p.dx && p.dsum)
#pragma unroll
      for (int c = 0; c < RUNS; ++c) fetch_ahead<WIDE, RUNS>(static_cast<const T*>(p.dsum) + row * p.ld_dsum, p.cols, THREADS, t, c, ds[c]);
    if (AHEAD && row + n_parts < p.rows) fetch(row + n_parts);
    double squares = 0.0, along = 0.0;
#pragma unroll
    for (int c = 0; c < RUNS; ++c)
#pragma unroll
      for (int k = 0; k < kRun; ++k) {
        const double d = (double)(float)rn[c].v[k];
        squares = fma(d, d, squares);
        along = fma((double)((float)g[c].v[k] * (float)dyn[c].v[k]), d, along);
      }
    squares = wave_sum64(squares);
    along = wave_sum64(along);
    if constexpr (THREADS > 64) {   // (two sets in turn: one barrier a row)
      if ((threadIdx.x & 63) == 0) {
        lds[turn][threadIdx.x >> 6][0] = squares;
        lds[turn][threadIdx.x >> 6][1] = along;
      }
      __syncthreads();
      squares = along = 0.0;
#pragma unroll
      for (int w = 0; w < THREADS / 64; ++w) {
        squares += lds[turn][w][0];
        along += lds[turn][w][1];
      }
      turn ^= 1;
    }
    const double rs = 1.0 / sqrt(squares / (double)p.cols + p.eps);
    const float mean = (float)(along * rs / (double)p.cols);
    // (an fp16 row is at least 2^-24 long, or none)
    const float two = std::is_same<T, _Float16>::value || (rs > 0x1p-125 && rs < 0x1p125) ? 1.f : rs > 1.0 ? 0x1p64f : 0x1p-64f;
    const float rstd = (float)(rs / (double)two);
#pragma unroll
    for (int c = 0; c < RUNS; ++c) {
      Run<T> v;
#pragma unroll
      for (int k = 0; k < kRun; ++k) {
        const float n = (float)rn[c].v[k] * two * rstd, y = (float)dyn[c].v[k];
        const float d = rstd * ((float)g[c].v[k] * y - n * mean);
        v.v[k] = (T)fmaf(d, two, p.dsum ? (float)ds[c].v[k] : -0.f);
        dg[c].v[k] = fmaf(y, n, dg[c].v[k]);
      }
      if (p.dx) store_run<WIDE>(static_cast<T*>(p.dx) + row * p.ld_dx, p.cols, THREADS, t, c, v);
    }
  }
  if (parts)
#pragma unroll
    for (int c = 0; c < RUNS; ++c) store_run<WIDE>(parts + (int64_t)part * p.cols, p.cols, THREADS, t, c, dg[c]);
}

// dgain: 64 columns a workgroup, its sixteen wavefronts take every sixteenth part, in order.
template <class T>
__global__ __launch_bounds__(1024) void norm_gain_grad_kernel(int cols, int n_parts, const float* __restrict__ parts, T* __restrict__ dgain) {
  __shared__ float lds[16][64];
  const int lane = threadIdx.x & 63, col = blockIdx.x * 64 + lane, wave = threadIdx.x >> 6;
  float s = 0.f;
  if (col < cols)
#pragma unroll 8
    for (int i = wave; i < n_parts; i += 16) s += parts[(int64_t)i * cols + col];
  lds[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && col < cols) {
    s = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += lds[w][lane];
    dgain[col] = (T)s;
  }
}

// f(threads, runs) as constants for rows of `cols`: a wavefront a row up to 1024 numbers, four up to 6144, sixteen from there.  Few
// runs a thread leave registers for more rows in flight: 16384 rows of 8192 bf16 numbers with a residual into integers 257 us with
// four runs in four wavefronts, 233 with one in sixteen.
// The quantiser (LEAN), whose rows take half the registers: four wavefronts up to 16384.
template <bool LEAN, class F>
static asd_status by_width(int cols, F f) {
  typedef std::integral_constant<int, 64> W1;
  typedef std::integral_constant<int, 256> W4;
  typedef std::integral_constant<int, 1024> W16;
  const auto runs = [&](int threads) { return (int)ceil_div(cols, threads * kRun); };
  if (runs(64) <= 1) return f(W1(), std::integral_constant<int, 1>());
  if (runs(64) <= 2) return f(W1(), std::integral_constant<int, 2>());
  if (runs(256) <= 1) return f(W4(), std::integral_constant<int, 1>());
  if (runs(256) <= 2) return f(W4(), std::integral_constant<int, 2>());
  if constexpr (LEAN) {
    if (runs(256) <= 4) return f(W4(), std::integral_constant<int, 4>());
    if (runs(256) <= 8) return f(W4(), std::integral_constant<int, 8>());
    return f(W16(), std::integral_constant<int, 4>());
  }
  if (runs(256) <= 3) return f(W4(), std::integral_constant<int, 3>());
  if (runs(1024) <= 1) return f(W16(), std::integral_constant<int, 1>());
  if (runs(1024) <= 2) return f(W16(), std::integral_constant<int, 2>());
  return f(W16(), std::integral_constant<int, 4>());
}

constexpr int kMaxNormCols = 32768;

template <class T, class O, bool NORM>
static asd_status run_norm(const asd_norm& p, hipStream_t st) {
  bool wide = p.cols % kRun == 0 && on16(p.x, p.ld_x, sizeof(T)) && ((uintptr_t)p.out & 15) == 0 && p.ld_out % kRun == 0;
  if (NORM)
    wide = wide && (!p.residual || on16(p.residual, p.ld_residual, sizeof(T))) && (!p.sum || on16(p.sum, p.ld_sum, sizeof(T))) &&
           ((uintptr_t)p.gain & 15) == 0;
  return by_width<!NORM && sizeof(T) == 2>(p.cols, [&](auto threads, auto runs) -> asd_status {
    constexpr int TH = decltype(threads)::value, R = decltype(runs)::value, PER = TH < 256 ? 256 / TH : 1;
    const dim3 grid = grid_of(ceil_div(p.rows, PER)), block(TH * PER);
    if (wide) hipLaunchKernelGGL((rms_norm_kernel<T, O, TH, R, NORM, true>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((rms_norm_kernel<T, O, TH, R, NORM, false>), grid, block, 0, st, p);
    ASD_HIP(hipGetLastError());
    return ASD_OK;
  });
}

template <class T>
static asd_status run_norm_to(const asd_norm& p, hipStream_t st) {
  switch (p.out_type) {
    case ASD_F32: return run_norm<T, float, true>(p, st);
    case ASD_BF16: return run_norm<T, __bf16, true>(p, st);
    case ASD_F16: return run_norm<T, _Float16, true>(p, st);
    default: return run_norm<T, int8_t, true>(p, st);
  }
}

asd_status launch_rms_norm(const asd_norm& p, hipStream_t st) {
  return p.type == ASD_F32 ? run_norm_to<float>(p, st) : p.type == ASD_BF16 ? run_norm_to<__bf16>(p, st) : run_norm_to<_Float16>(p, st);
}

asd_status launch_quantize_rows(const asd_norm& p, hipStream_t st) {
  return p.type == ASD_F32    ? run_norm<float, int8_t, false>(p, st)
         : p.type == ASD_BF16 ? run_norm<__bf16, int8_t, false>(p, st)
                              : run_norm<_Float16, int8_t, false>(p, st);
}

static asd_status check_norm_sizes(int rows, int cols, int type) {
  if (rows < 0 || cols < 1) return fail(ASD_EINVAL, "rows must be >= 0 and cols >= 1 (got %d, %d)", rows, cols);
  if (!float_type(type)) return fail(ASD_EINVAL, "type %d is not a number type", type);
  if (cols > kMaxNormCols) return fail(ASD_EUNSUPPORTED, "cols > %d (got %d)", kMaxNormCols, cols);
  return ASD_OK;
}

static asd_status check_norm(const asd_norm* p, bool norm) {
  if (!p) return fail(ASD_EINVAL, "arguments are NULL");
  ASD_TRY(check_norm_sizes(p->rows, p->cols, p->type));
  const int out_type = norm ? p->out_type : ASD_I8;
  if (!float_type(out_type) && out_type != ASD_I8) return fail(ASD_EINVAL, "unknown out_type %d", out_type);
  if (norm && !(p->eps >= 0.0 && p->eps < INFINITY)) return fail(ASD_EINVAL, "eps must be finite and >= 0");
  if (p->rows == 0) return ASD_OK;
  if (!p->x || !p->out) return fail(ASD_EINVAL, "%s is NULL", !p->x ? "x" : "out");
  if (out_type == ASD_I8 && !p->scale) return fail(ASD_EINVAL, "8-bit rows need scale");
  const int e = type_bytes(p->type);
  const MatArg m[] = {{"sum", norm ? p->sum : nullptr, p->rows, p->cols, p->ld_sum, e, true},
                      {"out", p->out, p->rows, p->cols, p->ld_out, type_bytes(out_type), true},
                      {"scale", out_type == ASD_I8 ? p->scale : nullptr, 1, p->rows, p->rows, 4, true},
                      {"x", p->x, p->rows, p->cols, p->ld_x, e, false},
                      {"residual", norm ? p->residual : nullptr, p->rows, p->cols, p->ld_residual, e, false},
                      {"gain", norm ? p->gain : nullptr, 1, p->cols, p->cols, e, false},
                      {"rows_used", p->rows_used, 1, 1, 1, 4, false}};
  return check_mats(m, 7, [](int i, int j) { return i == 0 && (j == 3 || j == 4); });
}

// Parts of dgain: as many workgroups as are on the chip at a time (two a CU), where each gets eight rows at least.
static int norm_grad_wgs(int rows, int cols) {
  const int per_wg = cols <= 2 * 64 * kRun ? 4 : 1;   // rows a workgroup takes at a time (by_width)
  return (int)std::max<int64_t>(1, std::min<int64_t>(512, ceil_div(rows, 8 * per_wg)));
}
static int norm_grad_parts(int rows, int cols) { return norm_grad_wgs(rows, cols) * (cols <= 2 * 64 * kRun ? 4 : 1); }

template <class T>
static asd_status run_norm_grad(const asd_norm_grad& p, hipStream_t st) {
  const bool wide = p.cols % kRun == 0 && on16(p.dy, p.ld_dy, sizeof(T)) && on16(p.sum, p.ld_sum, sizeof(T)) && (!p.gain || ((uintptr_t)p.gain & 15) == 0) &&
             (!p.dsum || on16(p.dsum, p.ld_dsum, sizeof(T))) && (!p.dx || on16(p.dx, p.ld_dx, sizeof(T)));
  float* parts = p.dgain ? static_cast<float*>(p.workspace) : nullptr;
  if (p.rows > 0) {
    ASD_TRY(by_width<false>(p.cols, [&](auto threads, auto runs) -> asd_status {
      constexpr int TH = decltype(threads)::value, R = decltype(runs)::value, PER = TH < 256 ? 256 / TH : 1;
      const dim3 grid((unsigned)norm_grad_wgs(p.rows, p.cols)), block(TH * PER);
      if (wide) hipLaunchKernelGGL((rms_norm_grad_kernel<T, TH, R, true>), grid, block, 0, st, p, parts);
      else hipLaunchKernelGGL((rms_norm_grad_kernel<T, TH, R, false>), grid, block, 0, st, p, parts);
      ASD_HIP(hipGetLastError());
      return ASD_OK;
    }));
  }
  if (p.dgain) {
    hipLaunchKernelGGL((norm_gain_grad_kernel<T>), dim3((unsigned)ceil_div(p.cols, 64)), dim3(1024), 0, st, p.cols,
                       p.rows > 0 ? norm_grad_parts(p.rows, p.cols) : 0, parts, static_cast<T*>(p.dgain));
    ASD_HIP(hipGetLastError());
  }
  return ASD_OK;
}

}  // namespace asd

using namespace asd;

extern "C" {

asd_status asd_rms_norm(const asd_norm* p, void* stream) {
  ASD_TRY(check_norm(p, true));
  return p->rows ? launch_rms_norm(*p, (hipStream_t)stream) : ASD_OK;
}

asd_status asd_quantize_rows(const asd_norm* p, void* stream) {
  ASD_TRY(check_norm(p, false));
  return p->rows ? launch_quantize_rows(*p, (hipStream_t)stream) : ASD_OK;
}

size_t asd_rms_norm_backward_workspace(const asd_norm_grad* p) {
  if (!p || !p->dgain || check_norm_sizes(p->rows, p->cols, p->type) != ASD_OK || p->rows == 0) return 0;
  return sizeof(float) * (size_t)norm_grad_parts(p->rows, p->cols) * (size_t)p->cols;
}

asd_status asd_rms_norm_backward(const asd_norm_grad* p, void* stream) {
  if (!p) return fail(ASD_EINVAL, "arguments are NULL");
  ASD_TRY(check_norm_sizes(p->rows, p->cols, p->type));
  if (!(p->eps >= 0.0 && p->eps < INFINITY)) return fail(ASD_EINVAL, "eps must be finite and >= 0");
  if (p->rows > 0 && (!p->dy || !p->sum)) return fail(ASD_EINVAL, "%s is NULL", !p->dy ? "dy" : "sum");
  const int e = type_bytes(p->type);
  const MatArg m[] = {{"dx", p->dx, p->rows, p->cols, p->ld_dx, e, true},
                      {"dgain", p->dgain, 1, p->cols, p->cols, e, true},
                      {"workspace", p->workspace, p->workspace && p->workspace_bytes ? 1 : 0, (int64_t)p->workspace_bytes, (int64_t)p->workspace_bytes, 1, true},
                      {"dy", p->dy, p->rows, p->cols, p->ld_dy, e, false},
                      {"sum", p->sum, p->rows, p->cols, p->ld_sum, e, false},
                      {"gain", p->gain, 1, p->cols, p->cols, e, false},
                      {"dsum", p->dsum, p->rows, p->cols, p->ld_dsum, e, false}};
  ASD_TRY(check_mats(m, 7, [](int i, int j) { return i == 0 && (j == 3 || j == 6); }));
  const size_t need = asd_rms_norm_backward_workspace(p);
  if (need && (!p->workspace || p->workspace_bytes < need || ((uintptr_t)p->workspace & 15)))
    return fail(ASD_EINVAL, "workspace: %zu bytes at a multiple of 16 are needed", need);
  const hipStream_t st = (hipStream_t)stream;
  return p->type == ASD_F32 ? run_norm_grad<float>(*p, st) : p->type == ASD_BF16 ? run_norm_grad<__bf16>(*p, st) : run_norm_grad<_Float16>(*p, st);
}

}  // extern "C"
