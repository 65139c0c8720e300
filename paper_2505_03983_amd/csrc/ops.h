// Shared by the operators' C entries (ops_norm.hip, ops_gemm.hip): argument checks and element types.
#pragma once
#include "common.h"

namespace asd {

inline int type_bytes(int t) { return t == ASD_F32 ? 4 : t == ASD_BF16 || t == ASD_F16 ? 2 : t == ASD_I8 ? 1 : 0; }
inline bool float_type(int t) { return t == ASD_F32 || t == ASD_BF16 || t == ASD_F16; }
inline bool half_type(int t) { return t == ASD_BF16 || t == ASD_F16; }

// A matrix argument: `rows` rows of `cols` elements of `bytes`, `ld` elements apart.
struct MatArg {
  const char* name;
  const void* p;
  int64_t rows, cols, ld;
  int bytes;
  bool out;
  const char* begin() const { return static_cast<const char*>(p); }
  const char* end() const { return begin() + ((rows - 1) * ld + cols) * bytes; }
  // no byte of the two is the same: one behind the other, or rows of one pitch between each other's (columns of one wider matrix)
  bool apart(const MatArg& o) const {
    if (begin() >= o.end() || o.begin() >= end()) return true;
    const int64_t pitch = ld * bytes;
    if (rows < 2 || o.rows < 2 || pitch != o.ld * o.bytes) return false;
    const int64_t at = ((o.begin() - begin()) % pitch + pitch) % pitch;   // where its rows start in this one's
    return at >= cols * bytes && at + o.cols * o.bytes <= pitch;
  }
};

// Pitches, alignment and overlaps of a call's matrices (NULL ones are left out).  may_share(a, b): an output and an input that
// may be the same array.
template <class Share>
inline asd_status check_mats(const MatArg* m, int n, Share may_share) {
  for (int i = 0; i < n; ++i) {
    if (!m[i].p || m[i].rows < 1) continue;
    if (m[i].ld < m[i].cols) return fail(ASD_EINVAL, "ld of %s is below its row length", m[i].name);
    if (m[i].rows > 1 && m[i].ld > ((int64_t)1 << 40) / m[i].rows) return fail(ASD_EINVAL, "ld of %s is out of range", m[i].name);
    if ((uintptr_t)m[i].p % m[i].bytes) return fail(ASD_EINVAL, "%s is not aligned to its elements", m[i].name);
  }
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < n; ++j) {
      if (i == j || !m[i].out || !m[i].p || !m[j].p || m[i].rows < 1 || m[j].rows < 1 || (m[j].out && j < i)) continue;
      if (m[i].apart(m[j])) continue;
      if (may_share(i, j) && m[i].p == m[j].p && (m[i].ld == m[j].ld || m[i].rows == 1)) continue;
      return fail(ASD_EINVAL, "%s overlaps %s", m[i].name, m[j].name);
    }
  return ASD_OK;
}
inline asd_status check_mats(const MatArg* m, int n) {
  return check_mats(m, n, [](int, int) { return false; });
}

// Rows at any 16 bytes: what the wide loads and stores ask for.
inline bool on16(const void* p, int64_t ld, int bytes) { return ((uintptr_t)p & 15) == 0 && (ld * bytes & 15) == 0; }

// n workgroups as a grid (a dimension times its threads stays below 2^32), and a workgroup's number in it.
inline dim3 grid_of(int64_t n) {
  const int64_t x = n < 65536 ? n : 65536;
  return dim3((unsigned)x, (unsigned)((n + x - 1) / x));
}
__device__ __forceinline__ int64_t workgroup() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// For the library's own launches: the operators without their argument checks.
asd_status launch_rms_norm(const asd_norm& p, hipStream_t st);
asd_status launch_quantize_rows(const asd_norm& p, hipStream_t st);
// likely: rows to expect, where the device knows their number (0: all): which tile suits, no bit of the results
// split: the workspace has room for partial sums, where few tiles have long ones
asd_status launch_linear8(const asd_linear8& p, hipStream_t st, bool split, int likely = 0);
asd_status launch_gated(const asd_gated& p, hipStream_t st, int likely = 0);
// out[m][n] = sum over k of x[m][k] w[n][k]: bf16 rows of whole 16 bytes, side by side, fp32 results
asd_status launch_linear_bf16(const void* x, const void* w, float* out, int rows, int cols, int channels, const int32_t* rows_used,
                              hipStream_t st, int likely);
// Microseconds of a product of `rows` rows with `channels` channels (both matrices' of a gated one) of kb bytes, on the kernel picked
// for `most` rows; and the number, below 8, of the kernel that a call of up to `most` rows takes where `rows` are likely.
double product_us(int rows, int most, int64_t channels, int64_t kb);
int product_pick(int rows, int most, int64_t channels, int64_t kb);

}  // namespace asd
