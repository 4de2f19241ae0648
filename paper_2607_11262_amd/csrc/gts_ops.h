// gts_ops.h — what the operators' host checks and kernels share: the launch
// functions, and the device helpers for 16-byte loads, grids and division by a
// number known at launch.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/gts.h"
#include "../../include/gts_ops.h"

namespace gts {

constexpr uint32_t kTableFreqs = GTS_OPS_MAX_DIM / 2;
struct TableFreqs {
  double f[kTableFreqs];
};

hipError_t launch_rotary(const gts_rotary_args& a, hipStream_t stream);
hipError_t launch_rotary_table(float* table, uint32_t n_positions, uint32_t rot_dim, const TableFreqs& f, double scale,
                               hipStream_t stream);
hipError_t launch_append(const gts_append_args& a, hipStream_t stream);
hipError_t launch_attention(const gts_attention_args& a, hipStream_t stream);
uint64_t attention_scratch(uint32_t batch, uint32_t tokens, uint32_t q_heads, uint32_t kv_heads, uint32_t dim);

#ifdef __HIPCC__
// A launch has less than 2^32 threads in each dimension: workgroups of 256 past
// 2^23 go on in further rows of the grid (the last row may pass their number).
constexpr uint32_t kGridRow = 1u << 23;
constexpr uint64_t kMostBlocks = (uint64_t)kGridRow * 65535;
inline dim3 grid_of(uint64_t blocks) {
  return blocks <= kGridRow ? dim3((uint32_t)blocks) : dim3(kGridRow, (uint32_t)((blocks + kGridRow - 1) / kGridRow));
}
__device__ __forceinline__ uint64_t block_number() { return (uint64_t)blockIdx.y * kGridRow + blockIdx.x; }

// n / d for n < 2^31 and 1 <= d < 2^31: one multiplication high and a shift
// (m = ceil(2^(32 + s) / d) - 2^32 with 2^s >= d; the sum with n keeps the
// 33rd bit of the multiplier).
struct FastDiv {
  uint32_t d, m, s;
  FastDiv() = default;
  explicit FastDiv(uint32_t div) : d(div) {
    s = 0;
    while ((1ull << s) < div) ++s;
    m = (uint32_t)(((1ull << 32) * ((1ull << s) - div)) / div + 1);
  }
  __device__ __forceinline__ uint32_t div(uint32_t n) const { return (uint32_t)(((uint64_t)__umulhi(n, m) + n) >> s); }
};

// N values of T that are loaded and stored as one access (N * sizeof(T) <= 16
// bytes, aligned to that).
template <typename T, int N>
struct alignas(N * sizeof(T)) Pack {
  T v[N];
};

// The sequence of new token t and its number within it; false when no
// sequence has it.  Every lane of a wave calls it with the same t: 64 bounds
// are compared at once, so 4096 sequences take two loads in a row.
__device__ __forceinline__ bool find_sequence(const gts_kv_batch& b, uint32_t t, uint32_t* seq, uint32_t* index,
                                              uint32_t* count) {
  if (!b.starts) {
    const uint32_t n = b.tokens / b.batch;
    *seq = t / n;
    *index = t - *seq * n;
    *count = n;
    return true;
  }
  const uint32_t lane = threadIdx.x & 63u;
  // largest lo in [0, batch] with starts[lo] <= t (0 if there is none)
  uint32_t lo = 0, n = b.batch + 1;
  while (n > 1) {
    const uint32_t step = (n + 63u) / 64u;
    const uint32_t at = lane * step;
    const bool le = at < n && (lane == 0 || b.starts[lo + at] <= (int32_t)t);
    const uint64_t m = __ballot(le);
    const uint32_t last = 63u - (uint32_t)__builtin_clzll(m);
    lo += last * step;
    n = n - last * step < step ? n - last * step : step;
  }
  if (lo >= b.batch) return false;
  const int32_t s0 = b.starts[lo], s1 = b.starts[lo + 1];
  if (s0 < 0 || s0 > (int32_t)t || s1 <= (int32_t)t || (uint32_t)s1 > b.tokens) return false;
  *seq = lo;
  *index = t - (uint32_t)s0;
  *count = (uint32_t)(s1 - s0);
  return true;
}
#endif

}  // namespace gts
