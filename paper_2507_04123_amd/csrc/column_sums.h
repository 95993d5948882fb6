// Sums that blocks of a launch have left per column, joined by a second launch in a fixed order: what the gradients of weights end with.
#pragma once
#include "common.h"

namespace {

// The sum of N values by halves: log2(N) additions behind each, where one after the other would be up to N.
template <int N> __device__ __forceinline__ float sum_by_halves(float (&v)[N]) {
#pragma unroll
  for (int d = N / 2; d > 0; d /= 2)
#pragma unroll
    for (int i = 0; i < d; ++i) v[i] += v[i + d];
  return v[0];
}

// out[c] = factor * the sum of column c over `parts` lines of `width` values; columns go to up to three arrays, one behind the other (any may be null).
struct Columns {
  const float* parts;
  int32_t lines, width;
  float* to[3];
  int32_t end[3];                // first column behind each array's
  const float* factor;           // of the first array; null: 1
};
// 32 columns a block, 32 threads a column, each with eight loads under way (beyond the last line: of the last one again, not counted).  Added by halves:
// of 1280 lines none has more than 13 additions behind it.
__global__ void __launch_bounds__(1024) k_column_sums(const Columns a) {
  __shared__ float part[32][33];
  const int32_t col = blockIdx.x * 32 + (threadIdx.x & 31), seg = threadIdx.x >> 5;
  float s = 0.0f;
  if (col < a.width) {
    for (int32_t b = seg; b < a.lines; b += 32 * 8) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = a.parts[(int64_t)min(b + 32 * i, a.lines - 1) * a.width + col];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = b + 32 * i < a.lines ? v[i] : 0.0f;
      s += sum_by_halves(v);
    }
  }
  part[seg][threadIdx.x & 31] = s;
  __syncthreads();
  if (seg == 0 && col < a.width) {
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = part[i][threadIdx.x];
    const float all = sum_by_halves(v);
    const int which = col < a.end[0] ? 0 : col < a.end[1] ? 1 : 2;
    float* const to = which == 0 ? a.to[0] : which == 1 ? a.to[1] : a.to[2];
    const int32_t at = col - (which == 0 ? 0 : which == 1 ? a.end[0] : a.end[1]);
    if (to) to[at] = which == 0 && a.factor ? all * *a.factor : all;
  }
}
static inline void emc2_column_sums(const Columns& a, hipStream_t stream) {
  hipLaunchKernelGGL(k_column_sums, dim3((unsigned)emc2_div_up(a.width, 32)), dim3(1024), 0, stream, a);
}

}  // namespace
