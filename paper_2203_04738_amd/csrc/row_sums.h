// Sums of the rows of an array of floats, column by column: what workgroups left of the gradients of parameters.
#pragma once
#include <hip/hip_runtime.h>

namespace mg {

// A workgroup has SUM_COLS columns side by side and goes through the rows in SUM_PARTS parts.
constexpr int SUM_COLS = 32, SUM_PARTS = 16, SUM_THREADS = SUM_COLS * SUM_PARTS;
inline unsigned sum_groups(long long columns) { return (unsigned)((columns + SUM_COLS - 1) / SUM_COLS); }

__device__ inline long long sum_column() { return (long long)blockIdx.x * SUM_COLS + threadIdx.x % SUM_COLS; }
// The sum of a column's n rows, `stride` apart, in the same order in every run; true in the thread that has it.  Every
// thread of the workgroup calls it.
__device__ inline bool sum_rows(const float* column, long long stride, long long n, bool exists, float& sum) {
  __shared__ float part[SUM_PARTS][SUM_COLS];
  const int col = threadIdx.x % SUM_COLS, k = threadIdx.x / SUM_COLS;
  const long long per = (n + SUM_PARTS - 1) / SUM_PARTS, from = k * per, to = from + per < n ? from + per : n;
  float v = 0.f;
  if (exists) {
    const float* p = column + from * stride;
#pragma unroll 8
    for (long long i = from; i < to; ++i, p += stride) v += *p;
  }
  part[k][col] = v;
  __syncthreads();
  if (k || !exists) return false;
  sum = part[0][col];
#pragma unroll
  for (int i = 1; i < SUM_PARTS; ++i) sum += part[i][col];
  return true;
}

}  // namespace mg
