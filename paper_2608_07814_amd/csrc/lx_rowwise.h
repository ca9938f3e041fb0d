// Rows of 8 values a lane, for kernels that treat each value by itself.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

namespace lx {

// f(row, distance to the next row of the U, column) for every group of 8 columns: TPR
// lanes a row, U rows under way at once; there is no division by the row length.
template <int U, class F>
__device__ __forceinline__ void for_rows(int64_t rows, int vecs, int tpr, F&& f) {
  const int lt = threadIdx.x & (tpr - 1), rpb = 256 / tpr;
  for (int64_t r = (int64_t)blockIdx.x * rpb * U + (int)threadIdx.x / tpr; r < rows; r += (int64_t)gridDim.x * rpb * U)
    for (int v = lt; v < vecs; v += tpr) f(r, rpb, v * 8);
}

// Lanes of a row for `vecs` groups of 8 values, workgroups for U rows at a time.
inline int row_lanes(int vecs) {
  int n = 1;
  while (n < vecs && n < 256) n *= 2;
  return n;
}
inline int row_grid(int64_t rows, int tpr, int U) {
  const int64_t per = 256 / tpr * U;
  return (int)std::min<int64_t>((rows + per - 1) / per, 1 << 16);
}

}  // namespace lx
