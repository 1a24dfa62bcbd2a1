// A grid of n workgroups in a row, whatever n.  The threads along one dimension
// have to fit 32 bits (a launch of more runs their number modulo 2^32 and
// reports nothing), so long rows go on along y, or z.  Kernels find their place
// by row_block and return past n.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dattri {

inline hipError_t row_grid(int64_t n, dim3* grid, int threads = 256, bool along_z = false) {
  const int64_t most = ((int64_t)1 << 31) / threads;
  if (n < 1 || n > most * 65535) return hipErrorInvalidValue;
  const int64_t x = n < most ? n : most;
  grid->x = (unsigned)x;
  (along_z ? grid->z : grid->y) = (unsigned)((n + x - 1) / x);
  return hipSuccess;
}
__device__ inline int64_t row_block() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

}  // namespace dattri
