#pragma once

#include <hip/hip_runtime.h>

namespace ax {

// out[c] = sum over r of part[r * cols + c], in a fixed order (zeros for no rows).
hipError_t launch_column_sum(const float* part, int rows, int cols, float* out, hipStream_t s);

}  // namespace ax
