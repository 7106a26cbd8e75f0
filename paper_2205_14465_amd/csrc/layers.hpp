// layers.hpp -- arguments and launchers of the layer and optimizer kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "elem.hpp"

namespace bc {

// ------------------------------------------------------------ layer norm
struct LnForward {
    const void *x, *weight, *bias;
    void* y;
    float *mean, *rstd;
    uint64_t rows, ldx, ldy;
    uint32_t cols;
    float inv_cols, eps;
};
struct LnBackward {
    const void *dy, *x, *weight;
    const float *mean, *rstd;
    void* dx;
    float* part;            // [parts][2][cols] column sums, NULL: not wanted
    uint64_t rows, lddy, ldx, lddx;
    uint32_t cols, parts;
    float inv_cols;
};
// Workgroups that leave column sums for a call of this shape.
uint32_t ln_parts(uint64_t rows, uint32_t cols, int dtype);
hipError_t launch_ln_forward(int dtype, int wdtype, const LnForward& a, hipStream_t s);
hipError_t launch_ln_backward(int dtype, int wdtype, const LnBackward& a, void* dweight, void* dbias, hipStream_t s);
// out0[c] = sum over r of part[r * stride + c], out1 likewise of the cols
// values after them; either may be NULL.
hipError_t launch_sum_parts(int dtype, const float* part, uint32_t parts, uint64_t stride, uint32_t cols, void* out0,
                            void* out1, hipStream_t s);

}  // namespace bc
