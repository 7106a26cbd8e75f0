// api_layers.hip -- the C ABI of the layer and optimizer operators
// (include/bytecomp.h): argument checks on the host, workspace carving, and
// the launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "../../include/bytecomp.h"
#include "launch.hpp"
#include "layers.hpp"

using namespace bc;

namespace {

constexpr uint64_t kMaxRows = 1ull << 31;

int status_of(hipError_t e) { return e == hipSuccess ? BC_OK : BC_E_HIP; }

// Whether p violates the alignment of `dtype`'s elements.
bool misaligned(const void* p, int dtype) { return ((uintptr_t)p & (dtype_bytes(dtype) - 1)) != 0; }

int check_layernorm(int dtype, int wdtype, uint64_t rows, uint64_t cols) {
    if (!dtype_ok(dtype) || (wdtype != dtype && wdtype != BC_F32)) return BC_E_DTYPE;
    if (rows >= kMaxRows || cols >= (1ull << 24)) return BC_E_SIZE;
    return BC_OK;
}

size_t layernorm_ws(uint64_t rows, uint64_t cols) {
    const uint32_t a = ln_parts(rows, (uint32_t)cols, BC_F32), b = ln_parts(rows, (uint32_t)cols, BC_F16);
    return (size_t)(a > b ? a : b) * 2 * cols * sizeof(float);
}

}  // namespace

extern "C" {

int bytecomp_layernorm_forward(int dtype, int wdtype, uint64_t rows, uint64_t cols, const void* x, uint64_t ldx,
                               const void* weight, const void* bias, double eps, void* y, uint64_t ldy, float* mean,
                               float* rstd, void* stream) {
    const CallRange range("bytecomp_layernorm_forward");
    if (const int rc = check_layernorm(dtype, wdtype, rows, cols)) return rc;
    if (!(eps >= 0.0) || std::isinf(eps)) return BC_E_VALUE;
    if (rows == 0 || cols == 0) return BC_OK;
    if (!x || !y) return BC_E_NULL;
    if (ldx < cols || ldy < cols) return BC_E_SIZE;
    if (misaligned(x, dtype) || misaligned(y, dtype) || misaligned(weight, wdtype) || misaligned(bias, wdtype) ||
        misaligned(mean, BC_F32) || misaligned(rstd, BC_F32))
        return BC_E_ALIGN;
    const LnForward a{x, weight, bias, y, mean, rstd, rows, ldx, ldy, (uint32_t)cols, (float)(1.0 / (double)cols),
                      (float)eps};
    hipStream_t s = (hipStream_t)stream;
    return finish_call(status_of(launch_ln_forward(dtype, wdtype, a, s)), s, nullptr);
}

int bytecomp_layernorm_workspace_size(uint64_t rows, uint64_t cols, size_t* bytes) {
    if (!bytes) return BC_E_NULL;
    if (const int rc = check_layernorm(BC_F32, BC_F32, rows, cols)) return rc;
    *bytes = layernorm_ws(rows, cols);
    return BC_OK;
}

int bytecomp_layernorm_backward(int dtype, int wdtype, uint64_t rows, uint64_t cols, const void* dy, uint64_t lddy,
                                const void* x, uint64_t ldx, const void* weight, const float* mean, const float* rstd,
                                void* dx, uint64_t lddx, void* dweight, void* dbias, void* ws, size_t ws_bytes,
                                void* stream) {
    const CallRange range("bytecomp_layernorm_backward");
    if (const int rc = check_layernorm(dtype, wdtype, rows, cols)) return rc;
    if (cols == 0 || (!dx && !dweight && !dbias)) return BC_OK;
    if (rows > 0 && (!dy || !x || !mean || !rstd)) return BC_E_NULL;
    if (lddy < cols || ldx < cols || (dx && lddx < cols)) return BC_E_SIZE;
    if (misaligned(dy, dtype) || misaligned(x, dtype) || misaligned(weight, wdtype) || misaligned(dx, dtype) ||
        misaligned(mean, BC_F32) || misaligned(rstd, BC_F32) || misaligned(dweight, wdtype) ||
        misaligned(dbias, wdtype) || misaligned(ws, BC_F32))
        return BC_E_ALIGN;
    const bool sums = dweight || dbias;
    if (sums && rows > 0 && (!ws || ws_bytes < layernorm_ws(rows, cols))) return BC_E_WORKSPACE;
    const LnBackward a{dy, x, weight, mean, rstd, dx, sums ? (float*)ws : nullptr, rows, lddy, ldx, lddx,
                       (uint32_t)cols, ln_parts(rows, (uint32_t)cols, dtype), (float)(1.0 / (double)cols)};
    hipStream_t s = (hipStream_t)stream;
    return finish_call(status_of(launch_ln_backward(dtype, wdtype, a, dweight, dbias, s)), s, nullptr);
}

}  // extern "C"
