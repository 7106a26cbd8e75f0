// act.hpp -- what the products of the linear layers share beside their tiles:
// activations with their slopes, and fp32 as planes of bfloat16.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "elem.hpp"

namespace bc {

// ------------------------------------------------------------- activations
// Both in fp32; `exact` keeps fp32's last places (fp32 tensors), otherwise the
// hardware's exponential and reciprocal do.  The hardware's exponential takes its
// argument t times log2(e), rounded to fp32: up to about |t| 2^-24 of its value off
// (2^-19 at t = 30), still far below a unit of fp16 or bfloat16.  dbias in fp32
// carries it, which sums what was never rounded to them.
constexpr float kSqrtHalf = 0.70710678118654752f;
constexpr float kTanhScale = 0.79788456080286536f;      // sqrt(2 / pi)
constexpr float kTanhCubic = 0.044715f;

// 1 / (1 + exp(-t))
template <bool exact>
__device__ __forceinline__ float logistic(float t) {
    if constexpr (exact) return 1.0f / (1.0f + expf(-t));
    else return __builtin_amdgcn_rcpf(1.0f + __expf(-t));
}

template <bool exact>
__device__ __forceinline__ float activate(int act, float z) {
    switch (act) {
        case BC_ACT_RELU: return z < 0.0f ? 0.0f : z;  // NaN stays
        case BC_ACT_GELU: return 0.5f * z * erfcf(-z * kSqrtHalf);
        // 0.5 (1 + tanh t) is the logistic function of 2 t
        case BC_ACT_GELU_TANH: return z * logistic<exact>(2.0f * kTanhScale * (z + kTanhCubic * z * z * z));
        case BC_ACT_SILU: return z * logistic<exact>(z);
        default: return z;
    }
}

template <bool exact>
__device__ __forceinline__ float act_slope(int act, float z) {
    switch (act) {
        case BC_ACT_RELU: return z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z;
        case BC_ACT_GELU:
            return 0.5f * erfcf(-z * kSqrtHalf) +
                   z * (0.5f * kTanhScale) * (exact ? expf(-0.5f * z * z) : __expf(-0.5f * z * z));
        case BC_ACT_GELU_TANH: {
            const float p = logistic<exact>(2.0f * kTanhScale * (z + kTanhCubic * z * z * z));
            // (where z z would pass fp32's range p (1 - p) has long been 0)
            return p + z * p * (1.0f - p) * (2.0f * kTanhScale) * (1.0f + 3.0f * kTanhCubic * fminf(z * z, 1e30f));
        }
        case BC_ACT_SILU: {
            const float p = logistic<exact>(z);
            return p + z * p * (1.0f - p);
        }
        default: return 1.0f;
    }
}

// ------------------------------------------------------------------- planes
template <typename T>
struct PlaneOf {
    typedef T type;
    static constexpr int P = 1;
};
template <>
struct PlaneOf<float> {
    typedef bf16_t type;
    static constexpr int P = 3;
};

// v rounded to a plane's type, toward zero where the nearest is an infinity (fp32
// numbers past bfloat16's largest: the next planes hold what is left of them).
template <typename E>
__device__ __forceinline__ E lead(float v) {
    if constexpr (__is_same(E, bf16_t)) {
        const uint32_t bits = __float_as_uint(v);
        if ((bits & 0x7fffffffu) - 0x7f7f8000u < 0x8000u) v = __uint_as_float(bits & 0xffff0000u);
    }
    return (E)v;
}

// v as P planes of eight elements at p, p + plane, ...
template <typename T>
__device__ __forceinline__ void store_planes(typename PlaneOf<T>::type* p, uint64_t plane, const float (&v)[8]) {
    typedef typename PlaneOf<T>::type E;
    typedef E vec __attribute__((ext_vector_type(8)));
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = v[i];
#pragma unroll
    for (int q = 0; q < PlaneOf<T>::P; ++q) {
        vec w;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w[i] = PlaneOf<T>::P > 1 && q == 0 ? lead<E>(rest[i]) : (E)rest[i];
            rest[i] -= (float)w[i];  // exact
        }
        *(vec*)(p + q * plane) = w;
    }
}

}  // namespace bc
