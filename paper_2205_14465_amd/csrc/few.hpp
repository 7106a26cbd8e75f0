// few.hpp -- fragments of the 16 x 16 matrix instructions straight from memory, for
// products of few rows.
#pragma once

#include "gemm.hpp"

namespace bc {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

template <typename T>
struct FewFrag {
    typedef typename Frag<T>::type type;
    static constexpr int kStep = 32;
    static __device__ __forceinline__ void load(const T* p, int left, type& f) {
        if (left >= 8) {
            __builtin_memcpy(&f, p, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = i < left ? p[i] : (T)0.0f;
        }
    }
    static __device__ __forceinline__ f32x4_t mma(type a, type b, f32x4_t c) {
        if constexpr (__is_same(T, f16_t)) return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
// fp32: four 16x16x4 instructions, the k of lane group g's element i being
// 4 g + i in both operands.
template <>
struct FewFrag<float> {
    typedef f32x4_t type;
    static constexpr int kStep = 16;
    static __device__ __forceinline__ void load(const float* p, int left, type& f) {
        if (left >= 4) {
            __builtin_memcpy(&f, p, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = i < left ? p[i] : 0.0f;
        }
    }
    static __device__ __forceinline__ f32x4_t mma(type a, type b, f32x4_t c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
};

}  // namespace bc
