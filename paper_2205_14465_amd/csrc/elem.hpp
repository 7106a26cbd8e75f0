// elem.hpp -- element types of the layer operators (layer norm, linear layer,
// orthogonalised updates): fp32, fp16 and bfloat16 in memory, fp32 in
// registers.  Rows may start at any element, so vector accesses assume no more
// than an element's alignment; gfx950 takes such global loads and stores whole.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/bytecomp.h"

namespace bc {

typedef _Float16 f16_t;
typedef __bf16 bf16_t;

inline size_t dtype_bytes(int dtype) { return dtype == BC_F32 ? 4 : 2; }
inline bool dtype_ok(int dtype) { return dtype == BC_F32 || dtype == BC_F16 || dtype == BC_BF16; }

// Elements of one 16-byte access.
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);

// V consecutive elements widened to fp32; the first `left` of them when
// fewer are left (the others 0, not read).  kWhole: left is at least V or at
// most 0, which the caller knows of all its lanes; without the branch for a part
// the compiler lets loads follow each other unwaited for.
template <bool kWhole = false, typename T, int V>
__device__ __forceinline__ void load_vec(const T* p, int left, float (&f)[V]) {
    if constexpr (kWhole) {
        typedef T vec __attribute__((ext_vector_type(V)));
        vec v = (T)0.0f;
        if (left > 0) __builtin_memcpy(&v, p, sizeof(v));
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = (float)v[i];
    } else if (left >= V) {
        typedef T vec __attribute__((ext_vector_type(V)));
        vec v;
        __builtin_memcpy(&v, p, sizeof(v));
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = (float)v[i];
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = i < left ? (float)p[i] : 0.0f;
    }
}

// The same without widening them: V elements as they lie.
template <typename T, int V>
struct Raw {
    typedef T vec __attribute__((ext_vector_type(V)));
    vec v;
    template <bool kWhole = false>
    __device__ __forceinline__ void load(const T* p, int left) {
        if constexpr (kWhole) {
            v = (T)0.0f;
            if (left > 0) __builtin_memcpy(&v, p, sizeof(v));
        } else if (left >= V) {
            __builtin_memcpy(&v, p, sizeof(v));
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = i < left ? p[i] : (T)0.0f;
        }
    }
};

// Whether a result of this many bytes is written with the non-temporal hint:
// past half of the L2s' 32 MB it would only push out what the launch still reads
// (with the hint, layer norm of 8192 x 1600 in bfloat16 10% faster, a linear
// layer of 8192 x 1600 x 6400 6%; 5 MB of fp32 1% slower).
inline bool streams(uint64_t bytes) { return bytes > (16ull << 20); }

// load_vec's counterpart: rounded once (nearest, ties to even) and written;
// nt: with the non-temporal hint.
template <typename T, int V>
__device__ __forceinline__ void store_vec(T* p, int left, const float (&f)[V], bool nt = false) {
    if (left >= V) {
        typedef T vec __attribute__((ext_vector_type(V)));
        typedef T loose __attribute__((ext_vector_type(V), aligned(sizeof(T))));
        vec v;
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (T)f[i];
        if (nt) {
            // the fences keep the compiler from joining the two stores, without the hint
            asm volatile("" ::: "memory");
            __builtin_nontemporal_store(v, (loose*)p);
            asm volatile("" ::: "memory");
        } else {
            __builtin_memcpy(p, &v, sizeof(v));
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < left) p[i] = (T)f[i];
    }
}

// Sum over the 64 lanes of a wave, in every lane.
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
    return x;
}

}  // namespace bc
