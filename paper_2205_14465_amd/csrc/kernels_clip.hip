// kernels_clip.hip -- the norm of a whole list of gradients and its clipping:
//   norm = sqrt(sum of g^2), or max |g|, over every element of the list,
//   c = norm > max_norm ? max_norm / norm : 1,  out = c g.
// The sum is taken in fp64, where the square of an element is exact: each thread
// adds its own in order, a workgroup its threads' in a fixed tree, the next
// launch the workgroups' in a fixed order.  The maximum is taken over the
// magnitudes' bits, so that a NaN is the largest.
//
// Both passes are bound by memory.  A workgroup takes a run of consecutive chunks
// and finds its first matrix by a search of the table with all its threads; the
// second pass walks its run backwards and meets what the caches kept of the first.
#include "common.hpp"
#include "experts.hpp"

#include <algorithm>
#include <cstring>

namespace bc {

namespace {

constexpr int kThreads = 256, kEach = kClipChunk / kThreads;

// The last matrix whose first chunk is c or before, empty ones (which share their
// first chunk with the next) passed over.  All threads call it.
__device__ __forceinline__ uint32_t matrix_of_chunk(const ClipDesc* __restrict__ d, uint32_t T, uint64_t c) {
    uint32_t lo = 0, n = T;  // the answer is in [lo, lo + n)
    while (n > 1) {
        const uint32_t each = (n + kThreads - 1) / kThreads;
        const uint32_t i = threadIdx.x * each;
        const int before = __syncthreads_count(i < n && d[lo + i].chunk0 <= c);
        const uint32_t at = (uint32_t)(before - 1) * each;
        n = n - at < each ? n - at : each;
        lo += at;
    }
    return lo;
}

// fn(descriptor, chunk of its own) for chunks [from, to), in order or backwards.
template <bool kBack, typename F>
__device__ __forceinline__ void for_chunks(const ClipDesc* __restrict__ d, uint32_t T, uint64_t from, uint64_t to, F fn) {
    if (from >= to) return;
    uint32_t t = matrix_of_chunk(d, T, kBack ? to - 1 : from);
    for (uint64_t i = from; i < to; ++i) {
        const uint64_t c = kBack ? to - 1 - (i - from) : i;
        if constexpr (kBack) {
            while (d[t].chunk0 > c) --t;
        } else {
            while (t + 1 < T && d[t + 1].chunk0 <= c) ++t;
        }
        fn(d[t], c - d[t].chunk0);
    }
}

struct Piece {
    uint64_t in, out;       // element offsets
    int left;               // elements of it, 0: none
};
__device__ __forceinline__ Piece piece_of(const ClipDesc& d, uint64_t chunk, int i) {
    const uint64_t p = chunk * kClipChunk + (uint32_t)i * kThreads + threadIdx.x;
    if (p >= d.pieces) return Piece{0, 0, 0};
    if (d.row_pieces == 0) {
        const uint64_t at = p * 8;
        return Piece{at, at, (int)(d.cols - at < 8 ? d.cols - at : 8)};
    }
    const uint64_t row = p / d.row_pieces, at = (p - row * d.row_pieces) * 8;
    return Piece{row * d.ld_in + at, row * d.ld_out + at, (int)(d.cols - at < 8 ? d.cols - at : 8)};
}

template <typename T>
__device__ __forceinline__ void fetch(const ClipDesc& d, uint64_t chunk, Raw<T, 8> (&v)[kEach], Piece (&p)[kEach]) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) p[i] = piece_of(d, chunk, i);
    // (whole pieces without a branch for parts, so that all loads are in flight at once)
    if ((d.cols & 7) == 0 || (d.row_pieces == 0 && (chunk + 1) * kClipChunk * 8 <= d.cols)) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) v[i].template load<true>((const T*)d.in + p[i].in, p[i].left);
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i) v[i].load((const T*)d.in + p[i].in, p[i].left);
    }
}

template <typename F>
__device__ __forceinline__ void with_type(uint32_t dtype, F fn) {
    if (dtype == BC_F32) fn(float{});
    else if (dtype == BC_F16) fn(f16_t{});
    else fn(bf16_t{});
}

__device__ __forceinline__ double block_reduce(double x, int kind) {
    __shared__ double sh[kThreads / 64];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const double y = __shfl_xor(x, o, 64);
        x = kind == BC_NORM_MAX ? __longlong_as_double(max(__double_as_longlong(x), __double_as_longlong(y))) : x + y;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
    __syncthreads();
    x = sh[0];
#pragma unroll
    for (int i = 1; i < kThreads / 64; ++i)
        x = kind == BC_NORM_MAX ? __longlong_as_double(max(__double_as_longlong(x), __double_as_longlong(sh[i]))) : x + sh[i];
    return x;
}

// The norm from the first pass's parts, by all threads of a workgroup.
__device__ __forceinline__ double norm_of(const Clip& a) {
    if (a.given) return *a.given;
    double x = 0.0;
    for (uint32_t i = threadIdx.x; i < a.parts; i += kThreads)
        x = a.kind == BC_NORM_MAX ? __longlong_as_double(max(__double_as_longlong(x), __double_as_longlong(a.part[i])))
                                  : x + a.part[i];
    x = block_reduce(x, a.kind);
    return a.kind == BC_NORM_MAX ? x : sqrt(x);
}

__global__ __launch_bounds__(kThreads) void clip_norm(Clip a) {
    const uint64_t from = a.chunks * blockIdx.x / gridDim.x, to = a.chunks * (blockIdx.x + 1) / gridDim.x;
    double sum[4] = {0.0, 0.0, 0.0, 0.0};
    uint32_t most = 0;
    for_chunks<false>(a.d, a.T, from, to, [&](const ClipDesc& d, uint64_t chunk) {
        with_type(d.dtype, [&](auto of) {
            Raw<decltype(of), 8> v[kEach];
            Piece p[kEach];
            fetch(d, chunk, v, p);
            if (a.kind == BC_NORM_MAX) {
#pragma unroll
                for (int i = 0; i < kEach; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint((float)v[i].v[j]) & 0x7fffffffu);
            } else {
#pragma unroll
                for (int i = 0; i < kEach; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const double x = (double)(float)v[i].v[j];
                        sum[j & 3] = fma(x, x, sum[j & 3]);
                    }
            }
        });
    });
    double x = a.kind == BC_NORM_MAX ? (double)__uint_as_float(most) : (sum[0] + sum[1]) + (sum[2] + sum[3]);
    if (a.kind == BC_NORM_MAX) x = fabs(x);  // (a NaN's sign)
    x = block_reduce(x, a.kind);
    if (threadIdx.x == 0) a.part[blockIdx.x] = x;
}

__global__ __launch_bounds__(kThreads) void norm_of_parts(Clip a) {
    const double norm = norm_of(a);
    if (threadIdx.x == 0) *a.norm = norm;
}

__global__ __launch_bounds__(kThreads) void clip_scale(Clip a) {
    const double norm = norm_of(a);
    const float c = norm > a.max_norm ? (float)(a.max_norm / norm) : 1.0f;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        if (a.norm) *a.norm = norm;
        if (a.factor) *a.factor = c;
    }
    const uint64_t from = a.chunks * blockIdx.x / gridDim.x, to = a.chunks * (blockIdx.x + 1) / gridDim.x;
    for_chunks<true>(a.d, a.T, from, to, [&](const ClipDesc& d, uint64_t chunk) {
        if (c == 1.0f && d.in == d.out) return;
        with_type(d.dtype, [&](auto of) {
            typedef decltype(of) E;
            Raw<E, 8> v[kEach];
            Piece p[kEach];
            fetch(d, chunk, v, p);
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = c * (float)v[i].v[j];
                store_vec((E*)d.out + p[i].out, p[i].left, f, a.nt);
            }
        });
    });
}

// 960 words of a table as arguments.
constexpr uint32_t kTableWords = 960;
struct TableWords {
    uint32_t w[kTableWords];
};
__global__ __launch_bounds__(kThreads) void write_table(uint32_t* to, TableWords t, uint32_t n) {
    for (uint32_t i = threadIdx.x; i < n; i += kThreads) to[i] = t.w[i];
}

}  // namespace

uint32_t clip_parts(uint64_t chunks) { return (uint32_t)std::min<uint64_t>(chunks, kClipParts); }

hipError_t launch_grad_norm(const Clip& a, hipStream_t s) {
    if (a.parts == 0) return hipSuccess;
    hipLaunchKernelGGL(clip_norm, dim3(a.parts), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_norm_of_parts(const Clip& a, hipStream_t s) {
    hipLaunchKernelGGL(norm_of_parts, dim3(1), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_clip(const Clip& a, hipStream_t s) {
    hipLaunchKernelGGL(clip_scale, dim3(std::max(1u, clip_parts(a.chunks))), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_write_table(void* to, const void* from, size_t bytes, hipStream_t s) {
    for (size_t at = 0; at < bytes; at += kTableWords * 4) {
        TableWords t{};
        const size_t n = std::min<size_t>(bytes - at, kTableWords * 4);
        std::memcpy(t.w, (const char*)from + at, n);
        hipLaunchKernelGGL(write_table, dim3(1), dim3(kThreads), 0, s, (uint32_t*)((char*)to + at), t, (uint32_t)(n / 4));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace bc
