// kernels_clip.hip -- the norm of a whole list of gradients and its clipping:
//   norm = sqrt(sum of g^2), or max |g|, over every element of the list,
//   c = norm > max_norm ? max_norm / norm : 1,  out = c g.
// The sum is taken in fp64, where the square of an element is exact: each thread
// adds its own in order, a workgroup its threads' in a fixed tree, the next
// launch the workgroups' in a fixed order.  The maximum is taken over the
// magnitudes' bits, so that a NaN is the largest.
//
// Both passes are bound by memory (1.56e9 fp32 elements: 1010 us for the norm, 6.2
// TB/s, and 2490 for the scaling to another place, 5.0, where a copy reaches 4.3 and an
// elementwise product of one array 5.9; in bfloat16 521 and 1250; ResNet-50's 161
// gradients of 25.6e6 elements: 20.9 us and 37.6, with nothing to scale 5.6; in bfloat16
// 18.2, 25.4 and 5.6).  A workgroup takes a run of consecutive chunks and finds its
// first matrix by a search of the table with all its threads; the second pass walks
// its run backwards and meets what the caches kept of the first.  Over a whole group of
// chunks a thread has 128 bytes of loads in flight whatever the type (with 64 of the
// 16-bit types the norm of the large list took 722 us in place of 524); of a 16-bit list
// of less than 33e6 elements a workgroup's run is shorter than a group (clip_parts), so
// that its chunks go by pieces, fewer in flight.  Rows' ends are left to a loop of their
// own, whose registers would cost a quarter of the waves in flight.
#include "common.hpp"
#include "experts.hpp"

#include <algorithm>
#include <cstring>

namespace bc {

namespace {

constexpr int kThreads = 256;
static_assert(kClipChunk == kThreads, "a piece of a chunk for every thread");
// Chunks whose loads are in flight at once: 128 bytes a thread.
template <typename T>
constexpr int kGroup = 16 / (int)sizeof(T);

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

// fn(descriptor, first chunk of its own, chunks) for the chunks [from, to), matrix
// by matrix, in order or backwards.
template <bool kBack, typename F>
__device__ __forceinline__ void for_matrices(const ClipDesc* __restrict__ d, uint32_t T, uint64_t from, uint64_t to, F fn) {
    if (from >= to) return;
    uint32_t t = matrix_of_chunk(d, T, kBack ? to - 1 : from);
    if constexpr (kBack) {
        while (true) {
            const uint64_t first = max(from, d[t].chunk0);
            if (first < to) fn(d[t], first - d[t].chunk0, to - first);
            if (first <= from) break;
            to = first;
            --t;
        }
    } else {
        while (true) {
            const uint64_t end = t + 1 < T ? min(to, d[t + 1].chunk0) : to;
            if (from < end) fn(d[t], from - d[t].chunk0, end - from);
            if (end >= to) break;
            from = end;
            ++t;
        }
    }
}

struct Piece {
    uint64_t in, out;       // element offsets
    uint32_t left;          // elements of it, 0: none
};
__device__ __forceinline__ Piece piece_of(const ClipDesc& d, uint64_t chunk) {
    const uint64_t p = chunk * kClipChunk + threadIdx.x;
    if (p >= d.pieces) return Piece{0, 0, 0};
    if (d.row_pieces == 0) {
        const uint64_t at = p * 8;
        return Piece{at, at, (uint32_t)min(d.cols - at, (uint64_t)8)};
    }
    const uint64_t row = d.pieces >> 32 ? p / d.row_pieces : (uint32_t)p / d.row_pieces;
    const uint64_t at = (p - row * d.row_pieces) * 8;
    return Piece{row * d.ld_in + at, row * d.ld_out + at, (uint32_t)min(d.cols - at, (uint64_t)8)};
}

// Whether chunks [chunk, chunk + n) are a whole group of a matrix that is one row.
template <typename T>
__device__ __forceinline__ bool whole_group(const ClipDesc& d, uint64_t chunk, uint32_t n) {
    return d.row_pieces == 0 && n == kGroup<T> && (chunk + n) * kClipChunk * 8 <= d.cols;
}

// The whole pieces of chunks [chunk, chunk + n), n no more than a group, all loads
// in flight at once; zeros in place of others.
template <typename T>
__device__ __forceinline__ void fetch(const ClipDesc& d, uint64_t chunk, uint32_t n, Raw<T, 8> (&v)[kGroup<T>]) {
    if (whole_group<T>(d, chunk, n)) {
        const T* at = (const T*)d.in + chunk * kClipChunk * 8;
#pragma unroll
        for (int i = 0; i < kGroup<T>; ++i) v[i].template load<true>(at + ((uint32_t)i * kThreads + threadIdx.x) * 8, 8);
    } else {
#pragma unroll
        for (int i = 0; i < kGroup<T>; ++i) {
            const Piece p = (uint32_t)i < n ? piece_of(d, chunk + i) : Piece{0, 0, 0};
            v[i].template load<true>((const T*)d.in + p.in, p.left == 8);
        }
    }
}

// fn(piece) for the chunks' pieces of fewer than eight elements, the ends of rows.
template <typename F>
__device__ __forceinline__ void for_ends(const ClipDesc& d, uint64_t chunk, uint32_t n, F fn) {
    if ((d.cols & 7) == 0 || (d.row_pieces == 0 && (chunk + n) * kClipChunk * 8 <= d.cols)) return;
#pragma unroll 1
    for (uint32_t i = 0; i < n; ++i) {
        const Piece p = piece_of(d, chunk + i);
        if (p.left > 0 && p.left < 8) fn(p);
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
    double part[kClipParts / kThreads];  // (all loads at once)
#pragma unroll
    for (uint32_t i = 0; i < kClipParts / kThreads; ++i) {
        const uint32_t at = threadIdx.x + i * kThreads;
        part[i] = at < a.parts ? a.part[at] : 0.0;
    }
#pragma unroll
    for (uint32_t i = 0; i < kClipParts / kThreads; ++i)
        x = a.kind == BC_NORM_MAX ? __longlong_as_double(max(__double_as_longlong(x), __double_as_longlong(part[i])))
                                  : x + part[i];
    x = block_reduce(x, a.kind);
    return a.kind == BC_NORM_MAX ? x : sqrt(x);
}

__global__ __launch_bounds__(kThreads) void clip_norm(Clip a) {
    const uint64_t from = a.chunks * blockIdx.x / gridDim.x, to = a.chunks * (blockIdx.x + 1) / gridDim.x;
    double sum[4] = {0.0, 0.0, 0.0, 0.0};
    uint32_t most = 0;
    for_matrices<false>(a.d, a.T, from, to, [&](const ClipDesc& d, uint64_t chunk, uint64_t n) {
        with_type(d.dtype, [&](auto of) {
            typedef decltype(of) E;
            for (uint64_t at = 0; at < n; at += kGroup<E>) {
                const uint32_t m = (uint32_t)min(n - at, (uint64_t)kGroup<E>);
                Raw<E, 8> v[kGroup<E>];
                fetch(d, chunk + at, m, v);
                if (a.kind == BC_NORM_MAX) {
#pragma unroll
                    for (int i = 0; i < kGroup<E>; ++i)
#pragma unroll
                        for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint((float)v[i].v[j]) & 0x7fffffffu);
                } else {
#pragma unroll
                    for (int i = 0; i < kGroup<E>; ++i)
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const double x = (double)(float)v[i].v[j];
                            sum[j & 3] = fma(x, x, sum[j & 3]);
                        }
                }
                for_ends(d, chunk + at, m, [&](const Piece& p) {
#pragma unroll 1
                    for (uint32_t j = 0; j < p.left; ++j) {
                        const float x = (float)((const E*)d.in)[p.in + j];
                        if (a.kind == BC_NORM_MAX) most = max(most, __float_as_uint(x) & 0x7fffffffu);
                        else sum[0] = fma((double)x, (double)x, sum[0]);
                    }
                });
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
    for_matrices<true>(a.d, a.T, from, to, [&](const ClipDesc& d, uint64_t chunk, uint64_t n) {
        if (c == 1.0f && d.in == d.out) return;
        with_type(d.dtype, [&](auto of) {
            typedef decltype(of) E;
            for (uint64_t end = n; end > 0;) {
                const uint32_t m = (uint32_t)min(end, (uint64_t)kGroup<E>);
                end -= m;
                if (whole_group<E>(d, chunk + end, m)) {
                    // 16 bytes a lane, side by side: of 32 bytes in two instructions, fp32's
                    // lines are written in halves (the elements above 2740 us in place of 2490)
                    constexpr int kEach = 16 / (int)sizeof(E), kLoads = 8;
                    const uint64_t at = (chunk + end) * kClipChunk * 8 + threadIdx.x * kEach;
                    Raw<E, kEach> v[kLoads];
#pragma unroll
                    for (int i = 0; i < kLoads; ++i) v[i].template load<true>((const E*)d.in + at + i * kThreads * kEach, 1);
#pragma unroll
                    for (int i = 0; i < kLoads; ++i) {
                        float f[kEach];
#pragma unroll
                        for (int j = 0; j < kEach; ++j) f[j] = c * (float)v[i].v[j];
                        store_vec((E*)d.out + at + i * kThreads * kEach, kEach, f, a.nt);
                    }
                    continue;
                }
                Raw<E, 8> v[kGroup<E>];
                fetch(d, chunk + end, m, v);
#pragma unroll
                for (int i = 0; i < kGroup<E>; ++i) {
                    const Piece p = (uint32_t)i < m ? piece_of(d, chunk + end + i) : Piece{0, 0, 0};
                    if (p.left != 8) continue;
                    float f[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] = c * (float)v[i].v[j];
                    store_vec((E*)d.out + p.out, 8, f, a.nt);
                }
                for_ends(d, chunk + end, m, [&](const Piece& p) {
#pragma unroll 1
                    for (uint32_t j = 0; j < p.left; ++j)
                        ((E*)d.out)[p.out + j] = (E)(c * (float)((const E*)d.in)[p.in + j]);
                });
            }
        });
    });
}

// 960 words of a table as arguments: a captured graph holds them itself, where a copy
// from the host would leave it with a pointer.
constexpr uint32_t kTableWords = 960;
struct TableWords {
    uint32_t w[kTableWords];
};
__global__ __launch_bounds__(kThreads) void write_table(uint32_t* to, TableWords t, uint32_t n) {
    for (uint32_t i = threadIdx.x; i < n; i += kThreads) to[i] = t.w[i];
}

}  // namespace

// A chunk a workgroup while there are no more chunks than CUs, then four (a group of
// fp32's, half of a 16-bit one) until there are kClipParts workgroups.
uint32_t clip_parts(uint64_t chunks) {
    return (uint32_t)std::min(std::min<uint64_t>(chunks, kClipParts), std::max<uint64_t>((chunks + 3) / 4, 256));
}

hipError_t launch_grad_norm(const Clip& a, hipStream_t s) {
    if (a.parts == 0) return hipSuccess;
    hipLaunchKernelGGL(clip_norm, dim3(a.parts), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_norm_of_parts(const Clip& a, hipStream_t s) {
    hipLaunchKernelGGL(norm_of_parts, dim3(1), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

// Five workgroups a CU, each of which adds the parts up first: from 768 to 2048 the
// 1.56e9 elements take the same time, ResNet-50's to another place 40.6 us with 768, 41.9
// with 1024, 37.6 with 1280 and 37.3 with 2048 (in bfloat16 31.0, 28.4, 25.4, 24.0), and
// with nothing to scale 5.9, 6.0, 5.6 and 7.5.
hipError_t launch_clip(const Clip& a, hipStream_t s) {
    const uint32_t blocks = std::max(1u, std::min(clip_parts(a.chunks), 1280u));
    hipLaunchKernelGGL(clip_scale, dim3(blocks), dim3(kThreads), 0, s, a);
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
