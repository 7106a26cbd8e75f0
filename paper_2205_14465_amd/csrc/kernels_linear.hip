// kernels_linear.hip -- the linear layer on the matrix cores: forward
//   z = x w^T + bias,  y = act(z) + residual
// and backward, with dz = dy act'(z),
//   dx = dz w,  dw = dz^T x,  dbias = sum over rows of dz.
//
// The products run in the tiles of gemm.hpp, which want both operands with the
// contracted axis contiguous, 16-byte pieces and whole steps of it.  The
// forward pass's fp16 and bfloat16 operands are usually so and are read where
// they lie; lay_out copies the others into the workspace (padding with zeros,
// turning for the backward pass, splitting fp32 into three bfloat16 planes, whose
// six leading products reach fp32's last places at more than twice the rate of
// the fp32 matrix instructions).  dz is formed in that pass from dy and z and,
// for fp16 and bfloat16, rounded to their type: each of its roundings is half a
// unit in the last place of one term of dx and dw, whose own results are
// rounded once to the same type.  dbias is the fp32 sum of the unrounded dz.
#include "gemm.hpp"
#include "launch.hpp"
#include "layers.hpp"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace bc {

namespace {

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

// ------------------------------------------------------------------ lay_out
// A workgroup 64 rows x 64 columns: read once, written flat from registers and
// turned through LDS, eight elements (16 bytes) of a plane at a time.  Bound by
// memory: for the backward pass of 8192 x 1600 x 6400 in bfloat16 83 us for the
// 510 MB of dy, z, x and w in and dz, dz^T, x^T and w^T out (6.2 TB/s).
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

template <typename T>
__global__ __launch_bounds__(256) void lay_out(LayOuts all) {
    typedef typename PlaneOf<T>::type E;
    const int which = blockIdx.x >= all.first[2] ? 2 : blockIdx.x >= all.first[1] ? 1 : 0;
    const LayOut& a = all.of[which];
    const uint32_t block = blockIdx.x - all.first[which];
    __shared__ float tile[64][65];
    __shared__ float sums[4][64];
    const uint64_t flat_ld = plane_cols(a.cols), turned_ld = plane_cols(a.rows);
    const uint32_t across = (uint32_t)(flat_ld / 64), by = block / across;
    const uint32_t r0 = by * 64, c0 = block % across * 64;
    const uint32_t lc = threadIdx.x % 8 * 8, c = c0 + lc;
    float v[2][8], z[2][8];
    auto fetch = [&](auto whole) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t r = r0 + threadIdx.x / 8 + 32 * i;
            const int left = r < a.rows && c < a.cols ? (int)(a.cols - c) : 0;
            load_vec<decltype(whole)::value>((const T*)a.in + (left > 0 ? r * a.ld_in + c : 0), left, v[i]);
            if (a.z) load_vec<decltype(whole)::value>((const T*)a.z + (left > 0 ? r * a.ld_z + c : 0), left, z[i]);
        }
    };
    if (a.cols % 8 == 0 || c0 + 64 <= a.cols) fetch(std::true_type{});
    else fetch(std::false_type{});
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t lr = threadIdx.x / 8 + 32 * i, r = r0 + lr;
        if (a.z)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                v[i][j] = r < a.rows && c + j < a.cols ? v[i][j] * act_slope<sizeof(T) == 4>(a.act, z[i][j]) : 0.0f;
        if (a.flat && r < a.rows && c < flat_ld)
            store_planes<T>((E*)a.flat + r * flat_ld + c, (uint64_t)a.rows * flat_ld, v[i]);
        if (a.turned || a.part)
#pragma unroll
            for (int j = 0; j < 8; ++j) tile[lr][lc + j] = v[i][j];
    }
    if (!a.turned && !a.part) return;
    __syncthreads();
    if (a.turned)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t tc = threadIdx.x / 8 + 32 * i, tr = threadIdx.x % 8 * 8;
            if (c0 + tc < a.cols && r0 + tr < turned_ld) {
                float w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = tile[tr + j][tc];
                store_planes<T>((E*)a.turned + (c0 + tc) * turned_ld + r0 + tr, (uint64_t)a.cols * turned_ld, w);
            }
        }
    if (a.part) {
        const int tc = threadIdx.x & 63, g = threadIdx.x >> 6;
        float s = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) s += tile[g * 16 + r][tc];
        sums[g][tc] = s;
        __syncthreads();
        if (g == 0 && c0 + tc < a.cols)
            a.part[(uint64_t)by * a.cols + c0 + tc] = (sums[0][tc] + sums[1][tc]) + (sums[2][tc] + sums[3][tc]);
    }
}

// ----------------------------------------------------------------- products
// Eight columns of a row of the result from the fp32 sums v, in place.
template <typename TO, bool forward>
__device__ __forceinline__ void finish_row(const Product& p, uint64_t m, uint32_t n, float (&v)[8]) {
    constexpr bool exact = sizeof(TO) == 4;
    const int left = (int)(p.cols - n);
    if constexpr (forward) {
        float t[8];
        if (p.bias) {
            load_vec((const TO*)p.bias + n, left, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += t[i];
        }
        if (p.z) store_vec((TO*)p.z + m * p.ld_z + n, left, v, p.nt);
        if (p.act != BC_ACT_NONE)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = activate<exact>(p.act, v[i]);
        if (p.residual) {
            load_vec((const TO*)p.residual + m * p.ld_residual + n, left, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += t[i];
        }
    }
    store_vec((TO*)p.out + m * p.ld_out + n, left, v, p.nt);
}

template <typename G, typename TO, bool forward>
__device__ __forceinline__ void product_tile(const Product& p, uint32_t index, char* lds) {
    typedef typename G::T T;
    const uint32_t tiles_m = (p.rows + G::kBM - 1) / G::kBM, tiles_n = (p.cols + G::kBN - 1) / G::kBN;
    uint32_t tm, tn;
    tile_of<8>(index, tiles_m, tiles_n, tm, tn);
    const uint32_t m0 = tm * G::kBM, n0 = tn * G::kBN;
    // this workgroup's steps along k
    const uint32_t from = (uint32_t)((uint64_t)p.steps * blockIdx.y / p.split);
    const uint32_t to = (uint32_t)((uint64_t)p.steps * (blockIdx.y + 1) / p.split);
    const uint64_t k0 = (uint64_t)from * kPlaneCols;
    const Operand<T> a{(const T*)p.a.p + m0 * p.a.ld + k0, (uint32_t)p.a.ld, p.a.plane, p.rows - m0};
    const Operand<T> b{(const T*)p.b.p + n0 * p.b.ld + k0, (uint32_t)p.b.ld, p.b.plane, p.cols - n0};
    G g;
    g.multiply(a, b, (to - from) * (kPlaneCols / G::kBK), lds);
    float* part = p.split > 1 ? p.part + (uint64_t)blockIdx.y * p.rows * p.cols : nullptr;
    g.finish(lds, [&](int row, int col, float (&v)[8]) {
        const uint64_t m = m0 + row;
        const uint32_t n = n0 + col;
        if (m >= p.rows || n >= p.cols) return;
        if (part) store_vec(part + m * p.cols + n, (int)(p.cols - n), v);
        else finish_row<TO, forward>(p, m, n, v);
    });
}

// One product.  Bound by the matrix cores in its main loop, by whole rounds of
// tiles over the chip and, forward, by the writes between them: 8192 x 1600 x 6400
// in bfloat16 211 to 222 us (760 to 800 TFLOP/s) with gelu and z kept, 162 to 167 and
// 188 to 212 us (1030 to 790) for the two products of its backward pass.  The two of
// a pair have a kernel of their own: choosing between them at run time costs the
// single one its arguments in scalar registers (8192x1600x6400 forward, bf16: 211
// us, against 227).
template <typename G, typename TO, bool forward>
__global__ __launch_bounds__(G::kThreads) void product(Product p) {
    extern __shared__ char lds[];
    product_tile<G, TO, forward>(p, blockIdx.x, lds);
}

template <typename G, typename TO>
__global__ __launch_bounds__(G::kThreads) void product_pair(Products all) {
    extern __shared__ char lds[];
    const bool second = blockIdx.x >= all.first;
    product_tile<G, TO, false>(all.of[second], blockIdx.x - (second ? all.first : 0), lds);
}

// The result from the sums of the parts of k, added in order.  Bound by its
// launch at the sizes that are split (777 x 515, two parts: 5 us).
template <typename TO, bool forward>
__global__ __launch_bounds__(256) void join_parts(Product p) {
    const uint32_t across = (p.cols + 7) / 8;
    const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x, m = i / across;
    const uint32_t n = (uint32_t)(i % across) * 8;
    if (m >= p.rows) return;
    const int left = (int)(p.cols - n);
    float v[8];
    load_vec(p.part + m * p.cols + n, left, v);
    for (uint32_t s = 1; s < p.split; ++s) {
        float t[8];
        load_vec(p.part + ((uint64_t)s * p.rows + m) * p.cols + n, left, t);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += t[j];
    }
    finish_row<TO, forward>(p, m, n, v);
}

template <typename G>
uint32_t tiles_of(const Product& p) {
    return ((p.rows + G::kBM - 1) / G::kBM) * ((p.cols + G::kBN - 1) / G::kBN);
}

// More LDS than a kernel may use by default; the attribute is per device and
// setting it again costs next to nothing.
template <typename G>
hipError_t allow_lds(const void* kernel) {
    return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, G::kLdsBytes);
}

template <typename G, typename TO, bool forward>
hipError_t launch_tiles(const Product& p, hipStream_t s) {
    hipError_t e = allow_lds<G>((const void*)product<G, TO, forward>);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((product<G, TO, forward>), dim3(tiles_of<G>(p), p.split), dim3(G::kThreads), G::kLdsBytes, s, p);
    e = hipGetLastError();
    if (e != hipSuccess || p.split == 1) return e;
    const uint64_t pieces = (uint64_t)p.rows * ((p.cols + 7) / 8);
    hipLaunchKernelGGL((join_parts<TO, forward>), dim3((uint32_t)((pieces + 255) / 256)), dim3(256), 0, s, p);
    return hipGetLastError();
}

template <typename G, typename TO>
hipError_t launch_both(const Product& p, const Product& q, hipStream_t s) {
    hipError_t e = allow_lds<G>((const void*)product_pair<G, TO>);
    if (e != hipSuccess) return e;
    const Products all{{p, q}, tiles_of<G>(p)};
    hipLaunchKernelGGL((product_pair<G, TO>), dim3(all.first + tiles_of<G>(q)), dim3(G::kThreads), G::kLdsBytes, s, all);
    return hipGetLastError();
}

// Tile shapes, small to large, and what product_cut knows of them (us): a tile's
// time for 64 along k with its compute unit nearly to itself, a compute unit's
// share of it when the chip is full, and a tile's start and epilogue.  From
// products of 768 x 768 x 1600 to 4096 x 4096 x 6400.
struct TileCost {
    uint32_t rows, cols;
    double alone, full, ends;
};
constexpr TileCost kCost16[3] = {{64, 64, 0.30, 0.193, 0.5}, {128, 128, 0.60, 0.53, 2.0}, {256, 256, 1.05, 1.50, 11.0}};
constexpr TileCost kCost32[3] = {{64, 64, 0.82, 0.95, 0.5}, {128, 128, 1.86, 2.56, 1.5}, {256, 128, 3.4, 4.68, 8.7}};

// The tiles of those costs.
template <typename T> struct Tiles {
    typedef GemmTile<T, 1, 64, 64, 64, 2, 2, 2> Small;
    typedef GemmTile<T, 1, 128, 128, 64, 2, 4, 2> Middle;
    typedef GemmTile<T, 1, 256, 256, 64, 2, 4, 2> Large;
};
template <> struct Tiles<float> {
    typedef GemmTile<bf16_t, 3, 64, 64, 32, 2, 2, 3> Small;
    typedef GemmTile<bf16_t, 3, 128, 128, 32, 2, 4, 3> Middle;
    typedef GemmTile<bf16_t, 3, 256, 128, 32, 4, 2, 2> Large;
};

template <typename T, typename TO, bool forward>
hipError_t launch_cut(int tile, const Product& p, hipStream_t s) {
    if (tile == 0) return launch_tiles<typename Tiles<T>::Small, TO, forward>(p, s);
    if (tile == 1) return launch_tiles<typename Tiles<T>::Middle, TO, forward>(p, s);
    return launch_tiles<typename Tiles<T>::Large, TO, forward>(p, s);
}

template <typename T>
hipError_t launch_pair_of(int tile, const Product& p, const Product& q, hipStream_t s) {
    if (tile == 0) return launch_both<typename Tiles<T>::Small, T>(p, q, s);
    return launch_both<typename Tiles<T>::Middle, T>(p, q, s);
}

// ----------------------------------------------------------------- few rows
// At most kFewRows rows of x: the weight's bytes are the cost, and every
// workgroup reads its 16 rows of w once, straight into the first operand of the
// 16x16x32 matrix instruction; its waves share out the inner axis and meet in
// LDS.  The second operand holds kGroups groups of 16 rows of x.  Bound by the
// loads that cols / 16 workgroups keep in flight: 16 rows in fp16, 1600 by 6400
// 8.5 us (2.4 TB/s), 6400 by 1600 13.7; in fp32, 4096 by 4096 20 (3.4 TB/s).
constexpr int kFewWaves = 8;
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

template <typename T, int kGroups>
__global__ __launch_bounds__(64 * kFewWaves) void few_rows(FewRows a) {
    typedef FewFrag<T> F;
    constexpr int kEach = F::kStep / 4;         // elements of a lane and step
    __shared__ float meet[kFewWaves][kGroups][16][17];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t n0 = blockIdx.x * 16;
    const uint32_t n = n0 + (lane & 15), kl = (lane >> 4) * kEach;
    const T* w = (const T*)a.w + (uint64_t)(n < a.cols ? n : a.cols - 1) * a.ldw;
    const T* x[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const uint32_t m = g * 16 + (lane & 15);
        x[g] = (const T*)a.x + (uint64_t)(m < a.rows ? m : a.rows - 1) * a.ldx;
    }
    f32x4_t acc[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) acc[g] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    const uint32_t steps = (a.inner + F::kStep - 1) / F::kStep;
    const uint32_t whole = a.inner / F::kStep;
    constexpr int kAhead = kGroups > 2 ? 2 : 4;
    uint32_t s = wave;
    // kAhead steps of loads go out before the first is used
    for (; s + (kAhead - 1) * kFewWaves < whole; s += kAhead * kFewWaves) {
        typename F::type fw[kAhead], fx[kAhead][kGroups];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t k = (s + u * kFewWaves) * F::kStep + kl;
            F::load(w + k, kEach, fw[u]);
#pragma unroll
            for (int g = 0; g < kGroups; ++g) F::load(x[g] + k, kEach, fx[u][g]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int g = 0; g < kGroups; ++g) acc[g] = F::mma(fw[u], fx[u][g], acc[g]);
    }
    for (; s < steps; s += kFewWaves) {
        const uint32_t k = s * F::kStep + kl;
        const int left = k < a.inner ? (int)(a.inner - k) : 0;
        typename F::type fw, fx;
        F::load(w + (left ? k : 0), left, fw);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            F::load(x[g] + (left ? k : 0), left, fx);
            acc[g] = F::mma(fw, fx, acc[g]);
        }
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
#pragma unroll
        for (int r = 0; r < 4; ++r) meet[wave][g][lane & 15][(lane >> 4) * 4 + r] = acc[g][r];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < 16 * 16 * kGroups; i += 64 * kFewWaves) {
        const uint32_t m = i / 16, c = n0 + i % 16;
        if (m >= a.rows || c >= a.cols) continue;
        float v = 0.0f;
#pragma unroll
        for (int q = 0; q < kFewWaves; ++q) v += meet[q][m / 16][m % 16][i % 16];
        if (a.bias) v += (float)((const T*)a.bias)[c];
        if (a.z) ((T*)a.z)[m * a.ldz + c] = (T)v;
        v = activate<sizeof(T) == 4>(a.act, v);
        if (a.residual) v += (float)((const T*)a.residual)[m * a.ld_residual + c];
        ((T*)a.y)[m * a.ldy + c] = (T)v;
    }
}

// At most four rows of x: a wave a row of w, which it reads whole kilobytes at a
// time, the loads of kFetch pieces in flight; products and sums in fp32.  Bound
// by the weight's bytes: one row of 6400 by 1600 columns in fp16 6.1 us (3.3
// TB/s), of 1600 by 6400 5.9, of 6400 by 6400 14.4 (5.7 TB/s, launch
// included).  Eight pieces take 6.0, 6.1 and 14.3, sixteen 6.0, 8.7 and
// 14.8: their registers cost more waves than they hide time.  Rows with a part
// at their end (a branch for each piece, waited for) do best with two: 5001 by
// 1601 6.3, with four 6.8.  few_rows, whose hundred workgroups read 64 bytes
// of a row at a time, takes 10.2 for 6400 by 1600.
constexpr uint32_t kDotRows = 4;

template <typename T, int kRows, bool kWhole>
__global__ __launch_bounds__(256) void dot_rows(FewRows a) {
    constexpr int V = kVec<T>, kFetch = kWhole ? 4 : 2;
    const int lane = threadIdx.x & 63;
    const uint32_t c = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (c >= a.cols) return;
    const T* w = (const T*)a.w + (uint64_t)c * a.ldw;
    float acc[kRows];
#pragma unroll
    for (int m = 0; m < kRows; ++m) acc[m] = 0.0f;
    for (uint32_t k0 = 0; k0 < a.inner; k0 += kFetch * 64 * V) {
        Raw<T, V> fw[kFetch], fx[kFetch][kRows];
#pragma unroll
        for (int u = 0; u < kFetch; ++u) {
            const uint32_t k = k0 + (u * 64 + lane) * V;
            const int left = k < a.inner ? (int)(a.inner - k) : 0;
            fw[u].template load<kWhole>(w + (left ? k : 0), left);
#pragma unroll
            for (int m = 0; m < kRows; ++m)
                fx[u][m].template load<kWhole>((const T*)a.x + (uint64_t)(m < (int)a.rows ? m : 0) * a.ldx + (left ? k : 0), left);
        }
#pragma unroll
        for (int u = 0; u < kFetch; ++u)
#pragma unroll
            for (int m = 0; m < kRows; ++m)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[m] = fmaf((float)fw[u].v[i], (float)fx[u][m].v[i], acc[m]);
    }
#pragma unroll
    for (int m = 0; m < kRows; ++m) acc[m] = wave_sum(acc[m]);
    // lane m finishes row m
    float v = acc[0];
#pragma unroll
    for (int m = 1; m < kRows; ++m) v = lane == m ? acc[m] : v;
    if (lane < (int)a.rows) {
        if (a.bias) v += (float)((const T*)a.bias)[c];
        if (a.z) ((T*)a.z)[lane * a.ldz + c] = (T)v;
        v = activate<sizeof(T) == 4>(a.act, v);
        if (a.residual) v += (float)((const T*)a.residual)[lane * a.ld_residual + c];
        ((T*)a.y)[lane * a.ldy + c] = (T)v;
    }
}

template <typename T, int kRows>
void launch_dot_rows(const FewRows& a, hipStream_t s) {
    const dim3 grid((a.cols + 3) / 4), block(256);
    if (a.inner % kVec<T> == 0) hipLaunchKernelGGL((dot_rows<T, kRows, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((dot_rows<T, kRows, false>), grid, block, 0, s, a);
}

template <typename T>
void few_rows_launch(const FewRows& a, hipStream_t s) {
    if (a.rows <= kDotRows) {
        if (a.rows == 1) launch_dot_rows<T, 1>(a, s);
        else if (a.rows == 2) launch_dot_rows<T, 2>(a, s);
        else launch_dot_rows<T, 4>(a, s);
        return;
    }
    const dim3 grid((a.cols + 15) / 16), block(64 * kFewWaves);
    if (a.rows <= 16) hipLaunchKernelGGL((few_rows<T, 1>), grid, block, 0, s, a);
    else if (a.rows <= 32) hipLaunchKernelGGL((few_rows<T, 2>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((few_rows<T, 4>), grid, block, 0, s, a);
}

}  // namespace

hipError_t launch_lay_outs(int dtype, LayOuts& a, hipStream_t s) {
    uint64_t n = 0;
    for (int i = 0; i < 3; ++i) {
        a.first[i] = (uint32_t)n;
        if (i < a.count) n += plane_cols(a.of[i].cols) / 64 * (plane_cols(a.of[i].rows) / 64);
        else a.first[i] = 0xFFFFFFFFu;
    }
    if (n == 0) return hipSuccess;
    if (n >= (1ull << 31)) return hipErrorInvalidValue;
    const dim3 grid((uint32_t)n), block(256);
    if (dtype == BC_F32) hipLaunchKernelGGL(lay_out<float>, grid, block, 0, s, a);
    else if (dtype == BC_F16) hipLaunchKernelGGL(lay_out<f16_t>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(lay_out<bf16_t>, grid, block, 0, s, a);
    return hipGetLastError();
}

constexpr double kUnits = 256.0;

static double tiles_at(const TileCost& c, const Shape& s) {
    return (double)((s.rows + c.rows - 1) / c.rows) * (double)((s.cols + c.cols - 1) / c.cols);
}

// The cheapest cut by the costs above.  Splitting k pays where tiles are fewer
// than compute units: its sums are written and read again (about 4 TB/s from
// the caches) and joined in a launch of their own.
static Cut cheapest_cut(int dtype, const Shape& s, double& least) {
    const TileCost* cost = dtype == BC_F32 ? kCost32 : kCost16;
    const uint64_t steps = plane_cols(s.k) / kPlaneCols;
    Cut best{0, 1};
    least = 1e30;
    for (int i = 0; i < 3; ++i) {
        const double tiles = tiles_at(cost[i], s);
        for (uint32_t split = 1; split <= 32 && (split == 1 || (split * 4 <= steps && tiles * split <= 512)); split *= 2) {
            const double each = (double)((steps + split - 1) / split);
            const double full = each * cost[i].full + cost[i].ends, n = tiles * split / kUnits;
            // the largest tiles come one to a unit, in whole rounds
            const double busy = i == 2 ? std::ceil(n) * full : n <= 1.0 ? 0.0 : (n + 0.5) * full;
            double t = std::max(each * cost[i].alone + cost[i].ends, busy);
            if (split > 1) t += 4.0 + 2.0 * 4.0 * (double)split * (double)s.rows * (double)s.cols / 4e6;
            if (t < least) {
                least = t;
                best = Cut{i, split};
            }
        }
    }
    return best;
}

Cut product_cut(int dtype, uint64_t rows, uint64_t cols, uint64_t k) {
    double least;
    return cheapest_cut(dtype, Shape{rows, cols, k}, least);
}

int pair_tile(int dtype, const Shape& a, const Shape& b) {
    const TileCost* cost = dtype == BC_F32 ? kCost32 : kCost16;
    double ta, tb, least = 1e30;
    cheapest_cut(dtype, a, ta);
    cheapest_cut(dtype, b, tb);
    int best = -1;
    for (int i = 0; i < 2; ++i) {  // the largest tiles fill the chip by themselves
        double alone = 0.0, busy = 0.0, longest = 0.0;
        for (const Shape* s : {&a, &b}) {
            const double steps = (double)(plane_cols(s->k) / kPlaneCols), full = steps * cost[i].full + cost[i].ends;
            alone = std::max(alone, steps * cost[i].alone + cost[i].ends);
            busy += tiles_at(cost[i], *s) * full / kUnits;
            longest = std::max(longest, full);
        }
        const double t = std::max(alone, busy + 0.5 * longest);
        if (t < least) {
            least = t;
            best = i;
        }
    }
    return least < ta + tb + 2.5 ? best : -1;
}

hipError_t launch_product(int dtype, int out_dtype, bool forward, const Cut& cut, const Product& given, hipStream_t s) {
    if (given.rows == 0 || given.cols == 0) return hipSuccess;
    Product p = given;
    p.split = cut.split;
    const int t = cut.tile;
    if (forward) {
        if (dtype == BC_F32) return launch_cut<float, float, true>(t, p, s);
        if (dtype == BC_F16) return launch_cut<f16_t, f16_t, true>(t, p, s);
        return launch_cut<bf16_t, bf16_t, true>(t, p, s);
    }
    if (dtype == BC_F32) return launch_cut<float, float, false>(t, p, s);
    if (dtype == BC_F16) {
        if (out_dtype == BC_F32) return launch_cut<f16_t, float, false>(t, p, s);
        return launch_cut<f16_t, f16_t, false>(t, p, s);
    }
    if (out_dtype == BC_F32) return launch_cut<bf16_t, float, false>(t, p, s);
    return launch_cut<bf16_t, bf16_t, false>(t, p, s);
}

hipError_t launch_pair(int dtype, int tile, const Product& first, const Product& second, hipStream_t s) {
    Product p = first, q = second;
    p.split = q.split = 1;
    const bool no_p = p.rows == 0 || p.cols == 0, no_q = q.rows == 0 || q.cols == 0;
    if (no_p || no_q) {
        const hipError_t e = launch_product(dtype, dtype, false, Cut{tile, 1}, p, s);
        return e != hipSuccess ? e : launch_product(dtype, dtype, false, Cut{tile, 1}, q, s);
    }
    if (dtype == BC_F32) return launch_pair_of<float>(tile, p, q, s);
    if (dtype == BC_F16) return launch_pair_of<f16_t>(tile, p, q, s);
    return launch_pair_of<bf16_t>(tile, p, q, s);
}

hipError_t launch_few_rows(int dtype, const FewRows& a, hipStream_t s) {
    if (dtype == BC_F32) few_rows_launch<float>(a, s);
    else if (dtype == BC_F16) few_rows_launch<f16_t>(a, s);
    else few_rows_launch<bf16_t>(a, s);
    return hipGetLastError();
}

}  // namespace bc
