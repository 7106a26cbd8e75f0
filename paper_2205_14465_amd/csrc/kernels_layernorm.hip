// kernels_layernorm.hip -- layer norm over the last axis, forward and backward.
//
// With mean m and variance s of a row of D elements (both over the row, the
// variance of the centred elements) and r = 1 / sqrt(s + eps):
//   xhat = (x - m) r,   y = xhat w + b
//   h = dy w,  dx = r (h - mean(h) - xhat mean(h xhat))
//   dw = sum over rows of dy xhat,  db = sum over rows of dy
// All arithmetic is fp32; y, dx, dw and db are rounded once, when written.
//
// Both passes are bound by memory: forward reads x and writes y, backward
// reads x and dy and writes dx, each once.  A row lives in the registers of the
// wave (or workgroup) that owns it, so the centred variance costs no second
// read.  Backward keeps the column sums of the rows it visits in registers as
// well; workgroups leave partial sums in the workspace, which a second small
// kernel adds in a fixed order (no atomics: results do not depend on timing).
#include "launch.hpp"
#include "layers.hpp"

namespace bc {

namespace {

constexpr int kLnBlock = 256;
constexpr int kLnWaves = kLnBlock / 64;

// Sum over the kGroup threads of a row: one wave, or the whole workgroup
// (through `sh`, which the caller leaves alone until the next barrier).
template <int kGroup>
__device__ __forceinline__ float group_sum(float x, float* sh) {
    x = wave_sum(x);
    if constexpr (kGroup > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
        __syncthreads();
        x = 0.0f;
#pragma unroll
        for (int i = 0; i < kGroup / 64; ++i) x += sh[i];
    }
    return x;
}

// Weights of N columns from c, `none` where the call has no weights.
template <bool kWhole, typename WT, int N>
__device__ __forceinline__ void load_weight(const void* w, uint32_t c, int left, float none, float (&f)[N]) {
    if (w) {
        load_vec<kWhole>((const WT*)w + c, left, f);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = none;
    }
}

// ---------------------------------------------------------------- forward
// kGroup threads a row (64: four rows a workgroup, kLnBlock: one), kPer
// vectors a thread; kWhole: rows are whole vectors, loaded without a branch for
// parts (8192 x 1600 in bfloat16 11.8 us, 4.4 TB/s, against 13.7 with it).  One
// token of 768: 3.9 us, the launch.  Rows following each other with their
// weights in registers, as in the backward pass, are 6% slower: the registers
// cost more waves than the weights cost loads.
template <typename T, typename WT, int kGroup, int kPer, bool kWhole>
__global__ __launch_bounds__(kLnBlock) void ln_forward(LnForward a) {
    constexpr int V = kVec<T>;
    __shared__ float sh[kLnWaves];
    const int j = threadIdx.x % kGroup;
    const uint64_t row = kGroup == 64 ? (uint64_t)blockIdx.x * kLnWaves + (threadIdx.x >> 6) : blockIdx.x;
    if (row >= a.rows) return;  // whole waves, and no barrier with kGroup == 64
    const T* x = (const T*)a.x + row * a.ldx;
    float v[kPer][V];
    float sum = 0.0f;
#pragma unroll
    for (int p = 0; p < kPer; ++p) {
        const int c = (p * kGroup + j) * V;
        load_vec<kWhole>(x + c, (int)a.cols - c, v[p]);
    }
#pragma unroll
    for (int p = 0; p < kPer; ++p)
#pragma unroll
        for (int i = 0; i < V; ++i) sum += v[p][i];
    const float mean = group_sum<kGroup>(sum, sh) * a.inv_cols;
    float sq = 0.0f;
#pragma unroll
    for (int p = 0; p < kPer; ++p) {
        const int left = (int)a.cols - (p * kGroup + j) * V;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float d = v[p][i] - mean;
            sq += i < left ? d * d : 0.0f;
        }
    }
    const float rstd = 1.0f / sqrtf(group_sum<kGroup>(sq, sh) * a.inv_cols + a.eps);
    if (j == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    T* y = (T*)a.y + row * a.ldy;
#pragma unroll
    for (int p = 0; p < kPer; ++p) {
        const int c = (p * kGroup + j) * V, left = (int)a.cols - c;
        if (left > 0) {
            float w[V], b[V], o[V];
            load_weight<kWhole, WT>(a.weight, c, left, 1.0f, w);
            load_weight<kWhole, WT>(a.bias, c, left, 0.0f, b);
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = (v[p][i] - mean) * rstd * w[i] + b[i];
            store_vec(y + c, left, o, a.nt);
        }
    }
}

// Rows too long for registers: a workgroup reads its row three times (the
// second and third from the caches).
constexpr int kWideBlock = 1024;

template <typename T, typename WT>
__global__ __launch_bounds__(kWideBlock) void ln_forward_wide(LnForward a) {
    constexpr int V = kVec<T>;
    __shared__ float sh[kWideBlock / 64];
    const uint64_t row = blockIdx.x;
    const T* x = (const T*)a.x + row * a.ldx;
    const uint32_t step = kWideBlock * V;
    float sum = 0.0f;
    for (uint32_t c = threadIdx.x * V; c < a.cols; c += step) {
        float v[V];
        load_vec(x + c, (int)(a.cols - c), v);
        float part = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) part += v[i];
        sum += part;
    }
    const float mean = group_sum<kWideBlock>(sum, sh) * a.inv_cols;
    float sq = 0.0f;
    for (uint32_t c = threadIdx.x * V; c < a.cols; c += step) {
        float v[V];
        load_vec(x + c, (int)(a.cols - c), v);
        float part = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float d = v[i] - mean;
            part += i < (int)(a.cols - c) ? d * d : 0.0f;
        }
        sq += part;
    }
    const float rstd = 1.0f / sqrtf(group_sum<kWideBlock>(sq, sh) * a.inv_cols + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    T* y = (T*)a.y + row * a.ldy;
    for (uint32_t c = threadIdx.x * V; c < a.cols; c += step) {
        const int left = (int)(a.cols - c);
        float v[V], w[V], b[V];
        load_vec(x + c, left, v);
        load_weight<false, WT>(a.weight, c, left, 1.0f, w);
        load_weight<false, WT>(a.bias, c, left, 0.0f, b);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (v[i] - mean) * rstd * w[i] + b[i];
        store_vec(y + c, left, v, a.nt);
    }
}

// --------------------------------------------------------------- backward
// A workgroup (kGroup == 64: each of its waves) visits rows a fixed step apart
// and adds their columns' dy xhat and dy in registers: thread j the vectors
// j, j + kGroup, ...  The next row's loads are in flight under the arithmetic of
// the last; weights stay in registers.  The waves of a workgroup then meet in
// LDS, and the workgroup's sums go to part[block] (cols of dw, then cols of db).
// Bound by memory and by the few waves that its registers leave to hide it:
// 8192 x 1600 in fp16 20 us, 3.9 TB/s, and 4 more for sum_parts (33 in all without
// the loads ahead); 1237 x 1001 in fp32 7 and 3.
template <typename T, typename WT, int kGroup, int kPer, bool kWhole>
__global__ __launch_bounds__(kLnBlock) void ln_backward(LnBackward a) {
    constexpr int V = kVec<T>;
    __shared__ float sh[kLnWaves];
    const int j = threadIdx.x % kGroup;
    const uint32_t unit = kGroup == 64 ? blockIdx.x * kLnWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : blockIdx.x;
    const uint32_t step = kGroup == 64 ? gridDim.x * kLnWaves : gridDim.x;
    float aw[kPer][V], ab[kPer][V], w[kPer][V];
    Raw<T, V> nx[kPer], ny[kPer];
    auto fetch = [&](uint64_t row) {
        const T* x = (const T*)a.x + row * a.ldx;
        const T* dy = (const T*)a.dy + row * a.lddy;
#pragma unroll
        for (int p = 0; p < kPer; ++p) {
            const int c = (p * kGroup + j) * V;
            nx[p].template load<kWhole>(x + c, (int)a.cols - c);
            ny[p].template load<kWhole>(dy + c, (int)a.cols - c);
        }
    };
    if (unit < a.rows) fetch(unit);
#pragma unroll
    for (int p = 0; p < kPer; ++p) {
        const int c = (p * kGroup + j) * V;
        load_weight<kWhole, WT>(a.weight, c, (int)a.cols - c, 1.0f, w[p]);
#pragma unroll
        for (int i = 0; i < V; ++i) aw[p][i] = ab[p][i] = 0.0f;
    }
    for (uint64_t row = unit; row < a.rows; row += step) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        float xh[kPer][V], h[kPer][V];
#pragma unroll
        for (int p = 0; p < kPer; ++p)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                xh[p][i] = (float)nx[p].v[i];
                h[p][i] = (float)ny[p].v[i];
            }
        if (row + step < a.rows) fetch(row + step);
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int p = 0; p < kPer; ++p) {
            const int left = (int)a.cols - (p * kGroup + j) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = h[p][i];
                // past the row's end dy and the weight are 0, but the mean is not
                xh[p][i] = i < left ? (xh[p][i] - mean) * rstd : 0.0f;
                aw[p][i] += d * xh[p][i];
                ab[p][i] += d;
                h[p][i] = i < left ? d * w[p][i] : 0.0f;
                s1 += h[p][i];
                s2 += h[p][i] * xh[p][i];
            }
        }
        if (!a.dx) continue;  // the same for every row
        s1 = group_sum<kGroup>(s1, sh) * a.inv_cols;
        s2 = group_sum<kGroup>(s2, sh) * a.inv_cols;
        T* dx = (T*)a.dx + row * a.lddx;
#pragma unroll
        for (int p = 0; p < kPer; ++p) {
            const int c = (p * kGroup + j) * V, left = (int)a.cols - c;
            if (left > 0) {
                float o[V];
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] = rstd * (h[p][i] - s1 - xh[p][i] * s2);
                store_vec(dx + c, left, o, a.nt);
            }
        }
    }
    if (!a.part) return;
    float* part = a.part + (uint64_t)blockIdx.x * 2 * a.cols;
    if constexpr (kGroup == 64) {
        __shared__ float4 meet[kLnWaves * 64 * kPer * V / 4];
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int p = 0; p < kPer; ++p)
#pragma unroll
                for (int q = 0; q < V / 4; ++q) {
                    const float* s = which ? &ab[p][4 * q] : &aw[p][4 * q];
                    meet[((wave * kPer + p) * (V / 4) + q) * 64 + j] = make_float4(s[0], s[1], s[2], s[3]);
                }
            __syncthreads();
            // thread i: vectors i, i + kLnBlock, ... of four columns
            for (int i = threadIdx.x; i < 64 * kPer * V / 4; i += kLnBlock) {
                float4 t = meet[i];
#pragma unroll
                for (int w = 1; w < kLnWaves; ++w) {
                    const float4 u = meet[w * 64 * kPer * V / 4 + i];
                    t.x += u.x; t.y += u.y; t.z += u.z; t.w += u.w;
                }
                const int lane = i % 64, q = i / 64 % (V / 4), p = i / 64 / (V / 4);
                const int c = (p * 64 + lane) * V + 4 * q;
                const float f[4] = {t.x, t.y, t.z, t.w};
                if (c < (int)a.cols) store_vec(part + which * a.cols + c, (int)a.cols - c, f);
            }
        }
    } else {
#pragma unroll
        for (int p = 0; p < kPer; ++p) {
            const int c = (p * kGroup + j) * V, left = (int)a.cols - c;
            if (left > 0) {
                store_vec(part + c, left, aw[p]);
                store_vec(part + a.cols + c, left, ab[p]);
            }
        }
    }
}

// Rows too long for registers: dx by a workgroup a row, in two reads (the
// second from the caches) ...
template <typename T, typename WT>
__global__ __launch_bounds__(kWideBlock) void ln_backward_wide(LnBackward a) {
    constexpr int V = kVec<T>;
    __shared__ float sh[kWideBlock / 64];
    const uint64_t row = blockIdx.x;
    const T* x = (const T*)a.x + row * a.ldx;
    const T* dy = (const T*)a.dy + row * a.lddy;
    T* dx = (T*)a.dx + row * a.lddx;
    const float mean = a.mean[row], rstd = a.rstd[row];
    const uint32_t step = kWideBlock * V;
    float s1 = 0.0f, s2 = 0.0f;
    for (uint32_t c = threadIdx.x * V; c < a.cols; c += step) {
        const int left = (int)(a.cols - c);
        float v[V], d[V], w[V];
        load_vec(x + c, left, v);
        load_vec(dy + c, left, d);
        load_weight<false, WT>(a.weight, c, left, 1.0f, w);
        float p1 = 0.0f, p2 = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float h = i < left ? d[i] * w[i] : 0.0f;
            p1 += h;
            p2 += h * (i < left ? (v[i] - mean) * rstd : 0.0f);
        }
        s1 += p1;
        s2 += p2;
    }
    s1 = group_sum<kWideBlock>(s1, sh) * a.inv_cols;
    s2 = group_sum<kWideBlock>(s2, sh) * a.inv_cols;
    for (uint32_t c = threadIdx.x * V; c < a.cols; c += step) {
        const int left = (int)(a.cols - c);
        float v[V], d[V], w[V];
        load_vec(x + c, left, v);
        load_vec(dy + c, left, d);
        load_weight<false, WT>(a.weight, c, left, 1.0f, w);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = rstd * (d[i] * w[i] - s1 - (v[i] - mean) * rstd * s2);
        store_vec(dx + c, left, v, a.nt);
    }
}

// ... and the column sums by workgroups of kLnBlock vectors of columns and a
// run of rows each.
template <typename T>
__global__ __launch_bounds__(kLnBlock) void ln_column_sums(LnBackward a) {
    constexpr int V = kVec<T>;
    const uint32_t c = (blockIdx.x * kLnBlock + threadIdx.x) * V;
    if (c >= a.cols) return;
    const int left = (int)(a.cols - c);
    const uint64_t per = (a.rows + gridDim.y - 1) / gridDim.y;
    const uint64_t lo = blockIdx.y * per, hi = lo + per < a.rows ? lo + per : a.rows;
    float aw[V], ab[V];
#pragma unroll
    for (int i = 0; i < V; ++i) aw[i] = ab[i] = 0.0f;
    for (uint64_t row = lo; row < hi; ++row) {
        float v[V], d[V];
        load_vec((const T*)a.x + row * a.ldx + c, left, v);
        load_vec((const T*)a.dy + row * a.lddy + c, left, d);
        const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            aw[i] += i < left ? d[i] * ((v[i] - mean) * rstd) : 0.0f;
            ab[i] += d[i];
        }
    }
    float* part = a.part + (uint64_t)blockIdx.y * 2 * a.cols;
    store_vec(part + c, left, aw);
    store_vec(part + a.cols + c, left, ab);
}

}  // namespace

// Column sums of `parts` rows of `cols` fp32 values `stride` apart, rounded
// once: a workgroup 32 columns, 32 threads a column, each adding every 32nd
// row in order, then a fixed tree.  Zero rows give zeros.
template <typename WT>
__global__ __launch_bounds__(1024) void sum_parts(const float* __restrict__ part, uint32_t parts, uint64_t stride,
                                                  uint32_t cols, WT* __restrict__ out0, WT* __restrict__ out1) {
    __shared__ float sh[32][33];
    const int cx = threadIdx.x & 31, ry = threadIdx.x >> 5;
    const uint32_t c = blockIdx.x * 32 + cx;
    WT* out = blockIdx.y ? out1 : out0;
    if (!out) return;
    const float* p = part + blockIdx.y * (uint64_t)cols;
    float s = 0.0f;
    if (c < cols)
#pragma unroll 4
        for (uint32_t r = ry; r < parts; r += 32) s += p[r * stride + c];
    sh[ry][cx] = s;
    __syncthreads();
    // thread (cx, ry) now adds for column ry, row group cx: 32 lanes of a wave
    float t = sh[cx][ry];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor(t, o, 32);
    const uint32_t col = blockIdx.x * 32 + ry;
    if (cx == 0 && col < cols) out[col] = (WT)t;
}

hipError_t launch_sum_parts(int dtype, const float* part, uint32_t parts, uint64_t stride, uint32_t cols, void* out0,
                            void* out1, hipStream_t s) {
    if (cols == 0 || (!out0 && !out1)) return hipSuccess;
    const dim3 grid((cols + 31) / 32, out1 ? 2 : 1), block(1024);
    if (dtype == BC_F32)
        hipLaunchKernelGGL(sum_parts<float>, grid, block, 0, s, part, parts, stride, cols, (float*)out0, (float*)out1);
    else if (dtype == BC_F16)
        hipLaunchKernelGGL(sum_parts<f16_t>, grid, block, 0, s, part, parts, stride, cols, (f16_t*)out0, (f16_t*)out1);
    else
        hipLaunchKernelGGL(sum_parts<bf16_t>, grid, block, 0, s, part, parts, stride, cols, (bf16_t*)out0,
                           (bf16_t*)out1);
    return hipGetLastError();
}

// Calls launch(part) for parts of the rows with fewer than 2^32 threads each, which
// is what HIP takes along an axis, at `threads` a row; from(r) is the call from row r on.
template <typename A, typename From, typename Launch>
static void by_rows(const A& a, uint32_t threads, From from, Launch launch) {
    const uint64_t most = (1ull << 31) / threads;
    for (uint64_t r = 0; r < a.rows; r += most) {
        A part = from(r);
        part.rows = a.rows - r < most ? a.rows - r : most;
        launch(part, (uint32_t)part.rows);
    }
}

// Rows of up to 64 * kPer vectors go to a wave, of up to kLnBlock * kPer to a
// workgroup, longer ones to the wide kernels.  Measured in bfloat16, us:
//   forward   8192 x 2048  wave 12.9, workgroup 14.0;  8192 x 4096  22.7, 22.4;
//             512 x 4096 (fp16)  6.3, 4.2;  2048 x 16384  workgroup 23.7, wide 30.0
//   backward  8192 x 2048  wave 23.6, workgroup 30.5;  8192 x 4096  66.5, 49.6;
//             2048 x 8192  workgroup 33.1, wide 54.4;  2048 x 16384  90.7, 89.2,
//             500 x 12001 (fp16)  48.4, 33.6;  fp32, 4096 x 8192  103, 133
template <typename T, typename WT, bool kWhole>
static void ln_forward_launch(const LnForward& all, hipStream_t s) {
    const uint32_t vecs = (all.cols + kVec<T> - 1) / kVec<T>;
    const auto from = [&](uint64_t r) {
        LnForward a = all;
        a.x = (const T*)a.x + r * a.ldx;
        a.y = (T*)a.y + r * a.ldy;
        if (a.mean) a.mean += r;
        if (a.rstd) a.rstd += r;
        return a;
    };
    const dim3 block(kLnBlock);
    if (vecs <= 256) {
        by_rows(all, 64, from, [&](const LnForward& a, uint32_t rows) {
            const dim3 waves((rows + kLnWaves - 1) / kLnWaves);
            if (vecs <= 64) hipLaunchKernelGGL((ln_forward<T, WT, 64, 1, kWhole>), waves, block, 0, s, a);
            else if (vecs <= 128) hipLaunchKernelGGL((ln_forward<T, WT, 64, 2, kWhole>), waves, block, 0, s, a);
            else hipLaunchKernelGGL((ln_forward<T, WT, 64, 4, kWhole>), waves, block, 0, s, a);
        });
    } else if (vecs <= 2048) {
        by_rows(all, kLnBlock, from, [&](const LnForward& a, uint32_t rows) {
            if (vecs <= 512) hipLaunchKernelGGL((ln_forward<T, WT, kLnBlock, 2, kWhole>), dim3(rows), block, 0, s, a);
            else if (vecs <= 1024) hipLaunchKernelGGL((ln_forward<T, WT, kLnBlock, 4, kWhole>), dim3(rows), block, 0, s, a);
            else hipLaunchKernelGGL((ln_forward<T, WT, kLnBlock, 8, kWhole>), dim3(rows), block, 0, s, a);
        });
    } else {
        by_rows(all, kWideBlock, from, [&](const LnForward& a, uint32_t rows) {
            hipLaunchKernelGGL((ln_forward_wide<T, WT>), dim3(rows), dim3(kWideBlock), 0, s, a);
        });
    }
}

// Vectors of the longest rows that the backward pass holds in registers: twice
// as many where two arrays of fp32 need no widening and no masks.
template <typename T>
static uint32_t ln_longest(uint32_t cols) { return sizeof(T) == 4 && cols % kVec<T> == 0 ? 2048 : 1024; }

template <typename T, typename WT, bool kWhole>
static void ln_backward_launch(const LnBackward& a, hipStream_t s) {
    const uint32_t vecs = (a.cols + kVec<T> - 1) / kVec<T>;
    const dim3 block(kLnBlock), grid(a.parts);
    if (vecs <= 64) hipLaunchKernelGGL((ln_backward<T, WT, 64, 1, kWhole>), grid, block, 0, s, a);
    else if (vecs <= 128) hipLaunchKernelGGL((ln_backward<T, WT, 64, 2, kWhole>), grid, block, 0, s, a);
    else if (vecs <= 256) hipLaunchKernelGGL((ln_backward<T, WT, 64, 4, kWhole>), grid, block, 0, s, a);
    else if (vecs <= 512) hipLaunchKernelGGL((ln_backward<T, WT, kLnBlock, 2, kWhole>), grid, block, 0, s, a);
    else if (vecs <= 1024) hipLaunchKernelGGL((ln_backward<T, WT, kLnBlock, 4, kWhole>), grid, block, 0, s, a);
    else if (vecs <= ln_longest<T>(a.cols)) {
        if constexpr (sizeof(T) == 4 && kWhole) hipLaunchKernelGGL((ln_backward<T, WT, kLnBlock, 8, true>), grid, block, 0, s, a);
    } else {
        const auto from = [&](uint64_t r) {
            LnBackward p = a;
            p.dy = (const T*)p.dy + r * p.lddy;
            p.x = (const T*)p.x + r * p.ldx;
            p.dx = (T*)p.dx + r * p.lddx;
            p.mean += r;
            p.rstd += r;
            return p;
        };
        if (a.dx)
            by_rows(a, kWideBlock, from, [&](const LnBackward& p, uint32_t rows) {
                hipLaunchKernelGGL((ln_backward_wide<T, WT>), dim3(rows), dim3(kWideBlock), 0, s, p);
            });
        if (a.part)
            hipLaunchKernelGGL((ln_column_sums<T>), dim3((vecs + kLnBlock - 1) / kLnBlock, a.parts), block, 0, s, a);
    }
}

// Workgroups that leave partial sums of columns.  (The wide kernel's take eight
// rows each at least: 500 x 12001 in fp16 33.6 us, with four the same, with 32
// rows 61.5.)
uint32_t ln_parts(uint64_t rows, uint32_t cols, int dtype) {
    const uint32_t V = dtype == BC_F32 ? 4 : 8, vecs = (cols + V - 1) / V;
    const bool held = vecs <= (dtype == BC_F32 ? ln_longest<float>(cols) : ln_longest<f16_t>(cols));
    const uint64_t units = vecs <= 256 ? (rows + kLnWaves - 1) / kLnWaves : held ? rows : (rows + 7) / 8;
    const uint64_t most = held ? 512 : 64;
    return (uint32_t)(units < most ? units : most);
}

template <typename T, typename WT>
static void ln_forward_any(const LnForward& a, hipStream_t s) {
    if (a.cols % kVec<T> == 0) ln_forward_launch<T, WT, true>(a, s);
    else ln_forward_launch<T, WT, false>(a, s);
}
template <typename T, typename WT>
static void ln_backward_any(const LnBackward& a, hipStream_t s) {
    if (a.cols % kVec<T> == 0) ln_backward_launch<T, WT, true>(a, s);
    else ln_backward_launch<T, WT, false>(a, s);
}

hipError_t launch_ln_forward(int dtype, int wdtype, const LnForward& a, hipStream_t s) {
    if (dtype == BC_F32) ln_forward_any<float, float>(a, s);
    else if (dtype == BC_F16 && wdtype == BC_F16) ln_forward_any<f16_t, f16_t>(a, s);
    else if (dtype == BC_F16) ln_forward_any<f16_t, float>(a, s);
    else if (wdtype == BC_BF16) ln_forward_any<bf16_t, bf16_t>(a, s);
    else ln_forward_any<bf16_t, float>(a, s);
    return hipGetLastError();
}

hipError_t launch_ln_backward(int dtype, int wdtype, const LnBackward& a, void* dweight, void* dbias, hipStream_t s) {
    if (a.rows) {
        if (dtype == BC_F32) ln_backward_any<float, float>(a, s);
        else if (dtype == BC_F16 && wdtype == BC_F16) ln_backward_any<f16_t, f16_t>(a, s);
        else if (dtype == BC_F16) ln_backward_any<f16_t, float>(a, s);
        else if (wdtype == BC_BF16) ln_backward_any<bf16_t, bf16_t>(a, s);
        else ln_backward_any<bf16_t, float>(a, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return launch_sum_parts(wdtype, a.part, a.parts, 2ull * a.cols, a.cols, dweight, dbias, s);
}

}  // namespace bc
