// kernels_ortho.hip -- updates orthogonalised by Newton-Schulz products, for
// lists of matrices: X_0 = U / (|U| + eps) with the Frobenius norm, then
//   A = X X^T,  B = b A + c A^2,  X <- a X + B X
// `steps` times, X with its shorter side as rows; and the optimizer step around
// it (momentum before, weights after).
//
// The work is three dependent products a step.  All matrices of the call share
// each launch (a tile finds its matrix by a search in the call's table), so a
// model's list costs 3 launches a step, and small matrices fill the chip
// together.  A and B are symmetric: only tiles on and above the diagonal are
// computed, and written twice.
//
// Precision: singular values under one grow by up to a per step, and with them
// every rounding made before, so 16-bit factors are not enough (in one fp16 part
// the result of a gradient with a few dominant directions is 2% off, in bfloat16
// 18%).  Every factor is kept as two fp16 parts (22 bits) scaled by powers of
// two to the middle of fp16's range, a product is three matrix-core products
// (leading x leading, leading x rest both ways), sums are fp32: the result is as
// close to the exact one as fp32 arithmetic's.
#include "gemm.hpp"
#include "launch.hpp"
#include "layers.hpp"

namespace bc {

namespace {

// The matrix that owns workgroup b, by the running counts in field F.
template <typename F>
__device__ __forceinline__ int owner(const Ortho* d, int T, uint32_t b, F first) {
    int lo = 0, hi = T - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first(d[mid]) <= b) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ void load_any(int dtype, const void* p, uint64_t i, int left, float (&v)[8]) {
    if (dtype == BC_F32) load_vec((const float*)p + i, left, v);
    else if (dtype == BC_F16) load_vec((const f16_t*)p + i, left, v);
    else load_vec((const bf16_t*)p + i, left, v);
}
__device__ __forceinline__ void store_any(int dtype, void* p, uint64_t i, int left, const float (&v)[8]) {
    if (dtype == BC_F32) store_vec((float*)p + i, left, v);
    else if (dtype == BC_F16) store_vec((f16_t*)p + i, left, v);
    else store_vec((bf16_t*)p + i, left, v);
}

// v as two fp16 planes at p and p + plane (16-byte aligned).
__device__ __forceinline__ void store_two(f16_t* p, uint64_t plane, const float (&v)[8]) {
    f16x8 hi, lo;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        hi[i] = (f16_t)v[i];
        lo[i] = (f16_t)(v[i] - (float)hi[i]);
    }
    *(f16x8*)p = hi;
    *(f16x8*)(p + plane) = lo;
}
__device__ __forceinline__ void load_two(const f16_t* p, uint64_t plane, float (&v)[8]) {
    const f16x8 hi = *(const f16x8*)p, lo = *(const f16x8*)(p + plane);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)hi[i] + (float)lo[i];
}

// Eight elements of the update U at (r, c); first: the momentum's new value is
// made and kept (later passes find it there).
template <bool first>
__device__ __forceinline__ void load_update(const OrthoCall& a, const Ortho& o, uint64_t r, uint32_t c, int left,
                                            float (&u)[8]) {
    load_any(a.in_dtype, o.in, left ? r * o.ld_in + c : 0, left, u);
    if (!a.muon) return;
    float m[8];
    float* at = o.momentum + (left ? r * o.ld_momentum + c : 0);
    load_vec(at, left, m);
    if constexpr (first) {
#pragma unroll
        for (int i = 0; i < 8; ++i) m[i] = a.momentum * m[i] + u[i];
        store_vec(at, left, m);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = a.nesterov ? a.momentum * m[i] + u[i] : m[i];
}

// Sums of squares in fp64 (no overflow or underflow from any fp32 value): a
// workgroup adds 64 x 64 tiles a fixed step apart, threads meet in a fixed tree.
__global__ __launch_bounds__(256) void ortho_norm(OrthoCall a) {
    __shared__ double sh[4];
    const Ortho& o = a.d[owner(a.d, a.T, blockIdx.x, [](const Ortho& x) { return x.part0; })];
    const uint32_t part = blockIdx.x - o.part0;
    const uint32_t across = (o.cols + 63) / 64, tiles = across * ((o.rows + 63) / 64);
    double sum = 0.0;
    for (uint32_t t = part; t < tiles; t += o.parts) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t r = t / across * 64 + threadIdx.x / 8 + 32 * i, c = t % across * 64 + threadIdx.x % 8 * 8;
            const int left = r < o.rows && c < o.cols ? (int)(o.cols - c) : 0;
            float u[8];
            load_update<true>(a, o, r, c, left, u);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += j < left ? (double)u[j] * (double)u[j] : 0.0;
        }
    }
    const double total = block_sum_f64(sum, sh);
    if (threadIdx.x == 0) ((double*)(a.ws + o.part))[part] = total;
}

// X_0 and its transpose as planes, a workgroup a 64 x 64 tile of U (columns
// and rows past the end as zeros, as far as the planes go).
__global__ __launch_bounds__(256) void ortho_start(OrthoCall a) {
    __shared__ double sh[4];
    __shared__ float tile[64][65];
    const Ortho& o = a.d[owner(a.d, a.T, blockIdx.x, [](const Ortho& x) { return x.tile0; })];
    const double mine = threadIdx.x < o.parts ? ((const double*)(a.ws + o.part))[threadIdx.x] : 0.0;
    const float scale = (float)((double)o.x_scale / (sqrt(block_sum_f64(mine, sh)) + (double)a.eps));
    const uint32_t t = blockIdx.x - o.tile0, across = (o.cols + 63) / 64;
    const uint32_t r0 = t / across * 64, c0 = t % across * 64;
    f16_t* flat = (f16_t*)(a.ws + (o.turned ? o.xt : o.x));
    f16_t* turned = (f16_t*)(a.ws + (o.turned ? o.x : o.xt));
    const uint64_t flat_ld = plane_cols(o.cols), turned_ld = plane_cols(o.rows);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t lr = threadIdx.x / 8 + 32 * i, lc = threadIdx.x % 8 * 8, r = r0 + lr, c = c0 + lc;
        const int left = r < o.rows && c < o.cols ? (int)(o.cols - c) : 0;
        float u[8];
        load_update<false>(a, o, r, c, left, u);
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = j < left ? u[j] * scale : 0.0f;  // 0 even where scale is infinite
        if (r < o.rows) store_two(flat + r * flat_ld + c, o.rows * flat_ld, u);
#pragma unroll
        for (int j = 0; j < 8; ++j) tile[lr][lc + j] = u[j];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t lc = threadIdx.x / 8 + 32 * i, lr = threadIdx.x % 8 * 8, c = c0 + lc, r = r0 + lr;
        if (c < o.cols) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = tile[lr + j][lc];
            store_two(turned + c * turned_ld + r, o.cols * turned_ld, v);
        }
    }
}

// ----------------------------------------------------------------- products
enum Stage { kGram, kPoly, kNext, kLast };

// Writes a symmetric m x m result (kGram, kPoly): the tile, and across the
// diagonal its mirror image.
template <int stage>
struct SymmetricEpilogue {
    f16_t* out;
    const f16_t* gram;          // kPoly
    uint64_t ld, plane;
    uint32_t m, m0, n0;
    float scale, gram_factor;
    __device__ __forceinline__ void row(int row, int col, float (&v)[8]) const {
        const uint32_t r = m0 + row, c = n0 + col;
        const bool there = r < m && c < ld;
        float g[8];
        if constexpr (stage == kPoly) {
            if (there) load_two(gram + r * ld + c, plane, g);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] *= scale;
            if constexpr (stage == kPoly) v[i] += gram_factor * g[i];
            if (c + i >= m) v[i] = 0.0f;
        }
        if (there) store_two(out + r * ld + c, plane, v);
    }
    __device__ __forceinline__ void column(int row, int col, float (&v)[8]) const {
        if (m0 == n0) return;
        // rows of this tile are whole: it lies above the diagonal
        const uint32_t r = m0 + row, c = n0 + col;
        if (c < m) store_two(out + c * ld + r, plane, v);
    }
};

// X <- a X + B X and its transpose.
struct NextEpilogue {
    f16_t *x, *xt;
    uint64_t x_ld, xt_ld;
    uint32_t m, n, m0, n0;
    float a, scale;
    __device__ __forceinline__ void row(int row, int col, float (&v)[8]) const {
        const uint32_t r = m0 + row, c = n0 + col;
        const bool there = r < m && c < x_ld;
        float g[8];
        if (there) load_two(x + r * x_ld + c, m * x_ld, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = there && c + i < n ? a * g[i] + v[i] * scale : 0.0f;
        if (there) store_two(x + r * x_ld + c, m * x_ld, v);
    }
    __device__ __forceinline__ void column(int row, int col, float (&v)[8]) const {
        const uint32_t r = m0 + row, c = n0 + col;  // rows past m hold zeros
        if (c < n && r < xt_ld) store_two(xt + c * xt_ld + r, n * xt_ld, v);
    }
};

template <typename G, int stage>
__global__ __launch_bounds__(G::kThreads) void ortho_product(OrthoCall a, int which, int from) {
    extern __shared__ char lds[];
    constexpr bool symmetric = stage == kGram || stage == kPoly;
    // workgroups are dealt to the eight compute dies in turn: a die gets a run
    // of consecutive tiles
    const uint32_t total = gridDim.x, q = total / 8, rest = total % 8, die = blockIdx.x % 8;
    const uint32_t b = die * q + (die < rest ? die : rest) + blockIdx.x / 8;
    const Ortho& o = a.d[owner(a.d, a.T, b, [which](const Ortho& x) { return symmetric ? x.sym0[which] : x.full0[which]; })];
    const uint64_t mp = plane_cols(o.m), np = plane_cols(o.n);
    const f16_t* x = (const f16_t*)(a.ws + o.x);
    f16_t* xt[2] = {(f16_t*)(a.ws + o.xt), (f16_t*)(a.ws + o.xt) + 2 * o.n * mp};
    f16_t* gram = (f16_t*)(a.ws + o.gram);
    f16_t* poly = (f16_t*)(a.ws + o.poly);
    uint32_t t = b - (symmetric ? o.sym0[which] : o.full0[which]), tm, tn;
    if constexpr (symmetric) {
        tn = (uint32_t)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
        while (tn * (tn + 1) / 2 > t) --tn;
        while ((tn + 1) * (tn + 2) / 2 <= t) ++tn;
        tm = t - tn * (tn + 1) / 2;
    } else {
        const bool tall = stage == kLast && o.turned;
        const uint32_t tiles_m = ((tall ? o.n : o.m) + G::kBM - 1) / G::kBM;
        const uint32_t tiles_n = ((tall ? o.m : o.n) + G::kBN - 1) / G::kBN;
        const uint32_t band = t / (8 * tiles_n), first = band * 8;
        const uint32_t high = tiles_m - first < 8 ? tiles_m - first : 8, in = t - first * tiles_n;
        tm = first + in % high;
        tn = in / high;
    }
    const uint32_t m0 = tm * G::kBM, n0 = tn * G::kBN;
    G g;
    auto rows_of = [](const f16_t* p, uint64_t ld, uint32_t rows, uint32_t at) {
        return Operand<f16_t>{p + at * ld, (uint32_t)ld, rows * ld, rows - at};
    };
    if constexpr (stage == kGram) {
        g.multiply(rows_of(x, np, o.m, m0), rows_of(x, np, o.m, n0), (int)(np / G::kBK), lds);
        const SymmetricEpilogue<stage> e{gram, nullptr, mp, o.m * mp, o.m, m0, n0,
                                         a.gram_scale / (o.x_scale * o.x_scale), 0.0f};
        g.finish_both_ways(lds, e);
    } else if constexpr (stage == kPoly) {
        g.multiply(rows_of(gram, mp, o.m, m0), rows_of(gram, mp, o.m, n0), (int)(mp / G::kBK), lds);
        const SymmetricEpilogue<stage> e{poly, gram, mp, o.m * mp, o.m, m0, n0,
                                         a.c * a.poly_scale / (a.gram_scale * a.gram_scale),
                                         a.b * a.poly_scale / a.gram_scale};
        g.finish_both_ways(lds, e);
    } else if constexpr (stage == kNext) {
        g.multiply(rows_of(poly, mp, o.m, m0), rows_of(xt[from], mp, o.n, n0), (int)(mp / G::kBK), lds);
        const NextEpilogue e{(f16_t*)x, xt[1 - from], np, mp, o.m, o.n, m0, n0, a.a, 1.0f / a.poly_scale};
        g.finish_both_ways(lds, e);
    } else {
        // the caller's orientation: X, or X^T <- a X^T + X^T B
        const f16_t* old = o.turned ? xt[from] : x;
        const uint64_t old_ld = o.turned ? mp : np, old_plane = o.turned ? o.n * mp : o.m * np;
        if (o.turned) g.multiply(rows_of(xt[from], mp, o.n, m0), rows_of(poly, mp, o.m, n0), (int)(mp / G::kBK), lds);
        else g.multiply(rows_of(poly, mp, o.m, m0), rows_of(xt[from], mp, o.n, n0), (int)(mp / G::kBK), lds);
        const float inv = 1.0f / o.x_scale, scale = 1.0f / a.poly_scale;
        g.finish(lds, [&](int row, int col, float (&v)[8]) {
            const uint64_t r = m0 + row;
            const uint32_t c = n0 + col;
            if (r >= o.rows || c >= o.cols) return;
            const int left = (int)(o.cols - c);
            float t[8];
            load_two(old + r * old_ld + c, old_plane, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (a.a * t[i] + v[i] * scale) * inv;
            if (a.muon) {
                load_any(a.out_dtype, o.out, r * o.ld_out + c, left, t);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = a.keep * t[i] - (a.lr * o.step_scale) * v[i];
            }
            store_any(a.out_dtype, o.out, r * o.ld_out + c, left, v);
        });
    }
}

typedef GemmTile<f16_t, 2, 128, 128, 32, 2, 2, 2> Small;
typedef GemmTile<f16_t, 2, 256, 256, 32, 2, 4, 2> Large;

template <typename G, int stage>
hipError_t launch_stage(const OrthoCall& c, int which, int from, hipStream_t s) {
    const hipError_t e = hipFuncSetAttribute((const void*)ortho_product<G, stage>,
                                             hipFuncAttributeMaxDynamicSharedMemorySize, G::kLdsBytes);
    if (e != hipSuccess) return e;
    const uint32_t grid = stage == kGram || stage == kPoly ? c.sym[which] : c.full[which];
    hipLaunchKernelGGL((ortho_product<G, stage>), dim3(grid), dim3(G::kThreads), G::kLdsBytes, s, c, which, from);
    return hipGetLastError();
}

template <int stage>
hipError_t launch_tiles(const OrthoCall& c, int from, hipStream_t s) {
    // large tiles move less data per product, small ones waste less at the
    // edges and in the last round: the smaller number of rounds times a round's time
    const uint32_t* count = stage == kGram || stage == kPoly ? c.sym : c.full;
    const uint32_t slots = (uint32_t)c.cus;
    const double small = (count[0] + 2 * slots - 1) / (2 * slots) * 2 * 1.2, large = (count[1] + slots - 1) / slots * 4;
    if (large <= small) return launch_stage<Large, stage>(c, 1, from, s);
    return launch_stage<Small, stage>(c, 0, from, s);
}

}  // namespace

hipError_t launch_orthogonalize(const OrthoCall& c, hipStream_t s) {
    hipLaunchKernelGGL(ortho_norm, dim3(c.parts), dim3(256), 0, s, c);
    hipLaunchKernelGGL(ortho_start, dim3(c.tiles), dim3(256), 0, s, c);
    hipError_t e = hipGetLastError();
    for (int i = 0; i < c.steps && e == hipSuccess; ++i) {
        e = launch_tiles<kGram>(c, 0, s);
        if (e == hipSuccess) e = launch_tiles<kPoly>(c, 0, s);
        if (e == hipSuccess) e = i + 1 < c.steps ? launch_tiles<kNext>(c, i & 1, s) : launch_tiles<kLast>(c, i & 1, s);
    }
    return e;
}

}  // namespace bc
