// kernels_ortho.hip -- updates orthogonalised by Newton-Schulz products, for
// lists of matrices: X_0 = U / (|U| + eps) with the Frobenius norm, then
//   A = X X^T,  B = b A + c A^2,  X <- (a I + B) X
// `steps` times, X with its shorter side m as rows and its longer side n as
// columns; and the optimizer step around it (momentum before, weights after).
//
// Two steps can share their long products, for everything else is a polynomial
// of A, m x m and symmetric: with P = a I + B the second step's Gram matrix is
// A' = P A P, and with B' from it
//   X <- (a I + B') (a I + B) X = (a^2 I + a (B + B') + B' B) X.
// That is 3/2 m^2 n + 5/2 m^3 multiply-adds for two steps (symmetric results
// half) instead of 3 m^2 n + m^3, and one pass over X instead of two.  More than
// two steps from one Gram matrix would lose digits: A's small eigenvalues are the
// squares of X's and grow by a^2 a step, their rounding with them.  Measured error
// of the result, with that of the same steps in fp32 products: 768 x 768 1.0e-6
// (2.4e-6); under a shorter side of 64, where fp32's is 1e-6, two steps give 1.5
// to 2 times that and results in fp32 are made step by step.  (In 64-bit sums of
// fp32 products five steps from one Gram matrix lose a factor of 13 where a few
// directions dominate.)
//
// All matrices of the call share each launch (a workgroup finds its matrix and
// tile in a list made with the call's table), so a model's list costs 3 launches
// a step or 7 for two, and small matrices fill the chip together.  Of a symmetric result only
// tiles on and above the diagonal are computed, and written twice.
//
// Precision: singular values under one grow by up to a per step, and with them
// every rounding made before, so 16-bit factors are not enough (in one fp16 part
// the result of a gradient with a few dominant directions is 2% off, in bfloat16
// 18%).  Every factor is kept as two fp16 parts scaled by powers of two to the
// top of fp16's range: 22 bits of each entry, or 2^-39 of |X| where an entry is
// so small beside it that its second part falls under fp16's smallest number (one
// entry 100 times the norm of the others: 1e-7 to 2e-7 off; scaled to the middle
// of the range, a typical entry near 1, 2e-6).  A product is three matrix-core
// products (leading x leading, leading x rest both ways), sums are fp32: the
// result is as close to the exact one as fp32 arithmetic's, until one entry is
// thousands of times the rest.
#include "gemm.hpp"
#include "launch.hpp"
#include "layers.hpp"

#include <algorithm>

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

// N elements of the update U at (r, c), fetched and then made: in the first
// pass the momentum's new value is made and kept, later passes find it there.
// (Fetches of several pieces go before the first store: the compiler cannot know
// that they do not overlap.)
template <typename T, int N>
struct Update {
    float g[N], m[N];
    float* at;
    int left;
    template <bool kWhole>
    __device__ __forceinline__ void fetch(const OrthoCall& a, const Ortho& o, uint64_t r, uint32_t c, int n) {
        left = n;
        load_vec<kWhole>((const T*)o.in + (left ? r * o.ld_in + c : 0), left, g);
        if (!a.muon) return;
        at = o.momentum + (left ? r * o.ld_momentum + c : 0);
        load_vec<kWhole>(at, left, m);
    }
    template <bool first>
    __device__ __forceinline__ void make(const OrthoCall& a) {
        if (!a.muon) return;
        if constexpr (first) {
#pragma unroll
            for (int i = 0; i < N; ++i) m[i] = a.momentum * m[i] + g[i];
            store_vec(at, left, m);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] = a.nesterov ? a.momentum * m[i] + g[i] : m[i];
    }
};

// Sums of squares in fp64 (no overflow or underflow from any fp32 value): the
// workgroups of a matrix take its pieces of four elements in turn, row after
// row, threads meet in a fixed tree.  Bound by memory: 61 million elements of
// a Muon step (G and M read, M written) 133 us, 5.5 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void ortho_norm(OrthoCall a) {
    __shared__ double sh[4];
    const Ortho o = a.d[owner(a.d, a.T, blockIdx.x, [](const Ortho& x) { return x.part0; })];
    const uint32_t part = blockIdx.x - o.part0, across = (o.cols + 3) / 4;
    const uint64_t pieces = (uint64_t)o.rows * across, step = (uint64_t)o.parts * 256;
    const bool whole = o.cols % 4 == 0;
    double sum = 0.0;
    constexpr int kFetch = 2;
    for (uint64_t q = (uint64_t)part * 256 + threadIdx.x; q < pieces; q += kFetch * step) {
        Update<T, 4> u[kFetch];
#pragma unroll
        for (int f = 0; f < kFetch; ++f) {
            const uint64_t at = q + f * step;
            const uint32_t r = pieces < (1ull << 32) ? (uint32_t)at / across : (uint32_t)(at / across);
            const uint32_t c = (uint32_t)(at - (uint64_t)r * across) * 4;
            const int n = at < pieces ? (int)(o.cols - c) : 0;
            if (whole) u[f].template fetch<true>(a, o, r, c, n);
            else u[f].template fetch<false>(a, o, r, c, n);
        }
#pragma unroll
        for (int f = 0; f < kFetch; ++f) {
            u[f].template make<true>(a);
#pragma unroll
            for (int j = 0; j < 4; ++j) sum += j < u[f].left ? (double)u[f].g[j] * (double)u[f].g[j] : 0.0;
        }
    }
    const double total = block_sum_f64(sum, sh);
    if (threadIdx.x == 0) ((double*)(a.ws + o.part))[part] = total;
}

// X_0 and its transpose as planes, a workgroup a 64 x 64 tile of U (columns and
// rows past the end as zeros, as far as the planes go).  Bound by memory: the same
// step (G and M read, eight bytes an element written) 202 us, 4.9 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void ortho_start(OrthoCall a) {
    __shared__ double sh[4];
    __shared__ float tile[64][65];
    if (blockIdx.x == 0)  // nobody has met yet
        for (uint32_t i = threadIdx.x; i < a.slots; i += 256) ((uint32_t*)(a.ws + a.meet))[i] = 0;
    const Ortho o = a.d[owner(a.d, a.T, blockIdx.x, [](const Ortho& x) { return x.tile0; })];
    const double mine = threadIdx.x < o.parts ? ((const double*)(a.ws + o.part))[threadIdx.x] : 0.0;
    // The scale in two factors, the first a power of two that keeps the second and
    // their products with U in fp32's range.  (A sum so small that its scale still
    // passes that range is eps alone, of a matrix of zeros.)
    double size = sqrt(block_sum_f64(mine, sh)) + a.eps;
    const float first = size < 0x1p-100 ? 0x1p64f : size > 0x1p100 ? 0x1p-64f : 1.0f;
    size *= first;
    const double second = (double)a.x_scale / size;  // infinite for 0, NaN for NaN
    const float scale = size > 0.0 && second > (double)__FLT_MAX__ ? __FLT_MAX__ : (float)second;
    const uint32_t across = (o.cols + 63) / 64;
    f16_t* flat = (f16_t*)(a.ws + (o.turned ? o.xt : o.x));
    f16_t* turned = (f16_t*)(a.ws + (o.turned ? o.x : o.xt));
    const uint64_t flat_ld = plane_cols(o.cols), turned_ld = plane_cols(o.rows);
    const uint32_t t = blockIdx.x - o.tile0;
    const uint32_t r0 = t / across * 64, c0 = t % across * 64;
    const bool whole = o.cols % 8 == 0 || c0 + 64 <= o.cols;
    Update<T, 8> u[2];
    const uint32_t lc = threadIdx.x % 8 * 8, c = c0 + lc;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t r = r0 + threadIdx.x / 8 + 32 * i;
        const int n = r < o.rows && c < o.cols ? (int)(o.cols - c) : 0;
        if (whole) u[i].template fetch<true>(a, o, r, c, n);
        else u[i].template fetch<false>(a, o, r, c, n);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t lr = threadIdx.x / 8 + 32 * i, r = r0 + lr;
        u[i].template make<false>(a);
        float (&v)[8] = u[i].g;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < u[i].left ? v[j] * first * scale : 0.0f;  // 0 even where scale is infinite
        if (r < o.rows) store_two(flat + r * flat_ld + c, o.rows * flat_ld, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) tile[lr][lc + j] = v[j];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t tc = threadIdx.x / 8 + 32 * i, tr = threadIdx.x % 8 * 8;
        if (c0 + tc < o.cols) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = tile[tr + j][tc];
            store_two(turned + (c0 + tc) * turned_ld + r0 + tr, o.cols * turned_ld, v);
        }
    }
}

// ----------------------------------------------------------------- products
enum Stage { kGram, kSym, kNext, kLast };

// What a launch computes: kSym: matrix `out` = alpha U V + beta U + gamma V of
// the symmetric matrices u and v; kGram: matrix `out`, kNext and kLast:
// X <- alpha X + beta U X, X^T read from its copy `from`.  The factors contain
// the scales of what they multiply.
struct StageArgs {
    int u, v, out, from;
    float alpha, beta, gamma;
};

// Writes a symmetric m x m result: the tile, and across the diagonal its
// mirror image.
struct SymmetricEpilogue {
    f16_t* out;
    const f16_t *u, *v;         // NULL where their factor is 0
    uint64_t ld, plane;
    uint32_t m, m0, n0;
    float alpha, beta, gamma;
    __device__ __forceinline__ void row(int row, int col, float (&x)[8]) const {
        const uint32_t r = m0 + row, c = n0 + col;
        const bool there = r < m && c < ld;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= alpha;
        if (there) {
            float g[8];
            if (u) {
                load_two(u + r * ld + c, plane, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] += beta * g[i];
            }
            if (v) {
                load_two(v + r * ld + c, plane, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] += gamma * g[i];
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i >= m) x[i] = 0.0f;
        if (there) store_two(out + r * ld + c, plane, x);
    }
    __device__ __forceinline__ void column(int row, int col, float (&x)[8]) const {
        if (m0 == n0) return;
        // rows of this tile are whole: it lies above the diagonal
        const uint32_t r = m0 + row, c = n0 + col;
        if (c < m) store_two(out + c * ld + r, plane, x);
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

// The sums of a tile's parts along k: each workgroup leaves its own in its slot
// and counts itself; the last one gets all of them, added in the order of the
// parts, and goes on (true).  Nobody waits.  (The release costs three of 512 x 4608
// with one of 2048 x 512 2.5%, 326 us against 317 where the stores' own way past the
// L2 and the wait alone order them.)
template <typename G>
__device__ __forceinline__ bool meet(G& g, const OrthoCall& a, const OrthoWork& w, char* lds) {
    constexpr uint32_t kTile = G::kBM * G::kBN;
    static_assert(kTile * sizeof(float) == kOrthoSlotBytes, "a slot holds a tile");
    uint32_t* met = (uint32_t*)(a.ws + a.meet) + w.met;
    float* sums = (float*)(a.ws + a.meet + kOrthoSlots * sizeof(uint32_t)) + (uint64_t)w.sums * kTile + threadIdx.x;
#pragma unroll
    for (int r = 0; r < 16; ++r)
        __hip_atomic_store(sums + w.part * kTile + r * G::kThreads, g.acc[0][0][r], __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's sums have left for where every die sees them
    __syncthreads();
    if (threadIdx.x == 0) {
        // releases the sums of the workgroup, which the barrier has put before it, and
        // acquires the others'
        const bool last = __hip_atomic_fetch_add(met, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) + 1 == w.parts;
        if (last) __hip_atomic_store(met, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // for the next launch
        *(uint32_t*)lds = last;
    }
    __syncthreads();
    const bool last = *(const uint32_t*)lds != 0;
    __syncthreads();  // the epilogue writes LDS
    if (!last) return false;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
#pragma unroll
    for (int r = 0; r < 16; ++r) g.acc[0][0][r] = sums[r * G::kThreads];
    for (uint32_t q = 1; q < w.parts; ++q)
#pragma unroll
        for (int r = 0; r < 16; ++r) g.acc[0][0][r] += sums[q * kTile + r * G::kThreads];
    return true;
}

// The product's tile, or this workgroup's part of it; whether to go on with it.
template <typename G>
__device__ __forceinline__ bool multiply(G& g, const OrthoCall& a, const OrthoWork& w, Operand<f16_t> u,
                                         Operand<f16_t> v, uint64_t k, char* lds) {
    const uint32_t steps = (uint32_t)(k / G::kBK);
    if constexpr (G::kBM == 64) {
        const uint32_t from = steps * w.part / w.parts, to = steps * (w.part + 1) / w.parts;
        u.p += from * G::kBK;
        v.p += from * G::kBK;
        g.multiply(u, v, (int)(to - from), lds);
        return w.parts == 1 || meet(g, a, w, lds);
    } else {
        g.multiply(u, v, (int)steps, lds);
        return true;
    }
}

// One tile of one product of one matrix (or a part of it along k).  Bound by the
// matrix cores on large matrices (a long product of two GPT-2-XL blocks, 5.9e11
// 16-bit operations, 820 us: 720 TFLOP/s with its epilogue), by the chain of a tile's steps and
// the launch on small ones (768 x 768: 9 to 11 us a product).
template <typename G, int stage>
__global__ __launch_bounds__(G::kThreads) void ortho_product(OrthoCall a, StageArgs s,
                                                             const OrthoWork* __restrict__ list) {
    extern __shared__ char lds[];
    constexpr bool symmetric = stage == kGram || stage == kSym;
    const OrthoWork work = list[blockIdx.x];
    if (work.matrix == kOrthoIdle) return;
    const uint32_t m = work.m, n = work.n;
    const uint64_t mp = plane_cols(m), np = plane_cols(n);
    f16_t* x = (f16_t*)(a.ws + ((uint64_t)work.x << 8));
    f16_t* xt[2];
    xt[0] = (f16_t*)(a.ws + ((uint64_t)work.xt << 8));
    xt[1] = xt[0] + 2 * n * mp;
    auto sym = [&](int i) { return (f16_t*)(a.ws + ((uint64_t)work.sym << 8)) + i * (2 * m * mp); };
    const bool tall = stage == kLast && a.d[work.matrix].turned;
    const uint32_t t = work.tile;
    uint32_t tm, tn;
    if constexpr (symmetric) {
        tn = (uint32_t)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
        while (tn * (tn + 1) / 2 > t) --tn;
        while ((tn + 1) * (tn + 2) / 2 <= t) ++tn;
        tm = t - tn * (tn + 1) / 2;
    } else {
        const uint32_t tiles_m = ((tall ? n : m) + G::kBM - 1) / G::kBM;
        const uint32_t tiles_n = ((tall ? m : n) + G::kBN - 1) / G::kBN;
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
        if (!multiply(g, a, work, rows_of(x, np, m, m0), rows_of(x, np, m, n0), np, lds)) return;
        const SymmetricEpilogue e{sym(s.out), nullptr, nullptr, mp, m * mp, m, m0, n0,
                                  s.alpha, 0.0f, 0.0f};
        g.finish_both_ways(lds, e);
    } else if constexpr (stage == kSym) {
        if (!multiply(g, a, work, rows_of(sym(s.u), mp, m, m0), rows_of(sym(s.v), mp, m, n0), mp, lds)) return;
        const SymmetricEpilogue e{sym(s.out), s.beta != 0.0f ? sym(s.u) : nullptr,
                                  s.gamma != 0.0f ? sym(s.v) : nullptr, mp, m * mp, m, m0, n0,
                                  s.alpha, s.beta, s.gamma};
        g.finish_both_ways(lds, e);
    } else if constexpr (stage == kNext) {
        if (!multiply(g, a, work, rows_of(sym(s.u), mp, m, m0), rows_of(xt[s.from], mp, n, n0), mp, lds)) return;
        const NextEpilogue e{x, xt[1 - s.from], np, mp, m, n, m0, n0, s.alpha, s.beta};
        g.finish_both_ways(lds, e);
    } else {
        // the caller's orientation: X, or its transpose, whose product is X^T U
        const Ortho o = a.d[work.matrix];
        const f16_t* old = tall ? xt[s.from] : x;
        const uint64_t old_ld = tall ? mp : np, old_plane = tall ? n * mp : m * np;
        const Operand<f16_t> u = tall ? rows_of(old, mp, n, m0) : rows_of(sym(s.u), mp, m, m0);
        const Operand<f16_t> v = tall ? rows_of(sym(s.u), mp, m, n0) : rows_of(xt[s.from], mp, n, n0);
        if (!multiply(g, a, work, u, v, mp, lds)) return;
        g.finish(lds, [&](int row, int col, float (&v)[8]) {
            const uint64_t r = m0 + row;
            const uint32_t c = n0 + col;
            if (r >= o.rows || c >= o.cols) return;
            const int left = (int)(o.cols - c);
            float t[8];
            load_two(old + r * old_ld + c, old_plane, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = s.alpha * t[i] + v[i] * s.beta;
            if (a.muon) {
                load_any(a.out_dtype, o.out, r * o.ld_out + c, left, t);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = a.keep * t[i] - (a.lr * o.step_scale) * v[i];
            }
            store_any(a.out_dtype, o.out, r * o.ld_out + c, left, v);
        });
    }
}

// Tile shapes and the model that picks among them (us): a tile's time for 32
// along k with its compute unit to itself, and a compute unit's share of it when
// the chip is full; a tile's start and epilogue.  From products of 768 x 768 x 768
// to 4096 x 4096 x 6400; a launch ends, on average, half a tile after its mean.
typedef GemmTile<f16_t, 2, 64, 64, 64, 2, 2, 2> Tile64;
typedef GemmTile<f16_t, 2, 64, 64, 64, 2, 2, 3> Tile64Deep;
typedef GemmTile<f16_t, 2, 128, 128, 64, 2, 4, 2> Tile128;
typedef GemmTile<f16_t, 2, 256, 256, 32, 2, 4, 2> Tile256;
constexpr double kAlone[kOrthoSides] = {0.32, 0.50, 1.55}, kFull[kOrthoSides] = {0.21, 0.63, 2.2};
constexpr double kEnds[kOrthoSides] = {1.5, 6.0, 40.0};
constexpr double kLaunch = 3.0, kMeet = 2.5;

double time_of(const OrthoLoad& l, int side, double chain, int cus) {
    const bool cut = side == 0 && l.longest > chain;
    const double longest = cut ? chain : l.longest, ends = kEnds[side] + (cut ? kMeet : 0.0);
    const double alone = longest * kAlone[side] + ends;
    const double full = (l.steps * kFull[side] + l.tiles * kEnds[side]) / cus;
    return kLaunch + std::max(alone, full + 0.5 * (longest * kFull[side] + ends));
}

template <typename G, int stage>
hipError_t launch_tiles(const OrthoCall& c, const OrthoGroup& g, int kind, const StageArgs& a, hipStream_t s) {
    // more LDS than a kernel may use by default; the attribute is per device
    // and setting it again costs next to nothing
    const hipError_t e = hipFuncSetAttribute((const void*)ortho_product<G, stage>,
                                             hipFuncAttributeMaxDynamicSharedMemorySize, G::kLdsBytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((ortho_product<G, stage>), dim3(g.workgroups[kind]), dim3(G::kThreads), G::kLdsBytes, s, c, a,
                       g.list[kind]);
    return hipGetLastError();
}

template <int stage>
hipError_t launch_stage(const OrthoPlan& p, const OrthoGroup& g, const StageArgs& a, hipStream_t s) {
    constexpr int kind = stage == kGram ? kOrthoGram : stage == kSym ? kOrthoSym : kOrthoFull;
    // A compute unit holds two workgroups of Tile64 or one of Tile64Deep, whose
    // loads run further ahead: one 768 x 768 matrix (144 tiles) 156 us against 184,
    // but ResNet-50's list, which has more tiles than units, 1% slower.
    if (g.side[kind] == 0 && g.workgroups[kind] <= (uint32_t)p.cus)
        return launch_tiles<Tile64Deep, stage>(p.c, g, kind, a, s);
    if (g.side[kind] == 0) return launch_tiles<Tile64, stage>(p.c, g, kind, a, s);
    if (g.side[kind] == 1) return launch_tiles<Tile128, stage>(p.c, g, kind, a, s);
    return launch_tiles<Tile256, stage>(p.c, g, kind, a, s);
}

template <typename T>
hipError_t launch_start(const OrthoPlan& p, hipStream_t s) {
    hipLaunchKernelGGL(ortho_norm<T>, dim3(p.c.parts), dim3(256), 0, s, p.c);
    hipLaunchKernelGGL(ortho_start<T>, dim3(p.c.tiles), dim3(256), 0, s, p.c);
    return hipGetLastError();
}

}  // namespace

void ortho_choose(OrthoGroup& g, bool may_pair, int cus) {
    double time[kOrthoKinds];
    for (int kind = 0; kind < kOrthoKinds; ++kind) {
        for (int i = 0; i < kOrthoSides; ++i) {
            const double t = time_of(g.load[kind][i], i, g.chain[kind], cus);
            if (i > 0 && !(t < time[kind])) continue;
            g.side[kind] = i;
            time[kind] = t;
        }
    }
    g.pairs = may_pair && 4 * time[kOrthoSym] + time[kOrthoFull] + time[kOrthoGram] + time[kOrthoSym] <
                              2 * (time[kOrthoGram] + time[kOrthoSym] + time[kOrthoFull]);
}

hipError_t launch_orthogonalize(const OrthoPlan& p, hipStream_t s) {
    const OrthoCall& c = p.c;
    hipError_t e = c.in_dtype == BC_F32   ? launch_start<float>(p, s)
                   : c.in_dtype == BC_F16 ? launch_start<f16_t>(p, s)
                                          : launch_start<bf16_t>(p, s);
    for (const OrthoGroup& g : p.group) {
        if (g.workgroups[kOrthoFull] == 0) continue;
        // out = alpha U V + beta U + gamma V, each matrix with the scale of its kind
        auto sym = [&](int u, SymScale ku, int v, SymScale kv, int out, SymScale ko, float alpha, float beta, float gamma) {
            const float *k = c.scale, to = k[ko];
            if (e == hipSuccess)
                e = launch_stage<kSym>(p, g, StageArgs{u, v, out, 0, alpha * to / (k[ku] * k[kv]), beta * to / k[ku],
                                                       gamma * to / k[kv]}, s);
        };
        int from = 0;
        for (int left = p.steps; left > 0 && e == hipSuccess;) {
            const bool two = g.pairs && left >= 2;
            e = launch_stage<kGram>(p, g, StageArgs{0, 0, 0, 0, c.scale[kScaleGram] / (c.x_scale * c.x_scale), 0.0f, 0.0f}, s);
            sym(0, kScaleGram, 0, kScaleGram, 1, kScalePoly, c.c, c.b, 0.0f);             // 1: B
            StageArgs next{1, 0, 0, from, c.a, 1.0f / c.scale[kScalePoly], 0.0f};
            if (two) {
                sym(1, kScalePoly, 0, kScaleGram, 2, kScaleTurn, 1.0f, 0.0f, c.a);        // 2: P A
                sym(2, kScaleTurn, 1, kScalePoly, 0, kScaleGram, 1.0f, c.a, 0.0f);        // 0: A' = P A P
                sym(0, kScaleGram, 0, kScaleGram, 2, kScalePoly, c.c, c.b, 0.0f);         // 2: B'
                sym(2, kScalePoly, 1, kScalePoly, 0, kScalePair, 1.0f, c.a, c.a);         // 0: B' B + a (B + B')
                next = StageArgs{0, 0, 0, from, c.a * c.a, 1.0f / c.scale[kScalePair], 0.0f};
            }
            left -= two ? 2 : 1;
            if (left == 0) {  // the caller's X has no scale
                next.alpha /= c.x_scale;
                next.beta /= c.x_scale;
            }
            if (e == hipSuccess)
                e = left > 0 ? launch_stage<kNext>(p, g, next, s) : launch_stage<kLast>(p, g, next, s);
            from = 1 - from;
        }
    }
    return e;
}

}  // namespace bc
