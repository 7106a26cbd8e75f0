// kernels_grouped.hip -- the linear layer grouped by expert: rows in runs, one run
// an expert, each expert with a weight of its own,
//   z = x w_e^T + bias_e,  y = act(z);  dz = dy act'(z),
//   dx = dz w_e,  dw_e = dz_e^T x_e,  dbias_e = sum over the expert's rows of dz.
//
// Where the runs begin is known to the device alone.  A launch has a workgroup
// for every tile that there can be; a tile finds its expert among the offsets by
// comparisons (experts.hpp), and those without rows end at once.  No operand is
// turned in memory: dx takes w and dw takes dz and x with k down their columns
// (run_tile.hpp).  16-bit operands are read where they lie, x through `source` if
// it is given; fp32 ones are laid out as three bfloat16 planes, as
// kernels_linear.hip does it.
#include "act.hpp"
#include "experts.hpp"
#include "launch.hpp"
#include "run_tile.hpp"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace bc {

namespace {

// ------------------------------------------------------------- whose tile
__device__ __forceinline__ uint32_t bounded(int32_t x, uint32_t rows) {
    return x < 0 ? 0 : (uint32_t)x < rows ? (uint32_t)x : rows;
}
__device__ __forceinline__ uint32_t offset_of(const Groups& g, uint32_t e) { return bounded(g.offsets[e], g.rows); }

// Tiles `kHigh` rows high before expert e's, from the offsets of the first
// expert and of this one.
template <uint32_t kHigh>
__device__ __forceinline__ uint32_t tiles_before(uint32_t first, uint32_t at, uint32_t e) { return at / kHigh - first / kHigh + e; }

// The rows of tile t: expert, first row, one past the expert's last.  False: none.
// The same in all lanes of a wave.
struct Run {
    uint32_t expert, from, to;
};
template <uint32_t kHigh>
__device__ __forceinline__ bool run_of(const Groups& g, uint32_t t, Run& r) {
    const uint32_t lane = threadIdx.x & 63, first = offset_of(g, 0);
    uint32_t n = 0;
    for (uint32_t e0 = 0; e0 < g.experts; e0 += 64) {
        const uint32_t e = e0 + lane;
        const bool before = e < g.experts && tiles_before<kHigh>(first, offset_of(g, e), e) <= t;
        n += __popcll(__ballot(before));
    }
    r.expert = __builtin_amdgcn_readfirstlane(n > 0 ? n - 1 : 0);
    const uint32_t at = offset_of(g, r.expert), to = offset_of(g, r.expert + 1);
    const uint32_t before = tiles_before<kHigh>(first, at, r.expert);
    r.from = at + (t - before) * kHigh;
    r.to = to;
    // (offsets that do not ascend give no rows, or rows of the call's)
    return t >= before && r.from >= at && r.from < to;
}

// The tiles there are, given the offsets.
template <uint32_t kHigh>
__device__ __forceinline__ uint32_t tiles_in_all(const Groups& g) {
    const uint32_t first = offset_of(g, 0), last = offset_of(g, g.experts);
    return tiles_before<kHigh>(first, last < first ? first : last, g.experts);
}

// ----------------------------------------------------------------- products
// Eight columns of a row of the result from the fp32 sums v.
template <typename TO, bool forward>
__device__ __forceinline__ void finish_row(const GroupedProduct& p, uint32_t e, uint64_t m, uint32_t n, float (&v)[8]) {
    constexpr bool exact = sizeof(TO) == 4;
    const int left = (int)(p.cols - n);
    if constexpr (forward) {
        if (p.bias) {
            float t[8];
            load_vec((const TO*)p.bias + e * p.ld_bias + n, left, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += t[i];
        }
        if (p.z) store_vec((TO*)p.z + m * p.ld_z + n, left, v, p.nt);
        if (p.act != BC_ACT_NONE)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = activate<exact>(p.act, v[i]);
    }
    store_vec((TO*)p.out + m * p.ld_out + n, left, v, p.nt);
}

// The experts' rows times their weight: forward with k along the rows of both,
// for dx with k down the columns of w.
template <typename G, typename TO, bool forward>
__global__ __launch_bounds__(G::kThreads) void rows_product(GroupedProduct p) {
    typedef RunTile<G, false, !forward> R;
    typedef typename G::T T;
    extern __shared__ char lds[];
    const uint32_t tiles_n = (p.cols + G::kBN - 1) / G::kBN, tiles_m = tiles_in_all<G::kBM>(p.g);
    if (blockIdx.x >= tiles_m * tiles_n) return;
    uint32_t tm, tn;
    tile_of<8>(blockIdx.x, tiles_m, tiles_n, tm, tn);
    Run run;
    if (!run_of<G::kBM>(p.g, tm, run)) return;
    const uint32_t m0 = run.from, n0 = tn * G::kBN;
    const bool gather = forward && p.source;
    const Side<T> a{(const T*)p.a.p + (gather ? 0 : m0 * p.a.ld), p.a.plane, (uint32_t)p.a.ld, run.to - m0};
    const Side<T> b{(const T*)p.b.p + run.expert * p.b.expert + (forward ? n0 * p.b.ld : n0), p.b.plane, (uint32_t)p.b.ld,
                    p.cols - n0};
    R g;
    g.template multiply<false>(a, b, p.k, lds, [&](int r) -> uint32_t {
        if (!gather) return (uint32_t)r * (uint32_t)p.a.ld * 2;
        const uint32_t row = (uint32_t)p.source[m0 + r];
        return row < p.a_rows ? row * (uint32_t)p.a.ld * 2 : kNowhere;
    }, nullptr);
    g.finish(lds, [&](int row, int col, float (&v)[8]) {
        const uint32_t m = m0 + row, n = n0 + col;
        if (m < run.to && n < p.cols) finish_row<TO, forward>(p, run.expert, m, n, v);
    });
}

// dw: every expert's tiles, over its rows.
template <typename G, typename TO, bool kTable>
__global__ __launch_bounds__(G::kThreads) void weights_product(GroupedProduct p) {
    typedef RunTile<G, true, true> R;
    typedef typename G::T T;
    extern __shared__ char lds[];
    const uint32_t tiles_m = (p.rows + G::kBM - 1) / G::kBM, tiles_n = (p.cols + G::kBN - 1) / G::kBN;
    // a die works on one expert at a time: its tiles one after the other
    const uint32_t each = tiles_m * tiles_n, total = each * p.g.experts, q = total / 8, rest = total % 8;
    const uint32_t die = blockIdx.x % 8, t = die * q + (die < rest ? die : rest) + blockIdx.x / 8;
    const uint32_t e = t / each, in = t - e * each, tm = in / tiles_n, tn = in - tm * tiles_n;
    const uint32_t first = offset_of(p.g, 0), from = offset_of(p.g, e), to = offset_of(p.g, e + 1);
    const uint32_t m0 = tm * G::kBM, n0 = tn * G::kBN;
    const Side<T> a{(const T*)p.a.p + (uint64_t)from * p.a.ld + m0, p.a.plane, (uint32_t)p.a.ld, p.rows - m0};
    const Side<T> b{(const T*)p.b.p + (kTable ? 0 : (uint64_t)from * p.b.ld) + n0, p.b.plane, (uint32_t)p.b.ld, p.cols - n0};
    const uint32_t* where = kTable ? p.where + (uint64_t)tiles_before<64>(first, from, e) * 64 : nullptr;
    // (offsets that do not ascend: no rows)
    R g;
    g.template multiply<kTable>(a, b, to > from && from >= first ? to - from : 0, lds, [](int) { return 0u; }, where);
    g.finish(lds, [&](int row, int col, float (&v)[8]) {
        const uint32_t m = m0 + row, n = n0 + col;
        if (m < p.rows && n < p.cols)
            store_vec((TO*)p.out + e * p.expert_out + m * p.ld_out + n, (int)(p.cols - n), v, p.nt);
    });
}

// Tile shapes, small to large.
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

template <typename G>
hipError_t launch_tiles(const void* kernel, const GroupedProduct& p, uint64_t grid, hipStream_t s) {
    hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, G::kLdsBytes);
    if (e != hipSuccess) return e;
    if (grid * G::kThreads >= (1ull << 32)) return hipErrorInvalidValue;
    void* args[] = {(void*)&p};
    return hipLaunchKernel(kernel, dim3((uint32_t)grid), dim3(G::kThreads), args, G::kLdsBytes, s);
}

template <typename G, typename TO>
hipError_t launch_kind(int kind, const GroupedProduct& p, hipStream_t s) {
    const uint64_t across = (p.cols + G::kBN - 1) / G::kBN;
    if (kind == kGroupedWeights) {
        const uint64_t grid = (uint64_t)p.g.experts * ((p.rows + G::kBM - 1) / G::kBM) * across;
        if (p.where) return launch_tiles<G>((const void*)weights_product<G, TO, true>, p, grid, s);
        return launch_tiles<G>((const void*)weights_product<G, TO, false>, p, grid, s);
    }
    const uint64_t grid = group_tiles(p.g.rows, p.g.experts, G::kBM) * across;
    if constexpr (std::is_same_v<TO, typename G::T> || G::P > 1) {
        if (kind == kGroupedForward) return launch_tiles<G>((const void*)rows_product<G, TO, true>, p, grid, s);
        return launch_tiles<G>((const void*)rows_product<G, TO, false>, p, grid, s);
    }
    return hipErrorInvalidValue;
}

// What a tile costs (us), as in kernels_linear.hip: 64 along k alone on its
// compute unit and on a full chip, and its start and epilogue.
struct TileCost {
    uint32_t rows, cols;
    double alone, full, ends;
};
constexpr TileCost kCost16[3] = {{64, 64, 0.30, 0.193, 0.5}, {128, 128, 0.60, 0.53, 2.0}, {256, 256, 1.05, 1.50, 11.0}};
constexpr TileCost kCost32[3] = {{64, 64, 0.82, 0.95, 0.5}, {128, 128, 1.86, 2.56, 1.5}, {256, 128, 3.4, 4.68, 8.7}};

int tile_for(int kind, int dtype, const GroupedProduct& p) {
    const TileCost* cost = dtype == BC_F32 ? kCost32 : kCost16;
    int best = 0;
    double least = 1e300;
    for (int i = 0; i < 3; ++i) {
        const TileCost& c = cost[i];
        const double rows = (double)p.g.rows, experts = (double)p.g.experts;
        const double across = std::ceil((double)p.cols / c.cols);
        double tiles, k;
        if (kind == kGroupedWeights) {
            tiles = experts * std::ceil((double)p.rows / c.rows) * across;
            k = rows / experts;
        } else {
            // half a tile of every run is past its end
            tiles = (rows / c.rows + std::fmin(experts, rows) * 0.5) * across;
            k = (double)p.k;
        }
        const double steps = std::ceil(k / 64.0), full = steps * c.full + c.ends, n = tiles / 256.0;
        const double busy = i == 2 ? std::ceil(n) * full : n <= 1.0 ? 0.0 : (n + 0.5) * full;
        const double t = std::fmax(steps * c.alone + c.ends, busy);
        if (t < least) {
            least = t;
            best = i;
        }
    }
    return best;
}

template <typename T, typename TO>
hipError_t launch_tile(int kind, int tile, const GroupedProduct& p, hipStream_t s) {
    if (tile == 0) return launch_kind<typename Tiles<T>::Small, TO>(kind, p, s);
    if (tile == 1) return launch_kind<typename Tiles<T>::Middle, TO>(kind, p, s);
    return launch_kind<typename Tiles<T>::Large, TO>(kind, p, s);
}

// ----------------------------------------------------------------- few rows
// The i-th expert that has rows, or -1.  The same in all lanes of a wave.
__device__ __forceinline__ int busy_expert(const Groups& g, uint32_t i, uint32_t& from, uint32_t& to) {
    const uint32_t lane = threadIdx.x & 63;
    for (uint32_t e0 = 0; e0 < g.experts; e0 += 64) {
        const uint32_t e = e0 + lane;
        uint32_t a = 0, b = 0;
        if (e < g.experts) {
            a = offset_of(g, e);
            b = offset_of(g, e + 1);
        }
        uint64_t busy = __ballot(b > a);
        const uint32_t n = (uint32_t)__popcll(busy);
        if (i < n) {
            for (; i > 0; --i) busy &= busy - 1;
            const int at = __builtin_ctzll(busy);
            from = (uint32_t)__builtin_amdgcn_readlane((int)a, at);
            to = (uint32_t)__builtin_amdgcn_readlane((int)b, at);
            return (int)(e0 + at);
        }
        i -= n;
    }
    return -1;
}

// A wave a row of w, kRows of the expert's rows at a time: products and sums in fp32.
constexpr int kFewAtOnce = 4;
template <typename T, bool kWhole>
__global__ __launch_bounds__(256) void grouped_few(GroupedFew a) {
    constexpr int V = kVec<T>, kFetch = kWhole ? 4 : 2;
    const int lane = threadIdx.x & 63;
    const uint32_t c = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t from, to;
    const int e = busy_expert(a.g, blockIdx.y, from, to);
    if (e < 0 || c >= a.cols) return;
    const T* w = (const T*)a.w + (uint32_t)e * a.expert_w + (uint64_t)c * a.ldw;
    for (uint32_t r0 = from; r0 < to; r0 += kFewAtOnce) {
        const T* x[kFewAtOnce];
        float acc[kFewAtOnce];
        bool there[kFewAtOnce];
#pragma unroll
        for (int m = 0; m < kFewAtOnce; ++m) {
            const uint32_t r = r0 + m < to ? r0 + m : r0;
            const uint32_t row = a.source ? (uint32_t)a.source[r] : r;
            there[m] = row < a.x_rows;  // a row from nowhere is zeros
            x[m] = (const T*)a.x + (uint64_t)(there[m] ? row : 0) * a.ldx;
            acc[m] = 0.0f;
        }
        auto rows = [&](auto count) {
            constexpr int kRows = decltype(count)::value;
            for (uint32_t k0 = 0; k0 < a.inner; k0 += kFetch * 64 * V) {
                Raw<T, V> fw[kFetch], fx[kFetch][kRows];
#pragma unroll
                for (int u = 0; u < kFetch; ++u) {
                    const uint32_t k = k0 + (u * 64 + lane) * V;
                    const int left = k < a.inner ? (int)(a.inner - k) : 0;
                    fw[u].template load<kWhole>(w + (left ? k : 0), left);
#pragma unroll
                    for (int m = 0; m < kRows; ++m) fx[u][m].template load<kWhole>(x[m] + (left ? k : 0), there[m] ? left : 0);
                }
#pragma unroll
                for (int u = 0; u < kFetch; ++u)
#pragma unroll
                    for (int m = 0; m < kRows; ++m)
#pragma unroll
                        for (int i = 0; i < V; ++i) acc[m] = fmaf((float)fw[u].v[i], (float)fx[u][m].v[i], acc[m]);
            }
        };
        if (to - r0 == 1) rows(std::integral_constant<int, 1>{});
        else if (to - r0 == 2) rows(std::integral_constant<int, 2>{});
        else rows(std::integral_constant<int, kFewAtOnce>{});
#pragma unroll
        for (int m = 0; m < kFewAtOnce; ++m) acc[m] = wave_sum(acc[m]);
        float v = acc[0];
#pragma unroll
        for (int m = 1; m < kFewAtOnce; ++m) v = lane == m ? acc[m] : v;
        const uint64_t r = r0 + lane;
        if (lane < kFewAtOnce && r < to) {
            if (a.bias) v += (float)((const T*)a.bias)[(uint32_t)e * a.ld_bias + c];
            if (a.z) ((T*)a.z)[r * a.ldz + c] = (T)v;
            ((T*)a.y)[r * a.ldy + c] = (T)activate<sizeof(T) == 4>(a.act, v);
        }
    }
}

// ---------------------------------------------------- what products are given
template <typename T>
__global__ __launch_bounds__(256) void lay_rows(LayRows a) {
    typedef typename PlaneOf<T>::type E;
    const uint64_t ld = plane_cols(a.cols), across = ld / 8, step = (uint64_t)gridDim.x * 256;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < a.count * across; i += step) {
        const uint64_t r = i / across;
        const uint32_t c = (uint32_t)(i - r * across) * 8;
        uint64_t at;
        bool there = c < a.cols;
        if (a.source) {
            const uint32_t row = (uint32_t)a.source[r];
            there = there && row < a.in_rows;
            at = row * a.ld;
        } else {
            const uint64_t m = r / a.group;
            at = m * a.matrix + (r - m * a.group) * a.ld;
        }
        float v[8];
        load_vec((const T*)a.in + (there ? at + c : 0), there ? (int)(a.cols - c) : 0, v);
        store_planes<T>((E*)a.out + r * ld + c, a.count * ld, v);
    }
}

// A workgroup 64 rows of one expert by 64 columns.
template <typename T>
__global__ __launch_bounds__(256) void grouped_slope(GroupedSlope a) {
    typedef typename PlaneOf<T>::type E;
    __shared__ float sums[4][64];
    Run run;
    const uint64_t ld = plane_cols(a.cols);
    const uint32_t across = (uint32_t)(ld / 64), tile = blockIdx.x / across, c0 = blockIdx.x % across * 64;
    const bool some = run_of<64>(a.g, tile, run);
    const uint32_t lc = threadIdx.x % 8 * 8, c = c0 + lc;
    float sum[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
    if (some) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint64_t r = run.from + threadIdx.x / 8 + 32 * i;
            const int left = r < run.to && c < a.cols ? (int)(a.cols - c) : 0;
            float v[8], z[8];
            load_vec((const T*)a.dy + (left > 0 ? r * a.ldd + c : 0), left, v);
            if (a.z) {
                load_vec((const T*)a.z + (left > 0 ? r * a.ldz + c : 0), left, z);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = j < left ? v[j] * act_slope<sizeof(T) == 4>(a.act, z[j]) : 0.0f;
            }
            if (a.dz && r < run.to) store_planes<T>((E*)a.dz + r * ld + c, (uint64_t)a.g.rows * ld, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += v[j];
        }
    }
    if (!a.part) return;
    // rows of the same columns: lanes eight apart, then the waves
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int o = 8; o < 64; o <<= 1) sum[j] += __shfl_xor(sum[j], o, 64);
    if ((threadIdx.x & 63) < 8)
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[threadIdx.x >> 6][lc + j] = sum[j];
    __syncthreads();
    const uint32_t col = c0 + threadIdx.x;
    if (threadIdx.x < 64 && col < a.cols)
        a.part[(uint64_t)tile * a.cols + col] =
            (sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]);
}

template <typename TO>
__global__ __launch_bounds__(256) void grouped_bias(GroupedSlope a, TO* out, uint64_t ld) {
    const uint32_t c = blockIdx.x * 256 + threadIdx.x, e = blockIdx.y;
    if (c >= a.cols) return;
    const uint32_t first = offset_of(a.g, 0), from = offset_of(a.g, e), to = offset_of(a.g, e + 1);
    float sum = 0.0f;
    if (from >= first && to > from) {
        const uint32_t t0 = tiles_before<64>(first, from, e), n = (to - from + 63) / 64;
        for (uint32_t t = 0; t < n; ++t) sum += a.part[(uint64_t)(t0 + t) * a.cols + c];
    }
    out[e * ld + c] = (TO)sum;
}

__global__ __launch_bounds__(256) void grouped_where(GroupedWhere a) {
    const uint32_t i = blockIdx.x * 256 + threadIdx.x;
    Run run;
    uint32_t at = kNowhere;
    if (run_of<64>(a.g, i / 64, run) && run.from + i % 64 < run.to) {
        const uint32_t row = (uint32_t)a.source[run.from + i % 64];
        if (row < a.x_rows) at = row * a.ld * 2;
    }
    if (i < 64 * (group_tiles(a.g.rows, a.g.experts, 64) + 1)) a.where[i] = at;
}

}  // namespace

hipError_t launch_grouped(int kind, int dtype, int out_dtype, const GroupedProduct& p, hipStream_t s) {
    if (p.cols == 0 || (kind == kGroupedWeights ? p.rows == 0 || p.g.experts == 0 : p.g.rows == 0)) return hipSuccess;
    const int t = tile_for(kind, dtype, p);
    if (dtype == BC_F32) return launch_tile<float, float>(kind, t, p, s);
    if (dtype == BC_F16) {
        if (out_dtype == BC_F32) return launch_tile<f16_t, float>(kind, t, p, s);
        return launch_tile<f16_t, f16_t>(kind, t, p, s);
    }
    if (out_dtype == BC_F32) return launch_tile<bf16_t, float>(kind, t, p, s);
    return launch_tile<bf16_t, bf16_t>(kind, t, p, s);
}

template <typename T>
static void few_of(const GroupedFew& a, hipStream_t s) {
    const dim3 grid((a.cols + 3) / 4, std::min(a.g.experts, a.g.rows));
    if (a.inner % kVec<T> == 0) hipLaunchKernelGGL((grouped_few<T, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((grouped_few<T, false>), grid, dim3(256), 0, s, a);
}

hipError_t launch_grouped_few(int dtype, const GroupedFew& a, hipStream_t s) {
    if (dtype == BC_F32) few_of<float>(a, s);
    else if (dtype == BC_F16) few_of<f16_t>(a, s);
    else few_of<bf16_t>(a, s);
    return hipGetLastError();
}

hipError_t launch_lay_rows(int dtype, const LayRows& a, hipStream_t s) {
    const uint64_t n = (a.count * (plane_cols(a.cols) / 8) + 255) / 256;
    if (n == 0) return hipSuccess;
    const dim3 grid((uint32_t)std::min<uint64_t>(n, 1u << 22)), block(256);
    if (dtype == BC_F32) hipLaunchKernelGGL(lay_rows<float>, grid, block, 0, s, a);
    else if (dtype == BC_F16) hipLaunchKernelGGL(lay_rows<f16_t>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(lay_rows<bf16_t>, grid, block, 0, s, a);
    return hipGetLastError();
}

hipError_t launch_grouped_slope(int dtype, const GroupedSlope& a, hipStream_t s) {
    const dim3 grid((uint32_t)(plane_cols(a.cols) / 64) * group_tiles(a.g.rows, a.g.experts, 64)), block(256);
    if (dtype == BC_F32) hipLaunchKernelGGL(grouped_slope<float>, grid, block, 0, s, a);
    else if (dtype == BC_F16) hipLaunchKernelGGL(grouped_slope<f16_t>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(grouped_slope<bf16_t>, grid, block, 0, s, a);
    return hipGetLastError();
}

hipError_t launch_grouped_bias(int out_dtype, const GroupedSlope& a, void* dbias, uint64_t ld, hipStream_t s) {
    const dim3 grid((a.cols + 255) / 256, a.g.experts), block(256);
    if (out_dtype == BC_F32) hipLaunchKernelGGL(grouped_bias<float>, grid, block, 0, s, a, (float*)dbias, ld);
    else if (out_dtype == BC_F16) hipLaunchKernelGGL(grouped_bias<f16_t>, grid, block, 0, s, a, (f16_t*)dbias, ld);
    else hipLaunchKernelGGL(grouped_bias<bf16_t>, grid, block, 0, s, a, (bf16_t*)dbias, ld);
    return hipGetLastError();
}

hipError_t launch_grouped_where(const GroupedWhere& a, hipStream_t s) {
    const uint32_t n = 64 * (group_tiles(a.g.rows, a.g.experts, 64) + 1);
    hipLaunchKernelGGL(grouped_where, dim3((n + 255) / 256), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace bc
