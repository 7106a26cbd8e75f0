// kernels_route.hip -- the router of a block of experts and the combination of
// the experts' results.
//
// Router: for each row x of logits, p = softmax(x); the k largest (ties to the
// lower expert), their weights p_j, or p_j over the chosen ones' sum; then the
// order of the choices by expert, and by row within an expert.  A logit of -inf
// has no probability and is never chosen.
//
// The order is a count: route_gate gives each choice its rank among those of
// the same expert in its block of rows (a bit mask of the block's rows for each
// expert, so that the rank is a count of bits and no order of atomics shows),
// route_scan adds the blocks' counts up, route_place adds what lies before; where the
// counts are few, every workgroup of route_add_place adds them up itself.
//
// Few bytes: what costs is the chain of launches and, within the first, of choices
// (16384 rows of 64 experts, k 2, bfloat16: 4.9, 2.5 and 3.3 us; 32768 of 1024, k 8, 99
// in all).  Up to 64 rows go in one launch and workgroup (one row, k 8: 5.6 us).
//
// Combination: out = residual + sum_j weight_j y[slot_j], the sum in fp32 in the
// order of j, and its gradient.  Bound by memory: a row's results are k whole
// rows elsewhere (8192x1600, k 2, bfloat16, with residual: 17.2 us, 6.1 TB/s; its
// gradient at 8000x1001 in fp16, in rows that are no whole pieces: 16.6, 4.8 TB/s).
#include "common.hpp"
#include "experts.hpp"

#include <algorithm>
#include <type_traits>

namespace bc {

namespace {

constexpr int kThreads = 256;

// Threads of a workgroup that chooses experts, G lanes a row: 64 rows at a time where
// that is at most 1024.
template <int G>
constexpr int kGate = G <= 16 ? 64 * G : 1024;

// Order of logits as unsigned numbers: -inf 0, then ascending; zeros are equal, a
// NaN is the largest.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 0xffffffffu;
    const uint32_t b = __float_as_uint(x + 0.0f);
    const uint32_t o = b & 0x80000000u ? ~b : b | 0x80000000u;
    return o - 0x007fffffu;  // -inf's
}

// A row of logits over G lanes, V consecutive ones each.
template <typename T, int V>
__device__ __forceinline__ void load_logits(const T* row, uint32_t experts, uint32_t lane, bool there, float (&x)[V]) {
    const uint32_t e = lane * V;
    const int left = there && e < experts ? (int)(experts - e) : 0;
    load_vec(row + (left > 0 ? e : 0), left, x);
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i >= left) x[i] = -INFINITY;
}

template <int G>
__device__ __forceinline__ float group_sum(float x) {
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
    return x;
}
// The logit of an order, but for a NaN's payload.
__device__ __forceinline__ float of_order(uint32_t o) {
    if (o == 0xffffffffu) return NAN;
    o += 0x007fffffu;
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}

// The largest x of G lanes, in all of them.  Within 16 lanes by the moves that cost no
// trip through LDS: neighbours, pairs, then halves and rows mirrored.
template <int G>
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
    auto with = [&](uint32_t y) { x = x > y ? x : y; };
    with(__builtin_amdgcn_mov_dpp(x, 0xb1, 0xf, 0xf, true));                      // lane ^ 1
    with(__builtin_amdgcn_mov_dpp(x, 0x4e, 0xf, 0xf, true));                      // lane ^ 2
    with(__builtin_amdgcn_mov_dpp(x, 0x141, 0xf, 0xf, true));                     // 7 - lane
    if constexpr (G > 8) with(__builtin_amdgcn_mov_dpp(x, 0x140, 0xf, 0xf, true));  // 15 - lane
    if constexpr (G > 16) with(__shfl_xor(x, 16, 64));
    if constexpr (G > 32) with(__shfl_xor(x, 32, 64));
    return x;
}

// exp(x - top), 0 for a logit that is masked out (also where all of them are).
__device__ __forceinline__ float chance(float x, float top) { return x == -INFINITY ? 0.0f : expf(x - top); }

// Writes a block's choices: weight and expert of its rows, and, in LDS, the mask of the
// rows of each expert.  A choice is the largest order over a row's lanes, of equals that
// of the first lane (lanes hold consecutive experts): each lane keeps its own largest at
// hand and looks for the next when it has lost it.
template <typename T, int G, int V>
__device__ __forceinline__ void gate_rows(const Route& a, uint64_t row0, uint32_t rows, uint32_t words, uint32_t* mask) {
    constexpr uint32_t kRows = kGate<G> / G;
    constexpr int kMine = (kMaxChoices + G - 1) / G;   // choices that a lane keeps
    const uint32_t lane = threadIdx.x % G, first = (threadIdx.x & 63) / G * G;
    for (uint32_t r0 = 0; r0 < rows; r0 += kRows) {
        const uint32_t r = r0 + threadIdx.x / G;
        const bool there = r < rows;
        const uint64_t row = row0 + (there ? r : 0);
        float x[V];
        load_logits<T, V>((const T*)a.logits + row * a.ld, a.experts, lane, there, x);
        uint32_t o[V], best = 0, at = 0;
        auto look = [&]() {
            best = 0;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (o[i] > best) {
                    best = o[i];
                    at = i;
                }
        };
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] = order_of(x[i]);
        look();
        float top = 0.0f, chosen = 0.0f, all = 1.0f, mine[kMine];
        int32_t e_mine[kMine];
#pragma unroll
        for (int s = 0; s < kMine; ++s) {
            mine[s] = 0.0f;
            e_mine[s] = -1;
            for (uint32_t jj = 0; jj < G && s * G + jj < a.k; ++jj) {
                const uint32_t most = group_max<G>(best);
                const bool found = most != 0;
                const uint64_t equal = __ballot(found && best == most) >> first & (G == 64 ? ~0ull : (1ull << (G & 63)) - 1);
                const uint32_t owner = found ? (uint32_t)__builtin_ctzll(equal) : 0;
                const uint32_t e = owner * V + (uint32_t)__shfl((int)at, (int)(first + owner), 64);
                const float value = of_order(most);
                if (s == 0 && jj == 0) {
                    top = found ? value : 0.0f;
                    float sum = 0.0f;
#pragma unroll
                    for (int i = 0; i < V; ++i) sum += chance(x[i], top);
                    all = group_sum<G>(sum);
                }
                const float p = found ? expf(value - top) : 0.0f;
                chosen += p;
                if (lane == jj) {
                    mine[s] = p;
                    e_mine[s] = found ? (int32_t)e : -1;
                }
                if (found && lane == owner) {
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (i == (int)at) o[i] = 0;
                    look();
                }
            }
        }
        // a row without a chosen expert has weights of 0 and nothing to divide by
        const float by = a.normalise ? chosen : all;
#pragma unroll
        for (int s = 0; s < kMine; ++s) {
            const uint32_t j = s * G + lane;
            if (!there || j >= a.k) continue;
            a.weight[row * a.k + j] = e_mine[s] < 0 ? 0.0f : mine[s] / by;
            a.expert[row * a.k + j] = e_mine[s];
            if (e_mine[s] >= 0) atomicOr(&mask[(uint32_t)e_mine[s] * words + r / 32], 1u << (r % 32));
        }
    }
}

// Rank of row r in the mask of one expert.
__device__ __forceinline__ uint32_t rank_of(const uint32_t* mask, uint32_t r) {
    uint32_t n = 0;
    for (uint32_t w = 0; w < r / 32; ++w) n += __popc(mask[w]);
    return n + __popc(mask[r / 32] & ((1u << (r % 32)) - 1));
}

template <typename T, int G, int V>
__global__ __launch_bounds__(kGate<G>) void route_gate(Route a) {
    constexpr uint32_t kThreads = kGate<G>;
    extern __shared__ uint32_t mask[];
    const uint64_t row0 = (uint64_t)blockIdx.x * a.block_rows;
    const uint32_t rows = a.rows - row0 < a.block_rows ? (uint32_t)(a.rows - row0) : a.block_rows;
    const uint32_t words = a.block_rows / 32;
    for (uint32_t i = threadIdx.x; i < a.experts * words; i += kThreads) mask[i] = 0;
    __syncthreads();
    gate_rows<T, G, V>(a, row0, rows, words, mask);
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < a.experts; e += kThreads) {
        uint32_t n = 0;
        for (uint32_t w = 0; w < words; ++w) n += __popc(mask[e * words + w]);
        a.count[a.add ? (uint64_t)blockIdx.x * a.experts + e : (uint64_t)e * a.blocks + blockIdx.x] = n;
    }
    for (uint32_t i = threadIdx.x; i < rows * a.k; i += kThreads) {
        const int32_t e = a.expert[row0 * a.k + i];
        a.slot[row0 * a.k + i] = e < 0 ? -1 : (int32_t)rank_of(mask + (uint32_t)e * words, i / a.k);
    }
}

// Exclusive sums of x over a workgroup; *total: the sum.
template <uint32_t kThreads>
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* total) {
    __shared__ uint32_t sh[kThreads / 64];
    const uint32_t lane = threadIdx.x & 63;
    uint32_t s = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = __shfl_up(s, o, 64);
        if (lane >= (uint32_t)o) s += y;
    }
    __syncthreads();
    if (lane == 63) sh[threadIdx.x >> 6] = s;
    __syncthreads();
    uint32_t before = 0, all = 0;
#pragma unroll
    for (uint32_t w = 0; w < kThreads / 64; ++w) {
        if (w < threadIdx.x >> 6) before += sh[w];
        all += sh[w];
    }
    *total = all;
    return before + s - x;
}

// A workgroup an expert: its blocks' counts become what lies before each of them.
__global__ __launch_bounds__(kThreads) void route_scan(Route a) {
    uint32_t* c = a.count + (uint64_t)blockIdx.x * a.blocks;
    uint32_t sum = 0;
    for (uint32_t b0 = 0; b0 < a.blocks; b0 += kThreads) {
        const uint32_t b = b0 + threadIdx.x;
        uint32_t total;
        const uint32_t before = block_scan<kThreads>(b < a.blocks ? c[b] : 0, &total);
        if (b < a.blocks) c[b] = sum + before;
        sum += total;
    }
    if (threadIdx.x == 0) a.count[(uint64_t)a.experts * a.blocks + blockIdx.x] = sum;
}

// Offsets of the experts from their totals, into LDS.
template <uint32_t kThreads, typename F>
__device__ __forceinline__ void offsets_of(uint32_t experts, uint32_t* offsets, F total_of) {
    uint32_t sum = 0;
    for (uint32_t e0 = 0; e0 < experts; e0 += kThreads) {
        const uint32_t e = e0 + threadIdx.x;
        uint32_t total;
        const uint32_t before = block_scan<kThreads>(e < experts ? total_of(e) : 0, &total);
        if (e < experts) offsets[e] = sum + before;
        sum += total;
    }
    if (threadIdx.x == 0) offsets[experts] = sum;
    __syncthreads();
}

// Slots and sources of a block's choices: before(e) of expert e's lie in other blocks.
template <typename F>
__device__ __forceinline__ void place_rows(const Route& a, const uint32_t* offsets, F before) {
    const uint64_t row0 = (uint64_t)blockIdx.x * a.block_rows;
    const uint32_t rows = a.rows - row0 < a.block_rows ? (uint32_t)(a.rows - row0) : a.block_rows;
    if (blockIdx.x == 0)
        for (uint32_t e = threadIdx.x; e <= a.experts; e += kThreads) a.offsets[e] = (int32_t)offsets[e];
    for (uint32_t i = threadIdx.x; i < rows * a.k; i += kThreads) {
        const uint64_t at = row0 * a.k + i;
        const int32_t e = a.expert[at];
        if (e < 0) continue;
        const uint32_t slot = offsets[e] + before((uint32_t)e) + (uint32_t)a.slot[at];
        a.slot[at] = (int32_t)slot;
        a.source[slot] = (int32_t)(row0 + i / a.k);
    }
}
__global__ __launch_bounds__(kThreads) void route_place(Route a) {
    __shared__ uint32_t offsets[kMaxExperts + 1];
    offsets_of<kThreads>(a.experts, offsets, [&](uint32_t e) { return a.count[(uint64_t)a.experts * a.blocks + e]; });
    place_rows(a, offsets, [&](uint32_t e) { return a.count[(uint64_t)e * a.blocks + blockIdx.x]; });
}

// The same from counts [blocks][experts] as route_gate has written them: `wide` threads
// side by side an expert each, the parts of a column added through LDS.  For up to
// kAddCounts counts: 64 experts, 256 rows 9.6 us in place of 11.5, 1024 rows 8.5 of 9.7;
// but 4096 rows 11.6 of 9.8 and 16384 24 of 10, as every workgroup reads the same lines.
constexpr uint32_t kAddCounts = 1024;
__global__ __launch_bounds__(kThreads) void route_add_place(Route a, uint32_t wide) {
    __shared__ uint32_t offsets[kMaxExperts + 1], before[kMaxExperts], all[kMaxExperts];
    const uint32_t parts = kThreads / wide, part = threadIdx.x / wide;
    for (uint32_t e = threadIdx.x % wide; e < a.experts; e += wide) {
        uint32_t sum = 0, mine = 0;
#pragma unroll 8
        for (uint32_t b = part; b < a.blocks; b += parts) {
            const uint32_t n = a.count[(uint64_t)b * a.experts + e];
            sum += n;
            if (b < blockIdx.x) mine += n;
        }
        before[part * wide + e] = mine;  // (more than `wide` experts: one part)
        all[part * wide + e] = sum;
    }
    __syncthreads();
    auto added = [&](const uint32_t* of, uint32_t e) {
        uint32_t n = 0;
        for (uint32_t p = 0; p < parts; ++p) n += of[p * wide + e];
        return n;
    };
    offsets_of<kThreads>(a.experts, offsets, [&](uint32_t e) { return added(all, e); });
    for (uint32_t e = threadIdx.x; e < a.experts; e += kThreads) all[e] = added(before, e);
    __syncthreads();
    place_rows(a, offsets, [&](uint32_t e) { return all[e]; });
}

// All of it in one workgroup.
template <typename T, int G, int V>
__global__ __launch_bounds__(kGate<G>) void route_small(Route a) {
    constexpr uint32_t kThreads = kGate<G>;
    extern __shared__ uint32_t mask[];
    __shared__ uint32_t offsets[kMaxExperts + 1];
    const uint32_t rows = (uint32_t)a.rows, words = a.block_rows / 32;
    for (uint32_t i = threadIdx.x; i < a.experts * words; i += kThreads) mask[i] = 0;
    __syncthreads();
    gate_rows<T, G, V>(a, 0, rows, words, mask);
    __syncthreads();
    offsets_of<kThreads>(a.experts, offsets, [&](uint32_t e) {
        uint32_t n = 0;
        for (uint32_t w = 0; w < words; ++w) n += __popc(mask[e * words + w]);
        return n;
    });
    for (uint32_t e = threadIdx.x; e <= a.experts; e += kThreads) a.offsets[e] = (int32_t)offsets[e];
    for (uint32_t i = threadIdx.x; i < rows * a.k; i += kThreads) {
        const int32_t e = a.expert[i];
        if (e < 0) {
            a.slot[i] = -1;
            continue;
        }
        const uint32_t slot = offsets[e] + rank_of(mask + (uint32_t)e * words, i / a.k);
        a.slot[i] = (int32_t)slot;
        a.source[slot] = (int32_t)(i / a.k);
    }
}

// dlogits: normalised over the chosen, w_e (dw_e - sum_j w_j dw_j) for them;
// otherwise p_e ([chosen] dw_e - sum_j p_j dw_j).  Logits of -inf get 0, whatever
// the sum is.  Bound by round trips to memory that follow each other: of every choice the
// expert and then, for one that is there, weight and dweight; the logits, which wait for
// none of these, are loaded behind them (8191 rows of 129, k 4, fp32: 7.4 us for 8.7 MB;
// normalised, without logits, 5.9).
template <typename T, int G, int V>
__device__ __forceinline__ void grad_row(const RouteGrad& a, uint64_t row, uint32_t lane) {
    const bool there = row < a.rows;
    float up[V], p[V];
    bool live[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        up[i] = p[i] = 0.0f;
        live[i] = false;
    }
    float dot = 0.0f;
    for (uint32_t j = 0; j < a.k; ++j) {
        const uint64_t at = there ? row * a.k + j : 0;
        const int32_t e = there ? a.expert[at] : -1;
        if (e < 0 || (uint32_t)e >= a.experts) continue;
        const float w = a.weight[at], d = a.dweight[at];
        dot += w * d;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if ((uint32_t)e == lane * V + i) {
                up[i] = d;
                p[i] = w;
                live[i] = true;
            }
    }
    if (!a.normalise) {
        float x[V], top = -INFINITY, sum = 0.0f;
        load_logits<T, V>((const T*)a.logits + (there ? row : 0) * a.ld, a.experts, lane, there, x);
#pragma unroll
        for (int i = 0; i < V; ++i) top = x[i] > top || x[i] != x[i] ? x[i] : top;
#pragma unroll
        for (int o = G / 2; o > 0; o >>= 1) {
            const float y = __shfl_xor(top, o, 64);
            top = y > top || y != y ? y : top;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            live[i] = x[i] != -INFINITY;
            sum += p[i] = chance(x[i], top);
        }
        sum = group_sum<G>(sum);
#pragma unroll
        for (int i = 0; i < V; ++i) p[i] /= sum;  // 0 / 0 where nothing is live
    }
    const uint32_t e = lane * V;
    if (!there || e >= a.experts) return;
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = live[i] ? p[i] * (up[i] - dot) : 0.0f;
    store_vec((T*)a.dlogits + row * a.ld_d + e, (int)(a.experts - e), p);
}

template <typename T, int G, int V>
__global__ __launch_bounds__(kThreads) void route_grad(RouteGrad a) {
    constexpr uint32_t kRows = kThreads / G;
    // (the lanes of a wave go round together: the sums need every one of them)
    for (uint64_t row0 = (uint64_t)blockIdx.x * kRows; row0 < a.rows; row0 += (uint64_t)gridDim.x * kRows)
        grad_row<T, G, V>(a, row0 + threadIdx.x / G, threadIdx.x % G);
}

// ------------------------------------------------------------ combination
// Elements of a lane's piece: 16 bytes, so that a wave's pieces lie side by side (in fp32,
// against eight elements in two loads: 8192x1600, k 2, 35.3 to 32.4 us and its gradient 53
// to 48; k 8 98 to 106 and 212 to 185).
template <typename T>
constexpr int kPiece = 16 / (int)sizeof(T);
// Lanes of a row: a power of two that its pieces fill, up to a workgroup.
template <typename T>
uint32_t row_lanes(uint32_t cols) {
    uint32_t n = 1;
    while (n < kThreads && n * kPiece<T> < cols) n *= 2;
    return n;
}

template <typename T, bool kWhole>
__device__ __forceinline__ void combine_row(const Combine& a, uint64_t row, uint32_t from, uint32_t step) {
    constexpr int V = kPiece<T>;
    for (uint32_t c = from; c < a.cols; c += step) {
        const int left = (int)(a.cols - c);
        float sum[V];
        if (a.residual) {
            load_vec<kWhole>((const T*)a.residual + row * a.ldr + c, left, sum);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i] = 0.0f;
        }
        for (uint32_t j = 0; j < a.k; ++j) {
            const uint32_t slot = (uint32_t)a.slot[row * a.k + j];
            if (slot >= a.slots) continue;  // none
            const float w = a.weight ? a.weight[row * a.k + j] : 1.0f;
            float y[V];
            load_vec<kWhole>((const T*)a.y + slot * a.ldy + c, left, y);
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i] += w * y[i];
        }
        store_vec((T*)a.out + row * a.ld_out + c, left, sum, a.nt);
    }
}

template <typename T, bool kWhole>
__global__ __launch_bounds__(kThreads) void combine(Combine a, uint32_t lanes) {
    const uint64_t step = (uint64_t)gridDim.x * kThreads / lanes;
    for (uint64_t row = ((uint64_t)blockIdx.x * kThreads + threadIdx.x) / lanes; row < a.rows; row += step)
        combine_row<T, kWhole>(a, row, threadIdx.x % lanes * kPiece<T>, lanes * kPiece<T>);
}

// dy[slot_j] = weight_j dout, dweight_j = <dout, y[slot_j]>: `lanes` lanes of a wave a
// row, its part of dout read once for each choice (from the caches after the first).
template <typename T, bool kWhole>
__global__ __launch_bounds__(kThreads) void combine_grad(CombineGrad a, uint32_t lanes) {
    constexpr int V = kPiece<T>;
    const uint32_t lane = threadIdx.x % lanes;
    const uint64_t step = (uint64_t)gridDim.x * kThreads / lanes;
    const uint64_t first = ((uint64_t)blockIdx.x * kThreads + threadIdx.x) / lanes;
    // (the lanes of a wave go round together: the sums need every one of them)
    for (uint64_t r = first; r < a.rows + first % (64 / lanes); r += step) {
        const bool there = r < a.rows;
        for (uint32_t j = 0; j < a.k; ++j) {
            const uint32_t slot = there ? (uint32_t)a.slot[r * a.k + j] : 0xffffffffu;
            float dot = 0.0f;
            if (slot < a.slots) {
                const float w = a.weight ? a.weight[r * a.k + j] : 1.0f;
                for (uint32_t c = lane * V; c < a.cols; c += lanes * V) {
                    const int left = (int)(a.cols - c);
                    float d[V], y[V];
                    load_vec<kWhole>((const T*)a.dout + r * a.ldd + c, left, d);
                    if (a.dweight) {
                        load_vec<kWhole>((const T*)a.y + slot * a.ldy + c, left, y);
#pragma unroll
                        for (int i = 0; i < V; ++i) dot = fmaf(d[i], y[i], dot);
                    }
                    if (a.dy) {
#pragma unroll
                        for (int i = 0; i < V; ++i) d[i] *= w;
                        store_vec((T*)a.dy + slot * a.lddy + c, left, d, a.nt);
                    }
                }
            }
            if (a.dweight) {
                for (uint32_t o = lanes / 2; o > 0; o >>= 1) dot += __shfl_xor(dot, (int)o, 64);
                if (lane == 0 && there) a.dweight[r * a.k + j] = dot;
            }
        }
    }
}

// Workgroups of a launch whose kernel goes round: HIP takes fewer than 2^32 threads.
uint32_t capped(uint64_t blocks) { return (uint32_t)std::min<uint64_t>(blocks, 1u << 22); }

// Calls fn(G, V) as constants for this many experts.
template <typename F>
hipError_t with_group(uint32_t experts, F fn) {
    using std::integral_constant;
    if (experts <= 8) return fn(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    if (experts <= 16) return fn(integral_constant<int, 8>{}, integral_constant<int, 2>{});
    if (experts <= 32) return fn(integral_constant<int, 8>{}, integral_constant<int, 4>{});
    if (experts <= 64) return fn(integral_constant<int, 8>{}, integral_constant<int, 8>{});
    if (experts <= 128) return fn(integral_constant<int, 16>{}, integral_constant<int, 8>{});
    if (experts <= 256) return fn(integral_constant<int, 32>{}, integral_constant<int, 8>{});
    if (experts <= 512) return fn(integral_constant<int, 64>{}, integral_constant<int, 8>{});
    return fn(integral_constant<int, 64>{}, integral_constant<int, 16>{});
}

template <typename T>
hipError_t route_of(const Route& a, hipStream_t s) {
    return with_group(a.experts, [&](auto g, auto v) {
        constexpr int G = decltype(g)::value, V = decltype(v)::value;
        const size_t lds = (size_t)a.experts * (a.block_rows / 32) * 4;
        if (a.blocks == 1) {
            hipLaunchKernelGGL((route_small<T, G, V>), dim3(1), dim3(kGate<G>), lds, s, a);
            return hipGetLastError();
        }
        hipLaunchKernelGGL((route_gate<T, G, V>), dim3(a.blocks), dim3(kGate<G>), lds, s, a);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (a.add) {
            uint32_t wide = 1;
            while (wide < kThreads && wide < a.experts) wide *= 2;
            hipLaunchKernelGGL(route_add_place, dim3(a.blocks), dim3(kThreads), 0, s, a, wide);
            return hipGetLastError();
        }
        hipLaunchKernelGGL(route_scan, dim3(a.experts), dim3(kThreads), 0, s, a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        hipLaunchKernelGGL(route_place, dim3(a.blocks), dim3(kThreads), 0, s, a);
        return hipGetLastError();
    });
}

template <typename T>
hipError_t route_grad_of(const RouteGrad& a, hipStream_t s) {
    return with_group(a.experts, [&](auto g, auto v) {
        constexpr int G = decltype(g)::value, V = decltype(v)::value;
        const uint64_t blocks = (a.rows + kThreads / G - 1) / (kThreads / G);
        hipLaunchKernelGGL((route_grad<T, G, V>), dim3(capped(blocks)), dim3(kThreads), 0, s, a);
        return hipGetLastError();
    });
}

template <typename T>
hipError_t combine_of(const Combine& a, hipStream_t s) {
    const uint32_t lanes = row_lanes<T>(a.cols);
    const uint64_t blocks = (a.rows * lanes + kThreads - 1) / kThreads;
    if (a.cols % kPiece<T> == 0) hipLaunchKernelGGL((combine<T, true>), dim3(capped(blocks)), dim3(kThreads), 0, s, a, lanes);
    else hipLaunchKernelGGL((combine<T, false>), dim3(capped(blocks)), dim3(kThreads), 0, s, a, lanes);
    return hipGetLastError();
}

template <typename T>
hipError_t combine_grad_of(const CombineGrad& a, hipStream_t s) {
    const uint32_t lanes = std::min(64u, row_lanes<T>(a.cols));
    const uint64_t blocks = (a.rows * lanes + kThreads - 1) / kThreads;
    if (a.cols % kPiece<T> == 0) hipLaunchKernelGGL((combine_grad<T, true>), dim3(capped(blocks)), dim3(kThreads), 0, s, a, lanes);
    else hipLaunchKernelGGL((combine_grad<T, false>), dim3(capped(blocks)), dim3(kThreads), 0, s, a, lanes);
    return hipGetLastError();
}

}  // namespace

// Rows of a workgroup of route_gate: 64, more where there would be more than 256
// workgroups and the masks of the experts (a bit a row) leave room.
uint32_t route_block_rows(uint64_t rows, uint32_t experts) {
    uint32_t n = 64;
    while (n < 1024 && (uint64_t)n * 2 * experts <= 32768ull * 8 && (rows + n - 1) / n > 256) n *= 2;
    return n;
}

hipError_t launch_route(int dtype, Route a, hipStream_t s) {
    a.add = (uint64_t)a.blocks * a.experts <= kAddCounts;
    if (dtype == BC_F32) return route_of<float>(a, s);
    if (dtype == BC_F16) return route_of<f16_t>(a, s);
    return route_of<bf16_t>(a, s);
}

hipError_t launch_route_grad(int dtype, const RouteGrad& a, hipStream_t s) {
    if (dtype == BC_F32) return route_grad_of<float>(a, s);
    if (dtype == BC_F16) return route_grad_of<f16_t>(a, s);
    return route_grad_of<bf16_t>(a, s);
}

hipError_t launch_combine(int dtype, const Combine& a, hipStream_t s) {
    if (dtype == BC_F32) return combine_of<float>(a, s);
    if (dtype == BC_F16) return combine_of<f16_t>(a, s);
    return combine_of<bf16_t>(a, s);
}

hipError_t launch_combine_grad(int dtype, const CombineGrad& a, hipStream_t s) {
    if (dtype == BC_F32) return combine_grad_of<float>(a, s);
    if (dtype == BC_F16) return combine_grad_of<f16_t>(a, s);
    return combine_grad_of<bf16_t>(a, s);
}

}  // namespace bc
