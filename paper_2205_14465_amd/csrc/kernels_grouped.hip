// kernels_grouped.hip -- the linear layer grouped by expert: rows in runs, one run
// an expert, each expert with a weight of its own,
//   z = x w_e^T + bias_e,  y = act(z);  dz = dy act'(z),
//   dx = dz w_e,  dw_e = dz_e^T x_e,  dbias_e = sum over the expert's rows of dz.
//
// Where the runs begin is known to the device alone.  A launch has a workgroup
// for every tile that there can be; a workgroup finds its tile's expert by counting the
// experts' tiles, and those without a tile end at once.  No operand is
// turned in memory: dx takes w and dw takes dz and x with k down their columns
// (run_tile.hpp).  Operands are read where they lie, x through `source` if it is
// given, but for 16-bit ones whose rows are no whole 16-byte pieces, which are laid
// out first.  fp32 ones are multiplied as fp32: three bfloat16 planes of every
// expert's weight (kernels_linear.hip) would move more bytes than their products
// take time, and few rows share each.
//
// With an activation, dz of 16-bit tensors is rounded to their type, which the matrix
// instructions take; as two parts it would be exact to fp32 and every product of the
// backward pass twice as long.  Each rounding is half a unit of one term, so that dx and
// dw, rounded once themselves, are 2.3e-3 off (2-norm) in bfloat16 where an exact dz
// would leave 1.7e-3, and 1.7e-3 off as fp32.  dbias sums the unrounded dz.
#include "act.hpp"
#include "experts.hpp"
#include "few.hpp"
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

// Inclusive sums over a wave.
__device__ __forceinline__ uint32_t sum_up_to(uint32_t x) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = __shfl_up(x, o, 64);
        if ((threadIdx.x & 63) >= (uint32_t)o) x += y;
    }
    return x;
}

// The rows and the column of a workgroup's tile of a product that is tiles_n tiles wide:
// the experts' tiles one expert after the other, an expert's down columns of at most
// kBand tiles, a die's workgroups consecutive ones.  Only tiles with rows count, so each
// lane counts those of some experts, and a scan places them: with an empty tile an expert,
// as run_of has it, no sum is needed, but all rows of one expert are then one die's work
// (fp32, 4096 rows, 128 experts of 512x512: spread evenly 50 us in place of 40, all with
// one expert 457 for 23; bfloat16, 1024 experts of 256x256 with 8 rows each 40 for 51).
constexpr uint32_t kBand = 8;
template <uint32_t kHigh>
__device__ __forceinline__ bool tile_run(const Groups& g, uint32_t block, uint32_t tiles_n, Run& r, uint32_t& tn) {
    const uint32_t lane = threadIdx.x & 63, per = (g.experts + 63) / 64;
    auto tiles_in = [](uint32_t at, uint32_t to) { return to > at ? (to - at + kHigh - 1) / kHigh : 0; };
    uint32_t n = 0, at = offset_of(g, min(lane * per, g.experts));
    for (uint32_t i = 1; i <= per; i += 4) {  // (past the last expert: no tiles)
        uint32_t to[4];
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) to[j] = offset_of(g, min(lane * per + min(i + j, per), g.experts));
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            n += tiles_in(at, to[j]);
            at = to[j];
        }
    }
    const uint32_t up_to = sum_up_to(n);
    // (offsets that do not ascend make more tiles than there can be: those are left out)
    const uint32_t tiles_m = min((uint32_t)__builtin_amdgcn_readlane((int)up_to, 63), group_tiles(g.rows, g.experts, kHigh));
    const uint32_t total = tiles_m * tiles_n, q = total / 8, rest = total % 8, die = block % 8;
    if (block / 8 >= q + (die < rest ? 1 : 0)) return false;
    const uint32_t t = die * q + (die < rest ? die : rest) + block / 8, row = t / tiles_n;
    const int owner = __popcll(__ballot(up_to <= row));
    uint32_t before = __builtin_amdgcn_readlane((int)(up_to - n), owner), e = (uint32_t)owner * per;
    if (per > 1) {  // which of the lane's experts: they have lanes of their own
        const uint32_t one = min(e + min(lane, per), g.experts), next = min(e + min(lane + 1, per), g.experts);
        const uint32_t m = tiles_in(offset_of(g, one), offset_of(g, next));
        const uint32_t sum = before + sum_up_to(m);
        const int nth = __popcll(__ballot(sum <= row));
        before = __builtin_amdgcn_readlane((int)(sum - m), nth);
        e += (uint32_t)nth;
    }
    e = min(e, g.experts - 1);
    const uint32_t first = offset_of(g, e), in = t - before * tiles_n;
    r.expert = e;
    r.to = offset_of(g, e + 1);
    const uint32_t high = tiles_in(first, r.to), rows = in / (kBand * tiles_n) * kBand;
    const uint32_t here = high - rows < kBand ? high - rows : kBand, i = in - rows * tiles_n;
    tn = i / here;
    r.from = first + (rows + i % here) * kHigh;
    return true;
}

// ----------------------------------------------------------------- products
// The activation for a 16-bit result: as activate<false>, with fused multiplications
// and the exponential's factor log2(e) among the constants, as the epilogue of large
// products is bound by these instructions.
__device__ __forceinline__ float quick_act(int act, float z) {
    constexpr float kLog2e = 1.44269504088896f;
    float t;
    if (act == BC_ACT_GELU_TANH) t = z * fmaf(z * z, -2.0f * kTanhScale * kTanhCubic * kLog2e, -2.0f * kTanhScale * kLog2e);
    else if (act == BC_ACT_SILU) t = -kLog2e * z;
    else return activate<false>(act, z);
    return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t));
}

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
            for (int i = 0; i < 8; ++i) v[i] = exact ? activate<true>(p.act, v[i]) : quick_act(p.act, v[i]);
    }
    store_vec((TO*)p.out + m * p.ld_out + n, left, v, p.nt);
}

// How the operands of a product lie: forward k along the rows of both, for dx
// down the columns of w, for dw down those of dz and x.
template <bool forward, int kPiece>
using RowsLie = Lie<false, !forward, false, kPiece>;
template <bool kTable, int kPiece>
using WeightsLie = Lie<true, true, kTable, kPiece>;

// Takes up the tile with rows `run` and columns n0 on of the experts' rows times
// their weight.
template <typename L, bool forward, typename R>
__device__ __forceinline__ void begin_rows(R& g, const GroupedProduct& p, const Run& run, uint32_t n0, char* lds) {
    typedef typename R::T T;
    const bool gather = forward && p.source;
    const uint32_t m0 = run.from;
    const uint32_t ld = (uint32_t)p.a.ld;
    const Side<T> a{(const T*)p.a.p + (gather ? 0 : m0 * p.a.ld), ld, run.to - m0};
    const Side<T> b{(const T*)p.b.p + run.expert * p.b.expert + (forward ? n0 * p.b.ld : n0), (uint32_t)p.b.ld, p.cols - n0};
    g.template begin<L>(a, b, p.k, nullptr, lds, [&](int r) -> uint32_t {
        if (!gather) return (uint32_t)r * ld * (uint32_t)sizeof(T);
        const uint32_t row = (uint32_t)p.source[m0 + r];
        return row < p.a_rows ? row * ld * (uint32_t)sizeof(T) : kNowhere;
    });
}

// The same for rows m0 and columns n0 on of expert e's dw.
template <typename L, typename R>
__device__ __forceinline__ void begin_weights(R& g, const GroupedProduct& p, uint32_t e, uint32_t m0, uint32_t n0, char* lds) {
    typedef typename R::T T;
    const uint32_t first = offset_of(p.g, 0), from = offset_of(p.g, e), to = offset_of(p.g, e + 1);
    const Side<T> a{(const T*)p.a.p + (uint64_t)from * p.a.ld + m0, (uint32_t)p.a.ld, p.rows - m0};
    const Side<T> b{(const T*)p.b.p + (L::kTable ? 0 : (uint64_t)from * p.b.ld) + n0, (uint32_t)p.b.ld, p.cols - n0};
    const uint32_t* where = L::kTable ? p.where + (uint64_t)tiles_before<64>(first, from, e) * 64 : nullptr;
    // (offsets that do not ascend: no rows)
    g.template begin<L>(a, b, to > from && from >= first ? to - from : 0, where, lds, [](int) { return 0u; });
}

// The experts' rows times their weight in tiles that leave room for others on a
// compute unit.  fp32, 2474 rows of 1001 to 515: 43 us, 60 TFLOP/s of 152: 387 tiles
// of 64x64 on 256 units, where the second round leaves half of them idle, and loads of
// single words (1004 to 516, whole pieces: 39).
template <typename G, typename TO, bool forward, int kPiece>
__device__ __forceinline__ void rows_tile(const GroupedProduct& p, uint32_t block, char* lds) {
    typedef RowsLie<forward, kPiece> L;
    const uint32_t tiles_n = (p.cols + G::kBN - 1) / G::kBN;
    Run run;
    uint32_t tn;
    if (!tile_run<G::kBM>(p.g, block, tiles_n, run, tn)) return;
    const uint32_t m0 = run.from, n0 = tn * G::kBN;
    RunTile<G, kPiece> g;
    begin_rows<L, forward>(g, p, run, n0, lds);
    g.template rest<L>(lds);
    g.template run<L>(lds);
    g.finish(lds, [&](int row, int col, float (&v)[8]) {
        const uint32_t m = m0 + row, n = n0 + col;
        if (m < run.to && n < p.cols) finish_row<TO, forward>(p, run.expert, m, n, v);
    });
}

// dw: every expert's tiles, over its rows.
template <typename G, typename TO, bool kTable, int kPiece>
__device__ __forceinline__ void weights_tile(const GroupedProduct& p, uint32_t block, char* lds) {
    typedef WeightsLie<kTable, kPiece> L;
    const uint32_t tiles_m = (p.rows + G::kBM - 1) / G::kBM, tiles_n = (p.cols + G::kBN - 1) / G::kBN;
    // an expert's tiles go to all dies, each a run of consecutive ones
    const uint32_t each = tiles_m * tiles_n, e = block / each, j = block - e * each;
    const uint32_t in = j % 8 * (each / 8) + (j % 8 < each % 8 ? j % 8 : each % 8) + j / 8;
    const uint32_t m0 = in / tiles_n * G::kBM, n0 = in % tiles_n * G::kBN;
    RunTile<G, kPiece> g;
    begin_weights<L>(g, p, e, m0, n0, lds);
    g.template rest<L>(lds);
    g.template run<L>(lds);
    g.finish(lds, [&](int row, int col, float (&v)[8]) {
        const uint32_t m = m0 + row, n = n0 + col;
        if (m < p.rows && n < p.cols)
            store_vec((TO*)p.out + e * p.expert_out + m * p.ld_out + n, (int)(p.cols - n), v, p.nt);
    });
}

template <typename G, typename TO, bool forward, int kPiece>
__global__ __launch_bounds__(G::kThreads) void rows_product(GroupedProduct p) {
    extern __shared__ char lds[];
    rows_tile<G, TO, forward, kPiece>(p, blockIdx.x, lds);
}

template <typename G, typename TO, bool kTable, int kPiece>
__global__ __launch_bounds__(G::kThreads) void weights_product(GroupedProduct p) {
    extern __shared__ char lds[];
    weights_tile<G, TO, kTable, kPiece>(p, blockIdx.x, lds);
}

// dbias: 64 columns of an expert, whose sums over 64 rows each the first four waves
// share out.
template <typename TO>
__device__ __forceinline__ void bias_columns(const GroupedBias& a, uint32_t block, float* sums) {
    const uint32_t across = (a.cols + 63) / 64, e = block / across;
    const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = block % across * 64 + lane;
    const uint32_t first = offset_of(a.g, 0), from = offset_of(a.g, e), to = offset_of(a.g, e + 1);
    float sum = 0.0f;
    if (wave < 4 && c < a.cols && from >= first && to > from) {
        const uint32_t t0 = tiles_before<64>(first, from, e), n = (to - from + 63) / 64;
        for (uint32_t t = wave; t < n; t += 4) sum += a.part[(uint64_t)(t0 + t) * a.cols + c];
    }
    if (wave < 4) sums[wave * 64 + lane] = sum;
    __syncthreads();
    if (wave == 0 && c < a.cols)
        ((TO*)a.out)[e * a.ld + c] = (TO)((sums[lane] + sums[64 + lane]) + (sums[128 + lane] + sums[192 + lane]));
}

// Both gradients' products where tiles of this size do not fill the chip, and dbias
// (8 experts' 2048 rows of 768 to 768 in fp32: 50 us with 256 rows each, 96 TFLOP/s of
// 152, with the tiles' first loads and epilogues in the open; 62 with 200 to 300, whose
// ends fill tiles badly):
// `split` workgroups of the first product (dx's with rows_first: the one whose k is the
// longer), those of the second up to `end`, then the bias's.
template <typename G, typename TO, bool kTable, int kPiece>
__global__ __launch_bounds__(G::kThreads) void grads_product(GroupedProduct px, GroupedProduct pw, GroupedBias bias, uint32_t split,
                                                             uint32_t end, bool rows_first) {
    extern __shared__ char lds[];
    if (blockIdx.x >= end) {
        bias_columns<TO>(bias, blockIdx.x - end, (float*)lds);
        return;
    }
    const bool first = blockIdx.x < split;
    const uint32_t block = first ? blockIdx.x : blockIdx.x - split;
    if (first == rows_first) rows_tile<G, typename G::T, false, kPiece>(px, block, lds);
    else weights_tile<G, TO, kTable, kPiece>(pw, block, lds);
}

// ---------------------------------------------------------- large products
// The largest tiles fill a compute unit, so nothing runs beside one's epilogue.
// Workgroups stay: before a tile's epilogue a workgroup takes up its next tile and
// asks for its first step, the other stage of LDS serves as the strips.
//
// They are bound by the matrix units at the clock that the power limit leaves (1.7 to
// 2.0 GHz, those units busy 35 to 52 % of all cycles) and by the epilogues between
// them: 16 experts' 16384 rows of 1600 to 6400 in bfloat16, y and z written, 443 to 480
// us, without z 410; 6400 to 1600 355, 940 TFLOP/s; both gradients of
// the first 765.  Half tiles with two workgroups a unit (128x256, 256x128, 32 along k),
// three stages of 32, reading ahead into the L2 and other heights of a band (2 to 16)
// were as fast or slower.

// The experts' tiles and rows, in LDS.
struct RunTable {
    uint32_t tiles[kMaxExperts + 1];   // before each expert
    uint32_t rows[kMaxExperts + 1];    // its first
    // experts by their rows, the most first (grads_large), or an expert's last tile, if at
    // most half of it has rows, counted apart: such tiles before each (rows_large)
    uint32_t order[kMaxExperts + 1];
    uint32_t next;                     // a workgroup's next tile
};
// Experts by their rows, where it takes few comparisons; fill_runs has run.
constexpr uint32_t kSortExperts = 128;
__device__ __forceinline__ void sort_runs(uint32_t experts, RunTable& t) {
    for (uint32_t e = threadIdx.x; e < experts; e += blockDim.x) {
        uint32_t at = e;
        if (experts <= kSortExperts) {
            const int32_t n = (int32_t)(t.rows[e + 1] - t.rows[e]);
            at = 0;
            for (uint32_t i = 0; i < experts; ++i) {
                const int32_t m = (int32_t)(t.rows[i + 1] - t.rows[i]);
                at += m > n || (m == n && i < e);
            }
        }
        t.order[at] = e;
    }
    __syncthreads();
}
__device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t& all) {  // over a wave
    const uint32_t s = sum_up_to(x);
    all = __shfl(s, 63, 64);
    return s - x;
}
template <uint32_t kHigh, bool kApart>
__device__ __forceinline__ void fill_runs(const Groups& g, RunTable& t) {
    if (threadIdx.x < 64) {
        uint32_t sum = 0, sum_low = 0, all;
        for (uint32_t e0 = 0; e0 <= g.experts; e0 += 64) {
            const uint32_t e = e0 + threadIdx.x;
            uint32_t at = 0, n = 0, low = 0;
            if (e <= g.experts) at = offset_of(g, e);
            if (e < g.experts) {
                const uint32_t to = offset_of(g, e + 1);
                n = to > at ? (to - at + kHigh - 1) / kHigh : 0;
                if (kApart && n > 0 && (to - at - 1) % kHigh < kHigh / 2) {
                    low = 1;
                    --n;
                }
            }
            const uint32_t before = sum + sum_before(n, all);
            sum += all;
            if (e <= g.experts) {
                t.tiles[e] = before;
                t.rows[e] = at;
            }
            if constexpr (kApart) {
                const uint32_t lows = sum_low + sum_before(low, all);
                sum_low += all;
                if (e <= g.experts) t.order[e] = lows;
            }
        }
    }
    __syncthreads();
}
// The last expert with counts[e] <= n, all lanes alike.
__device__ __forceinline__ uint32_t expert_at(const uint32_t* counts, uint32_t experts, uint32_t n) {
    const uint32_t lane = threadIdx.x & 63;
    uint32_t before = 0;
    for (uint32_t e0 = 0; e0 < experts; e0 += 64)
        before += __popcll(__ballot(e0 + lane < experts && counts[e0 + lane] <= n));
    return __builtin_amdgcn_readfirstlane(before - 1);
}
// Tile t of a product that is tiles_n tiles wide: as tile_run, without empty ones.
template <uint32_t kHigh>
__device__ __forceinline__ void run_in(const RunTable& table, uint32_t experts, uint32_t t, uint32_t tiles_n, Run& r,
                                       uint32_t& tn) {
    r.expert = expert_at(table.tiles, experts, t / tiles_n);
    const uint32_t before = __builtin_amdgcn_readfirstlane(table.tiles[r.expert]);
    const uint32_t next = __builtin_amdgcn_readfirstlane(table.tiles[r.expert + 1]);
    const uint32_t at = __builtin_amdgcn_readfirstlane(table.rows[r.expert]);
    r.to = __builtin_amdgcn_readfirstlane(table.rows[r.expert + 1]);
    const uint32_t high = next - before, in = t - before * tiles_n;
    const uint32_t first = in / (kBand * tiles_n) * kBand, here = high - first < kBand ? high - first : kBand;
    const uint32_t i = in - first * tiles_n;
    tn = i / here;
    r.from = at + (first + i % here) * kHigh;
}
// Tile t of those that are counted apart.
template <uint32_t kHigh>
__device__ __forceinline__ void low_run_in(const RunTable& table, uint32_t experts, uint32_t t, uint32_t tiles_n, Run& r,
                                           uint32_t& tn) {
    const uint32_t row = t / tiles_n;
    r.expert = expert_at(table.order, experts, row);
    const uint32_t at = __builtin_amdgcn_readfirstlane(table.rows[r.expert]);
    r.to = __builtin_amdgcn_readfirstlane(table.rows[r.expert + 1]);
    tn = t - row * tiles_n;
    r.from = at + (r.to - at) / kHigh * kHigh;
}

// LDS of a large product: two stages, and of the strips what one does not hold; the
// table comes behind (everything before is 16-byte aligned).
template <typename G>
constexpr int kLargeLds = G::kStageBytes + (G::kStageBytes > G::kEpiBytes ? G::kStageBytes : G::kEpiBytes);

// The first tile's first step has landed (its second may be on the way).
template <typename G>
__device__ __forceinline__ void wait_first() {
    wait_vmcnt<0>();
    lds_barrier();
}
// The epilogue, strips in the second stage.  The next tile's first step, asked for
// before, is waited for before the last stores: those are not waited for, as
// memory operations count down in order.
template <typename R, typename E>
__device__ __forceinline__ void finish_large(R& g, char* lds, const E& epi) {
    if (g.busy) g.template finish_blocks<0, R::kFM - 1>(lds + R::kStageBytes, epi);
    wait_vmcnt<0>();
    if (g.busy) g.template finish_blocks<R::kFM - 1, R::kFM>(lds + R::kStageBytes, epi);
    lds_barrier();  // every wave has read its strip, and its part of the next step is there
}

template <typename G, typename TO, bool forward>
__global__ __launch_bounds__(G::kThreads) void rows_large(GroupedProduct p) {
    typedef RowsLie<forward, 16> L;
    extern __shared__ char lds[];
    RunTable& table = *(RunTable*)(lds + kLargeLds<G>);
    fill_runs<G::kBM, true>(p.g, table);
    const uint32_t tiles_n = (p.cols + G::kBN - 1) / G::kBN;
    // (offsets that do not ascend make more tiles than there can be: those are left out)
    const uint32_t tiles_m = min((uint32_t)__builtin_amdgcn_readfirstlane(table.tiles[p.g.experts]),
                                 group_tiles(p.g.rows, p.g.experts, G::kBM));
    const uint32_t low_m = __builtin_amdgcn_readfirstlane(table.order[p.g.experts]);
    // a die's tiles are consecutive ones, expert by expert, dealt to its workgroups in turn;
    // those with no more than half their rows, which take less time, come last
    const uint32_t die = blockIdx.x % 8;
    const uint32_t total = tiles_m * tiles_n, q = total / 8, rest = total % 8;
    const uint32_t from = die * q + (die < rest ? die : rest), here = q + (die < rest ? 1 : 0);
    const uint32_t low_total = low_m * tiles_n, low_q = low_total / 8, low_rest = low_total % 8;
    const uint32_t low_from = die * low_q + (die < low_rest ? die : low_rest), to = here + low_q + (die < low_rest ? 1 : 0);
    uint32_t t = blockIdx.x / 8;
    if (t >= to) return;
    RunTile<G, 16> g;
    Run run;
    uint32_t tn;
    auto take = [&](uint32_t i) {
        if (i < here) run_in<G::kBM>(table, p.g.experts, from + i, tiles_n, run, tn);
        else low_run_in<G::kBM>(table, p.g.experts, low_from + i - here, tiles_n, run, tn);
        begin_rows<L, forward>(g, p, run, tn * G::kBN, lds);
    };
    take(t);
    g.template rest<L>(lds);
    wait_first<G>();
    for (;;) {
        g.template run<L, true>(lds);
        const Run done = run;
        const uint32_t m0 = run.from, n0 = tn * G::kBN;
        t += gridDim.x / 8;
        const bool more = t < to;
        if (more) take(t);
        finish_large(g, lds, [&](int row, int col, float (&v)[8]) {
            const uint32_t m = m0 + row, n = n0 + col;
            if (m < done.to && n < p.cols) finish_row<TO, forward>(p, done.expert, m, n, v);
        });
        if (!more) return;
        g.template rest<L>(lds);
    }
}

template <typename G, typename TO, bool kTable>
__global__ __launch_bounds__(G::kThreads) void weights_large(GroupedProduct p) {
    typedef WeightsLie<kTable, 16> L;
    extern __shared__ char lds[];
    const uint32_t tiles_m = (p.rows + G::kBM - 1) / G::kBM, tiles_n = (p.cols + G::kBN - 1) / G::kBN;
    const uint32_t each = tiles_m * tiles_n, all = each * p.g.experts;
    // workgroups take tiles in turn, and so experts one after the other; of an expert's,
    // the dies have a run of consecutive ones each
    auto place = [&](uint32_t b, uint32_t& e, uint32_t& m0, uint32_t& n0) {
        e = b / each;
        const uint32_t j = b - e * each, in = j % 8 * (each / 8) + (j % 8 < each % 8 ? j % 8 : each % 8) + j / 8;
        m0 = in / tiles_n * G::kBM;
        n0 = in % tiles_n * G::kBN;
    };
    uint32_t b = blockIdx.x, e, m0, n0;
    if (b >= all) return;
    RunTile<G, 16> g;
    place(b, e, m0, n0);
    begin_weights<L>(g, p, e, m0, n0, lds);
    g.template rest<L>(lds);
    wait_first<G>();
    for (;;) {
        g.template run<L, true>(lds);
        const uint32_t e1 = e, m1 = m0, n1 = n0;
        b += gridDim.x;
        const bool more = b < all;
        if (more) {
            place(b, e, m0, n0);
            begin_weights<L>(g, p, e, m0, n0, lds);
        }
        finish_large(g, lds, [&](int row, int col, float (&v)[8]) {
            const uint32_t m = m1 + row, n = n1 + col;
            if (m < p.rows && n < p.cols)
                store_vec((TO*)p.out + e1 * p.expert_out + m * p.ld_out + n, (int)(p.cols - n), v, p.nt);
        });
        if (!more) return;
        g.template rest<L>(lds);
    }
}

// dx's tiles and dw's, in one launch: each die's workgroups take its next tile when they
// have done theirs, so that the end of the first product's last round is filled with
// tiles of the second.  The product whose k is longer comes first, and of dw's tiles
// those of the experts with the most rows.
template <typename G, typename TO, bool kTable>
__global__ __launch_bounds__(G::kThreads) void grads_large(GroupedProduct px, GroupedProduct pw, uint32_t* counters) {
    typedef RowsLie<false, 16> LX;
    typedef WeightsLie<kTable, 16> LW;
    extern __shared__ char lds[];
    RunTable& table = *(RunTable*)(lds + kLargeLds<G>);
    fill_runs<G::kBM, false>(px.g, table);
    sort_runs(px.g.experts, table);
    const uint32_t die = blockIdx.x % 8, tiles_n = (px.cols + G::kBN - 1) / G::kBN;
    const uint32_t tiles_m = min((uint32_t)__builtin_amdgcn_readfirstlane(table.tiles[px.g.experts]),
                                 group_tiles(px.g.rows, px.g.experts, G::kBM));
    const uint32_t total = tiles_m * tiles_n, q = total / 8, rest = total % 8;
    const uint32_t from = die * q + (die < rest ? die : rest), rows_tiles = q + (die < rest ? 1 : 0);
    const uint32_t wide = (pw.cols + G::kBN - 1) / G::kBN, each = (pw.rows + G::kBM - 1) / G::kBM * wide;
    const uint32_t all = each * pw.g.experts, weights_tiles = all / 8 + (die < all % 8 ? 1 : 0);
    const bool rows_first = px.k >= pw.g.rows / pw.g.experts;
    RunTile<G, 16> g;
    Run run;
    uint32_t m0, n0;
    bool rows;
    // takes up the die's tile i, if there is one
    auto take = [&](uint32_t i) {
        if (i >= rows_tiles + weights_tiles) return false;
        rows = rows_first ? i < rows_tiles : i >= weights_tiles;
        if (rows != rows_first) i -= rows_first ? rows_tiles : weights_tiles;
        if (rows) {
            uint32_t tn;
            run_in<G::kBM>(table, px.g.experts, from + i, tiles_n, run, tn);
            m0 = run.from;
            n0 = tn * G::kBN;
            begin_rows<LX, false>(g, px, run, n0, lds);
            return true;
        }
        const uint32_t b = i * 8 + die;
        const uint32_t nth = b / each, j = b - nth * each;
        const uint32_t in = j % 8 * (each / 8) + (j % 8 < each % 8 ? j % 8 : each % 8) + j / 8;
        run.expert = __builtin_amdgcn_readfirstlane(table.order[nth]);
        m0 = in / wide * G::kBM;
        n0 = in % wide * G::kBN;
        begin_weights<LW>(g, pw, run.expert, m0, n0, lds);
        return true;
    };
    auto ask_rest = [&]() {
        if (rows) g.template rest<LX>(lds);
        else g.template rest<LW>(lds);
    };
    if (!take(blockIdx.x / 8)) return;
    ask_rest();
    wait_first<G>();
    for (;;) {
        // (its answer comes while the tile is at work)
        uint32_t next = 0, none = 0;
        asm volatile("" : "+v"(none));  // (of an address that all lanes share the compiler wants the answer at once)
        if (threadIdx.x == 0) next = atomicAdd(counters + die + none, 1u);
        if (rows) g.template run<LX, true>(lds);
        else g.template run<LW, true>(lds);
        if (threadIdx.x == 0) table.next = gridDim.x / 8 + next;
        __builtin_amdgcn_s_waitcnt(0xc07f);
        lds_barrier();
        const bool was_rows = rows;
        const uint32_t e1 = run.expert, to1 = run.to, m1 = m0, n1 = n0;
        const bool more = take(__builtin_amdgcn_readfirstlane(table.next));
        if (was_rows)
            finish_large(g, lds, [&](int row, int col, float (&v)[8]) {
                const uint32_t m = m1 + row, n = n1 + col;
                if (m < to1 && n < px.cols) finish_row<typename G::T, false>(px, e1, m, n, v);
            });
        else
            finish_large(g, lds, [&](int row, int col, float (&v)[8]) {
                const uint32_t m = m1 + row, n = n1 + col;
                if (m < pw.rows && n < pw.cols)
                    store_vec((TO*)pw.out + e1 * pw.expert_out + m * pw.ld_out + n, (int)(pw.cols - n), v, pw.nt);
            });
        if (!more) return;
        ask_rest();
    }
}

// Tile shapes, small to large.
template <typename T> struct Tiles {
    typedef GemmTile<T, 1, 64, 64, 64, 2, 2, 2> Small;
    typedef GemmTile<T, 1, 128, 128, 64, 2, 4, 2> Middle;
    typedef GemmTile<T, 1, 256, 256, 64, 2, 4, 2> Large;
};
// (fp32's matrix instructions take so long that a tile needs few bytes a step: the
// middle ones are large enough)
template <> struct Tiles<float> {
    typedef GemmTile<float, 1, 64, 64, 32, 2, 2, 2> Small;
    typedef GemmTile<float, 1, 128, 128, 32, 2, 4, 2> Middle;
    typedef Middle Large;
};

template <typename G>
hipError_t launch_large(const void* kernel, void** args, uint64_t tiles, hipStream_t s) {
    static_assert(G::kStages == 2, "the strips lie where the second stage is");
    int dev = 0;
    DevInfo di;
    hipError_t e = hipGetDevice(&dev);
    if (e == hipSuccess) e = device_info(dev, &di);
    constexpr int kLds = kLargeLds<G> + (int)sizeof(RunTable);
    if (e == hipSuccess) e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    if (e != hipSuccess) return e;
    // a whole number of workgroups for each die
    const uint32_t grid = (uint32_t)std::min<uint64_t>((tiles + 7) / 8 * 8, (uint64_t)(di.cus < 8 ? 8 : di.cus / 8 * 8));
    return hipLaunchKernel(kernel, dim3(grid), dim3(G::kThreads), args, kLds, s);
}

template <typename G>
hipError_t launch_tiles(const void* kernel, const GroupedProduct& p, uint64_t grid, hipStream_t s) {
    hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, G::kLdsBytes);
    if (e != hipSuccess) return e;
    if (grid * G::kThreads >= (1ull << 32)) return hipErrorInvalidValue;
    void* args[] = {(void*)&p};
    return hipLaunchKernel(kernel, dim3((uint32_t)grid), dim3(G::kThreads), args, G::kLdsBytes, s);
}

// The kernel for pieces of 4 bytes exists for fp32 alone.
template <typename G, typename TO, bool forward>
const void* rows_kernel(const GroupedProduct& p) {
    if constexpr (G::kElem == 4)
        if (!p.wide) return (const void*)rows_product<G, TO, forward, 4>;
    return (const void*)rows_product<G, TO, forward, 16>;
}
template <typename G, typename TO>
const void* weights_kernel(const GroupedProduct& p) {
    if constexpr (G::kElem == 4)
        if (!p.wide) return p.where ? (const void*)weights_product<G, TO, true, 4> : (const void*)weights_product<G, TO, false, 4>;
    return p.where ? (const void*)weights_product<G, TO, true, 16> : (const void*)weights_product<G, TO, false, 16>;
}
template <typename G, typename TO>
const void* grads_kernel(const GroupedProduct& x, const GroupedProduct& w) {
    if constexpr (G::kElem == 4)
        if (!x.wide || !w.wide)
            return w.where ? (const void*)grads_product<G, TO, true, 4> : (const void*)grads_product<G, TO, false, 4>;
    return w.where ? (const void*)grads_product<G, TO, true, 16> : (const void*)grads_product<G, TO, false, 16>;
}

template <typename G, typename TO>
hipError_t launch_kind(int kind, const GroupedProduct& p, hipStream_t s) {
    constexpr bool kLarge = G::kBM == 256;
    const uint64_t across = (p.cols + G::kBN - 1) / G::kBN;
    const uint64_t tiles = across * (kind == kGroupedWeights ? (uint64_t)p.g.experts * ((p.rows + G::kBM - 1) / G::kBM)
                                                             : group_tiles(p.g.rows, p.g.experts, G::kBM));
    if (kind == kGroupedWeights) {
        if constexpr (kLarge) {
            void* args[] = {(void*)&p};
            return launch_large<G>(p.where ? (const void*)weights_large<G, TO, true> : (const void*)weights_large<G, TO, false>, args,
                                   tiles, s);
        } else {
            return launch_tiles<G>(weights_kernel<G, TO>(p), p, tiles, s);
        }
    }
    if constexpr (std::is_same_v<TO, typename G::T>) {
        const bool forward = kind == kGroupedForward;
        if constexpr (kLarge) {
            void* args[] = {(void*)&p};
            return launch_large<G>(forward ? (const void*)rows_large<G, TO, true> : (const void*)rows_large<G, TO, false>, args,
                                   tiles, s);
        } else {
            return launch_tiles<G>(forward ? rows_kernel<G, TO, true>(p) : rows_kernel<G, TO, false>(p), p, tiles, s);
        }
    }
    return hipErrorInvalidValue;
}

// What a tile costs (us), as in kernels_linear.hip: 64 along k alone on its
// compute unit and on a full chip, and its start and epilogue (fp32: 0.6 TFLOP/s a unit,
// its matrix instructions' rate).
struct TileCost {
    uint32_t rows, cols;
    double alone, full, ends;
};
constexpr TileCost kCost16[3] = {{64, 64, 0.30, 0.193, 0.5}, {128, 128, 0.60, 0.53, 2.0}, {256, 256, 1.05, 1.50, 11.0}};
constexpr TileCost kCost32[3] = {{64, 64, 1.0, 0.95, 1.0}, {128, 128, 3.6, 3.6, 2.0}, {128, 128, 1e9, 1e9, 0.0}};

// A product in tiles of one size: rounds over the chip's 256 units, a tile's time alone
// and on a full chip.
struct Load {
    double rounds, alone, full;
};
Load load_of(int kind, const GroupedProduct& p, const TileCost& c) {
    const double rows = (double)p.g.rows, experts = (double)p.g.experts, across = std::ceil((double)p.cols / c.cols);
    const bool weights = kind == kGroupedWeights;
    // (half a tile of every run is past its end)
    const double tiles = weights ? experts * std::ceil((double)p.rows / c.rows) * across
                                 : (rows / c.rows + std::fmin(experts, rows) * 0.5) * across;
    const double steps = std::ceil((weights ? rows / experts : (double)p.k) / 64.0);
    return Load{tiles / 256.0, steps * c.alone + c.ends, steps * c.full + c.ends};
}
// The cheapest tile for one product; least: its time.
int tile_for(int kind, int dtype, const GroupedProduct& p, double& least) {
    const TileCost* cost = dtype == BC_F32 ? kCost32 : kCost16;
    int best = 0;
    least = 1e300;
    for (int i = 0; i < 3; ++i) {
        const Load l = load_of(kind, p, cost[i]);
        const double busy = i == 2 ? std::ceil(l.rounds) * l.full : l.rounds <= 1.0 ? 0.0 : (l.rounds + 0.5) * l.full;
        const double t = std::fmax(l.alone, busy);
        if (t < least) {
            least = t;
            best = i;
        }
    }
    return best;
}
// The same for both gradients' products in one launch.
int tile_for_both(int dtype, const GroupedProduct& rows, const GroupedProduct& weights, double& least) {
    const TileCost* cost = dtype == BC_F32 ? kCost32 : kCost16;
    int best = 0;
    least = 1e300;
    for (int i = 0; i < 3; ++i) {
        const Load x = load_of(kGroupedRows, rows, cost[i]), w = load_of(kGroupedWeights, weights, cost[i]);
        const double n = x.rounds + w.rounds, busy = x.rounds * x.full + w.rounds * w.full;
        const double t = std::fmax(std::fmax(x.alone, w.alone), n <= 1.0 ? 0.0 : busy + 0.5 * std::fmin(x.full, w.full));
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
// Bound by memory, w being read once (one token through two experts of 6400x1600 in
// fp16: 8.6 us for 41 MB, 4.8 TB/s).
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

// Sixteen rows of w by up to 16 kGroups of the expert's rows on the matrix cores: the
// waves share out the inner axis and meet in LDS.  w is read once for every 32 rows of
// its expert (64 rows of 8 experts 1600x6400 in fp16: 34 us for 164 MB, 4.8 TB/s).
constexpr int kFewWaves = 8;
template <typename T, int kGroups>
__device__ __forceinline__ void few_block(const GroupedFew& a, uint32_t e, uint32_t r0, uint32_t to, float* meet) {
    typedef FewFrag<T> F;
    constexpr int kEach = F::kStep / 4, kAhead = kGroups > 1 ? 2 : 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t n0 = blockIdx.x * 16, n = n0 + (lane & 15), kl = (lane >> 4) * kEach;
    const T* w = (const T*)a.w + e * a.expert_w + (uint64_t)(n < a.cols ? n : a.cols - 1) * a.ldw;
    const T* x[kGroups];
    bool there[kGroups];
    f32x4_t acc[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const uint32_t m = r0 + g * 16 + (lane & 15), r = m < to ? m : r0;
        const uint32_t row = a.source ? (uint32_t)a.source[r] : r;
        there[g] = row < a.x_rows;  // a row from nowhere is zeros
        x[g] = (const T*)a.x + (uint64_t)(there[g] ? row : 0) * a.ldx;
        acc[g] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const uint32_t steps = (a.inner + F::kStep - 1) / F::kStep, whole = a.inner / F::kStep;
    uint32_t s = wave;
    for (; s + (kAhead - 1) * kFewWaves < whole; s += kAhead * kFewWaves) {
        typename F::type fw[kAhead], fx[kAhead][kGroups];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t k = (s + u * kFewWaves) * F::kStep + kl;
            F::load(w + k, kEach, fw[u]);
#pragma unroll
            for (int g = 0; g < kGroups; ++g) F::load(x[g] + k, there[g] ? kEach : 0, fx[u][g]);
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
            F::load(x[g] + (left ? k : 0), there[g] ? left : 0, fx);
            acc[g] = F::mma(fw, fx, acc[g]);
        }
    }
    // [wave][group][row][17]
    __syncthreads();
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
#pragma unroll
        for (int r = 0; r < 4; ++r) meet[((wave * kGroups + g) * 16 + (lane & 15)) * 17 + (lane >> 4) * 4 + r] = acc[g][r];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < 256 * kGroups; i += 64 * kFewWaves) {
        const uint64_t r = r0 + i / 16;
        const uint32_t c = n0 + i % 16;
        if (r >= to || c >= a.cols) continue;
        float v = 0.0f;
#pragma unroll
        for (int q = 0; q < kFewWaves; ++q) v += meet[(q * kGroups * 16 + i / 16) * 17 + i % 16];
        if (a.bias) v += (float)((const T*)a.bias)[e * a.ld_bias + c];
        if (a.z) ((T*)a.z)[r * a.ldz + c] = (T)v;
        ((T*)a.y)[r * a.ldy + c] = (T)activate<sizeof(T) == 4>(a.act, v);
    }
}
template <typename T>
__global__ __launch_bounds__(64 * kFewWaves) void grouped_few_tiles(GroupedFew a) {
    __shared__ float meet[kFewWaves * 2 * 16 * 17];
    uint32_t from, to;
    const int e = busy_expert(a.g, blockIdx.y, from, to);
    if (e < 0) return;
    for (uint32_t r0 = from; r0 < to; r0 += 32) {
        if (to - r0 <= 16) few_block<T, 1>(a, (uint32_t)e, r0, to, meet);
        else few_block<T, 2>(a, (uint32_t)e, r0, to, meet);
    }
}

// ---------------------------------------------------- what products are given
template <typename T>
__device__ __forceinline__ void lay_rows(const LayRows& a, uint32_t block, uint32_t blocks) {
    const uint64_t ld = plane_cols(a.cols), across = ld / 8, step = (uint64_t)blocks * 256;
    for (uint64_t i = (uint64_t)block * 256 + threadIdx.x; i < a.count * across; i += step) {
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
        store_vec((T*)a.out + r * ld + c, 8, v);
    }
}

// A workgroup 64 rows of one expert by 128 columns; all its loads go out before the
// first is used.  Bound by memory: 16384 rows of 6400 in bfloat16, with z, 109 us, 5.8
// TB/s (as part of prepare).
constexpr uint32_t kSlopeCols = 128;
template <typename T>
__device__ __forceinline__ void slope_tile(const Groups& g, const GroupedSlope& a, uint32_t block) {
    constexpr int kPasses = 4;
    __shared__ float sums[4][kSlopeCols];
    Run run;
    const uint64_t ld = plane_cols(a.cols);
    const uint32_t across = (uint32_t)(ld + kSlopeCols - 1) / kSlopeCols, tile = block / across, c0 = block % across * kSlopeCols;
    const bool some = run_of<64>(g, tile, run);
    const uint32_t lc = threadIdx.x % 16 * 8, c = c0 + lc;
    float sum[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
    if (some) {
        Raw<T, 8> v[kPasses], z[kPasses];
        int left[kPasses];
        auto fetch = [&](auto whole) {
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                const uint64_t r = run.from + threadIdx.x / 16 + 16 * i;
                left[i] = r < run.to && c < a.cols ? (int)(a.cols - c) : 0;
                v[i].template load<decltype(whole)::value>((const T*)a.dy + (left[i] > 0 ? r * a.ldd + c : 0), left[i]);
                if (a.z) z[i].template load<decltype(whole)::value>((const T*)a.z + (left[i] > 0 ? r * a.ldz + c : 0), left[i]);
            }
        };
        if (a.cols % 8 == 0 || c0 + kSlopeCols <= a.cols) fetch(std::true_type{});
        else fetch(std::false_type{});
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const uint64_t r = run.from + threadIdx.x / 16 + 16 * i;
            float d[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                d[j] = (float)v[i].v[j];
                if (a.z) d[j] = j < left[i] ? d[j] * act_slope<sizeof(T) == 4>(a.act, (float)z[i].v[j]) : 0.0f;
                sum[j] += d[j];
            }
            if (a.dz && r < run.to && c < ld) store_vec((T*)a.dz + r * ld + c, 8, d);
        }
    }
    if (!a.part) return;
    // rows of the same columns: lanes sixteen apart, then the waves
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int o = 16; o < 64; o <<= 1) sum[j] += __shfl_xor(sum[j], o, 64);
    if ((threadIdx.x & 63) < 16)
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[threadIdx.x >> 6][lc + j] = sum[j];
    __syncthreads();
    const uint32_t col = c0 + threadIdx.x;
    if (threadIdx.x < kSlopeCols && col < a.cols)
        a.part[(uint64_t)tile * a.cols + col] =
            (sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]);
}

__device__ __forceinline__ void where_rows(const Groups& g, const GroupedWhere& a, uint32_t block) {
    const uint32_t i = block * 256 + threadIdx.x;
    Run run;
    uint32_t at = kNowhere;
    if (run_of<64>(g, i / 64, run) && run.from + i % 64 < run.to) {
        const uint32_t row = (uint32_t)a.source[run.from + i % 64];
        if (row < a.x_rows) at = row * a.row_bytes;
    }
    if (i < 64 * (group_tiles(g.rows, g.experts, 64) + 1)) a.where[i] = at;
}

template <typename T>
__global__ __launch_bounds__(256) void prepare(Prepare a) {
    const uint32_t b = blockIdx.x;
    if (b < a.first[0]) slope_tile<T>(a.g, a.slope, b);
    else if (b < a.first[1]) lay_rows<T>(a.lay[0], b - a.first[0], a.first[1] - a.first[0]);
    else if (b < a.first[2]) lay_rows<T>(a.lay[1], b - a.first[1], a.first[2] - a.first[1]);
    else if (b < a.first[3]) where_rows(a.g, a.where, b - a.first[2]);
    else if (threadIdx.x < kGroupedCounters) a.counters[threadIdx.x] = 0;
}

template <typename TO>
__global__ __launch_bounds__(256) void grouped_bias(GroupedBias a) {
    __shared__ float sums[256];
    bias_columns<TO>(a, blockIdx.x, sums);
}

}  // namespace

hipError_t launch_grouped(int kind, int dtype, int out_dtype, const GroupedProduct& p, hipStream_t s) {
    if (p.cols == 0 || (kind == kGroupedWeights ? p.rows == 0 || p.g.experts == 0 : p.g.rows == 0)) return hipSuccess;
    double least;
    const int t = tile_for(kind, dtype, p, least);
    if (dtype == BC_F32) return launch_tile<float, float>(kind, t, p, s);
    if (dtype == BC_F16) {
        if (out_dtype == BC_F32) return launch_tile<f16_t, float>(kind, t, p, s);
        return launch_tile<f16_t, f16_t>(kind, t, p, s);
    }
    if (out_dtype == BC_F32) return launch_tile<bf16_t, float>(kind, t, p, s);
    return launch_tile<bf16_t, bf16_t>(kind, t, p, s);
}

template <typename G, typename TO>
static hipError_t pair_of(GroupedProduct x, GroupedProduct w, GroupedBias bias, uint32_t* counters, hipStream_t s) {
    const uint64_t tiles_x = group_tiles(x.g.rows, x.g.experts, G::kBM) * ((uint64_t)(x.cols + G::kBN - 1) / G::kBN);
    const uint64_t tiles_w = (uint64_t)w.g.experts * ((w.rows + G::kBM - 1) / G::kBM) * ((w.cols + G::kBN - 1) / G::kBN);
    if constexpr (G::kBM == 256) {
        if (bias.out) {
            const hipError_t e = launch_grouped_bias(sizeof(TO) == 4 ? (int)BC_F32 : __is_same(TO, f16_t) ? (int)BC_F16 : (int)BC_BF16, bias, s);
            if (e != hipSuccess) return e;
        }
        void* args[] = {&x, &w, &counters};
        return launch_large<G>(w.where ? (const void*)grads_large<G, TO, true> : (const void*)grads_large<G, TO, false>, args,
                               tiles_x + tiles_w, s);
    } else {
        bool rows_first = x.k >= w.g.rows / w.g.experts;
        uint32_t split = (uint32_t)(rows_first ? tiles_x : tiles_w), end = (uint32_t)(tiles_x + tiles_w);
        const uint64_t grid = end + (bias.out ? (uint64_t)bias.g.experts * ((bias.cols + 63) / 64) : 0);
        const void* kernel = grads_kernel<G, TO>(x, w);
        const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, G::kLdsBytes);
        if (e != hipSuccess) return e;
        if (grid * G::kThreads >= (1ull << 32)) return hipErrorInvalidValue;
        void* args[] = {&x, &w, &bias, &split, &end, &rows_first};
        return hipLaunchKernel(kernel, dim3((uint32_t)grid), dim3(G::kThreads), args, G::kLdsBytes, s);
    }
}

template <typename T, typename TO>
static hipError_t pair_tile(int tile, const GroupedProduct& x, const GroupedProduct& w, const GroupedBias& bias,
                            uint32_t* counters, hipStream_t s) {
    if (tile == 0) return pair_of<typename Tiles<T>::Small, TO>(x, w, bias, counters, s);
    if (tile == 1) return pair_of<typename Tiles<T>::Middle, TO>(x, w, bias, counters, s);
    return pair_of<typename Tiles<T>::Large, TO>(x, w, bias, counters, s);
}

hipError_t launch_grouped_pair(int dtype, int out_dtype, const GroupedProduct& x, const GroupedProduct& w, const GroupedBias& bias,
                               uint32_t* counters, hipStream_t s) {
    double both = 0.0, tx = 0.0, tw = 0.0;
    const int of_x = tile_for(kGroupedRows, dtype, x, tx), of_w = tile_for(kGroupedWeights, dtype, w, tw);
    const int tile = tile_for_both(dtype, x, w, both);
    // (a launch of its own: 3 us, and the bias's another 3.  Where both products want the
    // largest tiles, as the experts' runs leave their rounds more ragged than the costs
    // say: 16 experts' 16384 rows of 1600 to 6400 872 to 847 us, all with 1024 rows 793 to 776)
    if ((tile == 2 && of_x == 2 && of_w == 2) || both < tx + tw + 3.0 + (bias.out && tile < 2 ? 3.0 : 0.0)) {
        if (dtype == BC_F32) return pair_tile<float, float>(tile, x, w, bias, counters, s);
        if (dtype == BC_F16) {
            if (out_dtype == BC_F32) return pair_tile<f16_t, float>(tile, x, w, bias, counters, s);
            return pair_tile<f16_t, f16_t>(tile, x, w, bias, counters, s);
        }
        if (out_dtype == BC_F32) return pair_tile<bf16_t, float>(tile, x, w, bias, counters, s);
        return pair_tile<bf16_t, bf16_t>(tile, x, w, bias, counters, s);
    }
    hipError_t e = bias.out ? launch_grouped_bias(out_dtype, bias, s) : hipSuccess;
    if (e == hipSuccess) e = launch_grouped(kGroupedRows, dtype, dtype, x, s);
    return e != hipSuccess ? e : launch_grouped(kGroupedWeights, dtype, out_dtype, w, s);
}

template <typename T>
static void few_of(const GroupedFew& a, hipStream_t s) {
    if (a.g.rows > (sizeof(T) == 4 ? 8 : 4)) {
        hipLaunchKernelGGL(grouped_few_tiles<T>, dim3((a.cols + 15) / 16, std::min(a.g.experts, a.g.rows)), dim3(64 * kFewWaves), 0, s, a);
        return;
    }
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

hipError_t launch_prepare(int dtype, Prepare& a, hipStream_t s) {
    uint64_t n = 0;
    if (a.slope.dz || a.slope.part) n += (plane_cols(a.slope.cols) + kSlopeCols - 1) / kSlopeCols * group_tiles(a.g.rows, a.g.experts, 64);
    for (int i = 0; i < 2; ++i) {
        a.first[i] = (uint32_t)n;
        if (a.lay[i].out) n += std::min<uint64_t>((a.lay[i].count * (plane_cols(a.lay[i].cols) / 8) + 255) / 256, 1u << 20);
    }
    a.first[2] = (uint32_t)n;
    if (a.where.where) n += (64 * (group_tiles(a.g.rows, a.g.experts, 64) + 1) + 255) / 256;
    a.first[3] = (uint32_t)n;
    if (a.counters) n += 1;
    a.first[4] = (uint32_t)n;
    if (n == 0) return hipSuccess;
    if (n * 256 >= (1ull << 32)) return hipErrorInvalidValue;
    const dim3 grid((uint32_t)n), block(256);
    if (dtype == BC_F32) hipLaunchKernelGGL(prepare<float>, grid, block, 0, s, a);
    else if (dtype == BC_F16) hipLaunchKernelGGL(prepare<f16_t>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(prepare<bf16_t>, grid, block, 0, s, a);
    return hipGetLastError();
}

hipError_t launch_grouped_bias(int out_dtype, const GroupedBias& a, hipStream_t s) {
    const dim3 grid((a.cols + 63) / 64 * a.g.experts), block(256);
    if (out_dtype == BC_F32) hipLaunchKernelGGL(grouped_bias<float>, grid, block, 0, s, a);
    else if (out_dtype == BC_F16) hipLaunchKernelGGL(grouped_bias<f16_t>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(grouped_bias<bf16_t>, grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace bc
