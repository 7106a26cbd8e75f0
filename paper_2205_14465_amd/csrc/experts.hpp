// experts.hpp -- arguments and launchers of the kernels of a block of experts
// (router, grouped linear layer, combination) and of the gradients' norm and
// clipping.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "layers.hpp"

namespace bc {

// ---------------------------------------------------------------- router
constexpr uint32_t kMaxExperts = 1024, kMaxChoices = 32;
struct Route {
    const void* logits;
    uint64_t ld;
    uint64_t rows;
    uint32_t experts, k;
    int normalise;
    float* weight;
    int32_t *expert, *slot, *source, *offsets;
    uint32_t* count;         // [experts][blocks], then [experts] totals; or [blocks][experts] (add)
    uint32_t blocks;         // workgroups of route_gate
    uint32_t block_rows;     // rows of each, a multiple of 64
    bool add;                // set by launch_route: the last launch adds the counts up
};
uint32_t route_block_rows(uint64_t rows, uint32_t experts);
hipError_t launch_route(int dtype, Route a, hipStream_t s);

struct RouteGrad {
    const void* logits;
    const float *weight, *dweight;
    const int32_t* expert;
    void* dlogits;
    uint64_t ld, ld_d, rows;
    uint32_t experts, k;
    int normalise;
};
hipError_t launch_route_grad(int dtype, const RouteGrad& a, hipStream_t s);

// ----------------------------------------------------------- combination
struct Combine {
    const void* y;           // [slots, cols]
    const int32_t* slot;     // [rows, k]
    const float* weight;     // [rows, k], or NULL: 1
    const void* residual;
    void* out;
    uint64_t ldy, ldr, ld_out, rows;
    uint32_t cols, k, slots;
    bool nt;
};
hipError_t launch_combine(int dtype, const Combine& a, hipStream_t s);

struct CombineGrad {
    const void *dout, *y;
    const int32_t* slot;
    const float* weight;
    void* dy;                // NULL: not wanted
    float* dweight;          // NULL: not wanted
    uint64_t ldd, ldy, lddy, rows;
    uint32_t cols, k, slots;
    bool nt;
};
hipError_t launch_combine_grad(int dtype, const CombineGrad& a, hipStream_t s);

// ------------------------------------------------- grouped linear layer
// Rows [offsets[e], offsets[e + 1]) of the call's `rows` are expert e's.
struct Groups {
    const int32_t* offsets;  // [experts + 1], ascending
    uint32_t experts, rows;
};
// Pieces of `high` rows: expert e has those from offsets[e] / high - offsets[0] /
// high + e on up to its successor's first, the last of which may be empty, so that a
// piece's expert is found by comparisons alone.  There are at most so many, which
// bounds the tiles with rows as well:
__host__ __device__ inline uint32_t group_tiles(uint32_t rows, uint32_t experts, uint32_t high) { return rows / high + experts; }

// A matrix for every expert, or one for all.
struct GroupedSide {
    const void* p;
    uint64_t ld, expert;     // elements from row to row, expert to expert
};
enum GroupedKind { kGroupedForward, kGroupedRows, kGroupedWeights };
struct GroupedProduct {
    Groups g;
    GroupedSide a, b;
    const int32_t* source;   // forward: rows of a; NULL: the call's own
    const uint32_t* where;   // weights: byte offsets of b's rows, the experts' padded to whole 64s; NULL: as they lie
    uint32_t a_rows;
    uint32_t rows, cols, k;  // of a result; rows and k where the experts' rows do not give them
    void* out;
    uint64_t ld_out, expert_out;
    const void* bias;
    void* z;
    uint64_t ld_bias, ld_z;
    int act;
    bool nt;
    bool wide;               // both operands' rows are whole 16-byte pieces (16-bit ones: always)
};
hipError_t launch_grouped(int kind, int dtype, int out_dtype, const GroupedProduct& p, hipStream_t s);
// dbias [experts][cols], rows ld apart, from the sums over 64 rows each of
// GroupedSlope.
struct GroupedBias {
    Groups g;
    const float* part;
    void* out;
    uint64_t ld;
    uint32_t cols;
};
hipError_t launch_grouped_bias(int out_dtype, const GroupedBias& a, hipStream_t s);
// Both gradients' products, none of them empty, and the bias's gradient where
// bias.out is given.  counters: kGroupedCounters words, zero (launch_prepare).
constexpr uint32_t kGroupedCounters = 8;
hipError_t launch_grouped_pair(int dtype, int out_dtype, const GroupedProduct& rows, const GroupedProduct& weights,
                               const GroupedBias& bias, uint32_t* counters, hipStream_t s);

// The forward pass for few rows, which needs no workspace: up to 64 in all; more in
// fp32, whose tiles are bound by the matrix instructions wherever rows fill them badly,
// and where 16-bit operands would be laid out first (weights in rows of no whole pieces,
// a gather from more than 2 GB).  us, this way and by tiles, with rows spread evenly (all
// with one expert): fp32, 8 experts of 1600x1600, 100 rows 25 (34) and 34 (32), 192 34
// (55) and 34 (32); 64 experts 128 rows 133 (44) and 189 (32), 500 164 (144) and 189
// (36); fp16, 64 experts of 768x768, 64 rows 15 and 13, of 1001x515 256 rows 32 and 36,
// 1024 47 and 38, 8 experts 128 rows 12 and 20, 256 19 and 20.  The limit goes by all
// experts, an expert's rows by one workgroup for 16 columns, 32 at a time: with very many
// experts, and the more so where one has all the rows, it is too high (at the limit, fp32,
// 128 experts of 768x768, 1088 rows 77 (167) and 86 (19); 1024 of 256x256, 8256 rows 147
// (582) and 99 (45); fp16, 128 of 769x769 99 (269) and 93 (69)).
inline uint64_t grouped_few_rows(int dtype, uint32_t experts, bool laid_out) {
    return 64 + (dtype == BC_F32 || laid_out ? 8ull * experts : 0);
}
struct GroupedFew {
    Groups g;
    const void *x, *w, *bias;
    const int32_t* source;
    void *y, *z;
    uint64_t ldx, ldw, expert_w, ld_bias, ldy, ldz;
    uint32_t x_rows, inner, cols;
    int act;
};
hipError_t launch_grouped_few(int dtype, const GroupedFew& a, hipStream_t s);

// What the products need first, in one launch; a part whose output is NULL is left out.
// Rows laid out as [count][plane_cols(cols)]: row r is row r % group of the matrix
// r / group, or row source[r] of the only one (zeros where there is none).
struct LayRows {
    const void* in;
    const int32_t* source;
    void* out;
    uint64_t ld, matrix, count, group;
    uint32_t cols, in_rows;
};
// dz = dy act'(z) of the experts' rows as [rows][plane_cols(cols)], and its
// sums over every tile of 64 rows.
struct GroupedSlope {
    const void *dy, *z;      // z NULL: dz = dy
    void* dz;                // NULL: sums only
    float* part;             // [group_tiles(rows, experts, 64)][cols], NULL: not wanted
    uint64_t ldd, ldz;
    uint32_t cols;
    int act;
};
// Byte offsets of the rows source[r] of a matrix, every expert's from a multiple of 64
// on, kNowhere in between.
struct GroupedWhere {
    const int32_t* source;
    uint32_t* where;         // [64 (group_tiles(rows, experts, 64) + 1)]
    uint32_t x_rows, row_bytes;
};
struct Prepare {
    Groups g;
    GroupedSlope slope;
    LayRows lay[2];
    GroupedWhere where;
    uint32_t* counters;      // set to zero
    uint32_t first[5];       // workgroups before lay[0], lay[1], where and counters, and in all
};
hipError_t launch_prepare(int dtype, Prepare& a, hipStream_t s);

// --------------------------------------------------- norm and clipping
// One matrix of a list (device table; compared by its bytes: no padding).
// Its elements are taken in pieces of eight of a row, kClipChunk pieces to a chunk.
struct ClipDesc {
    const void* in;
    void* out;
    uint64_t ld_in, ld_out, cols, pieces;
    uint64_t chunk0;         // chunks before this matrix's
    uint32_t row_pieces;     // pieces of a row; 0: one row
    uint32_t dtype;
};
static_assert(sizeof(ClipDesc) == 64, "ClipDesc layout");
constexpr uint32_t kClipChunk = 256, kClipParts = 2048;
struct Clip {
    const ClipDesc* d;
    uint32_t T;
    int kind;
    uint64_t chunks;
    double* part;            // [parts]
    uint32_t parts;          // workgroups of the norm's pass
    double max_norm;
    const double* given;     // the norm, computed elsewhere; NULL: from the parts
    double* norm;            // results; NULL: not wanted
    float* factor;
    bool nt;
};
uint32_t clip_parts(uint64_t chunks);
hipError_t launch_grad_norm(const Clip& a, hipStream_t s);   // parts
hipError_t launch_norm_of_parts(const Clip& a, hipStream_t s);
hipError_t launch_clip(const Clip& a, hipStream_t s);
// Writes a table into device memory by launches that carry it as arguments.
hipError_t launch_write_table(void* to, const void* from, size_t bytes, hipStream_t s);

}  // namespace bc
