// layers.hpp -- arguments and launchers of the layer and optimizer kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "elem.hpp"

namespace bc {

// ------------------------------------------------------------ layer norm
struct LnForward {
    const void *x, *weight, *bias;
    void* y;
    float *mean, *rstd;
    uint64_t rows, ldx, ldy;
    uint32_t cols;
    float inv_cols, eps;
    bool nt;                // y is written with the non-temporal hint
};
struct LnBackward {
    const void *dy, *x, *weight;
    const float *mean, *rstd;
    void* dx;
    float* part;            // [parts][2][cols] column sums, NULL: not wanted
    uint64_t rows, lddy, ldx, lddx;
    uint32_t cols, parts;
    float inv_cols;
    bool nt;                // dx likewise
};
// Workgroups that leave column sums for a call of this shape.
uint32_t ln_parts(uint64_t rows, uint32_t cols, int dtype);
hipError_t launch_ln_forward(int dtype, int wdtype, const LnForward& a, hipStream_t s);
hipError_t launch_ln_backward(int dtype, int wdtype, const LnBackward& a, void* dweight, void* dbias, hipStream_t s);
// out0[c] = sum over r of part[r * stride + c], out1 likewise of the cols
// values after them; either may be NULL.
hipError_t launch_sum_parts(int dtype, const float* part, uint32_t parts, uint64_t stride, uint32_t cols, void* out0,
                            void* out1, hipStream_t s);

// ---------------------------------------------------------- linear layer
// Operand planes of the product kernels (gemm.hpp): 16-bit elements, rows
// `ld` apart, a multiple of kPlaneCols long and zero past the operand's end.
constexpr uint32_t kPlaneCols = 64;
__host__ __device__ constexpr uint64_t plane_cols(uint64_t k) { return (k + kPlaneCols - 1) / kPlaneCols * kPlaneCols; }
// Planes of an element type: fp32 as three bfloat16 parts.
inline int planes_of(int dtype) { return dtype == BC_F32 ? 3 : 1; }

// An operand for the product kernels: planes in memory.
struct Planes {
    const void* p;
    uint64_t ld, plane;      // elements from row to row, from plane to plane
};

// A matrix laid out as planes: v = in, or in * act'(z) where z is given.
struct LayOut {
    const void *in, *z;
    uint64_t ld_in, ld_z;
    uint32_t rows, cols;
    void* flat;              // [P][rows][plane_cols(cols)], or NULL
    void* turned;            // [P][cols][plane_cols(rows)], or NULL
    float* part;             // [ceil(rows / 64)][cols] column sums of v, or NULL
    int act;
};
// Up to three matrices in one launch.
struct LayOuts {
    LayOut of[3];
    uint32_t first[3];       // workgroups before each (those past `count`: all)
    int count;
};
hipError_t launch_lay_outs(int dtype, LayOuts& a, hipStream_t s);

// out [rows, cols] = epilogue(A B^T), A [rows, k], B [cols, k] as planes.
struct Product {
    Planes a, b;
    uint32_t rows, cols, steps;   // steps of kPlaneCols along k
    void* out;
    uint64_t ld_out;
    // forward only: z = product + bias, out = act(z) + residual
    const void *bias, *residual;
    void* z;
    uint64_t ld_residual, ld_z;
    int act;
    bool nt;                      // out and z are written with the non-temporal hint
    float* part;                  // [split][rows][cols] sums of the parts of k, with split > 1
    uint32_t split;
};
// How a product of this shape is cut: the tiles' index and the parts of k (more
// than one where tiles are few and long; their sums then need
// split_bytes of workspace).
struct Cut {
    int tile;
    uint32_t split;
};
Cut product_cut(int dtype, uint64_t rows, uint64_t cols, uint64_t k);
inline uint64_t split_bytes(const Cut& c, uint64_t rows, uint64_t cols) {
    return c.split > 1 ? c.split * rows * cols * sizeof(float) : 0;
}
// The tile for two products of these shapes in one launch, or -1 where two
// launches are better.
struct Shape {
    uint64_t rows, cols, k;
};
int pair_tile(int dtype, const Shape& a, const Shape& b);
struct Products {
    Product of[2];
    uint32_t first;          // workgroups before the second
};
hipError_t launch_product(int dtype, int out_dtype, bool forward, const Cut& cut, const Product& p, hipStream_t s);
// Both gradients' products in one launch, neither split, both out in `dtype`.
hipError_t launch_pair(int dtype, int tile, const Product& first, const Product& second, hipStream_t s);

// The forward pass for few rows: x and w as the caller has them.
struct FewRows {
    const void *x, *w, *bias, *residual;
    void *y, *z;
    uint64_t ldx, ldw, ld_residual, ldy, ldz;
    uint32_t rows, inner, cols;
    int act;
};
// Up to so many rows, which then need no workspace.  (64 rows of 4096 by 4096 in
// fp32 38.7 us, by tiles, which take fp32 as planes, 61.2; in fp16 32 rows of 768
// by 768 4.2 and 6.1, of 1600 by 6400 11.3 and 14.6; 64 rows 5.9 and 6.2, 17.5 and
// 14.8, but of 6400 by 1600 30.7 and 14.1, with tiles cut along k and 3 MB of
// workspace: a small batch without one is worth that to its caller.)
constexpr uint32_t kFewRows = 64;
hipError_t launch_few_rows(int dtype, const FewRows& a, hipStream_t s);

// -------------------------------------------------- orthogonalised updates
// One matrix of a call (device table).  X is the matrix with its shorter side
// m as rows (turned: the caller's has it as columns), n the longer side.  The
// workspace holds, as two fp16 planes each, X [m][plane_cols(n)], X^T twice
// [n][plane_cols(m)] (a product reads one and writes the other), and three
// symmetric matrices [m][plane_cols(m)].
constexpr int kOrthoSides = 3;          // tiles 64, 128 and 256 wide
struct Ortho {
    const void* in;          // update, or gradient
    void* out;               // result, or weight
    float* momentum;         // NULL: the update is `in`
    uint64_t ld_in, ld_out, ld_momentum;
    uint64_t x, xt, sym, part;           // byte offsets in the workspace
    uint32_t rows, cols, m, n;
    uint32_t turned, parts;  // parts: partial sums of squares
    uint32_t part0;          // workgroups before this matrix's: of the norm,
    uint32_t tile0;          // of the 64 x 64 tiles of the start
    float step_scale;        // the update's factor beside the learning rate
    uint32_t group;          // OrthoPlan's group that it goes through the products with
};
// (the table is compared by its bytes: no padding)
static_assert(sizeof(Ortho) == 8 * 10 + 4 * 10, "Ortho layout");

// What a workgroup of a product launch computes: a tile of a matrix, or
// nothing (matrix kOrthoIdle).  It carries what all but the last product need of
// the matrix, so that a workgroup's operands are one load from its start.  A
// tile of long products is cut along k into parts: a workgroup each, whose sums
// lie from slot `sums` on, and the last to count itself at `met` adds them.
struct OrthoWork {
    uint32_t matrix, tile, m, n;
    uint32_t x, xt, sym;     // offsets in the workspace, in 256 bytes
    uint32_t part, parts, sums, met;
};
static_assert(sizeof(OrthoWork) == 44, "OrthoWork layout");
constexpr uint32_t kOrthoIdle = 0xFFFFFFFFu;

// The work of a launch with one tile side: tiles, and steps of 32 along k, in
// all and of the longest tile.
struct OrthoLoad {
    double tiles, steps, longest;
};
struct OrthoCall {
    const Ortho* d;
    char* ws;
    int T;
    int in_dtype, out_dtype;
    uint32_t parts, tiles;   // workgroups of the norm and of the start
    uint32_t slots;          // for sums of tiles cut along k: kOrthoSlots at most,
    uint64_t meet;           // from here on in the workspace, after as many counters
    double eps;
    float a, b, c;
    float x_scale;           // X is kept times this power of two
    float scale[4];          // of the symmetric matrices by what they hold (SymScale)
    bool muon, nesterov;
    float momentum, keep, lr;   // keep: 1 - lr * weight decay
};
enum SymScale { kScaleGram, kScalePoly, kScaleTurn, kScalePair };
// Products of a call by what bounds their work lists: X X^T, the symmetric
// m x m ones, and those with X's shape.
enum OrthoKind { kOrthoGram, kOrthoSym, kOrthoFull, kOrthoKinds };
// Matrices that go through the products together: [1] may take two steps from
// one Gram matrix, [0], the small ones of a call with fp32 results, keep more
// digits without (see kernels_ortho.hip).
constexpr uint32_t kOrthoPairs = 64;
// Tiles 64 wide may be cut along k into parts of at least kOrthoPart, whose sums
// meet in kOrthoSlots slots at most.
constexpr uint64_t kOrthoPart = 512, kOrthoSlots = 512, kOrthoSlotBytes = 64 * 64 * sizeof(float);
struct OrthoGroup {
    OrthoLoad load[kOrthoKinds][kOrthoSides];
    double chain[kOrthoKinds];         // the most steps of 32 that a 64-wide tile is left with
    int side[kOrthoKinds];             // the tile side chosen (ortho_choose)
    uint32_t workgroups[kOrthoKinds];  // and its launch's size (0: no matrix)
    const OrthoWork* list[kOrthoKinds];
    bool pairs;                        // two steps from one Gram matrix
};
struct OrthoPlan {
    OrthoCall c;
    int steps, cus;
    OrthoGroup group[2];               // [1]: the larger matrices
};
inline uint32_t ortho_group(const OrthoCall& c, uint32_t m) { return c.out_dtype != BC_F32 || m >= kOrthoPairs; }
// Picks tile sides and the schedule from the loads.
void ortho_choose(OrthoGroup& g, bool may_pair, int cus);
constexpr uint32_t kOrthoParts = 256;
hipError_t launch_orthogonalize(const OrthoPlan& p, hipStream_t s);

}  // namespace bc
