// api_experts.hip -- the C ABI of a block of experts and of the gradients' norm
// and clipping (include/bytecomp.h): argument checks on the host, workspace
// carving, and the launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "../../include/bytecomp.h"
#include "experts.hpp"
#include "launch.hpp"

using namespace bc;

namespace {

int status_of(hipError_t e) { return e == hipSuccess ? BC_OK : BC_E_HIP; }
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
bool misaligned(const void* p, int dtype) { return ((uintptr_t)p & (dtype_bytes(dtype) - 1)) != 0; }
bool misaligned4(const void* p) { return ((uintptr_t)p & 3) != 0; }

// ----------------------------------------------------------------- router
constexpr uint64_t kMaxTokens = 1ull << 29, kMaxSlots = 1ull << 31;

int check_route(uint64_t rows, uint32_t experts, uint32_t k) {
    if (experts < 1 || experts > kMaxExperts || k < 1 || k > kMaxChoices || k > experts) return BC_E_COUNT;
    if (rows >= kMaxTokens || rows * k >= kMaxSlots) return BC_E_SIZE;
    return BC_OK;
}

uint32_t route_blocks(uint64_t rows, uint32_t experts) {
    const uint32_t n = route_block_rows(rows, experts);
    return (uint32_t)((rows + n - 1) / n);
}

size_t route_ws(uint64_t rows, uint32_t experts) {
    const uint32_t blocks = route_blocks(rows, experts);
    return blocks <= 1 ? 0 : ((size_t)blocks + 1) * experts * sizeof(uint32_t);
}

// ------------------------------------------------------------ combination
constexpr uint64_t kMaxCols = 1ull << 24;

int check_combine(int dtype, uint64_t rows, uint64_t cols, uint32_t k, uint64_t slots) {
    if (!dtype_ok(dtype)) return BC_E_DTYPE;
    if (k < 1 || k > kMaxChoices) return BC_E_COUNT;
    if (rows >= kMaxTokens || rows * k >= kMaxSlots || slots >= kMaxSlots || cols >= kMaxCols) return BC_E_SIZE;
    return BC_OK;
}

// -------------------------------------------------- grouped linear layer
constexpr uint64_t kMaxGroupedRows = 1ull << 22, kMaxSide = 1ull << 20, kMaxElements = 1ull << 35;

int check_grouped(int dtype, uint64_t rows, uint64_t inner, uint64_t cols, uint32_t experts, uint64_t x_rows) {
    if (!dtype_ok(dtype)) return BC_E_DTYPE;
    if (experts < 1 || experts > kMaxExperts) return BC_E_COUNT;
    if (rows >= kMaxGroupedRows || x_rows >= (1ull << 31) || inner >= kMaxSide || cols >= kMaxSide) return BC_E_SIZE;
    // workgroups of a launch stay within 32 bits of threads
    const uint64_t i = plane_cols(inner), c = plane_cols(cols), wide = std::max(i, c);
    if ((rows + 64ull * experts) * wide >= kMaxElements || experts * (i / 64) * (c / 64) >= kMaxElements / 4096) return BC_E_SIZE;
    return BC_OK;
}

// Bytes of rows laid out for the tiles.
size_t laid_bytes(int dtype, uint64_t rows, uint64_t k) {
    return align256((size_t)(rows * plane_cols(k) * dtype_bytes(dtype)));
}

// Whether rows of k are whole 16-byte pieces.
bool whole(int dtype, const void* p, uint64_t ld, uint64_t k) {
    const uint64_t each = 16 / dtype_bytes(dtype);
    return k % each == 0 && ((uintptr_t)p & 15) == 0 && ld % each == 0;
}
// Whether the tiles can read rows of k where they lie: fp32 in any pieces.
bool readable(int dtype, const void* p, uint64_t ld, uint64_t k) {
    return dtype == BC_F32 || whole(dtype, p, ld, k);
}
// Byte offsets within a tile are 32-bit: row strides below this, in elements.
constexpr uint64_t kMaxStride = 1ull << 21;
// So are those of gathered rows.
constexpr uint64_t kGatherBytes = 0x7fffff00u;
bool in_reach(int dtype, bool gather, uint64_t x_rows, uint64_t ldx) {
    return !gather || x_rows * ldx * dtype_bytes(dtype) <= kGatherBytes;
}

// x laid out: its own rows, or, where the call takes fewer or they are too many
// for 32-bit offsets, the call's rows one after the other.
bool lay_own_rows(int dtype, bool gather, uint64_t rows, uint64_t x_rows, uint64_t inner) {
    return !gather || (x_rows <= rows && x_rows * plane_cols(inner) * dtype_bytes(dtype) <= kGatherBytes);
}

struct Carver {
    char* at;
    size_t used;
    void* take(size_t bytes) {
        char* p = at ? at + used : nullptr;
        used += align256(bytes);
        return p;
    }
};

size_t where_bytes(uint64_t rows, uint32_t experts) {
    return align256(64ull * (group_tiles((uint32_t)rows, experts, 64) + 1) * 4);
}
size_t part_bytes(uint64_t rows, uint32_t experts, uint64_t cols) {
    return align256((size_t)group_tiles((uint32_t)rows, experts, 64) * cols * 4);
}

size_t grouped_ws(int dtype, uint64_t rows, uint64_t inner, uint64_t cols, uint32_t experts, bool backward) {
    if (rows == 0) return 0;
    // (fp32: a gather from more than 2 GB lays x out, nothing does w)
    const size_t x = laid_bytes(dtype, rows, inner), w = dtype == BC_F32 ? 0 : laid_bytes(dtype, experts * cols, inner);
    if (!backward) return rows <= grouped_few_rows(dtype, experts, true) ? 0 : x + w;
    return x + w + laid_bytes(dtype, rows, cols) + part_bytes(rows, experts, cols) + where_bytes(rows, experts) +
           align256(kGroupedCounters * sizeof(uint32_t));
}

struct GroupedX {
    const void* x;
    uint64_t ld;
    const int32_t* source;
    uint64_t rows, call_rows, inner;
};
// x for the tiles; `source` becomes NULL where its rows now follow each other.
GroupedSide side_of_x(int dtype, GroupedX& x, uint32_t& a_rows, bool& wide, Carver& c, LayRows& lay) {
    const bool gather = x.source != nullptr;
    a_rows = (uint32_t)(gather ? x.rows : x.call_rows);
    if (readable(dtype, x.x, x.ld, x.inner) && in_reach(dtype, gather, x.rows, x.ld)) {
        wide = wide && whole(dtype, x.x, x.ld, x.inner);
        return GroupedSide{x.x, x.ld, 0};
    }
    const bool own = lay_own_rows(dtype, gather, x.call_rows, x.rows, x.inner);
    const uint64_t n = gather && own ? x.rows : x.call_rows, pc = plane_cols(x.inner);
    void* to = c.take(laid_bytes(dtype, n, x.inner));
    lay = LayRows{x.x, own ? nullptr : x.source, to, x.ld, 0, n, n, (uint32_t)x.inner, (uint32_t)x.rows};
    if (!own) {
        x.source = nullptr;
        a_rows = (uint32_t)x.call_rows;
    }
    return GroupedSide{to, pc, 0};
}
GroupedSide side_of_w(int dtype, const void* w, uint64_t ld, uint64_t expert, uint32_t experts, uint64_t cols, uint64_t inner,
                      bool& wide, Carver& c, LayRows& lay) {
    const bool aligned = whole(dtype, w, ld, inner) && expert * dtype_bytes(dtype) % 16 == 0;
    if (readable(dtype, w, ld, inner) && (dtype == BC_F32 || aligned)) {
        wide = wide && aligned;
        return GroupedSide{w, ld, expert};
    }
    const uint64_t pc = plane_cols(inner), n = experts * cols;
    void* to = c.take(laid_bytes(dtype, n, inner));
    lay = LayRows{w, nullptr, to, ld, expert, n, cols, (uint32_t)inner, 0};
    return GroupedSide{to, pc, cols * pc};
}

// ------------------------------------------------------ norm and clipping
constexpr int kMaxGrads = 1 << 20;
constexpr size_t kPartBytes = kClipParts * sizeof(double);

// A list's checks and its table.
int clip_table(const bc_grad* t, int T, bool scale, std::vector<ClipDesc>& d, uint64_t& chunks, uint64_t& bytes) {
    d.reserve((size_t)T);
    chunks = bytes = 0;
    for (int i = 0; i < T; ++i) {
        const bc_grad& g = t[i];
        if (!dtype_ok((int)g.dtype)) return BC_E_DTYPE;
        if (g.rows >= (1ull << 48) || g.cols >= (1ull << 48) || (g.rows && g.cols >= (1ull << 48) / g.rows)) return BC_E_SIZE;
        if (g.rows == 0 || g.cols == 0) continue;
        if (!g.grad || (scale && !g.out)) return BC_E_NULL;
        if (g.ld_grad < g.cols || (scale && g.ld_out < g.cols)) return BC_E_SIZE;
        if (misaligned(g.grad, (int)g.dtype) || (scale && misaligned(g.out, (int)g.dtype))) return BC_E_ALIGN;
        ClipDesc o;
        std::memset((void*)&o, 0, sizeof(o));
        o.in = g.grad;
        o.dtype = g.dtype;
        if (scale) o.out = g.out;
        // rows that follow each other are one
        if (g.rows == 1 || (g.ld_grad == g.cols && (!scale || g.ld_out == g.cols))) {
            o.cols = g.rows * g.cols;
            o.pieces = (o.cols + 7) / 8;
        } else {
            const uint64_t pieces = (g.cols + 7) / 8;
            if (pieces >= (1ull << 32)) return BC_E_SIZE;
            o.ld_in = g.ld_grad;
            o.ld_out = scale ? g.ld_out : 0;
            o.cols = g.cols;
            o.row_pieces = (uint32_t)pieces;
            o.pieces = g.rows * pieces;
        }
        o.chunk0 = chunks;
        chunks += (o.pieces + kClipChunk - 1) / kClipChunk;
        bytes += g.rows * g.cols * dtype_bytes((int)g.dtype);
        d.push_back(o);
    }
    return BC_OK;
}

size_t clip_ws(int T) { return kPartBytes + (size_t)T * sizeof(ClipDesc); }

// The launches of a call on its table: `run` gets the device table.  Under
// capture the table goes to the workspace by launches that carry it, so that the
// graph holds all it needs; otherwise it comes from the descriptor cache.
template <typename F>
int with_clip_table(const std::vector<ClipDesc>& d, void* ws, hipStream_t s, F run) {
    if (d.empty()) return status_of(run((const ClipDesc*)nullptr));
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(s, &capture) != hipSuccess) return BC_E_HIP;
    const size_t bytes = d.size() * sizeof(ClipDesc);
    if (capture != hipStreamCaptureStatusNone) {
        void* at = (char*)ws + kPartBytes;
        const hipError_t e = launch_write_table(at, d.data(), bytes, s);
        return status_of(e != hipSuccess ? e : run((const ClipDesc*)at));
    }
    try {
        return status_of(with_table(d.data(), bytes, 0, [](void*, void*) {}, s,
                                    [](void* f, const void* table) { return (*(F*)f)((const ClipDesc*)table); }, &run));
    } catch (const std::bad_alloc&) {
        return BC_E_SIZE;
    }
}

int check_clip(const bc_grad* t, int T, int kind, const void* ws, size_t ws_bytes) {
    if (T < 0 || T > kMaxGrads) return BC_E_COUNT;
    if (kind != BC_NORM_L2 && kind != BC_NORM_MAX) return BC_E_KIND;
    if (T > 0 && !t) return BC_E_NULL;
    if (!ws || ws_bytes < clip_ws(T)) return BC_E_WORKSPACE;
    if ((uintptr_t)ws & 15) return BC_E_ALIGN;
    return BC_OK;
}

}  // namespace

extern "C" {

int bytecomp_route_workspace_size(uint64_t rows, uint32_t experts, uint32_t k, size_t* bytes) {
    if (!bytes) return BC_E_NULL;
    if (const int rc = check_route(rows, experts, k)) return rc;
    *bytes = route_ws(rows, experts);
    return BC_OK;
}

int bytecomp_route_forward(int dtype, uint64_t rows, uint32_t experts, uint32_t k, const void* logits, uint64_t ld,
                           int normalise, float* weight, int32_t* expert, int32_t* slot, int32_t* source,
                           int32_t* offsets, void* ws, size_t ws_bytes, void* stream) {
    const CallRange range("bytecomp_route_forward");
    if (!dtype_ok(dtype)) return BC_E_DTYPE;
    if (const int rc = check_route(rows, experts, k)) return rc;
    if (!offsets || (rows > 0 && (!logits || !weight || !expert || !slot || !source))) return BC_E_NULL;
    if (ld < experts) return BC_E_SIZE;
    if (misaligned(logits, dtype) || misaligned4(weight) || misaligned4(expert) || misaligned4(slot) ||
        misaligned4(source) || misaligned4(offsets) || misaligned4(ws))
        return BC_E_ALIGN;
    const size_t need = route_ws(rows, experts);
    if (need > 0 && (!ws || ws_bytes < need)) return BC_E_WORKSPACE;
    const uint32_t blocks = route_blocks(rows, experts);
    const Route a{logits, ld, rows, experts, k, normalise != 0, weight, expert, slot, source, offsets, (uint32_t*)ws,
                  blocks > 0 ? blocks : 1, route_block_rows(rows, experts), false};
    hipStream_t s = (hipStream_t)stream;
    return finish_call(status_of(launch_route(dtype, a, s)), s, nullptr);
}

int bytecomp_route_backward(int dtype, uint64_t rows, uint32_t experts, uint32_t k, const void* logits, uint64_t ld,
                            int normalise, const float* weight, const int32_t* expert, const float* dweight,
                            void* dlogits, uint64_t ld_dlogits, void* stream) {
    const CallRange range("bytecomp_route_backward");
    if (!dtype_ok(dtype)) return BC_E_DTYPE;
    if (const int rc = check_route(rows, experts, k)) return rc;
    if (rows == 0) return BC_OK;
    if ((!normalise && !logits) || !weight || !expert || !dweight || !dlogits) return BC_E_NULL;
    if ((!normalise && ld < experts) || ld_dlogits < experts) return BC_E_SIZE;
    if (misaligned(logits, dtype) || misaligned4(weight) || misaligned4(expert) || misaligned4(dweight) ||
        misaligned(dlogits, dtype))
        return BC_E_ALIGN;
    const RouteGrad a{logits, weight, dweight, expert, dlogits, ld, ld_dlogits, rows, experts, k, normalise != 0};
    hipStream_t s = (hipStream_t)stream;
    return finish_call(status_of(launch_route_grad(dtype, a, s)), s, nullptr);
}

int bytecomp_combine_forward(int dtype, uint64_t rows, uint64_t cols, uint32_t k, uint64_t slots, const void* y,
                             uint64_t ldy, const int32_t* slot, const float* weight, const void* residual,
                             uint64_t ld_residual, void* out, uint64_t ld_out, void* stream) {
    const CallRange range("bytecomp_combine_forward");
    if (const int rc = check_combine(dtype, rows, cols, k, slots)) return rc;
    if (rows == 0 || cols == 0) return BC_OK;
    if (!slot || !out || (slots > 0 && !y)) return BC_E_NULL;
    if (ldy < cols || ld_out < cols || (residual && ld_residual < cols)) return BC_E_SIZE;
    if (misaligned(y, dtype) || misaligned4(slot) || misaligned4(weight) || misaligned(residual, dtype) ||
        misaligned(out, dtype))
        return BC_E_ALIGN;
    const Combine a{y, slot, weight, residual, out, ldy, ld_residual, ld_out, rows, (uint32_t)cols, k, (uint32_t)slots,
                    streams(rows * cols * dtype_bytes(dtype))};
    hipStream_t s = (hipStream_t)stream;
    return finish_call(status_of(launch_combine(dtype, a, s)), s, nullptr);
}

int bytecomp_combine_backward(int dtype, uint64_t rows, uint64_t cols, uint32_t k, uint64_t slots, const void* dout,
                              uint64_t ld_dout, const void* y, uint64_t ldy, const int32_t* slot, const float* weight,
                              void* dy, uint64_t lddy, float* dweight, void* stream) {
    const CallRange range("bytecomp_combine_backward");
    if (const int rc = check_combine(dtype, rows, cols, k, slots)) return rc;
    if (rows == 0 || (!dy && !dweight) || (cols == 0 && !dweight)) return BC_OK;
    if (!slot || (cols > 0 && (!dout || (dweight && slots > 0 && !y)))) return BC_E_NULL;
    if (ld_dout < cols || (dweight && ldy < cols) || (dy && lddy < cols)) return BC_E_SIZE;
    if (misaligned(dout, dtype) || misaligned(y, dtype) || misaligned4(slot) || misaligned4(weight) ||
        misaligned(dy, dtype) || misaligned4(dweight))
        return BC_E_ALIGN;
    const CombineGrad a{dout, y, slot, weight, dy, dweight, ld_dout, ldy, lddy, rows, (uint32_t)cols, k, (uint32_t)slots,
                        streams(rows * k * cols * dtype_bytes(dtype))};
    hipStream_t s = (hipStream_t)stream;
    return finish_call(status_of(launch_combine_grad(dtype, a, s)), s, nullptr);
}

int bytecomp_grouped_linear_workspace_size(int dtype, uint64_t rows, uint64_t x_rows, uint64_t inner, uint64_t cols,
                                           uint32_t experts, int backward, size_t* bytes) {
    if (!bytes) return BC_E_NULL;
    if (const int rc = check_grouped(dtype, rows, inner, cols, experts, x_rows)) return rc;
    *bytes = grouped_ws(dtype, rows, inner, cols, experts, backward != 0);
    return BC_OK;
}

int bytecomp_grouped_linear_forward(int dtype, uint64_t rows, uint64_t inner, uint64_t cols, uint32_t experts,
                                    const int32_t* offsets, const void* x, uint64_t ldx, const int32_t* source,
                                    uint64_t x_rows, const void* w, uint64_t ldw, uint64_t expert_w, const void* bias,
                                    uint64_t ld_bias, int act, void* y, uint64_t ldy, void* z, uint64_t ldz, void* ws,
                                    size_t ws_bytes, void* stream) {
    const CallRange range("bytecomp_grouped_linear_forward");
    if (const int rc = check_grouped(dtype, rows, inner, cols, experts, source ? x_rows : 0)) return rc;
    if (act < BC_ACT_NONE || act > BC_ACT_SILU) return BC_E_KIND;
    if (rows == 0 || cols == 0) return BC_OK;
    if (!offsets || !y || (inner > 0 && ((!x && (!source || x_rows > 0)) || !w))) return BC_E_NULL;
    if (ldx < inner || ldw < inner || expert_w < (cols - 1) * ldw + inner || (bias && ld_bias < cols) || ldy < cols ||
        (z && ldz < cols) || ldx >= kMaxStride || ldw >= kMaxStride)
        return BC_E_SIZE;
    if (misaligned(x, dtype) || misaligned(w, dtype) || misaligned(bias, dtype) || misaligned(y, dtype) ||
        misaligned(z, dtype) || misaligned4(offsets) || misaligned4(source) || ((uintptr_t)ws & 15))
        return BC_E_ALIGN;
    hipStream_t s = (hipStream_t)stream;
    const Groups g{offsets, experts, (uint32_t)rows};
    const bool lies = readable(dtype, x, ldx, inner) && in_reach(dtype, source, x_rows, ldx) && readable(dtype, w, ldw, inner) &&
                      (dtype == BC_F32 || expert_w % 8 == 0);
    if (rows <= grouped_few_rows(dtype, experts, !lies)) {
        const GroupedFew a{g, x, w, bias, source, y, z, ldx, ldw, expert_w, ld_bias, ldy, ldz,
                           (uint32_t)(source ? x_rows : rows), (uint32_t)inner, (uint32_t)cols, act};
        return finish_call(status_of(launch_grouped_few(dtype, a, s)), s, nullptr);
    }
    Carver c{(char*)ws, 0};
    GroupedX gx{x, ldx, source, x_rows, rows, inner};
    Prepare pre{};
    pre.g = g;
    GroupedProduct p{};
    p.g = g;
    p.wide = true;
    p.a = side_of_x(dtype, gx, p.a_rows, p.wide, c, pre.lay[0]);
    p.b = side_of_w(dtype, w, ldw, expert_w, experts, cols, inner, p.wide, c, pre.lay[1]);
    if (c.used > 0 && (!ws || ws_bytes < c.used)) return BC_E_WORKSPACE;
    p.source = gx.source;
    p.cols = (uint32_t)cols;
    p.k = (uint32_t)inner;
    p.out = y;
    p.ld_out = ldy;
    p.bias = bias;
    p.ld_bias = ld_bias;
    p.z = z;
    p.ld_z = ldz;
    p.act = act;
    p.nt = streams(rows * cols * dtype_bytes(dtype));
    hipError_t e = launch_prepare(dtype, pre, s);
    if (e == hipSuccess) e = launch_grouped(kGroupedForward, dtype, dtype, p, s);
    return finish_call(status_of(e), s, nullptr);
}

int bytecomp_grouped_linear_backward(int dtype, int gdtype, uint64_t rows, uint64_t inner, uint64_t cols,
                                     uint32_t experts, const int32_t* offsets, const void* dy, uint64_t lddy,
                                     const void* z, uint64_t ldz, int act, const void* x, uint64_t ldx,
                                     const int32_t* source, uint64_t x_rows, const void* w, uint64_t ldw,
                                     uint64_t expert_w, void* dx, uint64_t lddx, void* dw, uint64_t lddw,
                                     uint64_t expert_dw, void* dbias, uint64_t ld_dbias, void* ws, size_t ws_bytes,
                                     void* stream) {
    const CallRange range("bytecomp_grouped_linear_backward");
    if (const int rc = check_grouped(dtype, rows, inner, cols, experts, source ? x_rows : 0)) return rc;
    if (gdtype != dtype && gdtype != BC_F32) return BC_E_DTYPE;
    if (act < BC_ACT_NONE || act > BC_ACT_SILU) return BC_E_KIND;
    if (inner == 0) dx = dw = nullptr;
    if (cols == 0) dw = dbias = nullptr;
    if (rows == 0) dx = nullptr;
    if (!dx && !dw && !dbias) return BC_OK;
    if (!offsets || (rows > 0 && cols > 0 && (!dy || (act != BC_ACT_NONE && !z)))) return BC_E_NULL;
    if (rows > 0 && ((dw && !x && (!source || x_rows > 0)) || (dx && cols > 0 && !w))) return BC_E_NULL;
    if (lddy < cols || (act != BC_ACT_NONE && ldz < cols) || (dw && (ldx < inner || lddw < inner ||
                                                                    expert_dw < (cols - 1) * lddw + inner)) ||
        (dx && (ldw < inner || lddx < inner || (cols > 0 && expert_w < (cols - 1) * ldw + inner))) ||
        (dbias && ld_dbias < cols) || lddy >= kMaxStride || (dw && ldx >= kMaxStride) || (dx && ldw >= kMaxStride))
        return BC_E_SIZE;
    if (misaligned(dy, dtype) || misaligned(z, dtype) || misaligned(x, dtype) || misaligned(w, dtype) ||
        misaligned(dx, dtype) || misaligned(dw, gdtype) || misaligned(dbias, gdtype) || misaligned4(offsets) ||
        misaligned4(source) || ((uintptr_t)ws & 15))
        return BC_E_ALIGN;
    hipStream_t s = (hipStream_t)stream;
    Carver c{(char*)ws, 0};
    const Groups g{offsets, experts, (uint32_t)rows};
    const uint64_t pc = plane_cols(cols);
    // dz can be read as dy
    const bool same = act == BC_ACT_NONE && readable(dtype, dy, lddy, cols);
    Prepare pre{};
    pre.g = g;
    GroupedSlope& slope = pre.slope;
    slope = GroupedSlope{dy, act != BC_ACT_NONE ? z : nullptr, nullptr, nullptr, lddy, ldz, (uint32_t)cols, act};
    if (!same && (dx || dw)) slope.dz = c.take(laid_bytes(dtype, rows, cols));
    if (dbias) slope.part = (float*)c.take(part_bytes(rows, experts, cols));
    const GroupedSide dz = slope.dz ? GroupedSide{slope.dz, pc, 0} : GroupedSide{dy, lddy, 0};
    GroupedProduct px{}, pw{};
    px.g = pw.g = g;
    px.a = pw.a = dz;
    px.wide = pw.wide = slope.dz || whole(dtype, dy, lddy, cols);
    px.a_rows = (uint32_t)rows;
    if (dw) {
        GroupedX gx{x, ldx, source, x_rows, rows, inner};
        uint32_t n = 0;
        pw.b = side_of_x(dtype, gx, n, pw.wide, c, pre.lay[0]);
        if (gx.source) {
            pre.where = GroupedWhere{gx.source, (uint32_t*)c.take(where_bytes(rows, experts)), n,
                                     (uint32_t)(pw.b.ld * dtype_bytes(dtype))};
            pw.where = pre.where.where;
        }
        pw.rows = (uint32_t)cols;
        pw.cols = (uint32_t)inner;
        pw.out = dw;
        pw.ld_out = lddw;
        pw.expert_out = expert_dw;
        pw.nt = streams(experts * cols * inner * dtype_bytes(gdtype));
    }
    if (dx) {
        px.b = side_of_w(dtype, w, ldw, expert_w, experts, cols, inner, px.wide, c, pre.lay[1]);
        px.cols = (uint32_t)inner;
        px.k = (uint32_t)cols;
        px.out = dx;
        px.ld_out = lddx;
        px.nt = streams(rows * inner * dtype_bytes(dtype));
    }
    if (dx && dw) pre.counters = (uint32_t*)c.take(kGroupedCounters * sizeof(uint32_t));
    if (c.used > 0 && rows > 0 && (!ws || ws_bytes < c.used)) return BC_E_WORKSPACE;
    // (no rows: dw and dbias are zeros)
    hipError_t e = rows > 0 ? launch_prepare(dtype, pre, s) : hipSuccess;
    const GroupedBias bias{g, slope.part, dbias, ld_dbias, (uint32_t)cols};
    if (e == hipSuccess && dx && dw) {
        e = launch_grouped_pair(dtype, gdtype, px, pw, bias, pre.counters, s);
    } else {
        if (e == hipSuccess && dbias) e = launch_grouped_bias(gdtype, bias, s);
        if (e == hipSuccess && dx) e = launch_grouped(kGroupedRows, dtype, dtype, px, s);
        if (e == hipSuccess && dw) e = launch_grouped(kGroupedWeights, dtype, gdtype, pw, s);
    }
    return finish_call(status_of(e), s, nullptr);
}

int bytecomp_grad_norm_workspace_size(int T, size_t* bytes) {
    if (!bytes) return BC_E_NULL;
    if (T < 0 || T > kMaxGrads) return BC_E_COUNT;
    *bytes = clip_ws(T);
    return BC_OK;
}

int bytecomp_grad_norm(const bc_grad* t, int T, int kind, double* norm, void* ws, size_t ws_bytes, void* stream) {
    const CallRange range("bytecomp_grad_norm");
    if (const int rc = check_clip(t, T, kind, ws, ws_bytes)) return rc;
    if (!norm) return BC_E_NULL;
    if ((uintptr_t)norm & 7) return BC_E_ALIGN;
    std::vector<ClipDesc> d;
    Clip a{};
    uint64_t bytes = 0;
    try {
        if (const int rc = clip_table(t, T, false, d, a.chunks, bytes)) return rc;
    } catch (const std::bad_alloc&) {
        return BC_E_SIZE;
    }
    a.T = (uint32_t)d.size();
    a.kind = kind;
    a.part = (double*)ws;
    a.parts = clip_parts(a.chunks);
    a.norm = norm;
    hipStream_t s = (hipStream_t)stream;
    const int rc = with_clip_table(d, ws, s, [&](const ClipDesc* table) {
        a.d = table;
        const hipError_t e = launch_grad_norm(a, s);
        return e != hipSuccess ? e : launch_norm_of_parts(a, s);
    });
    return finish_call(rc, s, nullptr);
}

int bytecomp_clip_grads(const bc_grad* t, int T, int kind, double max_norm, const double* given, double* norm,
                        float* factor, void* ws, size_t ws_bytes, void* stream) {
    const CallRange range("bytecomp_clip_grads");
    if (const int rc = check_clip(t, T, kind, ws, ws_bytes)) return rc;
    if (!(max_norm >= 0.0)) return BC_E_VALUE;
    if (((uintptr_t)given & 7) || ((uintptr_t)norm & 7) || misaligned4(factor)) return BC_E_ALIGN;
    std::vector<ClipDesc> d;
    Clip a{};
    uint64_t bytes = 0;
    try {
        if (const int rc = clip_table(t, T, true, d, a.chunks, bytes)) return rc;
    } catch (const std::bad_alloc&) {
        return BC_E_SIZE;
    }
    a.T = (uint32_t)d.size();
    a.kind = kind;
    a.part = (double*)ws;
    a.parts = clip_parts(a.chunks);
    a.max_norm = max_norm;
    a.given = given;
    a.norm = norm;
    a.factor = factor;
    a.nt = streams(bytes);
    hipStream_t s = (hipStream_t)stream;
    const int rc = with_clip_table(d, ws, s, [&](const ClipDesc* table) {
        a.d = table;
        const hipError_t e = given ? hipSuccess : launch_grad_norm(a, s);
        return e != hipSuccess ? e : launch_clip(a, s);
    });
    return finish_call(rc, s, nullptr);
}

}  // extern "C"
