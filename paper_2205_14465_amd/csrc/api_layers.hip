// api_layers.hip -- the C ABI of the layer and optimizer operators
// (include/bytecomp.h): argument checks on the host, workspace carving, and
// the launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "../../include/bytecomp.h"
#include "launch.hpp"
#include "layers.hpp"

using namespace bc;

namespace {

constexpr uint64_t kMaxRows = 1ull << 31;

int status_of(hipError_t e) { return e == hipSuccess ? BC_OK : BC_E_HIP; }

// Whether p violates the alignment of `dtype`'s elements.
bool misaligned(const void* p, int dtype) { return ((uintptr_t)p & (dtype_bytes(dtype) - 1)) != 0; }

int check_layernorm(int dtype, int wdtype, uint64_t rows, uint64_t cols) {
    if (!dtype_ok(dtype) || (wdtype != dtype && wdtype != BC_F32)) return BC_E_DTYPE;
    if (rows >= kMaxRows || cols >= (1ull << 24)) return BC_E_SIZE;
    return BC_OK;
}

size_t layernorm_ws(uint64_t rows, uint64_t cols) {
    const uint32_t a = ln_parts(rows, (uint32_t)cols, BC_F32), b = ln_parts(rows, (uint32_t)cols, BC_F16);
    return (size_t)(a > b ? a : b) * 2 * cols * sizeof(float);
}

// ------------------------------------------------------------ linear layer
constexpr uint64_t kMaxDim = 1ull << 22;

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

int check_linear(int dtype, uint64_t rows, uint64_t inner, uint64_t cols) {
    if (!dtype_ok(dtype)) return BC_E_DTYPE;
    if (rows >= kMaxDim || inner >= kMaxDim || cols >= kMaxDim) return BC_E_SIZE;
    return BC_OK;
}

// Bytes of an operand of `rows` rows and k columns laid out as planes.
size_t planes_bytes(int dtype, uint64_t rows, uint64_t k) {
    return align256((size_t)(rows * plane_cols(k) * 2 * (uint64_t)planes_of(dtype)));
}

// Bytes for the sums of a product [rows, cols] whose k is split.
size_t sums_bytes(int dtype, uint64_t rows, uint64_t cols, uint64_t k) {
    return align256((size_t)split_bytes(product_cut(dtype, rows, cols, k), rows, cols));
}

size_t linear_ws(int dtype, uint64_t rows, uint64_t inner, uint64_t cols, bool backward) {
    if (!backward)
        return rows <= kFewRows ? 0
                                : planes_bytes(dtype, rows, inner) + planes_bytes(dtype, cols, inner) +
                                      sums_bytes(dtype, rows, cols, inner);
    return planes_bytes(dtype, rows, cols) + planes_bytes(dtype, cols, rows) + planes_bytes(dtype, inner, rows) +
           planes_bytes(dtype, inner, cols) + align256((size_t)((rows + 63) / 64 * cols * sizeof(float))) +
           std::max(sums_bytes(dtype, rows, inner, cols), sums_bytes(dtype, cols, inner, rows));
}

// Hands out the workspace piece by piece.
struct Carver {
    char* at;
    void* take(size_t bytes) {
        char* p = at;
        at += align256(bytes);
        return p;
    }
};

// Whether the product kernels can read an operand of k columns where it lies:
// 16-bit elements, whole steps, 16-byte pieces, offsets within 32 bits.
bool readable(int dtype, const void* p, uint64_t ld, uint64_t k) {
    return dtype != BC_F32 && k % kPlaneCols == 0 && ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && ld < (1ull << 23);
}

// An operand of `rows` rows and k columns for the product kernels: where it
// lies, or laid out at `c` by the call's lay_out launch.
Planes operand(int dtype, const void* p, uint64_t ld, uint64_t rows, uint64_t k, Carver& c, LayOuts& l) {
    if (readable(dtype, p, ld, k)) return Planes{p, ld, 0};
    void* to = c.take(planes_bytes(dtype, rows, k));
    l.of[l.count++] = LayOut{p, nullptr, ld, 0, (uint32_t)rows, (uint32_t)k, to, nullptr, nullptr, BC_ACT_NONE};
    return Planes{to, plane_cols(k), rows * plane_cols(k)};
}

// The transpose of a rows x cols matrix as an operand of cols rows.
Planes turned(int dtype, const void* p, uint64_t ld, uint64_t rows, uint64_t cols, Carver& c, LayOuts& l) {
    void* to = c.take(planes_bytes(dtype, cols, rows));
    l.of[l.count++] = LayOut{p, nullptr, ld, 0, (uint32_t)rows, (uint32_t)cols, nullptr, to, nullptr, BC_ACT_NONE};
    return Planes{to, plane_cols(rows), cols * plane_cols(rows)};
}

// -------------------------------------------------- orthogonalised updates
constexpr int kMaxMatrices = 1 << 20;

// The scales that keep X and the symmetric matrices (kernels_ortho.hip) at the
// top of fp16's range, where small entries beside large ones keep the most of
// their second part: bounds on their largest singular values, and so on their
// entries, rounded up to powers of two.  `reach` bounds X's within the steps, from
// [0, 1] at the start.  False: the coefficients are not finite, or reach passes 64.
bool ortho_scales(int steps, const double* k, float& x_scale, float* scale) {
    const double a = k[0], b = k[1], c = k[2];
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
    double reach = 1.0, most = 1.0;
    for (int i = 0; i + 1 < steps; ++i) {
        auto f = [&](double x) { return std::fabs(x * (a + x * x * (b + c * x * x))); };
        double next = f(reach);
        // f' = a + 3 b y + 5 c y^2 with y = x^2
        double y[2] = {-1.0, -1.0};
        if (c != 0.0) {
            const double d = 9.0 * b * b - 20.0 * a * c;
            if (d >= 0.0) {
                y[0] = (-3.0 * b + std::sqrt(d)) / (10.0 * c);
                y[1] = (-3.0 * b - std::sqrt(d)) / (10.0 * c);
            }
        } else if (b != 0.0) {
            y[0] = -a / (3.0 * b);
        }
        for (const double v : y)
            if (v > 0.0 && v < reach * reach) next = std::fmax(next, f(std::sqrt(v)));
        reach = next * 1.001;  // and what rounding adds
        most = std::fmax(most, reach);
        if (!(most <= 64.0)) return false;
    }
    // |b y + c y^2| for y up to the Gram matrix's largest eigenvalue
    auto p = [&](double y) { return std::fabs(y * (b + c * y)); };
    double poly = p(most * most);
    if (c != 0.0 && -b / (2.0 * c) > 0.0 && -b / (2.0 * c) < most * most) poly = std::fmax(poly, p(-b / (2.0 * c)));
    const double whole = std::fabs(a) + poly;  // of a I + the polynomial
    auto below = [](double x) {
        return (float)(0x1p15 / std::exp2(std::ceil(std::log2(std::fmax(x, 0x1p-40) * 1.001))));
    };
    const double bounds[4] = {most * most, poly, most * most * whole, whole * whole + a * a};
    for (int i = 0; i < 4; ++i) {
        if (!(bounds[i] <= 0x1p40)) return false;
        scale[i] = below(bounds[i]);
    }
    x_scale = below(most);
    return true;
}

// Tiles of a product, and steps of 32 along its k.
uint64_t ortho_tiles(const Ortho& o, int kind, int side) {
    const uint64_t w = 64u << side, a = (o.m + w - 1) / w, b = (o.n + w - 1) / w;
    return kind == kOrthoFull ? a * b : a * (a + 1) / 2;
}
uint64_t ortho_k(const Ortho& o, int kind) { return plane_cols(kind == kOrthoGram ? o.n : o.m); }
double ortho_steps(const Ortho& o, int kind) { return (double)ortho_k(o, kind) / 32.0; }
// The parts along k that leave chains of at most `chain` steps.
uint64_t ortho_parts(const Ortho& o, int kind, double chain) {
    return std::min((uint64_t)std::ceil(ortho_steps(o, kind) / chain),
                    std::max<uint64_t>(1, ortho_k(o, kind) / kOrthoPart));
}

// Workspace offsets and workgroup counts of one matrix; `at` advances.
void plan_matrix(uint64_t rows, uint64_t cols, uint64_t& at, OrthoPlan& p, Ortho& o) {
    auto take = [&](uint64_t bytes) {
        const uint64_t p = at;
        at += align256(bytes);
        return p;
    };
    o.rows = (uint32_t)rows;
    o.cols = (uint32_t)cols;
    o.turned = rows > cols;
    o.m = o.turned ? o.cols : o.rows;
    o.n = o.turned ? o.rows : o.cols;
    o.group = ortho_group(p.c, o.m);
    o.part0 = p.c.parts;
    o.tile0 = p.c.tiles;
    if (rows == 0 || cols == 0) return;
    const uint64_t m = o.m, n = o.n, mp = plane_cols(m), np = plane_cols(n);
    o.x = take(4 * m * np);
    o.xt = take(8 * n * mp);
    o.sym = take(12 * m * mp);
    const uint64_t tiles = plane_cols(rows) / 64 * (plane_cols(cols) / 64);
    o.parts = (uint32_t)(tiles < kOrthoParts ? tiles : kOrthoParts);
    o.part = take(8 * o.parts);
    p.c.parts += o.parts;
    p.c.tiles += (uint32_t)tiles;
    // (a matrix of as many tiles as there are units is not cut: its chain is no
    // longer than the mean)
    uint64_t slots = 0;
    for (int kind = 0; kind < kOrthoKinds; ++kind) {
        const uint64_t most = ortho_parts(o, kind, 1.0), n = ortho_tiles(o, kind, 0);
        if (most > 1 && n < kOrthoSlots / 2) slots = std::max(slots, n * most);
    }
    p.c.slots = (uint32_t)std::min(kOrthoSlots, p.c.slots + slots);
    for (int i = 0; i < kOrthoSides; ++i)
        for (int kind = 0; kind < kOrthoKinds; ++kind) {
            OrthoLoad& l = p.group[o.group].load[kind][i];
            const double steps = ortho_steps(o, kind);
            l.tiles += (double)ortho_tiles(o, kind, i);
            l.steps += (double)ortho_tiles(o, kind, i) * steps;
            l.longest = std::fmax(l.longest, steps);
        }
}

// What follows the matrices in the workspace: counters and slots for tiles cut
// along k.
void plan_meeting(uint64_t& at, OrthoPlan& p) {
    p.c.meet = at;
    if (p.c.slots) at += align256(kOrthoSlots * sizeof(uint32_t) + p.c.slots * kOrthoSlotBytes);
}

// How long a 64-wide tile's chain along k may be: about a compute unit's mean
// share of the launch (which makes at most twice as many parts as there are
// units), and where there are fewer tiles than units no shorter than one
// workgroup a unit allows.  (4781 x 188 in bfloat16 141 us against 184 uncut, three
// of 512 x 4608 with one of 2048 x 512 356 against 397; parts of 256 take 155 and
// 412, and two parts for 136 tiles, more than a workgroup a unit, 314 against 258.)
double ortho_chain(const OrthoPlan& p, const std::vector<Ortho>& table, uint32_t group, int kind) {
    const OrthoLoad& l = p.group[group].load[kind][0];
    double chain = std::fmax(l.steps / p.cus, kOrthoPart / 32.0);
    if (l.tiles > p.cus) return chain;
    for (; chain < l.longest; chain *= 1.1) {
        uint64_t n = 0;
        for (const Ortho& o : table)
            if (o.group == group) n += ortho_tiles(o, kind, 0) * ortho_parts(o, kind, chain);
        if (n <= (uint64_t)p.cus) break;
    }
    return chain;
}

// The workgroups of a launch, dealt to the eight compute dies in turn, each
// with an L2 of its own.  Where all tiles take about as long, the matrices' tiles
// one after the other are cut into eight runs of equal work, so that a die works
// on few matrices; otherwise each matrix of 16 tiles or more is cut into eight and
// smaller ones go whole to the least loaded die, the long tiles first.  `list`
// receives 8 x the longest die's count entries, the others' ends idle; returns
// that count.
uint32_t ortho_list(const OrthoPlan& p, const std::vector<Ortho>& table, uint32_t group, int kind,
                    std::vector<OrthoWork>& list) {
    constexpr int kDies = 8;
    std::vector<OrthoWork> die[kDies];
    const OrthoGroup& g = p.group[group];
    const int side = g.side[kind];
    const OrthoLoad& all = g.load[kind][side];
    uint32_t slots = 0, met = 0;
    // the parts of a tile follow each other on one die
    auto parts_of = [&](const Ortho& o) -> uint32_t {
        if (side != 0) return 1;
        const uint64_t parts = ortho_parts(o, kind, g.chain[kind]);
        return slots + parts * ortho_tiles(o, kind, 0) <= p.c.slots ? (uint32_t)parts : 1;
    };
    auto push = [&](std::vector<OrthoWork>& to, size_t i, uint64_t tile, uint32_t parts) {
        const Ortho& o = table[i];
        for (uint32_t q = 0; q < parts; ++q)
            to.push_back(OrthoWork{(uint32_t)i, (uint32_t)tile, o.m, o.n, (uint32_t)(o.x >> 8), (uint32_t)(o.xt >> 8),
                                   (uint32_t)(o.sym >> 8), q, parts, slots, met});
        if (parts == 1) return;
        slots += parts;
        met += 1;
    };
    if (all.longest * all.tiles <= 1.25 * all.steps) {
        double done = 0.0;
        for (size_t i = 0; i < table.size(); ++i) {
            if (table[i].group != group) continue;
            const uint64_t tiles = ortho_tiles(table[i], kind, side);
            const uint32_t parts = parts_of(table[i]);
            for (uint64_t t = 0; t < tiles; ++t) {
                push(die[std::min(kDies - 1, (int)(done * kDies / all.steps))], i, t, parts);
                done += ortho_steps(table[i], kind);
            }
        }
    } else {
        double load[kDies] = {};
        for (size_t i = 0; i < table.size(); ++i) {
            if (table[i].group != group) continue;
            const uint64_t tiles = ortho_tiles(table[i], kind, side);
            const uint32_t parts = parts_of(table[i]);
            const uint64_t pieces = tiles * parts >= 16 ? kDies : 1;
            for (uint64_t q = 0; q < pieces; ++q) {
                const int to = (int)(std::min_element(load, load + kDies) - load);
                const uint64_t lo = tiles * q / pieces, hi = tiles * (q + 1) / pieces;
                for (uint64_t t = lo; t < hi; ++t) push(die[to], i, t, parts);
                load[to] += (double)(hi - lo) * ortho_steps(table[i], kind);
            }
        }
    }
    size_t longest = 0;
    for (const auto& d : die) longest = std::max(longest, d.size());
    for (size_t q = 0; q < longest; ++q)
        for (const auto& d : die) list.push_back(q < d.size() ? d[q] : OrthoWork{kOrthoIdle, 0, 0, 0, 0, 0, 0, 0, 1, 0, 0});
    return (uint32_t)(kDies * longest);
}

int check_ortho(int T, int steps, const double* k, double eps, OrthoPlan& p) {
    OrthoCall& c = p.c;
    if (T < 0 || T > kMaxMatrices) return BC_E_COUNT;
    if (!k) return BC_E_NULL;
    if (steps < 1 || steps > 64 || !(eps >= 0.0) || std::isinf(eps)) return BC_E_VALUE;
    if (!ortho_scales(steps, k, c.x_scale, c.scale)) return BC_E_VALUE;
    c.a = (float)k[0];
    c.b = (float)k[1];
    c.c = (float)k[2];
    c.eps = eps;
    p.steps = steps;
    c.T = T;
    return BC_OK;
}

// get(i, rows, cols, o): matrix i's shape, pointers and strides, or its
// error.  The rest of the call: plan, table, launch.  Long products come first
// in the table, so that a launch ends on short ones.
template <typename Get>
int run_ortho(OrthoPlan& p, void* ws, size_t ws_bytes, hipStream_t s, Get get) {
    std::vector<Ortho> table;
    uint64_t at = 0, tiles = 0;
    try {
        std::vector<Ortho> given((size_t)p.c.T);
        std::memset((void*)given.data(), 0, given.size() * sizeof(Ortho));
        std::vector<std::pair<uint64_t, int>> order;
        for (int i = 0; i < p.c.T; ++i) {
            uint64_t rows = 0, cols = 0;
            Ortho& o = given[(size_t)i];
            if (const int rc = get(i, rows, cols, o)) return rc;
            if (rows >= kMaxDim || cols >= kMaxDim) return BC_E_SIZE;
            tiles += plane_cols(rows) / 64 * (plane_cols(cols) / 64);
            if (tiles >= (1ull << 28)) return BC_E_SIZE;  // workgroup counts stay within 32 bits
            o.rows = (uint32_t)rows;
            o.cols = (uint32_t)cols;
            if (rows && cols) order.push_back({rows > cols ? rows : cols, i});
        }
        std::sort(order.begin(), order.end(), [](const auto& x, const auto& y) {
            return x.first != y.first ? x.first > y.first : x.second < y.second;
        });
        for (const auto& [longer, i] : order) {
            table.push_back(given[(size_t)i]);
            Ortho& o = table.back();
            plan_matrix(o.rows, o.cols, at, p, o);
        }
    } catch (const std::bad_alloc&) {
        return BC_E_SIZE;
    }
    if (table.empty()) return BC_OK;
    plan_meeting(at, p);
    if (at >= (1ull << 40)) return BC_E_SIZE;  // offsets in 256 bytes stay within 32 bits
    if (!ws || ws_bytes < at) return BC_E_WORKSPACE;
    if ((uintptr_t)ws & 255) return BC_E_ALIGN;
    p.c.ws = (char*)ws;
    p.c.T = (int)table.size();
    int dev = 0;
    DevInfo di;
    hipError_t e = hipGetDevice(&dev);
    if (e == hipSuccess) e = device_info(dev, &di);
    if (e != hipSuccess) return BC_E_HIP;
    p.cus = di.cus;
    for (uint32_t g = 0; g < 2; ++g) {
        for (int kind = 0; kind < kOrthoKinds; ++kind) p.group[g].chain[kind] = ortho_chain(p, table, g, kind);
        ortho_choose(p.group[g], g == 1, p.cus);
    }
    // The table, then the work lists.  The lists follow from the table's bytes (shapes,
    // offsets and groups: the type of the results counts through the groups alone)
    // and the device, which together are what the copy is found again by.
    struct Ctx {
        OrthoPlan* p;
        hipStream_t s;
        std::vector<OrthoWork> list;
        size_t at;
    } ctx{&p, s, {}, table.size() * sizeof(Ortho)};
    try {
        for (uint32_t g = 0; g < 2; ++g)
            for (int kind = 0; kind < kOrthoKinds; ++kind)
                p.group[g].workgroups[kind] = ortho_list(p, table, g, kind, ctx.list);
        e = with_table(table.data(), ctx.at, ctx.list.size() * sizeof(OrthoWork),
                       [](void* c, void* extra) {
                           const Ctx* x = (const Ctx*)c;
                           std::memcpy(extra, x->list.data(), x->list.size() * sizeof(OrthoWork));
                       },
                       s,
                       [](void* c, const void* dev_table) {
                           Ctx* x = (Ctx*)c;
                           x->p->c.d = (const Ortho*)dev_table;
                           const OrthoWork* l = (const OrthoWork*)((const char*)dev_table + x->at);
                           for (OrthoGroup& g : x->p->group)
                               for (int kind = 0; kind < kOrthoKinds; ++kind) {
                                   g.list[kind] = l;
                                   l += g.workgroups[kind];
                               }
                           return launch_orthogonalize(*x->p, x->s);
                       },
                       &ctx);
    } catch (const std::bad_alloc&) {
        return BC_E_SIZE;
    }
    return finish_call(status_of(e), s, nullptr);
}

}  // namespace

extern "C" {

int bytecomp_layernorm_forward(int dtype, int wdtype, uint64_t rows, uint64_t cols, const void* x, uint64_t ldx,
                               const void* weight, const void* bias, double eps, void* y, uint64_t ldy, float* mean,
                               float* rstd, void* stream) {
    const CallRange range("bytecomp_layernorm_forward");
    if (const int rc = check_layernorm(dtype, wdtype, rows, cols)) return rc;
    if (!(eps >= 0.0) || std::isinf(eps)) return BC_E_VALUE;
    if (rows == 0 || cols == 0) return BC_OK;
    if (!x || !y) return BC_E_NULL;
    if (ldx < cols || ldy < cols) return BC_E_SIZE;
    if (misaligned(x, dtype) || misaligned(y, dtype) || misaligned(weight, wdtype) || misaligned(bias, wdtype) ||
        misaligned(mean, BC_F32) || misaligned(rstd, BC_F32))
        return BC_E_ALIGN;
    const LnForward a{x, weight, bias, y, mean, rstd, rows, ldx, ldy, (uint32_t)cols, (float)(1.0 / (double)cols),
                      (float)eps, streams(rows * cols * dtype_bytes(dtype))};
    hipStream_t s = (hipStream_t)stream;
    return finish_call(status_of(launch_ln_forward(dtype, wdtype, a, s)), s, nullptr);
}

int bytecomp_layernorm_workspace_size(uint64_t rows, uint64_t cols, size_t* bytes) {
    if (!bytes) return BC_E_NULL;
    if (const int rc = check_layernorm(BC_F32, BC_F32, rows, cols)) return rc;
    *bytes = layernorm_ws(rows, cols);
    return BC_OK;
}

int bytecomp_layernorm_backward(int dtype, int wdtype, uint64_t rows, uint64_t cols, const void* dy, uint64_t lddy,
                                const void* x, uint64_t ldx, const void* weight, const float* mean, const float* rstd,
                                void* dx, uint64_t lddx, void* dweight, void* dbias, void* ws, size_t ws_bytes,
                                void* stream) {
    const CallRange range("bytecomp_layernorm_backward");
    if (const int rc = check_layernorm(dtype, wdtype, rows, cols)) return rc;
    if (cols == 0 || (!dx && !dweight && !dbias)) return BC_OK;
    if (rows > 0 && (!dy || !x || !mean || !rstd)) return BC_E_NULL;
    if (lddy < cols || ldx < cols || (dx && lddx < cols)) return BC_E_SIZE;
    if (misaligned(dy, dtype) || misaligned(x, dtype) || misaligned(weight, wdtype) || misaligned(dx, dtype) ||
        misaligned(mean, BC_F32) || misaligned(rstd, BC_F32) || misaligned(dweight, wdtype) ||
        misaligned(dbias, wdtype) || misaligned(ws, BC_F32))
        return BC_E_ALIGN;
    const bool sums = dweight || dbias;
    if (sums && rows > 0 && (!ws || ws_bytes < layernorm_ws(rows, cols))) return BC_E_WORKSPACE;
    const LnBackward a{dy, x, weight, mean, rstd, dx, sums ? (float*)ws : nullptr, rows, lddy, ldx, lddx,
                       (uint32_t)cols, ln_parts(rows, (uint32_t)cols, dtype), (float)(1.0 / (double)cols),
                       streams(rows * cols * dtype_bytes(dtype))};
    hipStream_t s = (hipStream_t)stream;
    return finish_call(status_of(launch_ln_backward(dtype, wdtype, a, dweight, dbias, s)), s, nullptr);
}

int bytecomp_linear_workspace_size(int dtype, uint64_t rows, uint64_t inner, uint64_t cols, int backward,
                                   size_t* bytes) {
    if (!bytes) return BC_E_NULL;
    if (const int rc = check_linear(dtype, rows, inner, cols)) return rc;
    *bytes = linear_ws(dtype, rows, inner, cols, backward != 0);
    return BC_OK;
}

int bytecomp_linear_forward(int dtype, uint64_t rows, uint64_t inner, uint64_t cols, const void* x, uint64_t ldx,
                            const void* w, uint64_t ldw, const void* bias, int act, const void* residual,
                            uint64_t ld_residual, void* y, uint64_t ldy, void* z, uint64_t ldz, void* ws,
                            size_t ws_bytes, void* stream) {
    const CallRange range("bytecomp_linear_forward");
    if (const int rc = check_linear(dtype, rows, inner, cols)) return rc;
    if (act < BC_ACT_NONE || act > BC_ACT_SILU) return BC_E_KIND;
    if (rows == 0 || cols == 0) return BC_OK;
    if (!y || (inner > 0 && (!x || !w))) return BC_E_NULL;
    if (ldx < inner || ldw < inner || ldy < cols || (residual && ld_residual < cols) || (z && ldz < cols))
        return BC_E_SIZE;
    if (misaligned(x, dtype) || misaligned(w, dtype) || misaligned(bias, dtype) || misaligned(residual, dtype) ||
        misaligned(y, dtype) || misaligned(z, dtype) || ((uintptr_t)ws & 15))
        return BC_E_ALIGN;
    hipStream_t s = (hipStream_t)stream;
    if (rows <= kFewRows) {
        const FewRows a{x, w, bias, residual, y, z, ldx, ldw, ld_residual, ldy, ldz, (uint32_t)rows, (uint32_t)inner,
                        (uint32_t)cols, act};
        return finish_call(status_of(launch_few_rows(dtype, a, s)), s, nullptr);
    }
    size_t need = 0;
    if (!readable(dtype, x, ldx, inner)) need += planes_bytes(dtype, rows, inner);
    if (!readable(dtype, w, ldw, inner)) need += planes_bytes(dtype, cols, inner);
    const Cut cut = product_cut(dtype, rows, cols, inner);
    const size_t sums = align256((size_t)split_bytes(cut, rows, cols));
    need += sums;
    if (need > 0 && (!ws || ws_bytes < need)) return BC_E_WORKSPACE;
    Carver c{(char*)ws};
    Product p{};
    LayOuts l{};
    p.a = operand(dtype, x, ldx, rows, inner, c, l);
    p.b = operand(dtype, w, ldw, cols, inner, c, l);
    hipError_t e = launch_lay_outs(dtype, l, s);
    if (e == hipSuccess) {
        p.rows = (uint32_t)rows;
        p.cols = (uint32_t)cols;
        p.steps = (uint32_t)(plane_cols(inner) / kPlaneCols);
        p.out = y;
        p.ld_out = ldy;
        p.bias = bias;
        p.residual = residual;
        p.z = z;
        p.ld_residual = ld_residual;
        p.ld_z = ldz;
        p.act = act;
        p.nt = streams(rows * cols * dtype_bytes(dtype));
        p.part = (float*)c.take(sums);
        e = launch_product(dtype, dtype, true, cut, p, s);
    }
    return finish_call(status_of(e), s, nullptr);
}

int bytecomp_linear_backward(int dtype, int gdtype, uint64_t rows, uint64_t inner, uint64_t cols, const void* dy,
                             uint64_t lddy, const void* z, uint64_t ldz, int act, const void* x, uint64_t ldx,
                             const void* w, uint64_t ldw, void* dx, uint64_t lddx, void* dw, uint64_t lddw,
                             void* dbias, void* ws, size_t ws_bytes, void* stream) {
    const CallRange range("bytecomp_linear_backward");
    if (const int rc = check_linear(dtype, rows, inner, cols)) return rc;
    if (gdtype != dtype && gdtype != BC_F32) return BC_E_DTYPE;
    if (act < BC_ACT_NONE || act > BC_ACT_SILU) return BC_E_KIND;
    if (!dx && !dw && !dbias) return BC_OK;
    const bool any = rows > 0 && cols > 0 && inner > 0;
    if (rows > 0 && cols > 0 && (!dy || (act != BC_ACT_NONE && !z))) return BC_E_NULL;
    if (any && ((dw && !x) || (dx && !w))) return BC_E_NULL;
    if (lddy < cols || (act != BC_ACT_NONE && ldz < cols) || (dw && (ldx < inner || lddw < inner)) ||
        (dx && (ldw < inner || lddx < inner)))
        return BC_E_SIZE;
    if (misaligned(dy, dtype) || misaligned(z, dtype) || misaligned(x, dtype) || misaligned(w, dtype) ||
        misaligned(dx, dtype) || misaligned(dw, gdtype) || misaligned(dbias, gdtype) || ((uintptr_t)ws & 15))
        return BC_E_ALIGN;
    const bool same = act == BC_ACT_NONE && readable(dtype, dy, lddy, cols);  // dz can be read as dy
    const bool flat = dx && !same;
    size_t need = 0;
    if (flat) need += planes_bytes(dtype, rows, cols);
    if (dx) need += planes_bytes(dtype, inner, cols);
    if (dw) need += planes_bytes(dtype, cols, rows) + planes_bytes(dtype, inner, rows);
    const size_t part_bytes = align256((size_t)((rows + 63) / 64 * cols * sizeof(float)));
    if (dbias) need += part_bytes;
    // the products' split sums share their place: one product follows the other
    const Cut cut_x = product_cut(dtype, rows, inner, cols), cut_w = product_cut(dtype, cols, inner, rows);
    const size_t sums = std::max(dx ? align256((size_t)split_bytes(cut_x, rows, inner)) : 0,
                                 dw ? align256((size_t)split_bytes(cut_w, cols, inner)) : 0);
    need += sums;
    if (need > 0 && (!ws || ws_bytes < need)) return BC_E_WORKSPACE;
    hipStream_t s = (hipStream_t)stream;
    Carver c{(char*)ws};
    float* part = (float*)c.take(sums);
    LayOuts l{};
    Planes dz{}, dz_turned{}, w_turned{}, x_turned{};
    float* columns = nullptr;
    if (flat || dw || dbias) {
        LayOut& o = l.of[l.count++];
        o = LayOut{dy, act != BC_ACT_NONE ? z : nullptr, lddy, ldz, (uint32_t)rows, (uint32_t)cols, nullptr, nullptr,
                   nullptr, act};
        if (flat) o.flat = c.take(planes_bytes(dtype, rows, cols));
        if (dw) o.turned = c.take(planes_bytes(dtype, cols, rows));
        if (dbias) o.part = columns = (float*)c.take(part_bytes);
        dz = Planes{o.flat, plane_cols(cols), rows * plane_cols(cols)};
        dz_turned = Planes{o.turned, plane_cols(rows), cols * plane_cols(rows)};
    }
    if (!flat) dz = Planes{dy, lddy, 0};
    if (dx) w_turned = turned(dtype, w, ldw, cols, inner, c, l);
    if (dw) x_turned = turned(dtype, x, ldx, rows, inner, c, l);
    hipError_t e = launch_lay_outs(dtype, l, s);
    if (e == hipSuccess && dbias)
        e = launch_sum_parts(gdtype, columns, (uint32_t)((rows + 63) / 64), cols, (uint32_t)cols, dbias, nullptr, s);
    auto product = [&](const Planes& a, const Planes& b, uint64_t m, uint64_t k, void* out, uint64_t ld, int out_dtype) {
        Product p{};
        p.a = a;
        p.b = b;
        p.rows = (uint32_t)m;
        p.cols = (uint32_t)inner;
        p.steps = (uint32_t)(plane_cols(k) / kPlaneCols);
        p.out = out;
        p.ld_out = ld;
        p.nt = streams(m * inner * dtype_bytes(out_dtype));
        p.part = part;
        return p;
    };
    const Product px = product(dz, w_turned, rows, cols, dx, lddx, dtype);
    const Product pw = product(dz_turned, x_turned, cols, rows, dw, lddw, gdtype);
    // (the choice depends on the shape alone: each gradient is the same, whatever else is wanted)
    const int both = pair_tile(dtype, Shape{rows, inner, cols}, Shape{cols, inner, rows});
    if (e == hipSuccess && dx && dw && both >= 0 && gdtype == dtype) {
        e = launch_pair(dtype, both, px, pw, s);
    } else {
        if (e == hipSuccess && dx) e = launch_product(dtype, dtype, false, both >= 0 ? Cut{both, 1} : cut_x, px, s);
        if (e == hipSuccess && dw) e = launch_product(dtype, gdtype, false, both >= 0 ? Cut{both, 1} : cut_w, pw, s);
    }
    return finish_call(status_of(e), s, nullptr);
}

int bytecomp_orthogonalize_workspace_size(const uint64_t* rows, const uint64_t* cols, int T, size_t* bytes) {
    if (T < 0 || T > kMaxMatrices) return BC_E_COUNT;
    if (!bytes || (T > 0 && (!rows || !cols))) return BC_E_NULL;
    OrthoPlan p{};
    uint64_t at = 0;
    for (int i = 0; i < T; ++i) {
        if (rows[i] >= kMaxDim || cols[i] >= kMaxDim) return BC_E_SIZE;
        Ortho o{};
        plan_matrix(rows[i], cols[i], at, p, o);
    }
    plan_meeting(at, p);
    *bytes = (size_t)at;
    return BC_OK;
}

int bytecomp_orthogonalize(int dtype, const bc_update* t, int T, int steps, const double* coefficients, double eps,
                           void* ws, size_t ws_bytes, void* stream) {
    const CallRange range("bytecomp_orthogonalize");
    if (!dtype_ok(dtype)) return BC_E_DTYPE;
    OrthoPlan p{};
    OrthoCall& c = p.c;
    if (const int rc = check_ortho(T, steps, coefficients, eps, p)) return rc;
    if (T == 0) return BC_OK;
    if (!t) return BC_E_NULL;
    c.in_dtype = c.out_dtype = dtype;
    return run_ortho(p, ws, ws_bytes, (hipStream_t)stream, [&](int i, uint64_t& rows, uint64_t& cols, Ortho& o) {
        const bc_update& u = t[i];
        rows = u.rows;
        cols = u.cols;
        if (rows == 0 || cols == 0) return (int)BC_OK;
        if (!u.update || !u.out) return (int)BC_E_NULL;
        if (u.ld_update < cols || u.ld_out < cols) return (int)BC_E_SIZE;
        if (misaligned(u.update, dtype) || misaligned(u.out, dtype)) return (int)BC_E_ALIGN;
        o.in = u.update;
        o.out = u.out;
        o.ld_in = u.ld_update;
        o.ld_out = u.ld_out;
        return (int)BC_OK;
    });
}

int bytecomp_muon_step(int wdtype, int gdtype, const bc_param* t, int T, double lr, double momentum, int nesterov,
                       double weight_decay, int steps, const double* coefficients, double eps, void* ws,
                       size_t ws_bytes, void* stream) {
    const CallRange range("bytecomp_muon_step");
    if (!dtype_ok(wdtype) || !dtype_ok(gdtype)) return BC_E_DTYPE;
    OrthoPlan p{};
    OrthoCall& c = p.c;
    if (const int rc = check_ortho(T, steps, coefficients, eps, p)) return rc;
    if (!std::isfinite(lr) || !std::isfinite(momentum) || !std::isfinite(weight_decay)) return BC_E_VALUE;
    if (T == 0) return BC_OK;
    if (!t) return BC_E_NULL;
    c.in_dtype = gdtype;
    c.out_dtype = wdtype;
    c.muon = true;
    c.nesterov = nesterov != 0;
    c.momentum = (float)momentum;
    c.keep = (float)(1.0 - lr * weight_decay);
    c.lr = (float)lr;
    return run_ortho(p, ws, ws_bytes, (hipStream_t)stream, [&](int i, uint64_t& rows, uint64_t& cols, Ortho& o) {
        const bc_param& u = t[i];
        rows = u.rows;
        cols = u.cols;
        if (rows == 0 || cols == 0) return (int)BC_OK;
        if (!u.weight || !u.grad || !u.momentum) return (int)BC_E_NULL;
        if (u.ld_weight < cols || u.ld_grad < cols || u.ld_momentum < cols) return (int)BC_E_SIZE;
        if (misaligned(u.weight, wdtype) || misaligned(u.grad, gdtype) || misaligned(u.momentum, BC_F32))
            return (int)BC_E_ALIGN;
        if (!std::isfinite(u.scale)) return (int)BC_E_VALUE;
        o.in = u.grad;
        o.out = u.weight;
        o.momentum = u.momentum;
        o.ld_in = u.ld_grad;
        o.ld_out = u.ld_weight;
        o.ld_momentum = u.ld_momentum;
        o.step_scale = (float)u.scale;
        return (int)BC_OK;
    });
}

}  // extern "C"
