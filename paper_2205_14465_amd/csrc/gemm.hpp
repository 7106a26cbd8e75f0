// gemm.hpp -- one workgroup's tile of C = A B^T on the matrix cores of gfx950:
// A [M, K] and B [N, K] in 16-bit floating point with K contiguous, C in fp32
// registers, then handed to an epilogue row piece by row piece.
//
// Operands of more than 16 bits come as P planes whose sum is the value (a
// leading part, then what its rounding left, ...), and the tile adds the
// products of planes that reach fp32's last places:
//   P = 1: a0 b0
//   P = 2: a0 b0 + a0 b1 + a1 b0            (fp16: 22 bits of each operand)
//   P = 3: the same + a1 b1 + a0 b2 + a2 b0 (bfloat16: 24 bits)
// With an infinity or NaN among the values a0 b0 alone says what the sum is: the
// other products would make NaN of infinity times a zero part.
//
// Per step of kBK along K the tile's rows of A and B go from memory to LDS
// without passing registers (global_load_lds, 16 bytes a lane), up to kStages
// steps ahead of their use.  A lane's 16 bytes land at 16 * lane, so the
// swizzle that spreads a column of 16-byte chunks over the banks is applied to
// the global address: chunk c of row r lies at place c ^ swizzle(r) of the row.
// The matrix instruction (32x32x16) takes B's rows as its first operand, which
// leaves a lane four consecutive columns of one row of C at a time.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "elem.hpp"

namespace bc {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef f16_t f16x8 __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));

template <typename T>
struct Frag;
template <>
struct Frag<f16_t> {
    typedef f16x8 type;
    static __device__ __forceinline__ f32x16 mma(type a, type b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
};
template <>
struct Frag<bf16_t> {
    typedef bf16x8 type;
    static __device__ __forceinline__ f32x16 mma(type a, type b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
};

// Wait until at most n vector memory operations of this wave are in flight.
template <int n>
__device__ __forceinline__ void wait_vmcnt() {
    __builtin_amdgcn_s_waitcnt((n & 15) | ((n >> 4) << 14) | 0x0f70);
}
__device__ __forceinline__ void lds_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// One operand as a tile sees it: its first row and first k.
template <typename T>
struct Operand {
    const T* p;
    uint32_t ld;        // elements from row to row: ld * kBM * sizeof(T) < 2^32
    uint64_t plane;     // elements from plane to plane
    uint32_t rows;      // rows there are, >= 1 (a tile's rows past them read the last one)
};

template <typename T_, int P_, int BM_, int BN_, int BK_, int WM_, int WN_, int STAGES_>
struct GemmTile {
    typedef T_ T;
    static constexpr int P = P_, kBM = BM_, kBN = BN_, kBK = BK_, kWM = WM_, kWN = WN_, kStages = STAGES_;
    static constexpr int kWaves = kWM * kWN, kThreads = 64 * kWaves;
    static constexpr int kFM = kBM / kWM / 32, kFN = kBN / kWN / 32;     // 32x32 blocks of a wave
    static constexpr int kElem = sizeof(T);                             // bytes of an element
    static constexpr int kRow = kBK * kElem;                            // bytes of a row in LDS
    static constexpr int kChunks = kRow / 16;                           // 16-byte chunks of a row
    static constexpr int kRows = 64 / kChunks;                          // rows of one load instruction
    static constexpr int kLoadA = kBM / kRows / kWaves, kLoadB = kBN / kRows / kWaves;
    static constexpr int kLoads = P * (kLoadA + kLoadB);                // a step's loads of one wave
    static constexpr int kStageBytes = P * (kBM + kBN) * kRow;
    static constexpr int kEpiCols = kFN * 32, kEpiLd = kEpiCols + 4;     // a wave's strip of C in the epilogue
    static constexpr int kEpiBytes = kWaves * 32 * kEpiLd * 4;
    static constexpr int kLdsBytes = kStages * kStageBytes > kEpiBytes ? kStages * kStageBytes : kEpiBytes;
    static_assert(kRow == 64 || kRow == 128, "swizzles");
    static_assert(kLoadA * kRows * kWaves == kBM && kLoadB * kRows * kWaves == kBN, "loads cover the tile");

    f32x16 acc[kFM][kFN];
    // Tiles that have the registers add the products of lesser planes apart: two
    // thirds (P = 2) of the roundings at the size of the sum fall away.
    static constexpr bool kApart = P > 1 && kFM * kFN <= 4;
    static_assert(P < 3 || kApart, "bfloat16 planes hold infinities, which lesser products must not reach");

    static __device__ __forceinline__ int swizzle(int row) { return kRow == 128 ? (row >> 1) & 7 : (row >> 2) & 3; }

    // Products of `steps` steps of kBK into acc, which is cleared.
    __device__ __forceinline__ void multiply(const Operand<T>& a, const Operand<T>& b, int steps, char* lds) {
        const int lane = threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        uint32_t offa[kLoadA], offb[kLoadB];
#pragma unroll
        for (int i = 0; i < kLoadA; ++i) offa[i] = lane_offset(i * kWaves + wave, lane, a.rows, a.ld);
#pragma unroll
        for (int i = 0; i < kLoadB; ++i) offb[i] = lane_offset(i * kWaves + wave, lane, b.rows, b.ld);
        auto load = [&](int stage, int step) {
            char* to = lds + stage * kStageBytes + wave * 1024;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const __amdgpu_buffer_rsrc_t from = resource(a.p + p * a.plane);
#pragma unroll
                for (int i = 0; i < kLoadA; ++i)
                    copy16(from, offa[i], step * kRow, to + (p * kBM * kRow + i * kWaves * 1024));
            }
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const __amdgpu_buffer_rsrc_t from = resource(b.p + p * b.plane);
#pragma unroll
                for (int i = 0; i < kLoadB; ++i)
                    copy16(from, offb[i], step * kRow, to + ((P * kBM + p * kBN) * kRow + i * kWaves * 1024));
            }
        };
#pragma unroll
        for (int m = 0; m < kFM; ++m)
#pragma unroll
            for (int n = 0; n < kFN; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[m][n][r] = 0.0f;
        const int wm = wave / kWN, wn = wave % kWN;
        const int hi = lane >> 5, l31 = lane & 31, sw = swizzle(l31);
        const char* fa = lds + (wm * kFM * 32 + l31) * kRow;
        const char* fb = lds + (P * kBM + wn * kFN * 32 + l31) * kRow;
        // fragments of 16 along k, read while the matrix cores work on the last ones
        typename Frag<T>::type va[2][P][kFM], vb[2][P][kFN];
        auto read = [&](int set, int stage, int kk) {
            const int at = stage * kStageBytes + ((kk * 2 + hi) ^ sw) * 16;
#pragma unroll
            for (int p = 0; p < P; ++p) {
#pragma unroll
                for (int n = 0; n < kFN; ++n)
                    vb[set][p][n] = *(const typename Frag<T>::type*)(fb + at + (p * kBN + n * 32) * kRow);
#pragma unroll
                for (int m = 0; m < kFM; ++m)
                    va[set][p][m] = *(const typename Frag<T>::type*)(fa + at + (p * kBM + m * 32) * kRow);
            }
        };
        f32x16 lesser[kApart ? kFM : 1][kApart ? kFN : 1];
        if constexpr (kApart) {
#pragma unroll
            for (int m = 0; m < kFM; ++m)
#pragma unroll
                for (int n = 0; n < kFN; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r) lesser[m][n][r] = 0.0f;
        }
        auto mma = [&](int set) {
#pragma unroll
            for (int pa = 0; pa < P; ++pa)
#pragma unroll
                for (int pb = 0; pb + pa < P; ++pb)
#pragma unroll
                    for (int m = 0; m < kFM; ++m)
#pragma unroll
                        for (int n = 0; n < kFN; ++n) {
                            f32x16& to = kApart && pa + pb > 0 ? lesser[kApart ? m : 0][kApart ? n : 0] : acc[m][n];
                            to = Frag<T>::mma(vb[set][pb][n], va[set][pa][m], to);
                        }
        };
        constexpr int kKK = kBK / 16, kReads = P * (kFM + kFN), kMma = P * (P + 1) / 2 * kFM * kFN;
        static_assert(kKK % 2 == 0, "fragment sets alternate");
        if (steps > 0) {
#pragma unroll
            for (int i = 0; i < kStages; ++i)
                if (i < steps) load(i, i);
            // the first step's data has landed
            if (steps >= kStages) wait_vmcnt<(kStages - 1) * kLoads>();
            else wait_vmcnt<0>();
            lds_barrier();
            read(0, 0, 0);
        }
        int stage = 0;
        // One step: the matrix products of each 16 along k with the LDS reads of the
        // next 16 between them, one after each product so that a read is never
        // waited for at once.
        auto work = [&](auto loading, int step) {
            constexpr bool kLoad = decltype(loading)::value;
            const int after = stage + 1 == kStages ? 0 : stage + 1;
#pragma unroll
            for (int kk = 0; kk + 1 < kKK; ++kk) {
                read((kk + 1) & 1, stage, kk + 1);
                mma(kk & 1);
#pragma unroll
                for (int i = 0; i < kMma; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                 // a matrix product
                    if (i < kReads) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // an LDS read
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            // Every wave holds the last fragments of this step: its place in LDS is
            // free for the step kStages on, and the next step's data has landed.
            if (kLoad || step + 1 < steps) {
                if (kLoad || step + kStages <= steps) wait_vmcnt<(kStages - 2) * kLoads>();
                else wait_vmcnt<0>();
                __builtin_amdgcn_s_waitcnt(0xc07f);  // this wave's LDS reads are done
                lds_barrier();
                read(0, after, 0);
                if (kLoad) load(stage, step + kStages);
            }
            mma((kKK - 1) & 1);
            if (kLoad) {
#pragma unroll
                for (int i = 0; i < kMma; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    if (i < kReads) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    constexpr int kEach = (kLoads + kMma - 1) / kMma;
                    if (i * kEach < kLoads) __builtin_amdgcn_sched_group_barrier(0x010, kEach, 0);  // loads to LDS
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            stage = after;
        };
        int step = 0;
        for (; step + kStages < steps; ++step) work(Yes{}, step);
        for (; step < steps; ++step) work(No{}, step);
        if constexpr (kApart) {
#pragma unroll
            for (int m = 0; m < kFM; ++m)
#pragma unroll
                for (int n = 0; n < kFN; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float x = acc[m][n][r];
                        acc[m][n][r] = P < 3 || fabsf(x) < INFINITY ? x + lesser[m][n][r] : x;
                    }
        }
        lds_barrier();  // every wave has read its last fragments: the epilogue may write LDS
    }

    // epi(row, column, v): eight consecutive columns of a row of the tile, a
    // multiple of eight from its left edge.  A wave's strip of 32 rows passes
    // through LDS, so that eight lanes write 64 consecutive columns.
    template <typename E>
    __device__ __forceinline__ void finish(char* lds, const E& epi) {
        const int lane = threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int wm = wave / kWN, wn = wave % kWN;
        float* strip = (float*)lds + wave * 32 * kEpiLd;
        constexpr int kLanes = kEpiCols / 8, kPass = 64 / kLanes;
#pragma unroll
        for (int m = 0; m < kFM; ++m) {
            to_strip(strip, m, lane);
            // one copy of epi a block row: unrolled further, a large one keeps the
            // compiler from unrolling over m, and acc goes to scratch memory
#pragma unroll 1
            for (int r = 0; r < 32; r += kPass) {
                const int row = r + lane / kLanes, col = lane % kLanes * 8;
                float v[8];
                const float4 x = *(const float4*)(strip + row * kEpiLd + col);
                const float4 y = *(const float4*)(strip + row * kEpiLd + col + 4);
                v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
                v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
                epi((wm * kFM + m) * 32 + row, wn * kEpiCols + col, v);
            }
            asm volatile("" ::: "memory");
        }
    }

    // The same, and the block a second time by columns: epi.row(row, column, v)
    // may change v, epi.column(row, column, v) then gets eight consecutive rows
    // of a column as row() left them.
    template <typename E>
    __device__ __forceinline__ void finish_both_ways(char* lds, const E& epi) {
        const int lane = threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int wm = wave / kWN, wn = wave % kWN;
        float* strip = (float*)lds + wave * 32 * kEpiLd;
        constexpr int kLanes = kEpiCols / 8, kPass = 64 / kLanes;
#pragma unroll
        for (int m = 0; m < kFM; ++m) {
            to_strip(strip, m, lane);
#pragma unroll
            for (int r = 0; r < 32; r += kPass) {
                const int row = r + lane / kLanes, col = lane % kLanes * 8;
                float v[8];
                float* s = strip + row * kEpiLd + col;
                const float4 x = *(const float4*)s, y = *(const float4*)(s + 4);
                v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
                v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
                epi.row((wm * kFM + m) * 32 + row, wn * kEpiCols + col, v);
                *(float4*)s = make_float4(v[0], v[1], v[2], v[3]);
                *(float4*)(s + 4) = make_float4(v[4], v[5], v[6], v[7]);
            }
            asm volatile("" ::: "memory");
#pragma unroll
            for (int c = 0; c < kEpiCols; c += 16) {
                const int col = c + lane / 4, row = lane % 4 * 8;
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = strip[(row + i) * kEpiLd + col];
                epi.column((wm * kFM + m) * 32 + row, wn * kEpiCols + col, v);
            }
            asm volatile("" ::: "memory");
        }
    }

    // Block row m of the wave's part of C into its LDS strip of 32 rows.
    __device__ __forceinline__ void to_strip(float* strip, int m, int lane) {
#pragma unroll
        for (int n = 0; n < kFN; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(float4*)(strip + (lane & 31) * kEpiLd + n * 32 + q * 8 + (lane >> 5) * 4) =
                    make_float4(acc[m][n][4 * q], acc[m][n][4 * q + 1], acc[m][n][4 * q + 2], acc[m][n][4 * q + 3]);
    }

  protected:
    // Byte offset of what this lane loads with the wave's load instruction for
    // row group g.
    static __device__ __forceinline__ uint32_t lane_offset(int g, int lane, uint32_t rows, uint32_t ld) {
        const int row = g * kRows + lane / kChunks;
        const uint32_t there = (uint32_t)row < rows ? (uint32_t)row : rows - 1;
        return there * ld * 2 + (uint32_t)((lane % kChunks) ^ swizzle(row)) * 16;
    }
    // 16 bytes a lane from `from` + off (the lane's) + step (the wave's) to LDS
    // at `to` + 16 * lane.
    static __device__ __forceinline__ void copy16(__amdgpu_buffer_rsrc_t from, uint32_t off, int step, char* to) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, (int)off, step,
                                                 0, 0);
    }
    static __device__ __forceinline__ __amdgpu_buffer_rsrc_t resource(const T* p) {
        return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, -1, 0x00020000);
    }
    struct Yes { static constexpr bool value = true; };
    struct No { static constexpr bool value = false; };
};

// Tile of workgroup b of a grid of tiles_m x tiles_n.  Workgroups are dealt to
// the eight compute dies in turn, each die with an L2 of its own: a die gets a
// run of consecutive tiles, and the tiles run down columns `kGroup` tiles high,
// so that the tiles a die works on at a time share rows of A and B.
template <int kGroup>
__device__ __forceinline__ void tile_of(uint32_t b, uint32_t tiles_m, uint32_t tiles_n, uint32_t& tm, uint32_t& tn) {
    const uint32_t total = tiles_m * tiles_n, q = total / 8, r = total % 8, die = b % 8;
    const uint32_t t = die * q + (die < r ? die : r) + b / 8;
    const uint32_t band = t / (kGroup * tiles_n), first = band * kGroup;
    const uint32_t high = tiles_m - first < kGroup ? tiles_m - first : kGroup;
    const uint32_t in = t - first * tiles_n;
    tm = first + in % high;
    tn = in / high;
}

}  // namespace bc
