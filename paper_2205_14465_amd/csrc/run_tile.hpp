// run_tile.hpp -- the tile of gemm.hpp for operands that lie either way: each of
// the two has the contracted axis k along its rows, as there, or down its columns
// (an operand that a product takes transposed).
//
// An operand with k down its columns goes to LDS as it lies, a step's kBK rows of
// it, and the transposing LDS read hands each lane four consecutive k of one
// column: within 16 lanes, lane 4 j + q reads 8 bytes of row j, columns 4 q on, and
// lane i receives column i of rows 0 to 3.  Rows are a multiple of 128 bytes apart,
// so the 16-byte chunks of row r are swizzled by kTurn[r mod 4]: the four rows
// of a read, and the next sixteen columns, then lie in eight different pieces of 32
// bytes of 256.
//
// What is past an operand's end is loaded as zero: a lane's offset past the
// buffer's size reads 0.
#pragma once

#include "gemm.hpp"

namespace bc {

constexpr uint32_t kNowhere = 0x80000000u;   // a byte offset that reads zero

// One operand.  Rows (or columns) of the tile past `count` read zero.
template <typename T>
struct Side {
    const T* p;         // the tile's first row (column), first k
    uint64_t plane;     // elements from plane to plane
    uint32_t ld;        // elements from row to row in memory, < 2^21
    uint32_t count;     // rows (columns) there are from the tile's first on
};

// How a product's operands lie: whether k runs down A's and B's columns, and
// whether B's rows are wherever a table of byte offsets says.
template <bool TA_, bool TB_, bool kTable_ = false>
struct Lie {
    static constexpr bool TA = TA_, TB = TB_, kTable = kTable_;
};

template <typename B_>
struct RunTile : B_ {
    typedef B_ B;
    typedef typename B::T T;
    using B::P; using B::kBM; using B::kBN; using B::kBK; using B::kWN; using B::kStages; using B::kWaves;
    using B::kFM; using B::kFN; using B::kRow; using B::kChunks; using B::kRows; using B::kLoadA; using B::kLoadB;
    using B::kLoads; using B::kStageBytes; using B::kApart; using B::acc;
    typedef typename Frag<T>::type frag;
    typedef short s16x4 __attribute__((ext_vector_type(4)));

    static_assert((kBM & (kBM - 1)) == 0 && (kBN & (kBN - 1)) == 0 && kBM <= 512 && kBN <= 512, "whole rows in a load");

    // What a lane loads of the tile at hand.
    Side<T> a, b;
    uint32_t k;
    const uint32_t* where;
    uint32_t offa[kLoadA], offb[kLoadB], from_b[kLoadB];

    // Chunks' swizzle of row r in LDS, for rows of `width` elements.
    template <int width>
    static __device__ __forceinline__ int turn(int r) {
        return 2 * ((r & 3) | (width > 64 ? (r & 1) << 2 : 0));
    }
    // Row (or k) within the tile's step that load i of this wave brings to this
    // lane, and the lane's chunk of it.
    template <bool down, int width, int loads>
    static __device__ __forceinline__ int row_of(int i, int wave, int lane) {
        if constexpr (down) return (wave * loads + i) * (512 / width) + lane / (width / 8);
        else return (i * kWaves + wave) * kRows + lane / kChunks;
    }
    template <bool down, int width>
    static __device__ __forceinline__ int chunk_of(int r, int lane) {
        if constexpr (down) return lane % (width / 8) ^ turn<width>(r);
        else return lane % kChunks ^ B::swizzle(r);
    }
    __device__ __forceinline__ int steps() const { return (int)((k + kBK - 1) / kBK); }
    static __device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

    // Takes up a tile, k long, and asks for its first step; every wave must have read
    // what stage 0 held.  row_a(r): byte offset of row r of an operand A with k
    // along its rows (kNowhere: zeros).  where_: with a table, byte offsets of B's
    // rows, one for each k, valid up to a step past k.
    template <typename L, typename RowA>
    __device__ __forceinline__ void begin(const Side<T>& a_, const Side<T>& b_, uint32_t k_, const uint32_t* where_, char* lds,
                                          RowA row_a) {
        a = a_;
        b = b_;
        k = k_;
        where = where_;
        const int lane = threadIdx.x & 63, wave = wave_index();
#pragma unroll
        for (int i = 0; i < kLoadA; ++i) {
            const int r = row_of<L::TA, kBM, kLoadA>(i, wave, lane), c = chunk_of<L::TA, kBM>(r, lane);
            if constexpr (L::TA) {
                offa[i] = (uint32_t)c * 8 < a.count ? (uint32_t)r * a.ld * 2 + c * 16 : kNowhere;
            } else {
                const uint32_t at = (uint32_t)r < a.count ? row_a(r) : kNowhere;
                offa[i] = at == kNowhere ? kNowhere : at + c * 16;
            }
        }
#pragma unroll
        for (int i = 0; i < kLoadB; ++i) {
            const int r = row_of<L::TB, kBN, kLoadB>(i, wave, lane), c = chunk_of<L::TB, kBN>(r, lane);
            if constexpr (L::TB) {
                offb[i] = (uint32_t)c * 8 < b.count ? (L::kTable ? 0 : (uint32_t)r * b.ld * 2) + c * 16 : kNowhere;
                if (L::kTable && k > 0) from_b[i] = where[r];
            } else {
                offb[i] = (uint32_t)r < b.count ? (uint32_t)r * b.ld * 2 + c * 16 : kNowhere;
            }
        }
        ask<L>(lds, 0, 1);
    }
    // Asks for the next steps of the first kStages, when their stages are free.
    template <typename L>
    __device__ __forceinline__ void rest(char* lds) { ask<L>(lds, 1, kStages); }

    // The products over k into acc, after begin() and rest().  kLanded: every wave has
    // waited for its first step's loads, and met the others since.
    template <typename L, bool kLanded = false>
    __device__ __forceinline__ void run(char* lds) {
        const int steps = this->steps();
        const int lane = threadIdx.x & 63, wave = wave_index();
#pragma unroll
        for (int m = 0; m < kFM; ++m)
#pragma unroll
            for (int n = 0; n < kFN; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[m][n][r] = 0.0f;
        const int wm = wave / kWN, wn = wave % kWN;
        const int hi = lane >> 5, l31 = lane & 31;
        // where this lane's fragments lie in a stage
        const char* fa[kFM];
        const char* fb[kFN];
#pragma unroll
        for (int m = 0; m < kFM; ++m) fa[m] = lds + place<L::TA, kBM>(wm * kFM + m, lane);
#pragma unroll
        for (int n = 0; n < kFN; ++n) fb[n] = lds + P * kBM * kRow + place<L::TB, kBN>(wn * kFN + n, lane);
        frag va[2][P][kFM], vb[2][P][kFN];
        const int sw = B::swizzle(l31);
        auto read = [&](int set, int stage, int kk) {
            const int along = ((kk * 2 + hi) ^ sw) * 16;
#pragma unroll
            for (int p = 0; p < P; ++p) {
#pragma unroll
                for (int n = 0; n < kFN; ++n)
                    vb[set][p][n] = fetch<L::TB, kBN * 2>(fb[n] + stage * kStageBytes + p * kBN * kRow, kk, along);
#pragma unroll
                for (int m = 0; m < kFM; ++m)
                    va[set][p][m] = fetch<L::TA, kBM * 2>(fa[m] + stage * kStageBytes + p * kBM * kRow, kk, along);
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
        constexpr int kKK = kBK / 16, kMma = P * (P + 1) / 2 * kFM * kFN;
        constexpr int kReads = P * (kFM * (L::TA ? 2 : 1) + kFN * (L::TB ? 2 : 1)), kEachRead = (kReads + kMma - 1) / kMma;
        static_assert(kKK % 2 == 0, "fragment sets alternate");
        if (steps > 0) {
            if constexpr (!kLanded) {
                if (steps >= kStages) wait_vmcnt<(kStages - 1) * kLoads>();
                else wait_vmcnt<0>();
                lds_barrier();
            }
            read(0, 0, 0);
        }
        int stage = 0;
        // one step, as in gemm.hpp
        auto work = [&](auto loading, int step) {
            constexpr bool kLoad = decltype(loading)::value;
            const int after = stage + 1 == kStages ? 0 : stage + 1;
#pragma unroll
            for (int kk = 0; kk + 1 < kKK; ++kk) {
                read((kk + 1) & 1, stage, kk + 1);
                mma(kk & 1);
#pragma unroll
                for (int i = 0; i < kMma; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                                      // a matrix product
                    if (i * kEachRead < kReads) __builtin_amdgcn_sched_group_barrier(0x100, kEachRead, 0);  // LDS reads
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (kLoad || step + 1 < steps) {
                if (kLoad || step + kStages <= steps) wait_vmcnt<(kStages - 2) * kLoads>();
                else wait_vmcnt<0>();
                __builtin_amdgcn_s_waitcnt(0xc07f);  // this wave's LDS reads are done
                lds_barrier();
                read(0, after, 0);
                if (kLoad) load<L>(lds, stage, step + kStages);
            }
            mma((kKK - 1) & 1);
            if (kLoad) {
#pragma unroll
                for (int i = 0; i < kMma; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    if (i * kEachRead < kReads) __builtin_amdgcn_sched_group_barrier(0x100, kEachRead, 0);
                    constexpr int kEach = (kLoads + kMma - 1) / kMma;
                    if (i * kEach < kLoads) __builtin_amdgcn_sched_group_barrier(0x010, kEach, 0);  // loads to LDS
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            stage = after;
        };
        int step = 0;
        for (; step + kStages < steps - 1; ++step) work(typename B::Yes{}, step);
        if (step + kStages < steps) {
            mask_last<L>();
            work(typename B::Yes{}, step++);
        }
        for (; step < steps; ++step) work(typename B::No{}, step);
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
        lds_barrier();  // every wave has read its last fragments: LDS is free
    }

    // gemm.hpp's finish() in two parts: rows of blocks [from, to) of the wave's part of C.
    template <int from, int to, typename E>
    __device__ __forceinline__ void finish_blocks(char* lds, const E& epi) {
        const int lane = threadIdx.x & 63, wave = wave_index();
        const int wm = wave / kWN, wn = wave % kWN;
        float* strip = (float*)lds + wave * 32 * B::kEpiLd;
        constexpr int kLanes = B::kEpiCols / 8, kPass = 64 / kLanes;
#pragma unroll
        for (int m = from; m < to; ++m) {
            B::to_strip(strip, m, lane);
#pragma unroll 1
            for (int r = 0; r < 32; r += kPass) {
                const int row = r + lane / kLanes, col = lane % kLanes * 8;
                float v[8];
                const float4 x = *(const float4*)(strip + row * B::kEpiLd + col);
                const float4 y = *(const float4*)(strip + row * B::kEpiLd + col + 4);
                v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
                v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
                epi((wm * kFM + m) * 32 + row, wn * B::kEpiCols + col, v);
            }
            asm volatile("" ::: "memory");
        }
    }

  private:
    template <typename L>
    __device__ __forceinline__ void ask(char* lds, int from, int to) {
#pragma unroll
        for (int i = 0; i < kStages; ++i)
            if (i >= from && i < to && i < steps()) {
                if (i == steps() - 1) mask_last<L>();
                load<L>(lds, i, i);
            }
    }
    // The last step's loads: zeros past k.
    template <typename L>
    __device__ __forceinline__ void mask_last() {
        const int lane = threadIdx.x & 63, wave = wave_index();
        const uint32_t left = k - (uint32_t)(steps() - 1) * kBK;
#pragma unroll
        for (int i = 0; i < kLoadA; ++i) {
            const int r = row_of<L::TA, kBM, kLoadA>(i, wave, lane), c = chunk_of<L::TA, kBM>(r, lane);
            if ((L::TA ? (uint32_t)r : (uint32_t)c * 8) >= left) offa[i] = kNowhere;
        }
#pragma unroll
        for (int i = 0; i < kLoadB; ++i) {
            const int r = row_of<L::TB, kBN, kLoadB>(i, wave, lane), c = chunk_of<L::TB, kBN>(r, lane);
            if ((L::TB ? (uint32_t)r : (uint32_t)c * 8) >= left) offb[i] = kNowhere;
        }
    }
    template <typename L>
    __device__ __forceinline__ void load(char* lds, int stage, int step) {
        const int lane = threadIdx.x & 63, wave = wave_index();
        char* to = lds + stage * kStageBytes;
        uint32_t next[kLoadB];
        if constexpr (L::kTable) {
#pragma unroll
            for (int i = 0; i < kLoadB; ++i) next[i] = where[(uint32_t)(step + 1) * kBK + row_of<L::TB, kBN, kLoadB>(i, wave, lane)];
        }
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const __amdgpu_buffer_rsrc_t from = resource(a.p + p * a.plane + (L::TA ? (uint64_t)step * kBK * a.ld : 0));
#pragma unroll
            for (int i = 0; i < kLoadA; ++i)
                B::copy16(from, offa[i], L::TA ? 0 : step * kRow,
                          to + p * kBM * kRow + (L::TA ? wave * kLoadA + i : i * kWaves + wave) * 1024);
        }
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const __amdgpu_buffer_rsrc_t from =
                resource(b.p + p * b.plane + (L::TB && !L::kTable ? (uint64_t)step * kBK * b.ld : 0));
#pragma unroll
            for (int i = 0; i < kLoadB; ++i)
                B::copy16(from, L::kTable ? either(from_b[i], offb[i]) : offb[i], L::TB ? 0 : step * kRow,
                          to + (P * kBM + p * kBN) * kRow + (L::TB ? wave * kLoadB + i : i * kWaves + wave) * 1024);
        }
        if constexpr (L::kTable) {
#pragma unroll
            for (int i = 0; i < kLoadB; ++i) from_b[i] = next[i];
        }
    }
    static __device__ __forceinline__ uint32_t either(uint32_t row, uint32_t chunk) {
        return row == kNowhere || chunk == kNowhere ? kNowhere : row + chunk;
    }
    static __device__ __forceinline__ __amdgpu_buffer_rsrc_t resource(const T* p) {
        return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, 0x7fffffff, 0x00020000);
    }
    // Where a lane's fragments of block `block` (32 rows or columns) begin in a stage's operand.
    template <bool down, int width>
    static __device__ __forceinline__ int place(int block, int lane) {
        if constexpr (down) {
            const int r = (lane >> 5) * 8 + ((lane & 15) >> 2);   // its k
            const int chunk = block * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
            return r * width * 2 + (chunk ^ turn<width>(r)) * 16 + (lane & 1) * 8;
        } else {
            return (block * 32 + (lane & 31)) * kRow;
        }
    }
    // The transposing read.  Its pointer is restrict, which says no more than that it
    // has a scope of its own: for one without, the compiler waits for every load to
    // LDS in flight, also those of other stages.
    static __device__ __forceinline__ s16x4 turned(const char* __restrict__ p) {
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
    }
    // A fragment of 16 along k, from `at` of the lane's block; along: the swizzled
    // chunk of an operand with k along its rows.
    template <bool down, int row>
    static __device__ __forceinline__ frag fetch(const char* at, int kk, int along) {
        if constexpr (down) {
            const s16x4 v[2] = {turned(at + kk * 16 * row), turned(at + (kk * 16 + 4) * row)};
            frag f;
            __builtin_memcpy(&f, v, sizeof(f));
            return f;
        } else {
            return *(const frag*)(at + along);
        }
    }
};

}  // namespace bc
