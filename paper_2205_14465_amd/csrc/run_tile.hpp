// run_tile.hpp -- the tile of gemm.hpp for operands that lie either way: each of
// the two has the contracted axis k along its rows, as there, or down its columns
// (an operand that a product takes transposed); and for fp32 on the fp32 matrix
// instruction (32x32x2), two elements of k at a time.
//
// An operand with k down its columns goes to LDS as it lies, a step's kBK rows of
// it.  16-bit ones come back by the transposing LDS read, which hands each lane four
// consecutive k of one column: within 16 lanes, lane 4 j + q reads 8 bytes of row j,
// columns 4 q on, and lane i receives column i of rows 0 to 3.  Rows are a multiple
// of 128 bytes apart, so the 16-byte chunks of row r are swizzled by kTurn[r mod 4]:
// the four rows of a read, and the next sixteen columns, then lie in eight different
// pieces of 32 bytes of 256.  fp32 ones are read word by word, 32 columns of a row
// at a time.
//
// What is past an operand's end is loaded as zero: a lane's offset past the
// buffer's size reads 0.
#pragma once

#include "gemm.hpp"

namespace bc {

constexpr uint32_t kNowhere = 0x80000000u;   // a byte offset that reads zero

// A fragment: 16 bytes of a row of k for each lane, those of the upper half of the
// wave after those of the lower.
template <typename T>
struct RunFrag {
    typedef typename Frag<T>::type type;
    static constexpr int kProducts = 1;      // matrix instructions
    static __device__ __forceinline__ f32x16 mma(type a, type b, f32x16 c) { return Frag<T>::mma(a, b, c); }
};
typedef float f32x4v __attribute__((ext_vector_type(4)));
template <>
struct RunFrag<float> {
    typedef f32x4v type;
    static constexpr int kProducts = 4;
    // (element i of both halves: two of the fragment's eight k, the same in both operands)
    static __device__ __forceinline__ f32x16 mma(type a, type b, f32x16 c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
};

// One operand.  Rows (or columns) of the tile past `count` read zero.
template <typename T>
struct Side {
    const T* p;         // the tile's first row (column), first k
    uint32_t ld;        // elements from row to row in memory, < 2^21
    uint32_t count;     // rows (columns) there are from the tile's first on
};

// How a product's operands lie: whether k runs down A's and B's columns, whether B's
// rows are wherever a table of byte offsets says, and the bytes that a lane loads at a
// time: 16, where every row is made of whole such pieces, or 4 (fp32 only).
template <bool TA_, bool TB_, bool kTable_, int kPiece_>
struct Lie {
    static constexpr bool TA = TA_, TB = TB_, kTable = kTable_;
    static constexpr int kPiece = kPiece_;
};

template <typename B_, int kPiece>
struct RunTile : B_ {
    typedef B_ B;
    typedef typename B::T T;
    using B::kBM; using B::kBN; using B::kBK; using B::kWN; using B::kStages; using B::kWaves; using B::kElem;
    using B::kFM; using B::kFN; using B::kRow; using B::kStageBytes; using B::acc;
    typedef RunFrag<T> F;
    typedef typename F::type frag;
    typedef short s16x4 __attribute__((ext_vector_type(4)));

    static_assert(B::P == 1 && (kPiece == 16 || (kPiece == 4 && kElem == 4)), "pieces");
    static_assert((kBM & (kBM - 1)) == 0 && (kBN & (kBN - 1)) == 0, "whole rows in a load");
    // Load instructions of a wave and step.
    static constexpr int kLoadA = kBM * kRow / (64 * kPiece) / kWaves, kLoadB = kBN * kRow / (64 * kPiece) / kWaves;
    static constexpr int kLoads = kLoadA + kLoadB;
    static_assert(kLoadA * kWaves * 64 * kPiece == kBM * kRow && kLoadB * kWaves * 64 * kPiece == kBN * kRow, "loads cover the tile");
    static_assert((kStages - 1) * kLoads < 64, "the count of loads in flight has six bits");

    // What a lane loads of the tile at hand.
    Side<T> a, b;
    uint32_t k;
    const uint32_t* where;
    uint32_t offa[kLoadA], offb[kLoadB], from_b[kLoadB];
    bool busy;          // whether this wave took part in the last run()'s products

    // Chunks' swizzle of row r in LDS, for rows of `width` elements of k down columns.
    template <int width>
    static __device__ __forceinline__ int turn(int r) {
        return kElem == 4 ? 0 : 2 * ((r & 3) | (width > 64 ? (r & 1) << 2 : 0));
    }
    // Load i of this wave brings to LDS, from `index` x 64 pieces on, to this lane: row
    // (or k within the step) `row`, elements `at` on of it.
    template <bool down, int loads>
    static __device__ __forceinline__ int index_of(int i, int wave) { return down ? wave * loads + i : i * kWaves + wave; }
    struct Spot {
        int row, at;
    };
    template <bool down, int width, int loads>
    static __device__ __forceinline__ Spot spot_of(int i, int wave, int lane) {
        constexpr int kLong = down ? width * kElem : kRow;
        const int byte = (index_of<down, loads>(i, wave) * 64 + lane) * kPiece, row = byte / kLong, in = byte % kLong;
        const int chunk = in / 16 ^ (down ? turn<width>(row) : B::swizzle(row));
        return Spot{row, chunk * (16 / kElem) + in % 16 / kElem};
    }
    __device__ __forceinline__ int steps() const { return (int)((k + kBK - 1) / kBK); }
    static __device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
    // Which rows and columns of blocks are this wave's.  Waves w and w + 4 share a SIMD:
    // of the largest tile's, the upper four have the columns two on from the lower
    // ones', so that either half of the rows and either of the columns is one wave a SIMD.
    static __device__ __forceinline__ int wave_m(int wave) { return wave / kWN; }
    static __device__ __forceinline__ int wave_n(int wave) {
        return kBM == 256 && kWN == 4 ? wave % kWN ^ (wave / kWN & 1) * 2 : wave % kWN;
    }

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
            const Spot s = spot_of<L::TA, kBM, kLoadA>(i, wave, lane);
            if constexpr (L::TA) {
                offa[i] = (uint32_t)s.at < a.count ? ((uint32_t)s.row * a.ld + s.at) * kElem : kNowhere;
            } else {
                const uint32_t at = (uint32_t)s.row < a.count ? row_a(s.row) : kNowhere;
                offa[i] = at == kNowhere ? kNowhere : at + s.at * kElem;
            }
        }
#pragma unroll
        for (int i = 0; i < kLoadB; ++i) {
            const Spot s = spot_of<L::TB, kBN, kLoadB>(i, wave, lane);
            if constexpr (L::TB) {
                offb[i] = (uint32_t)s.at < b.count ? ((L::kTable ? 0 : (uint32_t)s.row * b.ld) + s.at) * kElem : kNowhere;
                if (L::kTable && k > 0) from_b[i] = where[s.row];
            } else {
                offb[i] = (uint32_t)s.row < b.count ? ((uint32_t)s.row * b.ld + s.at) * kElem : kNowhere;
            }
        }
        ask<L>(lds, 0, 1);
    }
    // Asks for the next steps of the first kStages, when their stages are free.
    template <typename L>
    __device__ __forceinline__ void rest(char* lds) { ask<L>(lds, 1, kStages); }

    // The products over k into acc, after begin() and rest().  kLanded: every wave has
    // waited for its first step's loads, and met the others since; and a wave whose part
    // of the tile is past the operands' ends loads, and waits, but has no products (16
    // experts' 16384 rows of 1600 to 6400, from 400 to 2100 an expert: 482 to 452 us,
    // with such tiles last).  Not with a table, whose loads the compiler then waits for
    // sooner (the weights' gradient of the same rows 500 to 532 us).
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
        const int wm = wave_m(wave), wn = wave_n(wave);
        busy = true;
        if constexpr (kLanded && !L::kTable) {
            busy = (uint32_t)wm * kFM * 32 < a.count && (uint32_t)wn * kFN * 32 < b.count;
            if (!busy) {
                attend<L>(lds, steps);
                return;
            }
        }
        const int hi = lane >> 5, l31 = lane & 31;
        // where this lane's fragments lie in a stage
        const char* fa[kFM];
        const char* fb[kFN];
#pragma unroll
        for (int m = 0; m < kFM; ++m) fa[m] = lds + place<L::TA, kBM>(wm * kFM + m, lane);
#pragma unroll
        for (int n = 0; n < kFN; ++n) fb[n] = lds + kBM * kRow + place<L::TB, kBN>(wn * kFN + n, lane);
        frag va[2][kFM], vb[2][kFN];
        const int sw = B::swizzle(l31);
        auto read = [&](int set, int stage, int kk) {
            const int along = ((kk * 2 + hi) ^ sw) * 16;
#pragma unroll
            for (int n = 0; n < kFN; ++n) vb[set][n] = fetch<L::TB, kBN * kElem>(fb[n] + stage * kStageBytes, kk, along);
#pragma unroll
            for (int m = 0; m < kFM; ++m) va[set][m] = fetch<L::TA, kBM * kElem>(fa[m] + stage * kStageBytes, kk, along);
        };
        auto mma = [&](int set) {
#pragma unroll
            for (int m = 0; m < kFM; ++m)
#pragma unroll
                for (int n = 0; n < kFN; ++n) acc[m][n] = F::mma(vb[set][n], va[set][m], acc[m][n]);
        };
        constexpr int kKK = kRow / 32, kMma = F::kProducts * kFM * kFN, kDown = kElem == 4 ? 4 : 2;
        constexpr int kReads = kFM * (L::TA ? kDown : 1) + kFN * (L::TB ? kDown : 1), kEachRead = (kReads + kMma - 1) / kMma;
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
        lds_barrier();  // every wave has read its last fragments: LDS is free
    }

    // gemm.hpp's finish() in two parts: rows of blocks [from, to) of the wave's part of C.
    template <int from, int to, typename E>
    __device__ __forceinline__ void finish_blocks(char* lds, const E& epi) {
        const int lane = threadIdx.x & 63, wave = wave_index();
        const int wm = wave_m(wave), wn = wave_n(wave);
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
    // run() without its products: the same loads, waits and barriers.
    template <typename L>
    __device__ __forceinline__ void attend(char* lds, int steps) {
        int stage = 0;
#pragma unroll 1
        for (int step = 0; step + 1 < steps; ++step) {
            if (step + kStages <= steps) wait_vmcnt<(kStages - 2) * kLoads>();
            else wait_vmcnt<0>();
            lds_barrier();
            if (step + kStages < steps) {
                if (step + kStages == steps - 1) mask_last<L>();
                load<L>(lds, stage, step + kStages);
            }
            stage = stage + 1 == kStages ? 0 : stage + 1;
        }
        lds_barrier();
    }
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
            const Spot s = spot_of<L::TA, kBM, kLoadA>(i, wave, lane);
            if ((uint32_t)(L::TA ? s.row : s.at) >= left) offa[i] = kNowhere;
        }
#pragma unroll
        for (int i = 0; i < kLoadB; ++i) {
            const Spot s = spot_of<L::TB, kBN, kLoadB>(i, wave, lane);
            if ((uint32_t)(L::TB ? s.row : s.at) >= left) offb[i] = kNowhere;
        }
    }
    template <typename L>
    __device__ __forceinline__ void load(char* lds, int stage, int step) {
        const int lane = threadIdx.x & 63, wave = wave_index();
        char* to = lds + stage * kStageBytes;
        uint32_t at[kLoadB];
#pragma unroll
        for (int i = 0; i < kLoadB; ++i) at[i] = L::kTable ? either(from_b[i], offb[i]) : offb[i];
        // the next step's rows, into the registers that have just been read and before this
        // step's loads, so that they are there when those still are not
        if constexpr (L::kTable) {
#pragma unroll
            for (int i = 0; i < kLoadB; ++i)
                from_b[i] = where[(uint32_t)(step + 1) * kBK + spot_of<L::TB, kBN, kLoadB>(i, wave, lane).row];
        }
        const __amdgpu_buffer_rsrc_t from_a = resource(a.p + (L::TA ? (uint64_t)step * kBK * a.ld : 0));
#pragma unroll
        for (int i = 0; i < kLoadA; ++i)
            copy(from_a, offa[i], L::TA ? 0 : step * kRow, to + index_of<L::TA, kLoadA>(i, wave) * 64 * kPiece);
        const __amdgpu_buffer_rsrc_t rows_b = resource(b.p + (L::TB && !L::kTable ? (uint64_t)step * kBK * b.ld : 0));
#pragma unroll
        for (int i = 0; i < kLoadB; ++i)
            copy(rows_b, at[i], L::TB ? 0 : step * kRow, to + kBM * kRow + index_of<L::TB, kLoadB>(i, wave) * 64 * kPiece);
    }
    static __device__ __forceinline__ void copy(__amdgpu_buffer_rsrc_t from, uint32_t off, int step, char* to) {
        auto* lds = (__attribute__((address_space(3))) void*)to;
        if constexpr (kPiece == 16) __builtin_amdgcn_raw_ptr_buffer_load_lds(from, lds, 16, (int)off, step, 0, 0);
        else __builtin_amdgcn_raw_ptr_buffer_load_lds(from, lds, 4, (int)off, step, 0, 0);
    }
    static __device__ __forceinline__ uint32_t either(uint32_t row, uint32_t chunk) {
        return row == kNowhere || chunk == kNowhere ? kNowhere : row + chunk;
    }
    // (p is the same in all lanes, which the compiler does not see everywhere: a load for
    // each different pointer would be a loop)
    static __device__ __forceinline__ __amdgpu_buffer_rsrc_t resource(const T* p) {
        const uint64_t at = (uint64_t)p;
        const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)at), hi = __builtin_amdgcn_readfirstlane((int)(at >> 32));
        return __builtin_amdgcn_make_buffer_rsrc((void*)((uint64_t)hi << 32 | lo), 0, 0x7fffffff, 0x00020000);
    }
    // Where a lane's fragments of block `block` (32 rows or columns) begin in a stage's operand.
    template <bool down, int width>
    static __device__ __forceinline__ int place(int block, int lane) {
        if constexpr (!down) {
            return (block * 32 + (lane & 31)) * kRow;
        } else if constexpr (kElem == 4) {
            return (lane >> 5) * 4 * width * 4 + (block * 32 + (lane & 31)) * 4;
        } else {
            const int r = (lane >> 5) * 8 + ((lane & 15) >> 2);   // its k
            const int chunk = block * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
            return r * width * 2 + (chunk ^ turn<width>(r)) * 16 + (lane & 1) * 8;
        }
    }
    // The transposing read.  Its pointer is restrict, which says no more than that it
    // has a scope of its own: for one without, the compiler waits for every load to
    // LDS in flight, also those of other stages.
    static __device__ __forceinline__ s16x4 turned(const char* __restrict__ p) {
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
    }
    // Fragment kk of a step, from `at` of the lane's block; along: the swizzled chunk of an
    // operand with k along its rows; row: bytes of one with k down its columns.
    template <bool down, int row>
    static __device__ __forceinline__ frag fetch(const char* at, int kk, int along) {
        if constexpr (!down) {
            return *(const frag*)(at + along);
        } else if constexpr (kElem == 4) {
            frag f;
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = *(const float*)(at + (kk * 8 + i) * row);
            return f;
        } else {
            const s16x4 v[2] = {turned(at + kk * 16 * row), turned(at + (kk * 16 + 4) * row)};
            frag f;
            __builtin_memcpy(&f, v, sizeof(f));
            return f;
        }
    }
};

}  // namespace bc
