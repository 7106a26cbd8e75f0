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

template <typename B_, bool TA, bool TB>
struct RunTile : B_ {
    typedef B_ B;
    typedef typename B::T T;
    using B::P; using B::kBM; using B::kBN; using B::kBK; using B::kWN; using B::kStages; using B::kWaves;
    using B::kFM; using B::kFN; using B::kRow; using B::kChunks; using B::kRows; using B::kLoadA; using B::kLoadB;
    using B::kLoads; using B::kStageBytes; using B::kApart; using B::acc;
    typedef typename Frag<T>::type frag;
    typedef short s16x4 __attribute__((ext_vector_type(4)));

    // Operands with k down their columns: bytes of a row in LDS, rows of a load instruction.
    static constexpr int kRowA = kBM * 2, kRowB = kBN * 2, kDownA = 512 / kBM, kDownB = 512 / kBN;
    static_assert(!TA || (kBM & (kBM - 1)) == 0, "whole rows in a load");
    static_assert(!TB || (kBN & (kBN - 1)) == 0, "whole rows in a load");
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

    // Products over k into acc, which is cleared.  row_a(r): byte offset of row r
    // of an operand A with k along its rows (kNowhere: zeros).  where_b: byte offsets
    // of the rows of an operand B with k down its columns, one for each k, valid
    // up to a step past k (kTable; then B's rows are wherever they say).
    template <bool kTable, typename RowA>
    __device__ __forceinline__ void multiply(const Side<T>& a, const Side<T>& b, uint32_t k, char* lds, RowA row_a,
                                             const uint32_t* __restrict__ where_b) {
        const int steps = (int)((k + kBK - 1) / kBK);
        const int lane = threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        uint32_t offa[kLoadA], offb[kLoadB], from_b[kLoadB];
#pragma unroll
        for (int i = 0; i < kLoadA; ++i) {
            const int r = row_of<TA, kBM, kLoadA>(i, wave, lane), c = chunk_of<TA, kBM>(r, lane);
            if constexpr (TA) {
                offa[i] = (uint32_t)c * 8 < a.count ? (uint32_t)r * a.ld * 2 + c * 16 : kNowhere;
            } else {
                const uint32_t at = (uint32_t)r < a.count ? row_a(r) : kNowhere;
                offa[i] = at == kNowhere ? kNowhere : at + c * 16;
            }
        }
#pragma unroll
        for (int i = 0; i < kLoadB; ++i) {
            const int r = row_of<TB, kBN, kLoadB>(i, wave, lane), c = chunk_of<TB, kBN>(r, lane);
            if constexpr (TB) {
                offb[i] = (uint32_t)c * 8 < b.count ? (kTable ? 0 : (uint32_t)r * b.ld * 2) + c * 16 : kNowhere;
                if (kTable && steps > 0) from_b[i] = where_b[r];
            } else {
                offb[i] = (uint32_t)r < b.count ? (uint32_t)r * b.ld * 2 + c * 16 : kNowhere;
            }
        }
        // the last step's loads: zeros past k
        auto mask_last = [&]() {
            const uint32_t left = k - (uint32_t)(steps - 1) * kBK;
#pragma unroll
            for (int i = 0; i < kLoadA; ++i) {
                const int r = row_of<TA, kBM, kLoadA>(i, wave, lane), c = chunk_of<TA, kBM>(r, lane);
                if ((TA ? (uint32_t)r : (uint32_t)c * 8) >= left) offa[i] = kNowhere;
            }
#pragma unroll
            for (int i = 0; i < kLoadB; ++i) {
                const int r = row_of<TB, kBN, kLoadB>(i, wave, lane), c = chunk_of<TB, kBN>(r, lane);
                if ((TB ? (uint32_t)r : (uint32_t)c * 8) >= left) offb[i] = kNowhere;
            }
        };
        auto load = [&](int stage, int step) {
            char* to = lds + stage * kStageBytes;
            uint32_t next[kLoadB];
            if constexpr (kTable) {
#pragma unroll
                for (int i = 0; i < kLoadB; ++i) next[i] = where_b[(uint32_t)(step + 1) * kBK + row_of<TB, kBN, kLoadB>(i, wave, lane)];
            }
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const __amdgpu_buffer_rsrc_t from = resource(a.p + p * a.plane + (TA ? (uint64_t)step * kBK * a.ld : 0));
#pragma unroll
                for (int i = 0; i < kLoadA; ++i)
                    B::copy16(from, offa[i], TA ? 0 : step * kRow,
                              to + p * kBM * kRow + (TA ? wave * kLoadA + i : i * kWaves + wave) * 1024);
            }
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const __amdgpu_buffer_rsrc_t from = resource(b.p + p * b.plane + (TB && !kTable ? (uint64_t)step * kBK * b.ld : 0));
#pragma unroll
                for (int i = 0; i < kLoadB; ++i)
                    B::copy16(from, kTable ? either(from_b[i], offb[i]) : offb[i], TB ? 0 : step * kRow,
                              to + (P * kBM + p * kBN) * kRow + (TB ? wave * kLoadB + i : i * kWaves + wave) * 1024);
            }
            if constexpr (kTable) {
#pragma unroll
                for (int i = 0; i < kLoadB; ++i) from_b[i] = next[i];
            }
        };
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
        for (int m = 0; m < kFM; ++m) fa[m] = lds + place<TA, kBM>(wm * kFM + m, lane);
#pragma unroll
        for (int n = 0; n < kFN; ++n) fb[n] = lds + P * kBM * kRow + place<TB, kBN>(wn * kFN + n, lane);
        frag va[2][P][kFM], vb[2][P][kFN];
        const int sw = B::swizzle(l31);
        auto read = [&](int set, int stage, int kk) {
            const int along = ((kk * 2 + hi) ^ sw) * 16;
#pragma unroll
            for (int p = 0; p < P; ++p) {
#pragma unroll
                for (int n = 0; n < kFN; ++n)
                    vb[set][p][n] = fetch<TB, kRowB>(fb[n] + stage * kStageBytes + p * kBN * kRow, kk, along);
#pragma unroll
                for (int m = 0; m < kFM; ++m)
                    va[set][p][m] = fetch<TA, kRowA>(fa[m] + stage * kStageBytes + p * kBM * kRow, kk, along);
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
        constexpr int kReads = P * (kFM * (TA ? 2 : 1) + kFN * (TB ? 2 : 1)), kEachRead = (kReads + kMma - 1) / kMma;
        static_assert(kKK % 2 == 0, "fragment sets alternate");
        if (steps > 0) {
#pragma unroll
            for (int i = 0; i < kStages; ++i)
                if (i < steps) {
                    if (i == steps - 1) mask_last();
                    load(i, i);
                }
            if (steps >= kStages) wait_vmcnt<(kStages - 1) * kLoads>();
            else wait_vmcnt<0>();
            lds_barrier();
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
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                                          // a matrix product
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
                if (kLoad) load(stage, step + kStages);
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
            mask_last();
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
        lds_barrier();  // every wave has read its last fragments: the epilogue may write LDS
    }

  private:
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
    // A fragment of 16 along k, from `at` of the lane's block; along: the swizzled
    // chunk of an operand with k along its rows.
    template <bool down, int row>
    static __device__ __forceinline__ frag fetch(const char* at, int kk, int along) {
        if constexpr (down) {
            typedef __attribute__((address_space(3))) s16x4 lds_vec;
            s16x4 v[2];
            v[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_vec*)(at + kk * 16 * row));
            v[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_vec*)(at + (kk * 16 + 4) * row));
            frag f;
            __builtin_memcpy(&f, v, sizeof(f));
            return f;
        } else {
            return *(const frag*)(at + along);
        }
    }
};

}  // namespace bc
