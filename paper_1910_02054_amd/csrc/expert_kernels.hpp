// expert_kernels.hpp -- products of the experts' rows with their weights, and the weights'
// gradient: tiles of both operands in LDS, sums in the matrix cores' registers.
//
// A step of the sum takes 128 bytes of its axis (64 elements of 16 bits, 32 of fp32).  An operand's tile
// comes in one of two layouts, as it lies in memory:
//   along    its rows run along the summed axis (x; weights that lie [out, in]): tile rows of 128 bytes
//   across   they run across it (weights that lie [in, out]; both operands of the gradient): one
//            tile row for each place of the axis, which the matrix instruction wants transposed;
//            ds_read_b64_tr_b16 does that for 16 bits, fp32's fragments are single words anyway
// The 16-byte chunks of a tile row are exchanged by a few bits of the row, so that the lanes of a fragment read
// different banks; the copy to LDS writes chunks in the lanes' order, so the exchange is in the address that a
// lane reads from memory.  (A ds_read_b128 takes lanes 0 to 3, 12 to 15 and 20 to 27 in one cycle, 4 to 11, 16 to
// 19 and 28 to 31 in the next, and likewise the upper half; the exchanges keep those apart, and the counters show
// no conflict.)
//
// The first operand of a matrix instruction is the columns' side (weights, dy), the second the rows' (x):
// a lane then holds neighbouring columns of one row of the result.
#pragma once

#include <type_traits>

#include "row_ops.hpp"
#include "zero_operators.h"

namespace zo {

#define ZO_LDS(T, p) ((__attribute__((address_space(3))) T*)(p))

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef u32x2 u32x2_e2 __attribute__((aligned(2)));

constexpr int kStepBytes = 128;  // of the summed axis

// The rows of a matrix (ZERO's `*_slots`): `mode` 0, 1 or n; a slot's row for n is slot * mul >> shift.
struct SlotMap {
    int32_t mode;
    uint32_t mul;
    int32_t shift;
    // Of an entry of order that lies in [0, slots).
    __device__ __forceinline__ int64_t row(uint32_t slot) const {
        return mode <= 1 ? slot : (uint32_t)((uint64_t)slot * mul >> shift);
    }
};

// Row i of the experts' order in a matrix, -1 where order names none.
__device__ __forceinline__ int64_t row_at(const int32_t* order, const SlotMap& map, int64_t slots, uint32_t i) {
    if (map.mode == 0)
        return i;
    const uint32_t slot = (uint32_t)order[i];
    return slot < (uint64_t)slots ? map.row(slot) : -1;
}

struct ExpertCall {
    const int32_t* offsets;
    const int32_t* order;
    const void* x;
    int64_t ld_x;
    const void* w;         // the weights, or dy
    int64_t ld_w;
    void* out;             // y, or dweight
    int64_t ld_out;
    float* partial;        // [parts, cols_in, cols_out]
    int64_t slots;
    int32_t experts;
    int32_t cols_in, cols_out;
    int32_t part;          // rows of a part of the weights' gradient's sums; 0: an expert's rows are one part
    SlotMap x_map, out_map;  // of x, and of y or dy
};

__device__ const u32x4 zero_chunk = {0, 0, 0, 0};

// ---------------------------------------------------------------------------
// Fragments: 16 bytes a lane, lane l's row is l % 16, its places of the axis are chunk l / 16 of
// the half step kk.
// ---------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (T::kPer == 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, (uint32_t)a[j]),
                                                     __builtin_bit_cast(float, (uint32_t)b[j]), c, 0, 0, 0);
        return c;
    } else if constexpr (T::kLowest == F16::kLowest) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                      0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    }
}

// Along: the exchange of the chunks of tile row r.  On the columns' side a pair of fragments takes 32 rows so that
// a lane's 4 + 4 results are neighbours: fragment f, lane row a is tile row 32 (f / 2) + 8 (a / 4) + 4 (f % 2) + a
// % 4.
template <bool PAIRED>
__device__ __forceinline__ int along_exchange(int r) {
    return PAIRED ? (r & 3) | (r >> 3 & 1) << 2 : r & 7;
}

// Across: the exchange of the chunks of the tile row of place k, for rows of CHUNKS chunks.
template <typename T, int CHUNKS>
__device__ __forceinline__ int across_exchange(int k) {
    if constexpr (T::kPer == 4)
        return ((k >> 2 & 3) << 2) & (CHUNKS - 1);
    else
        return (((k & 3) | (k >> 3 & 1) << 2) << 1) & (CHUNKS - 1);
}

// One side of a wave's fragments: byte offsets in the tile, once for each fragment or half step.
template <typename T, bool ALONG, bool PAIRED, int TILE, int COUNT>
struct Side {
    static constexpr int kRow = ALONG ? kStepBytes : TILE * (int)sizeof(typename T::elem);  // bytes of a tile row
    static constexpr int kChunks = kRow / 16;
    int at[ALONG ? 2 : COUNT];
    // first: the wave's first row (along) or column (across) in the tile
    __device__ __forceinline__ Side(int first, int lane) {
        const int a = lane & 15, g = lane >> 4;
        if constexpr (ALONG) {
            const int r = first + (PAIRED ? 8 * (a >> 2) + (a & 3) : a);
            const int c = g ^ along_exchange<PAIRED>(r);
#pragma unroll
            for (int kk = 0; kk < 2; ++kk)
                at[kk] = r * kRow + (c ^ 4 * kk) * 16;
        } else if constexpr (T::kPer == 4) {
#pragma unroll
            for (int f = 0; f < COUNT; ++f) {
                const int n = first + 16 * f + a, k = 4 * g;
                at[f] = k * kRow + ((n >> 2) ^ across_exchange<T, kChunks>(k)) * 16 + (n & 3) * 4;
            }
        } else {
#pragma unroll
            for (int f = 0; f < COUNT; ++f) {
                const int n = first + 16 * f + 4 * (a & 3), k = 8 * g + (a >> 2);
                at[f] = k * kRow + ((n >> 3) ^ across_exchange<T, kChunks>(k)) * 16 + (n & 7) * 2;
            }
        }
    }
    __device__ __forceinline__ u32x4 load(const char* tile, int f, int kk) const {
        if constexpr (ALONG) {
            const int step = PAIRED ? (f >> 1) * 32 * kRow + (f & 1) * 4 * kRow : f * 16 * kRow;
            // rows 4 apart in a pair have the same exchange
            return *reinterpret_cast<const u32x4*>(tile + at[kk] + step);
        } else if constexpr (T::kPer == 4) {
            u32x4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                v[j] = *reinterpret_cast<const uint32_t*>(tile + at[f] + (16 * kk + j) * kRow);
            return v;
        } else {
            const char* p = tile + at[f] + 32 * kk * kRow;
            const auto lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(ZO_LDS(i16x4, p));
            const auto hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(ZO_LDS(i16x4, p + 4 * kRow));
            const u32x2 l = __builtin_bit_cast(u32x2, lo), h = __builtin_bit_cast(u32x2, hi);
            return u32x4{l.x, l.y, h.x, h.y};
        }
    }
};

template <int BM_, int BN_, int WM_, int WN_, int STAGES_>
struct TileShape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, kStages = STAGES_;
    static constexpr int kThreads = 64 * WM * WN, kTm = BM / WM / 16, kTn = BN / WN / 16;
    static constexpr int kRowsBytes = BM * kStepBytes, kColsBytes = BN * kStepBytes, kStage = kRowsBytes + kColsBytes;
    static constexpr int kRowLoads = kRowsBytes / 16 / kThreads, kColLoads = kColsBytes / 16 / kThreads;  // a thread's
    static constexpr int kCopies = kRowLoads + kColLoads;
    static constexpr int kPerCu = 160 * 1024 / (kStages * kStage + 14 * 1024);  // workgroups, by their LDS
    static constexpr int kWaves = kPerCu * WM * WN / 4;                  // of a SIMD
    static_assert(kRowLoads * 16 * kThreads == kRowsBytes && kColLoads * 16 * kThreads == kColsBytes, "whole loads");
};

// Long sums in fp32: what kFoldSteps steps have added up goes into sums of its own, so that no chain of roundings is
// longer than 512 products and one for each 512 behind them (in one chain 8193 products of 0.9 were off by 7e-5 of their
// sum, 262144 by 2e-3).  The 16-bit types add 32 products at a time: up to 131072 of them their roundings of 2^-24
// stay below the result's own, 2^-12 or 2^-9.
constexpr int kFoldSteps = 16;

template <typename T, typename S>
struct Folded {
    static constexpr bool kUsed = T::kPer == 4;
    f32x4 sum[kUsed ? S::kTm : 1][kUsed ? S::kTn : 1];
    __device__ __forceinline__ Folded() {
        if constexpr (kUsed)
#pragma unroll
            for (int m = 0; m < S::kTm; ++m)
#pragma unroll
                for (int n = 0; n < S::kTn; ++n)
                    sum[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // Behind step s of a tile.
    __device__ __forceinline__ void fold(int s, f32x4 (&acc)[S::kTm][S::kTn]) {
        if constexpr (kUsed)
            if (s % kFoldSteps == kFoldSteps - 1) {
#pragma unroll
                for (int m = 0; m < S::kTm; ++m)
#pragma unroll
                    for (int n = 0; n < S::kTn; ++n) {
                        sum[m][n] += acc[m][n];
                        acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
                    }
            }
    }
    __device__ __forceinline__ void join(f32x4 (&acc)[S::kTm][S::kTn]) const {
        if constexpr (kUsed)
#pragma unroll
            for (int m = 0; m < S::kTm; ++m)
#pragma unroll
                for (int n = 0; n < S::kTn; ++n)
                    acc[m][n] += sum[m][n];
    }
};

// The step's part of a wave's results.
template <typename T, typename S, typename XS, typename WS>
__device__ __forceinline__ void multiply(const char* stage, const XS& xs, const WS& ws, f32x4 (&acc)[S::kTm][S::kTn]) {
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
        u32x4 xf[S::kTm], wf[S::kTn];
#pragma unroll
        for (int n = 0; n < S::kTn; ++n)
            wf[n] = ws.load(stage + S::kRowsBytes, n, kk);
#pragma unroll
        for (int m = 0; m < S::kTm; ++m)
            xf[m] = xs.load(stage, m, kk);
#pragma unroll
        for (int m = 0; m < S::kTm; ++m)
#pragma unroll
            for (int n = 0; n < S::kTn; ++n)
                acc[m][n] = mma<T>(wf[n], xf[m], acc[m][n]);
    }
}

// 16 bytes straight to LDS: lane l's land at base + 16 l.  Written as an instruction because the compiler holds
// every ds_read_tr behind all copies that it knows of (s_waitcnt vmcnt(0) before the step's first fragment: of the
// simplest kernel 16384 x 8 slots 1024 to 4096 bf16 took 1612 us, 1300 with this); wait_stage has the waits.
// There is no output register.  m0 is named as overwritten: the compiler sets it once for several instructions of its
// own that want the same value, and would not set it again behind this one.  (It warns that it does not keep a
// reserved register's value across the statement, which is what is wanted.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy_to_lds(const void* from, uint32_t base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(base), "v"(from) : "m0", "memory");
}

// 4 bytes, lane l's to base + 4 l.
__device__ __forceinline__ void copy_word_to_lds(const void* from, uint32_t base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(base), "v"(from) : "m0", "memory");
}
#pragma clang diagnostic pop

__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)ZO_LDS(const void, p); }

// Until at most LEFT of this wave's loads are under way, and all waves have come here: with 0 (or the loads of the
// later stages) left, a stage's copies have landed, and what was read from the stage to be filled next has been.
template <int LEFT>
__device__ __forceinline__ void wait_stage() {
    static_assert(LEFT < 64, "vmcnt has six bits");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((LEFT & 15) | (LEFT >> 4) << 14 | 7 << 4 | 0 << 8);  // vmcnt, no expcnt, lgkmcnt 0
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// The tiles that a workgroup takes, one after another, as one run of steps: the copies of a tile's first steps are
// under way before the tile before it has ended, and its results are stored while they land.
//   next_step()          prepares the copies of the run's next step; false: there is none.  What one call asks of
//                        LDS for a step kStages later is there: all waves have met since
//   copy(i, stage)       issues copy i of that step, into the stage at LDS address `stage`
//   tile_steps()         the steps of the next tile, below 0: none
//   finish(acc)          stores a tile's results
// A step is two halves of kTm groups of products, one of the rows' fragments with all of the columns'.  Fragments
// are read kLead groups before they are needed, so kLead groups before a step's end its stage is free for the
// copies of step s + kStages: there all waves meet, and step s + 1 has landed.  EARLY: copies of a stage that is
// free sooner, those of the columns' first half where its rows are places of the axis; they begin kLead groups
// before the half's end, and the columns' second half need not have landed before.  Copies 0 to EARLY - 1 are
// these, the last EARLY those of the second half. Without DMA a step's copies go to registers a step earlier, and
// put(stage) writes them to LDS where all waves have met.
//
// What bounds it, 16384 x 8 slots 1024 to 4096 bf16 (1137 to 1185 us from card to card, 967 to 928 TFLOP/s; batched
// library products of equal sizes 1086): the products with their fragments' reads alone 733 us, as fast as the library's
// 8192^3; the copies alone 547; both 985 to 1020, since LDS serves reads and copies by turns and a step's copies have a
// step's time to land; the stores the rest.  In steps taken, on one card: a workgroup a tile 1300; tiles in a run 1245;
// whole lines stored 1186; the early halves 1146.  Tried and left: steps of 64 bytes in four stages (half lines copied:
// 1315), lines touched ahead for L2 (1229), four waves of 128 by 128 (2830: one wave a SIMD), stores past the caches, a
// raised wave priority and groups of 4 or 16 row tiles (no difference).
template <typename T, typename S, bool DMA, int EARLY, typename XS, typename WS, typename NEXT, typename COPY, typename PUT,
          typename STEPS, typename FINISH>
__device__ __forceinline__ void multiply_tiles(char* tiles, uint32_t lds, const XS& xs, const WS& ws, NEXT next_step,
                                               COPY copy, PUT put, STEPS tile_steps, FINISH finish) {
    constexpr int kLead = S::kTm / 2, kGroups = 2 * S::kTm;
    static_assert(S::kTm % 2 == 0 && S::kTn % kLead == 0, "two halves, whole fragments a group");
    constexpr int kReads = S::kTn / kLead, kCopyRate = (S::kCopies - EARLY + kLead - 1) / kLead;
    constexpr int kEarlyRate = (EARLY + kLead - 1) / kLead;
    static_assert(DMA || (EARLY == 0 && S::kStages == 2));
    bool more = false;
#pragma unroll
    for (int s = 0; s < S::kStages; ++s) {
        more = next_step();
        if (more)
#pragma unroll
            for (int i = 0; i < S::kCopies; ++i)
                copy(i, lds + s * S::kStage);
        if (!DMA && more)
            put(tiles + s * S::kStage);
    }
    if (DMA && more)
        wait_stage<(S::kStages - 1) * S::kCopies + EARLY>();
    else
        wait_stage<0>();
    if constexpr (!DMA) {
        more = more && next_step();  // behind the wait: it may need what all waves brought in the first step
        if (more)
#pragma unroll
            for (int i = 0; i < S::kCopies; ++i)
                copy(i, 0);
    }
    u32x4 xf[S::kTm], wf[S::kTn], wn[S::kTn];
#pragma unroll
    for (int n = 0; n < S::kTn; ++n)
        wf[n] = ws.load(tiles + S::kRowsBytes, n, 0);
#pragma unroll
    for (int m = 0; m < kLead; ++m)
        xf[m] = xs.load(tiles, m, 0);
    int at = 0;  // the stage of the step
    for (int steps; (steps = tile_steps()) >= 0;) {
        f32x4 acc[S::kTm][S::kTn];
#pragma unroll
        for (int m = 0; m < S::kTm; ++m)
#pragma unroll
            for (int n = 0; n < S::kTn; ++n)
                acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        Folded<T, S> folded;
        for (int s = 0; s < steps; ++s) {
            const char* from = tiles + at * S::kStage;
            const uint32_t stage = lds + at * S::kStage;
#pragma unroll
            for (int q = 0; q < kGroups; ++q) {
                const int m = q % S::kTm, ahead = (q + kLead) % kGroups;
                // waits in the order of the loads: later ones that are under way can only make them longer
                if (EARLY > 0 && q == S::kTm - kLead) {
                    if (more)
                        wait_stage<(S::kStages - 1) * S::kCopies>();
                    else
                        wait_stage<0>();
                    more = more && next_step();
                }
                if (q == kGroups - kLead) {
                    if (DMA && more)
                        wait_stage<(S::kStages - 2) * S::kCopies + 2 * EARLY>();
                    else
                        wait_stage<0>();
                    if (!DMA && more)
                        put(tiles + at * S::kStage);
                    at = at + 1 == S::kStages ? 0 : at + 1;
                    from = tiles + at * S::kStage;
                    if (EARLY == 0)
                        more = more && next_step();
                }
                xf[ahead % S::kTm] = xs.load(from, ahead % S::kTm, ahead / S::kTm);
                if (m >= kLead) {
#pragma unroll
                    for (int i = 0; i < kReads; ++i)
                        wn[(m - kLead) * kReads + i] =
                            ws.load(from + S::kRowsBytes, (m - kLead) * kReads + i, ahead / S::kTm);
                    if (more) {
                        if (q < S::kTm) {
#pragma unroll
                            for (int i = (m - kLead) * kEarlyRate; i < (m - kLead + 1) * kEarlyRate && i < EARLY; ++i)
                                copy(i, stage);
                        } else {
#pragma unroll
                            for (int i = EARLY + (m - kLead) * kCopyRate;
                                 i < EARLY + (m - kLead + 1) * kCopyRate && i < S::kCopies; ++i)
                                copy(i, stage);
                        }
                    }
                }
#pragma unroll
                for (int n = 0; n < S::kTn; ++n)
                    acc[m][n] = mma<T>(wf[n], xf[m], acc[m][n]);
                __builtin_amdgcn_sched_barrier(0);
                if (m == S::kTm - 1)
#pragma unroll
                    for (int n = 0; n < S::kTn; ++n)
                        wf[n] = wn[n];
            }
            folded.fold(s, acc);
        }
        folded.join(acc);
        finish(acc);
    }
}

// Four neighbouring results of a row, of which those before column `cols` exist.
template <typename T>
__device__ __forceinline__ void store_results(typename T::elem* p, int col, int cols, const float* f) {
    if (col + 4 <= cols) {
        if constexpr (T::kPer == 4) {
            store_vec<T, false>(p + col, T::pack(f));
        } else {
            const float g[8] = {f[0], f[1], f[2], f[3], f[0], f[1], f[2], f[3]};
            const u32x4 v = T::pack(g);
            *reinterpret_cast<u32x2_e2*>(p + col) = u32x2{v.x, v.y};
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (col + j < cols)
                p[col + j] = T::of_f32(f[j]);
    }
}

// A lane's value of the lane eight away in its row of 16.
__device__ __forceinline__ uint32_t from_other_half(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xF, 0xF, true);  // row_ror:8
}

// A wave's results: out(m) is the row of its m-th (null: none), `first` its first column.  A lane has some columns
// of row l % 16.  Where 128 bytes of all rows exist they are stored as whole lines, eight lanes to a line: the
// lanes of rows r and r + 8 exchange halves of their lines (stored 32 bytes at a time the product above took 26 us
// more).
template <typename T, typename S, bool PAIRED, typename OUT>
__device__ __forceinline__ void store_tile(const f32x4 (&acc)[S::kTm][S::kTn], int first, int cols, int lane, OUT out) {
    const int g = lane >> 4;
    constexpr int kLine = T::kPer == 4 ? 2 : 4;  // fragments of a line
    if (S::kTn % kLine == 0 && first + 16 * S::kTn <= cols) {
        const bool high = lane & 8;
        // a lane's two chunks of 16 bytes of a line, in bytes from its start
        const int at0 = T::kPer == 4 ? (PAIRED ? 32 * g : 16 * g) : PAIRED ? 16 * g : 32 * (g & 1) + 16 * (g >> 1);
        const int at1 = at0 + (T::kPer == 4 && PAIRED ? 16 : 64);
        const int at = (high ? at1 : at0) / (int)sizeof(typename T::elem) + first;
#pragma unroll
        for (int m = 0; m < S::kTm; ++m) {
            typename T::elem* const p0 = out(16 * m + (lane & 7));
            typename T::elem* const p1 = out(16 * m + (lane & 7) + 8);
#pragma unroll
            for (int n = 0; n < S::kTn; n += kLine) {
                u32x4 c0, c1;
                if constexpr (T::kPer == 4) {
                    c0 = __builtin_bit_cast(u32x4, acc[m][n]);
                    c1 = __builtin_bit_cast(u32x4, acc[m][n + 1]);
                } else {
                    const float f[16] = {
                        acc[m][n].x,     acc[m][n].y,     acc[m][n].z,     acc[m][n].w,
                        acc[m][n + 1].x, acc[m][n + 1].y, acc[m][n + 1].z, acc[m][n + 1].w,
                        acc[m][n + 2].x, acc[m][n + 2].y, acc[m][n + 2].z, acc[m][n + 2].w,
                        acc[m][n + 3].x, acc[m][n + 3].y, acc[m][n + 3].z, acc[m][n + 3].w,
                    };
                    c0 = T::pack(f);
                    c1 = T::pack(f + 8);
                    if constexpr (!PAIRED) {  // four columns of two fragments each become eight of one
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const auto r0 = __builtin_amdgcn_permlane16_swap(c0[i], c0[i + 2], false, false);
                            const auto r1 = __builtin_amdgcn_permlane16_swap(c1[i], c1[i + 2], false, false);
                            c0[i] = r0[0];
                            c0[i + 2] = r0[1];
                            c1[i] = r1[0];
                            c1[i + 2] = r1[1];
                        }
                    }
                }
                u32x4 low, up;  // of rows l % 8 and l % 8 + 8
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t other = from_other_half(high ? c0[i] : c1[i]);
                    low[i] = high ? other : c0[i];
                    up[i] = high ? c1[i] : other;
                }
                const int col = at + 16 * n;
                if (p0)
                    store_vec<T, false>(p0 + col, low);
                if (p1)
                    store_vec<T, false>(p1 + col, up);
            }
        }
        return;
    }
#pragma unroll
    for (int m = 0; m < S::kTm; ++m) {
        typename T::elem* const p = out(16 * m + (lane & 15));
        if (!p)
            continue;
#pragma unroll
        for (int n = 0; n < S::kTn; ++n) {
            const float f[4] = {acc[m][n].x, acc[m][n].y, acc[m][n].z, acc[m][n].w};
            store_results<T>(p, first + (PAIRED ? 32 * (n / 2) + 8 * g + 4 * (n % 2) : 16 * n + 4 * g), cols, f);
        }
    }
}

// ---------------------------------------------------------------------------
// Which tiles a workgroup takes.  The host knows no expert's number of rows, so every workgroup adds up the
// experts' tiles first; where there are more workgroups than tiles, those past the last have nothing to do.
// Workgroups go to the eight dies in turn, so that numbering gives each die a run of the tiles: eight rows' tiles
// by all columns' tiles, whose operands its L2 then serves.
// ---------------------------------------------------------------------------
struct TilePlace {
    int expert;
    int first, end;    // rows of the experts' order
    int col_tile;
};

struct TileTable {
    uint32_t upto[ZERO_ROUTE_MAX_EXPERTS];  // row tiles, or parts, of the experts up to this one
    int32_t begin[ZERO_ROUTE_MAX_EXPERTS + 1];  // their first rows; never falling
};

// tiles(rows), and cost(rows) into `costs` (may be null), are added up.
template <typename TILES, typename COST>
__device__ __forceinline__ void fill_tile_table(TileTable& table, uint32_t* costs, const ExpertCall& a, TILES tiles, COST cost) {
    const int lane = threadIdx.x & 63, slots = (int)a.slots;
    auto row = [&](int e) {
        const int o = a.offsets[e];
        return o < 0 ? 0 : o > slots ? slots : o;
    };
    if (threadIdx.x < 64) {
        int begin = row(0);
        uint32_t before = 0, spent = 0;
        if (lane == 0)
            table.begin[0] = begin;
        for (int e0 = 0; e0 < a.experts; e0 += 64) {
            const int e = e0 + lane;
            int end = e < a.experts ? row(e + 1) : 0;
            end = end < begin ? begin : end;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int o = __shfl_up(end, d);
                end = lane >= d && o > end ? o : end;
            }
            const int previous = __shfl_up(end, 1), rows = end - (lane ? previous : begin);
            uint32_t n = e < a.experts ? tiles(rows) : 0, c = e < a.experts && costs ? cost(rows) : 0;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const uint32_t o = __shfl_up(n, d), q = __shfl_up(c, d);
                n += lane >= d ? o : 0;
                c += lane >= d ? q : 0;
            }
            if (e < a.experts) {
                table.begin[e + 1] = end;
                table.upto[e] = before + n;
                if (costs)
                    costs[e] = spent + c;
            }
            begin = __shfl(end, 63);
            before += __shfl(n, 63);
            spent += __shfl(c, 63);
        }
    }
    __syncthreads();
}

__device__ __forceinline__ uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }

// Tile `id` of rows by cols: row tiles in groups of eight by all columns' tiles, whose operands a die's L2 serves.
__device__ __forceinline__ void grouped_tile(uint32_t id, uint32_t rows, uint32_t cols, uint32_t& row, uint32_t& col) {
    constexpr uint32_t kGroup = 8;
    const uint32_t per = kGroup * cols, group = id / per, rest = id - group * per;
    const uint32_t rows_in = rows - group * kGroup < kGroup ? rows - group * kGroup : kGroup;
    col = rest / rows_in;
    row = group * kGroup + rest - col * rows_in;
}

// The first expert whose entry of a rising table is above `value`.
__device__ __forceinline__ int expert_above(const uint32_t* upto, int experts, uint32_t value) {
    const int lane = threadIdx.x & 63;
    for (int e0 = 0; e0 < experts; e0 += 64) {
        const int e = e0 + lane;
        const uint64_t found = __ballot(e < experts && upto[e < experts ? e : 0] > value);
        if (found)
            return e0 + __ffsll((unsigned long long)found) - 1;
    }
    return experts - 1;
}

__device__ __forceinline__ uint32_t die_order(uint32_t id, uint32_t count) {
    const uint32_t each = (count + 7) / 8;
    const uint32_t t = (id & 7) * each + (id >> 3);
    return (id >> 3) < each ? t : count;
}

template <int BM>
__device__ __forceinline__ TilePlace tile_place(const TileTable& table, int experts, uint32_t row_tiles, uint32_t col_tiles,
                                                uint32_t id) {
    uint32_t row_tile, col_tile;
    grouped_tile(id, row_tiles, col_tiles, row_tile, col_tile);
    TilePlace out;
    out.expert = expert_above(table.upto, experts, row_tile);
    const uint32_t before = out.expert > 0 ? uniform(table.upto[out.expert - 1]) : 0;
    out.first = uniform(table.begin[out.expert]) + (row_tile - before) * BM;
    out.end = uniform(table.begin[out.expert + 1]);
    out.col_tile = (int)col_tile;
    return out;
}

// ---------------------------------------------------------------------------
// y = x * weight, a workgroup a tile, for experts of few rows: every weight is read once, and the loads that a compute
// unit has under way bound it: three of four stages.  48 slots of 64 experts 4096 to 1024 bf16, one set of weights again
// and again: 36 to 42 us where they meet up to 32 experts, 256 tiles; 52 to 65 from 33 on, where some compute units have
// two; sets in turn 49 to 58.  Two slots of 8 experts 14336 to 4096, 64 tiles: 88 us, 2.7 TB/s; one of 4096 to 14336, 112
// tiles: 21 us, 5.5.
// ALONG: the weights lie [out, in].  DMA: every row of x and of the weights is made of aligned chunks of 16 bytes, which
// go straight to LDS; else they pass through the registers, where their ends are seen to, one step ahead (512 slots of 64
// experts 4096 to 1024 bf16: 100 us, 128 where rows are 2 bytes off a word; 64 of 8, 4095 to 1023 fp32: 368, aligned 87).
// ---------------------------------------------------------------------------
// (Two waves a SIMD are asked for in fp32 so that the sums stay in registers that additions take too: kept in the
// accumulation registers they went back and forth every step, 64 slots of 8 experts 4096 to 1024: 95 us and 87.)
template <typename T, typename S, bool ALONG, bool DMA>
__global__ __launch_bounds__(S::kThreads, T::kPer == 4 ? 2 : 1) void k_expert_product(const ExpertCall a, uint32_t first, uint32_t launched) {
    using elem = typename T::elem;
    constexpr int kPer = T::kPer, kStep = kStepBytes / (int)sizeof(elem);
    constexpr int kXChunks = kStepBytes / 16, kChunks = ALONG ? kXChunks : S::BN / kPer;  // of the tiles' rows
    constexpr int kXRows = S::kThreads / kXChunks, kWRows = S::kThreads / kChunks;  // tile rows of one load of all threads
    constexpr int kStages = DMA ? S::kStages : 2;
    __shared__ __attribute__((aligned(1024))) char tiles[kStages * S::kStage];

    static_assert(sizeof(TileTable) <= sizeof(tiles), "the table lies where the tiles will");
    TileTable& table = *reinterpret_cast<TileTable*>(tiles);
    fill_tile_table(table, nullptr, a, [](int rows) { return ((uint32_t)rows + S::BM - 1) / S::BM; }, [](int) { return 0u; });
    const uint32_t col_tiles = ((uint32_t)a.cols_out + S::BN - 1) / S::BN;
    const uint32_t row_tiles = uniform(table.upto[a.experts - 1]), all = row_tiles * col_tiles;
    if (first >= all)
        return;
    const uint32_t here = all - first < launched ? all - first : launched, in_run = die_order(blockIdx.x, here);
    if (in_run >= here)
        return;
    const TilePlace place = tile_place<S::BM>(table, a.experts, row_tiles, col_tiles, first + in_run);
    __syncthreads();
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int n0 = place.col_tile * S::BN, depth = a.cols_in, steps = (depth + kStep - 1) / kStep;
    const elem* const x = static_cast<const elem*>(a.x);
    const elem* const w = static_cast<const elem*>(a.w) +
                          (int64_t)place.expert * (ALONG ? a.cols_out : a.cols_in) * a.ld_w;
    const elem* const zeros = reinterpret_cast<const elem*>(&zero_chunk);

    // what this thread loads: chunk `xc` of its rows of x, `wc` of its rows of the weights
    const elem* px[S::kRowLoads];
    const elem* pw[S::kColLoads];
    int wc[S::kColLoads];
    const int xr = t / kXChunks, xc = ((t % kXChunks) ^ along_exchange<false>(xr)) * kPer;
#pragma unroll
    for (int j = 0; j < S::kRowLoads; ++j) {  // rows past the run's are not stored
        const uint32_t i = (uint32_t)place.first + xr + j * kXRows;  // may pass 2^31
        const int64_t row = row_at(a.order, a.x_map, a.slots, i < (uint32_t)place.end ? i : place.end - 1);
        px[j] = x + (row < 0 ? 0 : row) * a.ld_x;  // none: stored as zeros
        if constexpr (DMA)
            px[j] += xc;
    }
#pragma unroll
    for (int j = 0; j < S::kColLoads; ++j) {
        const int r = t / kChunks + j * kWRows;
        if constexpr (ALONG) {
            wc[j] = ((t % kXChunks) ^ along_exchange<true>(r)) * kPer;
            const int n = n0 + r < a.cols_out ? n0 + r : a.cols_out - 1;  // columns past the last are not stored
            pw[j] = w + n * a.ld_w;
            if constexpr (DMA)
                pw[j] += wc[j];
        } else {
            wc[j] = n0 + ((t % kChunks) ^ across_exchange<T, kChunks>(r)) * kPer;
            pw[j] = w + r * a.ld_w;
            if constexpr (DMA)
                pw[j] += wc[j] < a.cols_out ? wc[j] : a.cols_out - kPer;
        }
    }
    const int64_t w_step = ALONG ? 1 : a.ld_w;  // elements of the weights for a place of the axis
    const uint32_t lds = lds_address(tiles) + wave * 1024;
    u32x4 rx[DMA ? 1 : S::kRowLoads], rw[DMA ? 1 : S::kColLoads];

    // WHOLE: the step lies before the end of the axis
    auto copy = [&](int step, auto whole) __attribute__((always_inline)) {
        constexpr bool WHOLE = decltype(whole)::value;
        const int k0 = step * kStep;
        const uint32_t stage = lds + step % kStages * S::kStage;
#pragma unroll
        for (int j = 0; j < S::kRowLoads; ++j)
            copy_to_lds(WHOLE || k0 + xc < depth ? px[j] + k0 : zeros, stage + j * S::kThreads * 16);
#pragma unroll
        for (int j = 0; j < S::kColLoads; ++j) {
            const int place_of = ALONG ? wc[j] : t / kChunks + j * kWRows;
            copy_to_lds(WHOLE || k0 + place_of < depth ? pw[j] + k0 * w_step : zeros,
                        stage + S::kRowsBytes + j * S::kThreads * 16);
        }
    };
    auto fetch = [&](int step) __attribute__((always_inline)) {
        const int k0 = step * kStep;
        if constexpr (DMA) {
            if (k0 + kStep <= depth)
                copy(step, std::true_type());
            else
                copy(step, std::false_type());
        } else {
#pragma unroll
            for (int j = 0; j < S::kRowLoads; ++j)
                rx[j] = load_row<T>(px[j], k0 + xc, depth, 0);
#pragma unroll
            for (int j = 0; j < S::kColLoads; ++j) {
                if constexpr (ALONG) {
                    rw[j] = load_row<T>(pw[j], k0 + wc[j], depth, 0);
                } else {
                    rw[j] = u32x4{0, 0, 0, 0};
                    if (k0 + t / kChunks + j * kWRows < depth)
                        rw[j] = load_row<T>(pw[j] + k0 * w_step, wc[j], a.cols_out, 0);
                }
            }
        }
    };
    auto put = [&](int step) __attribute__((always_inline)) {
        if constexpr (!DMA) {
            char* const stage = tiles + step % kStages * S::kStage + t * 16;
#pragma unroll
            for (int j = 0; j < S::kRowLoads; ++j)
                *reinterpret_cast<u32x4*>(stage + j * S::kThreads * 16) = rx[j];
#pragma unroll
            for (int j = 0; j < S::kColLoads; ++j)
                *reinterpret_cast<u32x4*>(stage + S::kRowsBytes + j * S::kThreads * 16) = rw[j];
        }
    };

    const int wm = wave % S::WM, wn = wave / S::WM;
    const Side<T, true, false, S::BM, S::kTm> xs(wm * S::kTm * 16, lane);
    const Side<T, ALONG, ALONG, S::BN, S::kTn> ws(wn * S::kTn * 16, lane);
    f32x4 acc[S::kTm][S::kTn];
#pragma unroll
    for (int m = 0; m < S::kTm; ++m)
#pragma unroll
        for (int n = 0; n < S::kTn; ++n)
            acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};

    Folded<T, S> folded;
    constexpr int kAhead = kStages - 1;  // stages under way
#pragma unroll
    for (int s = 0; s < kAhead; ++s)
        if (s < steps) {
            fetch(s);
            put(s);
        }
    for (int s = 0; s < steps; ++s) {
        // the last steps have nothing behind them, so their loads are the last
        if (kAhead > 1 && s + kAhead <= steps)
            wait_stage<(kAhead - 1) * (S::kRowLoads + S::kColLoads)>();
        else
            wait_stage<0>();
        if (s + kAhead < steps)
            fetch(s + kAhead);
        multiply<T, S>(tiles + s % kStages * S::kStage, xs, ws, acc);
        folded.fold(s, acc);
        if (s + kAhead < steps)
            put(s + kAhead);
    }
    folded.join(acc);

    if (a.x_map.mode && !a.out_map.mode) {  // rows without a slot; in the slots' order they are not stored
#pragma unroll
        for (int m = 0; m < S::kTm; ++m) {
            const uint32_t i = (uint32_t)place.first + (wm * S::kTm + m) * 16 + (lane & 15);
            if (row_at(a.order, a.x_map, a.slots, i < (uint32_t)place.end ? i : place.end - 1) < 0)
#pragma unroll
                for (int n = 0; n < S::kTn; ++n)
                    acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    elem* const y = static_cast<elem*>(a.out);
    store_tile<T, S, ALONG>(acc, n0 + wn * S::kTn * 16, a.cols_out, lane, [&](int m) -> elem* {
        const uint32_t i = (uint32_t)place.first + wm * S::kTm * 16 + m;
        if (i >= (uint32_t)place.end)
            return nullptr;
        const int64_t row = row_at(a.order, a.out_map, a.slots, i);
        return row < 0 ? nullptr : y + row * a.ld_out;
    });
}

// ---------------------------------------------------------------------------
// The same in a run of tiles for each workgroup.  Rows of any alignment pass through registers (131072 slots 1024
// to 4096 bf16: 1135 us aligned, 1832 where rows are 4 bytes off a line, 2939 where they are 2 off, whose loads the memory
// pipeline takes apart; read as whole words and shifted 2580 and 2059, where these were 1795 and 2833, left).
// ---------------------------------------------------------------------------
template <typename T, typename S, bool ALONG, bool DMA>
__global__ __launch_bounds__(S::kThreads, S::kWaves) void k_expert_product_run(const ExpertCall a) {
    using elem = typename T::elem;
    constexpr int kPer = T::kPer, kStep = kStepBytes / (int)sizeof(elem);
    constexpr int kXChunks = kStepBytes / 16, kChunks = ALONG ? kXChunks : S::BN / kPer;  // of the tiles' rows
    constexpr int kXRows = S::kThreads / kXChunks, kWRows = S::kThreads / kChunks;  // tile rows of one load of all threads
    // Tiles whose entries of order are held: copies run up to kStages tiles ahead of the products (where a tile
    // has one step; through registers one tile more), the entries kStages tiles ahead of the copies.
    constexpr int kRing = S::kStages <= 3 ? 8 : 16;
    static_assert(kRing > 2 * S::kStages + (DMA ? 0 : 1) && S::BM % 64 == 0);
    __shared__ __attribute__((aligned(1024))) char tiles[S::kStages * S::kStage];
    __shared__ int32_t slots_of[kRing][S::BM];
    __shared__ TileTable table;

    fill_tile_table(table, nullptr, a, [](int rows) { return ((uint32_t)rows + S::BM - 1) / S::BM; }, [](int) { return 0u; });
    const uint32_t col_tiles = ((uint32_t)a.cols_out + S::BN - 1) / S::BN;
    const uint32_t row_tiles = uniform(table.upto[a.experts - 1]), all = row_tiles * col_tiles;
    // a die's workgroups take a run of the tiles in turn
    const uint32_t each = (all + 7) / 8, stride = gridDim.x / 8, die = blockIdx.x & 7;
    const uint32_t first = die * each + blockIdx.x / 8, last = (die + 1) * each < all ? (die + 1) * each : all;
    if (first >= last)
        return;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int depth = a.cols_in, steps = (depth + kStep - 1) / kStep;
    const elem* const zeros = reinterpret_cast<const elem*>(&zero_chunk);
    const bool ordered = a.x_map.mode | a.out_map.mode;
    auto place_of = [&](uint32_t id) { return tile_place<S::BM>(table, a.experts, row_tiles, col_tiles, id); };

    // The entries of order of a tile; each wave copies 64 of them.
    auto look_up = [&](uint32_t id, int ring) __attribute__((always_inline)) {
        if (ordered && id < last) {
            const TilePlace p = place_of(id);
            const int r = wave % (S::BM / 64) * 64;
            const uint32_t i = (uint32_t)p.first + r + lane;  // may pass 2^31
            copy_word_to_lds(a.order + (i < (uint32_t)p.end ? i : p.end - 1), lds_address(&slots_of[ring][r]));
        }
    };
    // The row of a matrix of row r of a tile whose entries of order lie in `ring`, -1: none
    auto row_of = [&](const SlotMap& map, const TilePlace& p, int ring, int r) __attribute__((always_inline)) -> int64_t {
        const uint32_t i = (uint32_t)p.first + r;
        if (map.mode == 0)
            return i < (uint32_t)p.end ? i : p.end - 1;
        const uint32_t slot = (uint32_t)slots_of[ring][r];
        return slot < (uint64_t)a.slots ? map.row(slot) : -1;
    };

    // the tile whose copies are issued, and the step of it
    uint32_t copy_id = first;
    int copy_step = 0, copy_ring = 0;
    const elem* px[S::kRowLoads];
    const int xr = t / kXChunks, xc = ((t % kXChunks) ^ along_exchange<false>(xr)) * kPer;
    // the exchange looks at four bits of the row, so a thread's rows of the weights' tile have one chunk, or two
    // in turn
    constexpr int kColumns = ALONG || kWRows % 16 == 0 ? 1 : 2;
    static_assert(kWRows * kColumns % 16 == 0);
    int wc[kColumns];  // across: the columns
    const int wr = t / kChunks, wk = ALONG ? ((t % kChunks) ^ along_exchange<true>(wr)) * kPer : wr;
    const elem* pw = nullptr;
    int w_room = 0;  // ALONG: the weights' rows behind the first
    int k0 = 0;
    auto next_step = [&]() __attribute__((always_inline)) -> bool {
        if (copy_step == steps) {
            copy_step = 0;
            copy_id += stride;
            copy_ring = (copy_ring + 1) % kRing;
        }
        if (copy_id >= last)
            return false;
        if (copy_step == 0) {
            const TilePlace p = place_of(copy_id);
            const int n0 = p.col_tile * S::BN;
            const elem* const w = static_cast<const elem*>(a.w) +
                                  (int64_t)p.expert * (ALONG ? a.cols_out : a.cols_in) * a.ld_w;
#pragma unroll
            for (int j = 0; j < S::kRowLoads; ++j) {  // rows past the run's are not stored
                const int64_t row = row_of(a.x_map, p, copy_ring, xr + j * kXRows);
                px[j] = static_cast<const elem*>(a.x) + (row < 0 ? 0 : row) * a.ld_x + (DMA ? xc : 0);  // none: stored as zeros
            }
            if constexpr (ALONG) {  // columns past the last are not stored
                const int n = n0 + wr < a.cols_out ? n0 + wr : a.cols_out - 1;
                pw = w + n * a.ld_w + (DMA ? wk : 0);
                w_room = a.cols_out - 1 - n;
            } else {
                pw = w + wr * a.ld_w;
#pragma unroll
                for (int j = 0; j < kColumns; ++j) {
                    const int c = n0 + ((t % kChunks) ^ across_exchange<T, kChunks>(wr + j * kWRows)) * kPer;
                    wc[j] = !DMA || c < a.cols_out ? c : a.cols_out - kPer;
                }
                if constexpr (DMA && kColumns == 1)
                    pw += wc[0];
            }
            look_up(copy_id + S::kStages * stride, (copy_ring + S::kStages) % kRing);
        }
        k0 = copy_step * kStep;
        ++copy_step;
        return true;
    };
    // the first half of the weights' copies, x's, the others; across a half is half of the places
    constexpr int kEarly = ALONG || !DMA ? 0 : S::kColLoads / 2;
    u32x4 held[DMA ? 1 : S::kCopies];
    auto copy = [&](int i, uint32_t stage) __attribute__((always_inline)) {
        if (i >= kEarly && i < kEarly + S::kRowLoads) {
            i -= kEarly;
            if constexpr (!DMA)
                held[i] = load_row<T>(px[i], k0 + xc, depth, 0);
            else
                copy_to_lds(k0 + xc < depth ? px[i] + k0 : zeros, stage + i * S::kThreads * 16);
        } else {
            const int j = i < kEarly ? i : i - S::kRowLoads;
            const elem* from = pw;
            if constexpr (ALONG)
                from += (w_room < j * kWRows ? w_room : j * kWRows) * a.ld_w + (DMA ? k0 : 0);
            else
                from += (k0 + j * kWRows) * a.ld_w + (DMA && kColumns > 1 ? wc[j % kColumns] : 0);
            if constexpr (!DMA && ALONG)
                held[i] = load_row<T>(from, k0 + wk, depth, 0);
            else if constexpr (!DMA)
                held[i] = load_row<T>(from, wc[j % kColumns], k0 + j * kWRows + wk < depth ? a.cols_out : 0, 0);
            else
                copy_to_lds(k0 + (ALONG ? 0 : j * kWRows) + wk < depth ? from : zeros, stage + S::kRowsBytes + j * S::kThreads * 16);
        }
    };

    auto put = [&](char* stage) __attribute__((always_inline)) {
        if constexpr (!DMA)
#pragma unroll
            for (int i = 0; i < S::kCopies; ++i)
                *reinterpret_cast<u32x4*>(stage + (i * S::kThreads + t) * 16) = held[i];
    };
    uint32_t id = first;
    int ring = 0;
    bool begun = false;
    auto tile_steps = [&]() __attribute__((always_inline)) -> int {
        if (begun) {
            id += stride;
            ring = (ring + 1) % kRing;
        }
        begun = true;
        return id < last ? steps : -1;
    };
    const int wm = wave % S::WM, wn = wave / S::WM;
    const Side<T, true, false, S::BM, S::kTm> xs(wm * S::kTm * 16, lane);
    const Side<T, ALONG, ALONG, S::BN, S::kTn> ws(wn * S::kTn * 16, lane);
    auto finish = [&](f32x4 (&acc)[S::kTm][S::kTn]) __attribute__((always_inline)) {
        const TilePlace p = place_of(id);
        if (a.x_map.mode && !a.out_map.mode) {  // rows without a slot; in the slots' order they are not stored
#pragma unroll
            for (int m = 0; m < S::kTm; ++m)
                if (row_of(a.x_map, p, ring, (wm * S::kTm + m) * 16 + (lane & 15)) < 0)
#pragma unroll
                    for (int n = 0; n < S::kTn; ++n)
                        acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        elem* const y = static_cast<elem*>(a.out);
        store_tile<T, S, ALONG>(acc, p.col_tile * S::BN + wn * S::kTn * 16, a.cols_out, lane, [&](int m) -> elem* {
            const int r = wm * S::kTm * 16 + m;
            if ((uint32_t)p.first + r >= (uint32_t)p.end)
                return nullptr;
            const int64_t row = row_of(a.out_map, p, ring, r);
            return row < 0 ? nullptr : y + row * a.ld_out;
        });
    };
    if (ordered) {
        for (int i = 0; i < S::kStages; ++i)
            look_up(first + i * stride, i);
        wait_stage<0>();
    }
    multiply_tiles<T, S, DMA, kEarly>(tiles, lds_address(tiles) + wave * 1024, xs, ws, next_step, copy, put,
                                                    tile_steps, finish);
}

// ---------------------------------------------------------------------------
// dweight = x^T * dy, a tile of one expert's matrix for a workgroup.  An expert's rows are cut into parts of
// `part` rows; where they are more than one, each leaves its sums in the workspace and k_expert_join adds them up.
// ---------------------------------------------------------------------------
struct PartPlace {
    int expert;
    int begin, end;  // rows of the experts' order
    uint32_t sums;   // which of the workspace's matrices it leaves its sums in
    bool only;       // of its expert: it has the results themselves
};

__device__ __forceinline__ uint32_t parts_of(uint32_t rows, int part) {
    return part == 0 || rows <= (uint32_t)part ? 1 : (rows + part - 1) / part;
}

__device__ __forceinline__ PartPlace part_place(const TileTable& table, const ExpertCall& a, uint32_t id) {
    PartPlace p;
    p.expert = expert_above(table.upto, a.experts, id);
    const uint32_t nth = id - (p.expert > 0 ? uniform(table.upto[p.expert - 1]) : 0);
    const int begin = uniform(table.begin[p.expert]), end = uniform(table.begin[p.expert + 1]);
    const uint32_t all = parts_of(end - begin, a.part);
    p.begin = begin + (int)nth * a.part;
    p.end = nth + 1 == all ? end : p.begin + a.part;
    p.sums = id;
    p.only = all == 1;
    return p;
}

// Where the results of a tile from (row, col) go.
template <typename T, typename S>
__device__ __forceinline__ void store_sums(const ExpertCall& a, const PartPlace& p, const f32x4 (&acc)[S::kTm][S::kTn], int row0,
                                           int col, int lane) {
    if (p.only) {
        typename T::elem* const to = static_cast<typename T::elem*>(a.out) + (int64_t)p.expert * a.cols_in * a.ld_out;
        store_tile<T, S, false>(acc, col, a.cols_out, lane, [&](int i) -> typename T::elem* {
            return row0 + i < a.cols_in ? to + (row0 + i) * a.ld_out : nullptr;
        });
    } else {
        float* const to = a.partial + (int64_t)p.sums * a.cols_in * a.cols_out;
        store_tile<F32, S, false>(acc, col, a.cols_out, lane, [&](int i) -> float* {
            return row0 + i < a.cols_in ? to + (int64_t)(row0 + i) * a.cols_out : nullptr;
        });
    }
}

// DMA: rows of x and dy are made of aligned chunks, which go straight to LDS.  Both halves of both operands'
// copies are early ones.  Bound as the product is (16384 x 8 slots 4096 by 1024 bf16 1245 to 1297 us from card to card, 883
// to 848 TFLOP/s): the products alone 773 us, the copies alone 798; all fragments are read transposed, which takes twice
// the LDS cycles.  Experts' loads differ, so the dies take equal shares of the steps, not of the tiles.
template <typename T, typename S, bool DMA>
__global__ __launch_bounds__(S::kThreads, S::kWaves) void k_expert_weight_back(const ExpertCall a) {
    using elem = typename T::elem;
    static_assert(S::BM == S::BN, "a thread's rows of x and dy are the same slots");
    constexpr int kPer = T::kPer, kStep = kStepBytes / (int)sizeof(elem);
    constexpr int kChunks = S::BN / kPer, kRows = S::kThreads / kChunks, kLoads = S::kColLoads;
    constexpr int kColumns = kRows % 16 == 0 ? 1 : 2;  // the exchange looks at four bits of the row
    static_assert(kRows * kColumns % 16 == 0 && kLoads % (2 * kColumns) == 0 && kStep <= 64);
    constexpr int kRing = 8;  // steps whose entries of order are held
    static_assert(S::kStages == 2, "entries of order come two steps before the copies");
    __shared__ __attribute__((aligned(1024))) char tiles[S::kStages * S::kStage];
    __shared__ int32_t slots_of[kRing][64];
    __shared__ TileTable table;

    __shared__ uint32_t costs[ZERO_ROUTE_MAX_EXPERTS];
    // Of a part's beginning and end, in steps (16384 slots of four of 64 experts, 1024 by 256 bf16: 139 us, 163 with 0 and
    // 136 with 16; 4096 of 8, 1600 by 6400 f16: 144, 154 and 144).
    constexpr uint32_t kTileCost = 4;
    fill_tile_table(table, costs, a, [&](int rows) { return parts_of(rows, a.part); },
                    [&](int rows) { return ((uint32_t)rows + kStep - 1) / kStep + kTileCost * parts_of(rows, a.part); });
    const uint32_t m_tiles = ((uint32_t)a.cols_in + S::BM - 1) / S::BM, n_tiles = ((uint32_t)a.cols_out + S::BN - 1) / S::BN;
    const uint32_t of_part = m_tiles * n_tiles, all = uniform(table.upto[a.experts - 1]) * of_part;
    // A die's workgroups take a run of the tiles in turn, an eighth of the steps.
    const uint32_t total = uniform(costs[a.experts - 1]);
    auto die_begin = [&](uint32_t die) -> uint32_t {
        if (die == 8)
            return all;
        const uint32_t at = (uint32_t)((uint64_t)total * die / 8);
        const int e = expert_above(costs, a.experts, at);
        const uint32_t before = e > 0 ? uniform(costs[e - 1]) : 0, own = uniform(costs[e]) - before;
        const uint32_t part = e > 0 ? uniform(table.upto[e - 1]) : 0, parts = uniform(table.upto[e]) - part;
        return part * of_part + (uint32_t)((uint64_t)(at - before) * (parts * of_part) / own);
    };
    const uint32_t stride = gridDim.x / 8, die = blockIdx.x & 7;
    const uint32_t first = die_begin(die) + blockIdx.x / 8, last = die_begin(die + 1);
    if (first >= last)
        return;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const uint32_t slots = (uint32_t)a.slots;
    const elem* const zeros = reinterpret_cast<const elem*>(&zero_chunk);
    const bool ordered = a.x_map.mode | a.out_map.mode;

    // The steps of the tiles in turn.
    struct Cursor {
        uint32_t id;
        int step, steps;
        PartPlace place;
    };
    auto steps_of = [&](const PartPlace& p) __attribute__((always_inline)) -> int {
        return (int)(((uint32_t)(p.end - p.begin) + kStep - 1) / kStep);
    };
    auto settle = [&](Cursor& c) __attribute__((always_inline)) {  // past tiles without steps
        while (c.id < last) {
            c.place = part_place(table, a, c.id / of_part);
            c.steps = steps_of(c.place);
            if (c.steps > 0)
                return;
            c.id += stride;
        }
    };
    auto advance = [&](Cursor& c) __attribute__((always_inline)) {
        if (++c.step == c.steps) {
            c.step = 0;
            c.id += stride;
            settle(c);
        }
    };

    // The entries of order come to LDS before the copies that need them.  (Loaded into registers they would have
    // to be waited for, and with them, in the order of the loads, all copies issued before.)
    Cursor look{first, 0, 0, {}};
    settle(look);
    int look_ring = 0;
    auto look_up = [&](int by) __attribute__((always_inline)) {  // by wave `by`, or all
        if (!ordered || look.id >= last)
            return;
        const uint32_t i = (uint32_t)look.place.begin + (uint32_t)look.step * kStep + lane;  // may pass 2^31
        if (by < 0 || by == wave)
            copy_word_to_lds(a.order + (i < (uint32_t)look.place.end ? i : look.place.end - 1), lds_address(slots_of[look_ring]));
        look_ring = (look_ring + 1) % kRing;
        advance(look);
    };
    for (int i = 0; i < 2 * S::kStages; ++i)
        look_up(-1);
    wait_stage<0>();

    Cursor from{first, 0, 0, {}};
    settle(from);
    int ring = 0, turn = 0;
    const elem *x = nullptr, *dy = nullptr;
    const int cr = t / kChunks;
    int xc[kColumns], wc[kColumns];  // columns of this thread's chunks; without DMA, in the tile
    int x_col = 0, dy_col = 0;       // the tile's first ones
    int rows_left = 0;
    uint32_t base = 0;
    uint32_t slot[kLoads];
    uint32_t tile_now = ~0u;
    auto next_step = [&]() __attribute__((always_inline)) -> bool {
        if (from.id >= last)
            return false;
        if (from.id != tile_now) {
            tile_now = from.id;
            uint32_t m, n;
            grouped_tile(from.id % of_part, m_tiles, n_tiles, m, n);
#pragma unroll
            for (int j = 0; j < kColumns; ++j) {  // rows and columns past the last are not stored
                const int c = ((t % kChunks) ^ across_exchange<T, kChunks>(cr + j * kRows)) * kPer;
                if constexpr (DMA) {
                    const int xi = (int)m * S::BM + c, wi = (int)n * S::BN + c;
                    xc[j] = xi < a.cols_in ? xi : a.cols_in - kPer;
                    wc[j] = wi < a.cols_out ? wi : a.cols_out - kPer;
                } else {  // the same registers for both
                    xc[j] = wc[j] = c;
                }
            }
            if constexpr (!DMA) {
                x_col = (int)m * S::BM;
                dy_col = (int)n * S::BN;
            }
        }
        x = static_cast<const elem*>(a.x);
        dy = static_cast<const elem*>(a.w);
        base = (uint32_t)from.place.begin + (uint32_t)from.step * kStep;
        rows_left = (int)((uint32_t)from.place.end - base);
        if (ordered) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j)
                slot[j] = (uint32_t)slots_of[ring][cr + j * kRows];
            ring = (ring + 1) % kRing;
        }
        look_up(turn);
        turn = turn + 1 == S::kThreads / 64 ? 0 : turn + 1;
        advance(from);
        return true;
    };
    // first the halves that are free sooner: x's and dy's first copies
    constexpr int kHalf = kLoads / 2;
    u32x4 held[DMA ? 1 : S::kCopies];
    auto copy = [&](int i, uint32_t stage) __attribute__((always_inline)) {
        const int half = i / (2 * kHalf), j = half * kHalf + i % kHalf;
        const bool is_x = i % (2 * kHalf) < kHalf;
        const int r = cr + j * kRows;
        const bool there = r < rows_left && (!ordered || slot[j] < slots);
        const SlotMap& map = is_x ? a.x_map : a.out_map;
        const uint32_t row = map.mode == 0 ? base + r : (uint32_t)map.row(slot[j]);
        const elem* p = is_x ? x + (int64_t)row * a.ld_x : dy + (int64_t)row * a.ld_w;
        const int c = is_x ? x_col + xc[j % kColumns] : dy_col + wc[j % kColumns];
        if constexpr (DMA)
            copy_to_lds(there ? p + c : zeros, stage + (is_x ? 0 : S::kRowsBytes) + j * S::kThreads * 16);
        else
            held[is_x ? j : kLoads + j] = load_row<T>(p, c, there ? is_x ? a.cols_in : a.cols_out : 0, 0);
    };
    auto put = [&](char* stage) __attribute__((always_inline)) {
        if constexpr (!DMA)
#pragma unroll
            for (int i = 0; i < S::kCopies; ++i)
                *reinterpret_cast<u32x4*>(stage + (i * S::kThreads + t) * 16) = held[i];
    };

    uint32_t id = first;
    bool begun = false;
    auto tile_steps = [&]() __attribute__((always_inline)) -> int {
        id += begun ? stride : 0;
        begun = true;
        return id < last ? steps_of(part_place(table, a, id / of_part)) : -1;
    };
    const int wm = wave % S::WM, wn = wave / S::WM;
    const Side<T, false, false, S::BM, S::kTm> xs(wm * S::kTm * 16, lane);
    const Side<T, false, false, S::BN, S::kTn> ws(wn * S::kTn * 16, lane);
    auto finish = [&](f32x4 (&acc)[S::kTm][S::kTn]) __attribute__((always_inline)) {
        uint32_t m, n;
        grouped_tile(id % of_part, m_tiles, n_tiles, m, n);
        store_sums<T, S>(a, part_place(table, a, id / of_part), acc, (int)m * S::BM + wm * S::kTm * 16,
                         (int)n * S::BN + wn * S::kTn * 16, lane);
    };
    multiply_tiles<T, S, DMA, DMA ? 2 * kHalf : 0>(tiles, lds_address(tiles) + wave * 1024, xs, ws, next_step, copy,
                                                          put, tile_steps, finish);
}

constexpr int kJoinBlock = 256;

// dweight of the experts of several parts from the parts' sums, in the parts' order; a thread four elements in
// turn, a row of workgroups an expert.
template <typename T>
__global__ __launch_bounds__(kJoinBlock) void k_expert_join(const ExpertCall a) {
    __shared__ TileTable table;
    fill_tile_table(table, nullptr, a, [&](int rows) { return parts_of(rows, a.part); }, [](int) { return 0u; });
    const int e = (int)blockIdx.y;
    const uint32_t first = e > 0 ? table.upto[e - 1] : 0, last = table.upto[e];
    if (last - first == 1)
        return;
    const int64_t all = (int64_t)a.cols_in * a.cols_out;
    const int64_t i = ((int64_t)blockIdx.x * kJoinBlock + threadIdx.x) * 4;
    if (i >= all)
        return;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    const float* const from = a.partial + first * all + i;
    const int count = all - i < 4 ? (int)(all - i) : 4;
    if (count == 4 && all % 4 == 0) {
        for (uint32_t s = 0; s < last - first; ++s) {
            float f[4];
            F32::unpack(load_vec<F32, false>(from + s * all), f);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                sum[j] += f[j];
        }
    } else {
        for (uint32_t s = 0; s < last - first; ++s)
            for (int j = 0; j < count; ++j)
                sum[j] += from[s * all + j];
    }
    typename T::elem* const out = static_cast<typename T::elem*>(a.out) + (int64_t)e * a.cols_in * a.ld_out;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < count)
            out[(i + j) / a.cols_out * a.ld_out + (i + j) % a.cols_out] = T::of_f32(sum[j]);
}

// ---------------------------------------------------------------------------
// A token's slots joined: a thread has a vector of the token's columns and goes through the slots.
// ---------------------------------------------------------------------------
constexpr int kMixBlock = 256;

__device__ __forceinline__ bool has_expert(const int32_t* index, int64_t slot, int experts) {
    if (!index)
        return true;
    const int e = index[slot];
    return e >= 0 && (experts == 0 || e < experts);
}

template <typename T>
__global__ __launch_bounds__(kMixBlock) void k_expert_mix(const zero_expert_mix_args_t a, int lanes, int64_t first) {
    using elem = typename T::elem;
    constexpr int kPer = T::kPer, kBatch = 4;
    const int64_t id = first + (int64_t)blockIdx.x * kMixBlock + threadIdx.x;
    const int64_t token = id / lanes;
    const int col = (int)(id - token * lanes) * kPer, cols = (int)a.cols;
    if (token >= a.tokens)
        return;
    float sum[kPer] = {};
    if (a.base)
        T::unpack(load_row<T>(static_cast<const elem*>(a.base) + token * a.ld_base, col, cols, 0), sum);
    const elem* y = static_cast<const elem*>(a.y) + token * a.k * a.ld_y;
    for (int i0 = 0; i0 < a.k; i0 += kBatch) {
        u32x4 v[kBatch];
        float w[kBatch];
        bool there[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int64_t slot = token * a.k + i0 + i;
            there[i] = i0 + i < a.k && has_expert(a.index, slot, a.experts);
            w[i] = there[i] && a.weight ? a.weight[slot] : 1.f;
            if (there[i])
                v[i] = load_row<T>(y + (i0 + i) * a.ld_y, col, cols, 0);
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
            if (there[i]) {
                float f[kPer];
                T::unpack(v[i], f);
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    sum[j] = __builtin_fmaf(w[i], f[j], sum[j]);
            }
    }
    store_row<T>(static_cast<elem*>(a.out) + token * a.ld_out, col, cols, T::pack(sum));
}

// Its gradients, a wave a slot.
template <typename T>
__global__ __launch_bounds__(kMixBlock) void k_expert_mix_back(const zero_expert_mix_backward_args_t a, int64_t first) {
    using elem = typename T::elem;
    constexpr int kPer = T::kPer;
    const int lane = threadIdx.x & 63, cols = (int)a.cols;
    const int64_t slot = first + (int64_t)blockIdx.x * (kMixBlock / 64) + threadIdx.x / 64;
    if (slot >= a.tokens * a.k)
        return;
    const bool there = has_expert(a.index, slot, a.experts);
    const float w = there ? (a.weight ? a.weight[slot] : 1.f) : 0.f;
    const elem* const dout = static_cast<const elem*>(a.dout) + slot / a.k * a.ld_dout;
    const elem* const y = static_cast<const elem*>(a.y) + slot * a.ld_y;
    elem* const dy = static_cast<elem*>(a.dy) + slot * a.ld_dy;
    float dot = 0.f;
    for (int col = lane * kPer; col < cols; col += 64 * kPer) {
        float d[kPer], f[kPer];
        u32x4 v = {0, 0, 0, 0};
        if (there)
            v = load_row<T>(dout, col, cols, 0);
        T::unpack(v, d);
        if (there && a.dweight) {
            T::unpack(load_row<T>(y, col, cols, 0), f);
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                dot = __builtin_fmaf(d[j], f[j], dot);
        }
        if (a.dy) {
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                d[j] = there ? w * d[j] : 0.f;
            store_row<T>(dy, col, cols, T::pack(d));
        }
    }
    if (a.dweight) {
        dot = seg_reduce<64>(dot, Add());
        if (lane == 0)
            a.dweight[slot] = dot;
    }
}

}  // namespace zo
