// expert_kernels.hpp -- products of the experts' rows with their weights, and the weights'
// gradient: tiles of both operands in LDS, sums in the matrix cores' registers.
//
// A step of the sum takes 128 bytes of its axis (64 elements of 16 bits, 32 of fp32).  An operand's tile
// comes in one of two layouts, as it lies in memory:
//   along    its rows run along the summed axis (x; weights that lie [out, in]): tile rows of 128 bytes
//   across   they run across it (weights that lie [in, out]; both operands of the gradient): one
//            tile row for each place of the axis, which the matrix instruction wants transposed;
//            ds_read_b64_tr_b16 does that for 16 bits, fp32's fragments are single words anyway
// The 16-byte chunks of a tile row are exchanged by a few bits of the row, so that the lanes of a fragment
// read different banks; the copy to LDS writes chunks in the lanes' order, so the exchange is in the address
// that a lane reads from memory.
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
    float* partial;        // [splits, experts, cols_in, cols_out]
    int64_t slots;
    int32_t experts;
    int32_t cols_in, cols_out;
    int32_t splits;
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

// Along: the exchange of the chunks of tile row r.  On the columns' side a pair of fragments takes 32 rows so that a lane's
// 4 + 4 results are neighbours: fragment f, lane row a is tile row 32 (f / 2) + 8 (a / 4) + 4 (f % 2) + a % 4.
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

// One side of a wave's fragments: byte offsets in the tile, once for each fragment or few.
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
            at[0] = r * kRow + c * 16;
            at[1] = r * kRow + (c ^ 4) * 16;
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
    static_assert(kRowLoads * 16 * kThreads == kRowsBytes && kColLoads * 16 * kThreads == kColsBytes, "whole loads");
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

// 16 bytes straight to LDS: lane l's land at base + 16 l.  Written as an instruction because the compiler holds every
// ds_read_tr behind all copies that it knows of (s_waitcnt vmcnt(0) before the step's first fragment: 16384 x 8 slots
// 1024 to 4096 bf16 1612 us); wait_stage has the waits.  There is no output register, and nothing else in these kernels uses m0.
__device__ __forceinline__ void copy_to_lds(const void* from, uint32_t base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(base), "v"(from) : "memory");
}

__device__ __forceinline__ uint32_t lds_address(char* p) { return (uint32_t)(uintptr_t)ZO_LDS(char, p); }

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

// Four neighbouring results of a row (or eight), of which those before column `cols` exist.
template <typename T, int COUNT>
__device__ __forceinline__ void store_results(typename T::elem* p, int col, int cols, const float* f) {
    if (col + COUNT <= cols) {
        if constexpr (T::kPer == 4) {
#pragma unroll
            for (int j = 0; j < COUNT; j += 4)
                store_vec<T, false>(p + col + j, T::pack(f + j));
        } else if constexpr (COUNT == 8) {
            store_vec<T, false>(p + col, T::pack(f));
        } else {
            float g[8];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                g[j] = g[j + 4] = f[j];
            const u32x4 v = T::pack(g);
            *reinterpret_cast<u32x2_e2*>(p + col) = u32x2{v.x, v.y};
        }
    } else {
#pragma unroll
        for (int j = 0; j < COUNT; ++j)
            if (col + j < cols)
                p[col + j] = T::of_f32(f[j]);
    }
}

// A wave's results: out(m) is the row of its m-th (null: none), `first` its first column.
template <typename T, typename S, bool PAIRED, typename OUT>
__device__ __forceinline__ void store_tile(const f32x4 (&acc)[S::kTm][S::kTn], int first, int cols, int lane, OUT out) {
    const int g = lane >> 4;
#pragma unroll
    for (int m = 0; m < S::kTm; ++m) {
        typename T::elem* const p = out(16 * m + (lane & 15));
        if (!p)
            continue;
        if constexpr (PAIRED) {
#pragma unroll
            for (int n = 0; n < S::kTn; n += 2) {
                const float f[8] = {acc[m][n].x,     acc[m][n].y,     acc[m][n].z,     acc[m][n].w,
                                    acc[m][n + 1].x, acc[m][n + 1].y, acc[m][n + 1].z, acc[m][n + 1].w};
                store_results<T, 8>(p, first + 16 * n + 8 * g, cols, f);
            }
        } else {
#pragma unroll
            for (int n = 0; n < S::kTn; ++n) {
                const float f[4] = {acc[m][n].x, acc[m][n].y, acc[m][n].z, acc[m][n].w};
                store_results<T, 4>(p, first + 16 * n + 4 * g, cols, f);
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Which tile a workgroup takes.  The host knows no expert's number of rows, so it launches as many as there
// can be; each workgroup adds up the experts' tiles, and those past the last have nothing to do.
// Workgroups go to the eight dies in turn, so that numbering gives each die a run of the tiles: eight
// rows' tiles by all columns' tiles, whose operands its L2 then serves.
// ---------------------------------------------------------------------------
struct TilePlace {
    int expert;
    int first, end;    // rows of the experts' order
    int col_tile;
};

__device__ __forceinline__ uint32_t die_order(uint32_t id, uint32_t count) {
    const uint32_t each = (count + 7) / 8;
    const uint32_t t = (id & 7) * each + (id >> 3);
    return (id >> 3) < each ? t : count;
}

template <int BM>
__device__ __forceinline__ bool find_tile(const ExpertCall& a, uint32_t first, uint32_t launched, uint32_t col_tiles,
                                          TilePlace& out) {
    const int lane = threadIdx.x & 63;
    const int slots = (int)a.slots;
    auto tiles_of = [&](int e, int& lo, int& hi) -> uint32_t {
        lo = hi = 0;
        if (e < a.experts) {
            lo = a.offsets[e];
            hi = a.offsets[e + 1];
        }
        lo = lo < 0 ? 0 : lo > slots ? slots : lo;
        hi = hi < lo ? lo : hi > slots ? slots : hi;
        return ((uint32_t)(hi - lo) + BM - 1) / BM;
    };
    int lo, hi;
    uint32_t total = 0;
    for (int e = lane; e < (a.experts + 63) / 64 * 64; e += 64)
        total += tiles_of(e, lo, hi);
    total = seg_reduce<64>(total, [](uint32_t p, uint32_t q) { return p + q; });
    total = __builtin_amdgcn_readfirstlane(total);
    const uint32_t all = total * col_tiles;
    if (first >= all)
        return false;
    const uint32_t here = all - first < launched ? all - first : launched;
    const uint32_t in_run = die_order(blockIdx.x, here);
    if (in_run >= here)
        return false;
    const uint32_t id = first + in_run;
    constexpr uint32_t kGroup = 8;
    const uint32_t per = kGroup * col_tiles, group = id / per, rest = id - group * per;
    const uint32_t rows_in = total - group * kGroup < kGroup ? total - group * kGroup : kGroup;
    const uint32_t col_tile = rest / rows_in, row_tile = group * kGroup + rest - col_tile * rows_in;
    uint32_t before = 0;
    for (int e0 = 0; e0 < a.experts; e0 += 64) {
        const uint32_t t = tiles_of(e0 + lane, lo, hi);
        uint32_t upto = t;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t o = __shfl_up(upto, d);
            upto += lane >= d ? o : 0;
        }
        const uint32_t mine = row_tile - (before + upto - t);  // this workgroup's place among the expert's tiles
        const uint64_t found = __ballot(mine < t);
        if (found) {
            const int l = __ffsll((unsigned long long)found) - 1;
            out.expert = e0 + l;
            out.first = __shfl(lo, l) + __shfl((int)mine, l) * BM;
            out.end = __shfl(hi, l);
            out.first = __builtin_amdgcn_readfirstlane(out.first);
            out.end = __builtin_amdgcn_readfirstlane(out.end);
            out.col_tile = (int)col_tile;
            return true;
        }
        before += __shfl(upto, 63);
    }
    return false;
}

// ---------------------------------------------------------------------------
// y = x * weight.  ALONG: the weights lie [out, in].  DMA: every row of x and of the weights is made of
// aligned chunks of 16 bytes, which go straight to LDS; else they pass through the registers, where their ends are seen to.
// ---------------------------------------------------------------------------
template <typename T, typename S, bool ALONG, bool DMA>
__global__ __launch_bounds__(S::kThreads) void k_expert_product(const ExpertCall a, uint32_t first, uint32_t launched) {
    using elem = typename T::elem;
    constexpr int kPer = T::kPer, kStep = kStepBytes / (int)sizeof(elem);
    constexpr int kChunks = ALONG ? 8 : S::BN / kPer;             // chunks of a row of the weights' tile
    constexpr int kXRows = S::kThreads / 8, kWRows = S::kThreads / kChunks;  // tile rows of one load of all threads
    __shared__ __attribute__((aligned(1024))) char tiles[S::kStages * S::kStage];

    TilePlace place;
    const uint32_t col_tiles = ((uint32_t)a.cols_out + S::BN - 1) / S::BN;
    if (!find_tile<S::BM>(a, first, launched, col_tiles, place))
        return;
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
    const int xr = t / 8, xc = ((t & 7) ^ along_exchange<false>(xr)) * kPer;
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
            wc[j] = ((t & 7) ^ along_exchange<true>(r)) * kPer;
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
        const uint32_t stage = lds + step % S::kStages * S::kStage;
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
            char* const stage = tiles + step % S::kStages * S::kStage + t * 16;
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

    constexpr int kAhead = DMA ? S::kStages - 1 : 1;  // stages under way
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
        multiply<T, S>(tiles + s % S::kStages * S::kStage, xs, ws, acc);
        if (s + kAhead < steps)
            put(s + kAhead);
    }

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
// dweight = x^T * dy, a tile of one expert's matrix for a workgroup, the expert's rows in `splits` parts
// whose sums k_expert_join adds up.
// ---------------------------------------------------------------------------
template <typename T, typename S, bool DMA>
__global__ __launch_bounds__(S::kThreads) void k_expert_weight_back(const ExpertCall a, uint32_t first,
                                                                    uint32_t launched) {
    using elem = typename T::elem;
    static_assert(S::BM == S::BN, "a thread's rows of x and dy are the same slots");
    constexpr int kPer = T::kPer, kStep = kStepBytes / (int)sizeof(elem);
    constexpr int kChunks = S::BN / kPer, kRows = S::kThreads / kChunks, kLoads = S::kColLoads;
    __shared__ __attribute__((aligned(1024))) char tiles[2 * S::kStage];

    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const uint32_t m_tiles = ((uint32_t)a.cols_in + S::BM - 1) / S::BM, n_tiles = ((uint32_t)a.cols_out + S::BN - 1) / S::BN;
    uint32_t id = die_order(blockIdx.x, launched);
    if (id >= launched)
        return;
    id += first;
    const uint32_t part = id / (m_tiles * n_tiles), tile = id - part * (m_tiles * n_tiles);
    const int m0 = (int)(tile / n_tiles) * S::BM, n0 = (int)(tile % n_tiles) * S::BN;
    const int expert = (int)(part / (uint32_t)a.splits), split = (int)(part % (uint32_t)a.splits);
    const int slots = (int)a.slots;
    int lo = __builtin_amdgcn_readfirstlane(a.offsets[expert]), hi = __builtin_amdgcn_readfirstlane(a.offsets[expert + 1]);
    lo = lo < 0 ? 0 : lo > slots ? slots : lo;
    hi = hi < lo ? lo : hi > slots ? slots : hi;
    const int run = (int)(((uint32_t)(hi - lo) + kStep * a.splits - 1) / (kStep * a.splits)) * kStep;  // whole steps
    const int64_t from = lo + (int64_t)run * split;
    const int begin = from < hi ? (int)from : hi, end = hi - begin < run ? hi : begin + run;
    const int steps = (end - begin + kStep - 1) / kStep;
    const elem* const x = static_cast<const elem*>(a.x);
    const elem* const dy = static_cast<const elem*>(a.w);
    const elem* const zeros = reinterpret_cast<const elem*>(&zero_chunk);

    int xc[kLoads], wc[kLoads];  // columns of this thread's chunks
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
        const int c = ((t % kChunks) ^ across_exchange<T, kChunks>(t / kChunks + j * kRows)) * kPer;
        xc[j] = m0 + c;
        wc[j] = n0 + c;
        if constexpr (DMA) {  // rows and columns past the last are not stored
            xc[j] = xc[j] < a.cols_in ? xc[j] : a.cols_in - kPer;
            wc[j] = wc[j] < a.cols_out ? wc[j] : a.cols_out - kPer;
        }
    }
    const uint32_t lds = lds_address(tiles) + wave * 1024;
    const bool ordered = a.x_map.mode | a.out_map.mode;
    // entries of order for a step's rows, a step before they are needed; -1: no row
    int32_t slot[kLoads];
    auto look_up = [&](int step) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const uint32_t i = (uint32_t)begin + (uint32_t)step * kStep + t / kChunks + j * kRows;  // may pass 2^31
            slot[j] = i < (uint32_t)end ? (ordered ? a.order[i] : 0) : -1;
        }
    };
    u32x4 rx[DMA ? 1 : kLoads], rw[DMA ? 1 : kLoads];
    auto fetch = [&](int step) __attribute__((always_inline)) {
        const uint32_t stage = lds + (step & 1) * S::kStage;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int64_t i = begin + (int64_t)step * kStep + t / kChunks + j * kRows;
            const bool there = (uint32_t)slot[j] < (uint32_t)slots;
            const elem* const px = x + (a.x_map.mode ? a.x_map.row(slot[j]) : i) * a.ld_x;
            const elem* const pw = dy + (a.out_map.mode ? a.out_map.row(slot[j]) : i) * a.ld_w;
            if constexpr (DMA) {
                copy_to_lds(there ? px + xc[j] : zeros, stage + j * S::kThreads * 16);
                copy_to_lds(there ? pw + wc[j] : zeros, stage + S::kRowsBytes + j * S::kThreads * 16);
            } else {
                rx[j] = rw[j] = u32x4{0, 0, 0, 0};
                if (there) {
                    rx[j] = load_row<T>(px, xc[j], a.cols_in, 0);
                    rw[j] = load_row<T>(pw, wc[j], a.cols_out, 0);
                }
            }
        }
    };
    auto put = [&](int step) __attribute__((always_inline)) {
        if constexpr (!DMA) {
            char* const stage = tiles + (step & 1) * S::kStage + t * 16;
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                *reinterpret_cast<u32x4*>(stage + j * S::kThreads * 16) = rx[j];
                *reinterpret_cast<u32x4*>(stage + S::kRowsBytes + j * S::kThreads * 16) = rw[j];
            }
        }
    };

    const int wm = wave % S::WM, wn = wave / S::WM;
    const Side<T, false, false, S::BM, S::kTm> xs(wm * S::kTm * 16, lane);
    const Side<T, false, false, S::BN, S::kTn> ws(wn * S::kTn * 16, lane);
    f32x4 acc[S::kTm][S::kTn];
#pragma unroll
    for (int m = 0; m < S::kTm; ++m)
#pragma unroll
        for (int n = 0; n < S::kTn; ++n)
            acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};

    if (steps > 0) {
        look_up(0);
        fetch(0);
        put(0);
        look_up(1);
    }
    for (int s = 0; s < steps; ++s) {
        wait_stage<0>();
        if (s + 1 < steps) {
            fetch(s + 1);
            look_up(s + 2);
        }
        multiply<T, S>(tiles + (s & 1) * S::kStage, xs, ws, acc);
        if (s + 1 < steps)
            put(s + 1);
    }

    const int col = n0 + wn * S::kTn * 16;
    if (a.splits > 1) {
        float* const p = a.partial + ((int64_t)split * a.experts + expert) * a.cols_in * a.cols_out;
        store_tile<F32, S, false>(acc, col, a.cols_out, lane, [&](int m) -> float* {
            const int row = m0 + wm * S::kTm * 16 + m;
            return row < a.cols_in ? p + (int64_t)row * a.cols_out : nullptr;
        });
    } else {
        elem* const p = static_cast<elem*>(a.out) + (int64_t)expert * a.cols_in * a.ld_out;
        store_tile<T, S, false>(acc, col, a.cols_out, lane, [&](int m) -> elem* {
            const int row = m0 + wm * S::kTm * 16 + m;
            return row < a.cols_in ? p + row * a.ld_out : nullptr;
        });
    }
}

constexpr int kJoinBlock = 256;

// dweight from the parts' sums, in the parts' order; a thread an element.
template <typename T>
__global__ __launch_bounds__(kJoinBlock) void k_expert_join(const float* partial, int splits, int64_t all, int cols,
                                                            typename T::elem* out, int64_t ld) {
    const int64_t i = (int64_t)blockIdx.x * kJoinBlock + threadIdx.x;
    if (i >= all)
        return;
    float sum = 0.f;
    for (int s = 0; s < splits; ++s)
        sum += partial[s * all + i];
    out[i / cols * ld + i % cols] = T::of_f32(sum);
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
