// route_kernels.hpp -- routing of tokens to experts: choice and weights, the slots'
// order by expert, the gradient of the logits.
//
// A token's row is short (at most 1024 logits), so its bytes are read in a moment and the
// choice bounds the kernel: k rounds of a maximum over the row.  LPT lanes hold a
// token with VPL keys each, in registers, and a wave holds 64 / LPT tokens, whose rounds
// run side by side.  A lane's experts are a run of neighbours inside one group, runs
// rising with the lane, so the lowest lane that holds the maximum holds the lowest such expert.
//
// Measured at 16384 tokens of 256 experts (8 of them from 4 of 8 groups, sigmoid, bias): 15.9 us, of which a round takes
// 0.7, the sigmoids 2.7 and the groups 1.6 (the logits' 17 MB are 2.5 us at the copy kernel's rate); the ordering of their
// slots 3.6 and 7.9 in two launches; the gradient 8.9, softmax over all experts 15.2 (below).
#pragma once

#include "row_ops.hpp"
#include "zero_operators.h"

namespace zo {

constexpr int kRouteBlock = 256;
constexpr float kLog2e = 1.44269504088896340736f;

// Keys as integers that order as the floats do, -0 as +0; 0 is "never chosen" (-inf, NaN).
__device__ __forceinline__ uint32_t order_bits(float f) {
    const uint32_t b = __builtin_bit_cast(uint32_t, f + 0.0f);
    const uint32_t u = b >> 31 ? ~b : b | 0x80000000u;
    return f > -__builtin_inff() ? u : 0u;
}

__device__ __forceinline__ float order_value(uint32_t u) {
    if (u == 0)
        return -__builtin_inff();
    return __builtin_bit_cast(float, u >> 31 ? u & 0x7FFFFFFFu : ~u);
}

// Division and exponential correctly as written: a key decides a choice, and its value is defined
// by these operations.
__device__ __forceinline__ float sigmoid(float z) { return 1.0f / (1.0f + expf(-z)); }

// N consecutive elements from `col`, -inf at or past `end`.
template <typename T, int N>
__device__ __forceinline__ void load_keys(const typename T::elem* p, int col, int end, float* f) {
    if (col + N <= end) {
        typename T::elem e[N];
        __builtin_memcpy(e, p + col, sizeof e);
#pragma unroll
        for (int j = 0; j < N; ++j)
            f[j] = T::to_f32(e[j]);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            f[j] = col + j < end ? T::to_f32(p[col + j]) : -__builtin_inff();
    }
}

// The two largest of a run of lanes (a power of two up to 32, the same in the whole grid: with two groups
// or more a group has half a wave at most).
struct Top2 {
    uint32_t a, b;
};

__device__ __forceinline__ Top2 top2(uint32_t a0, uint32_t b0, uint32_t a1, uint32_t b1) {
    const uint32_t lo = a0 < a1 ? a0 : a1, b = b0 > b1 ? b0 : b1;
    return Top2{a0 < a1 ? a1 : a0, lo > b ? lo : b};
}

template <int CTRL>
__device__ __forceinline__ Top2 top2_dpp(Top2 t) {
    return top2(t.a, t.b, dpp<CTRL>(t.a), dpp<CTRL>(t.b));
}

__device__ __forceinline__ Top2 top2_swap(Top2 t) {
    const auto a = __builtin_amdgcn_permlane16_swap(t.a, t.a, false, false);
    const auto b = __builtin_amdgcn_permlane16_swap(t.b, t.b, false, false);
    return top2(a[0], b[0], a[1], b[1]);
}

__device__ __forceinline__ Top2 run_top2(Top2 t, int lanes) {
    if (lanes >= 2)
        t = top2_dpp<0xB1>(t);
    if (lanes >= 4)
        t = top2_dpp<0x4E>(t);
    if (lanes >= 8)
        t = top2_dpp<0x141>(t);
    if (lanes >= 16)
        t = top2_dpp<0x140>(t);
    if (lanes >= 32)
        t = top2_swap(t);
    return t;
}

// 2^shift lanes hold a group of `size` experts: groups << shift <= LPT, size <= VPL << shift; k <= LPT.
template <typename T, int LPT, int VPL>
__global__ __launch_bounds__(kRouteBlock) void k_route(const zero_route_args_t a, int size, int shift,
                                                        int64_t first) {
    constexpr int kTokens = kRouteBlock / LPT;
    __shared__ int32_t chosen[kTokens][LPT];
    const int lane = threadIdx.x % LPT, token = threadIdx.x / LPT, first_bit = (threadIdx.x & 63) - lane;
    const int64_t row = first + (int64_t)blockIdx.x * kTokens + token;
    const bool there = row < a.rows;
    const typename T::elem* logits = static_cast<const typename T::elem*>(a.logits) + row * a.ld_logits;
    const float inf = __builtin_inff();
    const bool soft = a.score == ZERO_SCORE_SOFTMAX;

    const int per_group = 1 << shift, group = lane >> shift;
    const int from = group * size + (lane & (per_group - 1)) * VPL;  // this lane's experts: [from, end)
    int end = (group + 1) * size;
    end = end < from + VPL ? end : from + VPL;
    if (!there || group >= a.groups)
        end = from;

    float z[VPL];
    uint32_t key[VPL];
    bool bad = false;
    load_keys<T, VPL>(logits, from, end, z);
    float b[VPL] = {};
    if (a.bias)
        load_keys<F32, VPL>(a.bias, from, end, b);
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
        const bool out = z[j] == -inf || b[j] == -inf;
        z[j] = out ? -inf : z[j];
        bad |= z[j] != z[j];
        key[j] = out ? 0u : order_bits((soft ? z[j] : sigmoid(z[j])) + b[j]);
    }
    chosen[token][lane] = -1;

    if (a.groups > 1) {
        Top2 t{0, 0};
#pragma unroll
        for (int j = 0; j < VPL; ++j)
            t = top2(t.a, t.b, key[j], 0);
        t = run_top2(t, per_group);
        const uint32_t mine = a.group_top == 2 ? order_bits(order_value(t.a) + order_value(t.b)) : t.a;
        int ahead = 0;  // groups that come before this one
        for (int g = 0; g < a.groups; ++g) {
            const uint32_t other = __shfl(mine, g << shift, LPT);
            ahead += other > mine || (other == mine && g < group);
        }
        const bool stays = mine != 0 && ahead < a.top_groups;
#pragma unroll
        for (int j = 0; j < VPL; ++j)
            key[j] = stays ? key[j] : 0u;
    }
    __syncthreads();

    // bits of this token's lanes before this one
    const uint64_t before = (((uint64_t)1 << lane) - 1) << first_bit;
    for (int i = 0; i < a.k; ++i) {
        uint32_t m = key[0];
#pragma unroll
        for (int j = 1; j < VPL; ++j)
            m = MaxU()(m, key[j]);
        const uint32_t top = seg_reduce<LPT>(m, MaxU());
        const bool has = m == top && top != 0;
        const uint64_t who = __ballot(has);
        if (has && (who & before) == 0) {
            int at = 0;
#pragma unroll
            for (int j = VPL - 1; j >= 0; --j)
                at = key[j] == top ? j : at;
            chosen[token][i] = from + at;
#pragma unroll
            for (int j = 0; j < VPL; ++j)
                key[j] = at == j ? 0u : key[j];
        }
    }
    __syncthreads();

    // lane i has slot i
    const int at = lane < a.k ? chosen[token][lane] : -1;
    const float zi = at >= 0 ? T::to_f32(logits[at]) : -inf;
    float w;
    if (soft) {
        float m, total;
        if (a.renormalise) {
            m = seg_reduce<LPT>(zi, Max());
            total = seg_reduce<LPT>(at >= 0 ? exp2_fast((zi - m) * kLog2e) : 0.f, Add());
        } else {
            m = z[0];
#pragma unroll
            for (int j = 1; j < VPL; ++j)
                m = fmaxf(m, z[j]);
            m = seg_reduce<LPT>(m, Max());
            total = 0.f;
#pragma unroll
            for (int j = 0; j < VPL; ++j)
                total += z[j] == -inf ? 0.f : exp2_fast((z[j] - m) * kLog2e);
            total = seg_reduce<LPT>(total, Add());
        }
        w = exp2_fast((zi - m) * kLog2e) / total;
    } else {
        w = at >= 0 ? sigmoid(zi) : 0.f;
        if (a.renormalise)
            w /= fmaxf(seg_reduce<LPT>(w, Add()), 0x1p-126f);
    }
    const bool nan = seg_reduce<LPT>((uint32_t)bad, MaxU()) != 0;
    if (there && lane < a.k) {
        a.index[row * a.k + lane] = at;
        a.weight[row * a.k + lane] = at < 0 ? 0.f : nan ? __builtin_nanf("") : w * (float)a.scale;
    }
}

// ---------------------------------------------------------------------------
// Order of the slots: a counting sort by expert, slots without one last.  The slots are
// cut into one run of chunks a workgroup; k_route_count leaves each run's counts, from which
// every workgroup of k_route_order takes its own places (a few kilobytes from L2:
// less than a kernel of its own would cost).
// ---------------------------------------------------------------------------
constexpr int kOrderBlock = 512, kOrderWaves = kOrderBlock / 64;
constexpr int kOrderKeys = ZERO_ROUTE_MAX_EXPERTS + 1;  // the experts, and "none"
constexpr int kOrderOwn = (kOrderKeys + kOrderBlock - 1) / kOrderBlock;  // keys a thread scans

__device__ __forceinline__ int slot_key(const int32_t* index, int64_t s, int experts) {
    const uint32_t e = (uint32_t)index[s];
    return e < (uint32_t)experts ? (int)e : experts;
}

// counts[b][key] over the run of workgroup b: slots [b * run, (b + 1) * run).
__global__ __launch_bounds__(kOrderBlock) void k_route_count(const int32_t* index, int64_t slots, int experts,
                                                             int64_t run, int32_t* counts) {
    __shared__ int32_t n[kOrderKeys];
    for (int e = threadIdx.x; e <= experts; e += kOrderBlock)
        n[e] = 0;
    __syncthreads();
    const int64_t from = blockIdx.x * run, end = from + run < slots ? from + run : slots;
#pragma unroll 4
    for (int64_t s = from + threadIdx.x; s < end; s += kOrderBlock)
        atomicAdd(&n[slot_key(index, s, experts)], 1);
    __syncthreads();
    for (int e = threadIdx.x; e <= experts; e += kOrderBlock)
        counts[(int64_t)blockIdx.x * (experts + 1) + e] = n[e];
}

// counts may be NULL where the grid is one workgroup.  run is a multiple of kOrderBlock, OWN * kOrderBlock
// at least the keys.
template <int OWN>
__global__ __launch_bounds__(kOrderBlock) void k_route_order(const int32_t* index, int64_t slots, int experts,
                                                             int64_t run, const int32_t* counts, int32_t* offsets,
                                                             int32_t* order) {
    __shared__ int32_t place[kOrderWaves][kOrderKeys];  // counts of each wave's slots, then their places
    __shared__ int32_t sums[kOrderWaves];
    const int keys = experts + 1, wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    const int64_t part = run / kOrderWaves;  // a wave's slots: neighbours, in the order of the waves
    const int64_t from = blockIdx.x * run + wave * part;
    const int64_t end = from + part < slots ? from + part : slots;
    constexpr int kBatch = 4;  // keys under way at a time; a wave's first batch stays in its registers
    auto load_keys = [&](int* key, int64_t s0) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int64_t s = s0 + 64 * i + lane;
            key[i] = s < end ? slot_key(index, s, experts) : -1;
        }
    };
    int first[kBatch];
    load_keys(first, from);

    for (int e = threadIdx.x; e < keys; e += kOrderBlock)
#pragma unroll
        for (int w = 0; w < kOrderWaves; ++w)
            place[w][e] = 0;
    __syncthreads();
    for (int64_t s0 = from; s0 < end; s0 += 64 * kBatch) {
        int key[kBatch];
        if (s0 == from) {
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                key[i] = first[i];
        } else {
            load_keys(key, s0);
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
            if (key[i] >= 0)
                atomicAdd(&place[wave][key[i]], 1);
    }
    __syncthreads();

    // this thread's keys: all slots of each, and those of the workgroups before this one
    int32_t all[OWN], prior[OWN];
#pragma unroll
    for (int j = 0; j < OWN; ++j) {
        const int e = threadIdx.x * OWN + j;
        all[j] = prior[j] = 0;
        if (counts && e < keys) {
            // sixteen loads under way; the last batch reads the last run again where there are none
            const int runs = (int)gridDim.x, before = (int)blockIdx.x;
            const int32_t* p = counts + e;
            for (int b0 = 0; b0 < runs; b0 += 16, p += 16 * keys) {
                int32_t c[16];
                if (b0 + 16 <= runs) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        c[i] = p[i * keys];
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        c[i] = p[(b0 + i < runs ? i : runs - 1 - b0) * keys];
                        c[i] = b0 + i < runs ? c[i] : 0;
                    }
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    all[j] += c[i];
                    prior[j] += b0 + i < before ? c[i] : 0;
                }
            }
        }
    }
    int32_t mine = 0;
#pragma unroll
    for (int j = 0; j < OWN; ++j) {
        const int e = threadIdx.x * OWN + j;
        if (!counts && e < keys) {
#pragma unroll
            for (int w = 0; w < kOrderWaves; ++w)
                all[j] += place[w][e];
        }
        mine += all[j];
    }
    int32_t upto = mine;  // inclusive sum over the workgroup's threads
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int32_t o = __shfl_up(upto, d);
        upto += lane >= d ? o : 0;
    }
    if (lane == 63)
        sums[wave] = upto;
    __syncthreads();
    int32_t at = upto - mine;
    for (int w = 0; w < wave; ++w)
        at += sums[w];
#pragma unroll
    for (int j = 0; j < OWN; ++j) {
        const int e = threadIdx.x * OWN + j;
        if (e < keys) {
            if (blockIdx.x == 0)
                offsets[e] = at;  // of the last key: the slots that have an expert
            int32_t p = at + prior[j];
#pragma unroll
            for (int w = 0; w < kOrderWaves; ++w) {
                const int32_t c = place[w][e];
                place[w][e] = p;
                p += c;
            }
        }
        at += all[j];
    }
    __syncthreads();

    const int bits = 32 - __builtin_clz(keys);
    for (int64_t s0 = from; s0 < end; s0 += 64 * kBatch) {
        int key[kBatch];
        if (s0 == from) {
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                key[i] = first[i];
        } else {
            load_keys(key, s0);
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int e = key[i];
            uint64_t same = __ballot(e >= 0);  // lanes with this lane's key
            for (int b = 0; b < bits; ++b) {
                const bool bit = e >> b & 1;
                const uint64_t m = __ballot(bit);
                same &= bit ? m : ~m;
            }
            const int rank = __popcll(same & (((uint64_t)1 << lane) - 1));
            int32_t base = 0;
            if (e >= 0 && rank == 0)
                base = atomicAdd(&place[wave][e], (int)__popcll(same));
            base = __shfl(base, e >= 0 ? __ffsll((unsigned long long)same) - 1 : lane);
            if (e >= 0)
                order[base + rank] = e < experts ? (int32_t)(s0 + 64 * i + lane) : -1;
        }
    }
}

// ---------------------------------------------------------------------------
// Gradient of the logits: the row goes through LDS, where the chosen experts' few terms are
// put between zeros, and out in whole vectors.  Of the 8.9 us at 16384 tokens of 256 f32 experts the
// rows' bytes are 2.5; the rest is a token's chain of latencies: index, gathered logit, sums across the lanes,
// LDS and its two barriers, then the first store.  Softmax over all experts reads the row three
// times, from the caches after the first: 15.2 us.
// ---------------------------------------------------------------------------
template <typename T, int LPT>
__global__ __launch_bounds__(kRouteBlock) void k_route_back(const zero_route_backward_args_t a, int64_t first) {
    using elem = typename T::elem;
    constexpr int kTokens = kRouteBlock / LPT, kPer = T::kPer;
    extern __shared__ float rows_lds[];  // [kTokens][experts]
    const int lane = threadIdx.x % LPT, token = threadIdx.x / LPT, experts = a.experts;
    const int64_t row = first + (int64_t)blockIdx.x * kTokens + token;
    const bool there = row < a.rows;
    const elem* logits = static_cast<const elem*>(a.logits) + row * a.ld_logits;
    float* grad = rows_lds + token * experts;
    const float inf = __builtin_inff();
    for (int e = lane; e < experts; e += LPT)
        grad[e] = 0.f;

    int at = -1;
    if (there && lane < a.k)
        at = a.index[row * a.k + lane];
    const bool has = (uint32_t)at < (uint32_t)experts;
    const float d = has ? a.dweight[row * a.k + lane] * (float)a.scale : 0.f;
    const float zi = has ? T::to_f32(logits[at]) : -inf;
    const bool whole = a.score == ZERO_SCORE_SOFTMAX && !a.renormalise;
    float m = 0.f, total = 1.f, mean = 0.f, g;
    auto in_row = [&](int e) { return e < experts && !(a.bias && a.bias[e] == -inf); };
    if (a.score == ZERO_SCORE_SOFTMAX) {
        if (!whole) {
            m = seg_reduce<LPT>(zi, Max());
            total = seg_reduce<LPT>(has ? exp2_fast((zi - m) * kLog2e) : 0.f, Add());
        } else {
            m = -inf;
            if (there)
                for (int e = lane; e < experts; e += LPT)
                    m = fmaxf(m, in_row(e) ? T::to_f32(logits[e]) : -inf);
            m = seg_reduce<LPT>(m, Max());
            float s = 0.f;
            if (there)
                for (int e = lane; e < experts; e += LPT) {
                    const float z = T::to_f32(logits[e]);
                    s += in_row(e) && z != -inf ? exp2_fast((z - m) * kLog2e) : 0.f;
                }
            total = seg_reduce<LPT>(s, Add());
        }
        const float p = has ? exp2_fast((zi - m) * kLog2e) / total : 0.f;
        mean = seg_reduce<LPT>(p * d, Add());
        g = whole ? p * d : p * (d - mean);
    } else {
        const float e = has ? expf(-zi) : 0.f, s = has ? 1.0f / (1.0f + e) : 0.f;
        float t = d;
        if (a.renormalise) {
            const float sum = fmaxf(seg_reduce<LPT>(s, Add()), 0x1p-126f);
            t = (d - seg_reduce<LPT>(d * s, Add()) / sum) / sum;
        }
        // 1 - s as e^-z s: from s, rounded beside 1, nothing of it is left from z = 17 on.  (Where e^-z is
        // past fp32, s is 0.)
        g = t * s * (fminf(e, 0x1.fffffep127f) * s);
    }
    __syncthreads();
    if (has)
        grad[at] = g;
    __syncthreads();
    if (!there)
        return;
    elem* out = static_cast<elem*>(a.dlogits) + row * a.ld_dlogits;
    for (int c = lane * kPer; c < experts; c += LPT * kPer) {
        float f[kPer];
#pragma unroll
        for (int j = 0; j < kPer; ++j)
            f[j] = c + j < experts ? grad[c + j] : 0.f;
        if (whole) {
            float z[kPer];
            T::unpack(load_row<T>(logits, c, experts, T::kLowest), z);
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                if (z[j] != -inf && in_row(c + j))
                    f[j] -= exp2_fast((z[j] - m) * kLog2e) / total * mean;
        }
        store_row<T>(out, c, experts, T::pack(f));
    }
}

}  // namespace zo
