// distill_kernels.hpp -- distillation from a teacher's top logits: a row's loss and the
// gradient of its student logits.
//
// With c = log2(e) / tau and m the row's maximum, q_tau[v] = 2^(c z_v - c m) / S; the
// gradient is q's multiple but at the teacher's few tokens and the label.  So a row
// needs its maximum, one or two sums (of temperature tau for the soft term, of 1 for the hard
// one), and k gathered logits; then one pass writes multiples of q, and the few tokens are
// written once more with their whole value.
//
// A workgroup takes a row.  In the step it is read once and kept in registers (NV 16-byte
// vectors a thread) until its gradient is written, so HBM sees one read and one write; each
// wave sums against its own maximum, so that maximum and sums cross the workgroup together,
// behind one barrier.
#pragma once

#include "row_ops.hpp"
#include "zero_operators.h"

namespace zo {

enum DistillMode { kDistillStep, kDistillLoss, kDistillBack };

// What a call's rows share, computed on the host.
struct DistillScalars {
    float c, c1;         // log2(e) / temperature, log2(e)
    float soft_loss;     // soft * temperature^2 * ln 2: the loss of one bit of the sum
    float soft_grad;     // soft * temperature
    float hard;
    float scale;
};

constexpr int kMarkBits = 65536;  // tokens modulo this are marked to find those listed twice

template <int NT>
struct DistillLds {
    float wave_max[NT / 64], wave_sum[NT / 64], wave_sum1[NT / 64], wave_top[NT / 64];
    int32_t wave_any[NT / 64];
    int32_t twice, label_listed;
    int32_t token[ZERO_DISTILL_MAX_K];                       // -1: absent
    float z[ZERO_DISTILL_MAX_K], teacher[ZERO_DISTILL_MAX_K];  // the entries' logits, both sides'
    uint32_t marks[kMarkBits / 32];
};

__device__ __forceinline__ float any_f32(const void* p, int64_t i, int dtype) {
    return dtype == ZERO_F32   ? static_cast<const float*>(p)[i]
           : dtype == ZERO_F16 ? F16::to_f32(static_cast<const uint16_t*>(p)[i])
                               : BF16::to_f32(static_cast<const uint16_t*>(p)[i]);
}

// The exponents x = c (f - m) of terms 2^x summed against a maximum m.  binary16 values take one
// fused operation, c f - cm with cm = c m rounded once: its error is the same in every term and in
// their sum, so their quotients do not have it.  In the other types c times the lowest value
// leaves fp32's range, so there the difference comes first.  A row or wave of nothing but -inf
// is summed against 0.
template <typename T>
struct Against {
    static constexpr bool kFused = T::kLowest == F16::kLowest;
    float c, m, cm;
    __device__ __forceinline__ Against(float c_, float m_)
        : c(c_), m(m_ == -__builtin_inff() ? 0.f : m_), cm(c * m) {}
    __device__ __forceinline__ float operator()(float f) const {
        return kFused ? __builtin_fmaf(f, c, -cm) : (f - m) * c;
    }
    // A sum against `from`, taken against this, which is not less.  A sum of 0 is that of nothing but
    // -inf, which has no maximum to go by.
    __device__ __forceinline__ float moved(float sum, const Against& from) const {
        return sum == 0.f ? 0.f : sum * exp2_fast(kFused ? from.cm - cm : (from.m - m) * c);
    }
};

// How the soft and the hard term share the exponentials of an element.
enum DistillKind {
    kOneSum,   // one temperature: tau = 1, or one of the terms alone
    kSquare,   // tau = 2: 2^x of temperature 1 is the square of that of temperature 2
    kTwoSums,  // an exponential for each
};

// Keeps the packed row in its registers between two passes over it: without it the compiler holds
// the first pass's fp32 values for the second, at twice the registers or more.
__device__ __forceinline__ void keep_packed(u32x4& v) { asm volatile("" : "+v"(v)); }

// This thread's maximum of PER packed values.
template <typename T>
__device__ __forceinline__ float max_of(u32x4 v, float m) {
    if constexpr (T::kLowest == F16::kLowest) {
        typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
        const f16x8 h = __builtin_bit_cast(f16x8, v);
        const auto a = __builtin_elementwise_max(h.lo, h.hi);
        const auto b = __builtin_elementwise_max(a.lo, a.hi);
        return fmaxf(fmaxf(m, (float)b.x), (float)b.y);
    } else {
        float f[T::kPer];
        T::unpack(v, f);
#pragma unroll
        for (int j = 0; j < T::kPer; ++j)
            m = fmaxf(m, f[j]);
        return m;
    }
}

template <typename T, int KIND>
__device__ __forceinline__ void add_terms(u32x4 v, const Against<T>& x, const Against<T>& x1, float& s, float& s1) {
    float f[T::kPer];
    T::unpack(v, f);
#pragma unroll
    for (int j = 0; j < T::kPer; ++j) {
        const float e = exp2_fast(x(f[j]));
        s += e;
        if constexpr (KIND == kSquare)
            s1 = __builtin_fmaf(e, e, s1);
        if constexpr (KIND == kTwoSums)
            s1 += exp2_fast(x1(f[j]));
    }
}

// The gradient without the teacher's own terms: a 2^x + a1 2^x1.
template <typename T, int KIND>
__device__ __forceinline__ float share(float f, const Against<T>& x, const Against<T>& x1, float a, float a1) {
    const float e = exp2_fast(x(f));
    if constexpr (KIND == kSquare)
        return e * __builtin_fmaf(a1, e, a);
    if constexpr (KIND == kTwoSums)
        return __builtin_fmaf(a1, exp2_fast(x1(f)), a * e);
    return a * e;
}

template <typename T, int KIND>
__device__ __forceinline__ u32x4 share_of(u32x4 v, const Against<T>& x, const Against<T>& x1, float a, float a1) {
    float f[T::kPer];
    T::unpack(v, f);
#pragma unroll
    for (int j = 0; j < T::kPer; ++j)
        f[j] = share<T, KIND>(f[j], x, x1, a, a1);
    return T::pack(f);
}

// NV > 0: the row lies in the registers, NV vectors a thread; NV = 0: it is read as it is needed.
template <typename T, int NT, int NV, int MODE, int KIND>
__device__ __forceinline__ void distill_row(const zero_distill_args_t& a, const DistillScalars& k, DistillLds<NT>& lds,
                                            int64_t row, float weight, int label) {
    using elem = typename T::elem;
    constexpr int kPer = T::kPer, kWaves = NT / 64;
    constexpr bool kInRegisters = NV > 0;
    const int t = threadIdx.x, wave = t / 64, lane = t & 63, vocab = (int)a.vocab, entries = a.k;
    const float inf = __builtin_inff();
    const elem* z = static_cast<const elem*>(a.logits) + row * a.ld_logits;
    elem* dz = static_cast<elem*>(a.dlogits) + row * a.ld_dlogits;
    const bool has_label = label >= 0;

    // the row, on its way while the teacher's list is read
    u32x4 v[kInRegisters ? NV : 1];
    if constexpr (kInRegisters) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * NT) * kPer;
            v[i] = u32x4{T::kLowest, T::kLowest, T::kLowest, T::kLowest};
            if (c < vocab)
                v[i] = load_row<T>(z, c, vocab, T::kLowest);
        }
    }

    // the teacher's entries; `top` is their largest logit
    float top = -inf;
    bool any = false;
    for (int j = t; j < entries; j += NT) {
        const int token = a.teacher_index[row * entries + j];
        const float x = any_f32(a.teacher_logits, row * entries + j, a.teacher_dtype);
        const bool present = token >= 0 && token < vocab && x != -inf;
        lds.token[j] = present ? token : -1;
        lds.teacher[j] = x;
        lds.z[j] = present ? T::to_f32(z[token]) : 0.f;
        any |= present;
        if (present)
            top = fmaxf(top, x);  // a NaN loses here and counts in the sum
    }
    const float z_label = has_label ? T::to_f32(z[label]) : 0.f;
    if constexpr (MODE != kDistillLoss) {
        for (int i = t; i < kMarkBits / 32; i += NT)
            lds.marks[i] = 0;
        if (t == 0)
            lds.twice = lds.label_listed = 0;
    }

    // the row's maximum and sums, of this thread, then of its wave
    float m = -inf, s = 0.f, s1 = 0.f;
    if constexpr (MODE == kDistillBack) {
    } else if constexpr (kInRegisters) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            m = max_of<T>(v[i], m);
        m = seg_reduce<64>(m, Max());
        const Against<T> x(k.c, m), x1(k.c1, m);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            keep_packed(v[i]);
            add_terms<T, KIND>(v[i], x, x1, s, s1);
        }
    } else {
        for (int c = t * kPer; c < vocab; c += NT * kPer) {
            const u32x4 u = load_row<T>(z, c, vocab, T::kLowest);
            const float up = max_of<T>(u, m);
            const Against<T> x(k.c, up), x1(k.c1, up);
            if (up > m) {
                s = x.moved(s, Against<T>(k.c, m));
                s1 = x1.moved(s1, Against<T>(k.c1, m));
                m = up;
            }
            add_terms<T, KIND>(u, x, x1, s, s1);
        }
        const float up = seg_reduce<64>(m, Max());
        s = Against<T>(k.c, up).moved(s, Against<T>(k.c, m));
        s1 = Against<T>(k.c1, up).moved(s1, Against<T>(k.c1, m));
        m = up;
    }
    if constexpr (MODE != kDistillBack) {
        s = seg_reduce<64>(s, Add());
        s1 = KIND == kOneSum ? 0.f : seg_reduce<64>(s1, Add());
    }
    top = seg_reduce<64>(top, Max());
    any = __ballot(any) != 0;
    if (lane == 0) {
        lds.wave_max[wave] = m;
        lds.wave_sum[wave] = s;
        lds.wave_sum1[wave] = s1;
        lds.wave_top[wave] = top;
        lds.wave_any[wave] = any;
    }
    __syncthreads();

    // of the row: every wave for itself, a lane a wave
    const int w = lane % kWaves;
    top = seg_reduce<kWaves>(lds.wave_top[w], Max());
    const bool has_soft = k.soft_grad != 0.f && __ballot(lds.wave_any[w] != 0) != 0;
    if constexpr (MODE == kDistillBack) {
        m = a.stats[3 * row];
        s = a.stats[3 * row + 1];
        s1 = a.stats[3 * row + 2];
    } else {
        m = seg_reduce<kWaves>(lds.wave_max[w], Max());
    }
    const Against<T> x(k.c, m), x1(k.c1, m);
    if constexpr (MODE != kDistillBack) {
        const float wm = lds.wave_max[w];
        s = seg_reduce<kWaves>(x.moved(lds.wave_sum[w], Against<T>(k.c, wm)), Add());
        s1 = KIND == kOneSum ? s : seg_reduce<kWaves>(x1.moved(lds.wave_sum1[w], Against<T>(k.c1, wm)), Add());
        if (MODE == kDistillLoss && a.stats && t == 0) {
            a.stats[3 * row] = m;
            a.stats[3 * row + 1] = s;
            a.stats[3 * row + 2] = s1;
        }
    }

    // the teacher's softmax, by every wave for itself
    auto entry = [&](int j) { return (lds.teacher[j] - top) * k.c; };
    float sum = 0.f;
    if (has_soft)
        for (int j = lane; j < entries; j += 64)
            sum += lds.token[j] >= 0 ? exp2_fast(entry(j)) : 0.f;
    sum = seg_reduce<64>(sum, Add());
    const float over = has_soft ? 1.f / sum : 0.f;

    if constexpr (MODE != kDistillBack) {
        if (wave == 0) {
            float loss = 0.f;
            if (has_soft) {
                const float bits = log2_fast(s) - log2_fast(sum);
                for (int j = lane; j < entries; j += 64) {
                    const float p = lds.token[j] >= 0 ? exp2_fast(entry(j)) * over : 0.f;
                    if (p != 0.f)  // log2 p - log2 q
                        loss += p * ((entry(j) - x(lds.z[j])) + bits);
                }
                loss = seg_reduce<64>(loss, Add()) * k.soft_loss;
            }
            if (has_label) {
                // at temperature 1 kSquare has twice the exponent of temperature 2
                const float xl = KIND == kSquare ? 2.f * x(z_label) : KIND == kTwoSums ? x1(z_label) : x(z_label);
                loss += k.hard * 0.6931471805599453f * (log2_fast(s1) - xl);
            }
            if (lane == 0)
                a.loss[row] = weight * loss;
        }
    }

    if constexpr (MODE != kDistillLoss) {
        float up = weight * k.scale;
        if (MODE == kDistillBack && a.dloss)
            up *= a.dloss[row];
        const float soft_up = has_soft ? up * k.soft_grad : 0.f, hard_up = has_label ? up * k.hard : 0.f;
        float f = has_soft ? soft_up / s : 0.f, f1 = has_label ? hard_up / s1 : 0.f;
        if constexpr (KIND == kOneSum) {
            f += f1;
            f1 = 0.f;
        }
        if (!has_soft && !has_label) {  // no term: nothing of the row counts
            for (int c = t * kPer; c < vocab; c += NT * kPer)
                store_row<T>(dz, c, vocab, u32x4{0, 0, 0, 0});
            return;
        }
        for (int j = t; j < entries && has_soft; j += NT) {
            const int token = lds.token[j];
            if (token >= 0) {
                const uint32_t bit = 1u << (token & 31);
                if (atomicOr(&lds.marks[token % kMarkBits / 32], bit) & bit)
                    lds.twice = 1;
                if (token == label)
                    lds.label_listed = 1;
            }
        }
        if constexpr (kInRegisters) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * NT) * kPer;
                keep_packed(v[i]);
                if (c < vocab)
                    store_row<T>(dz, c, vocab, share_of<T, KIND>(v[i], x, x1, f, f1));
            }
        } else {
            for (int c = t * kPer; c < vocab; c += NT * kPer)
                store_row<T>(dz, c, vocab,
                             share_of<T, KIND>(load_row<T>(z, c, vocab, T::kLowest), x, x1, f, f1));
        }
        // the tokens with a term of their own, over what was just stored: the barrier orders the
        // workgroup's stores before these
        __syncthreads();
        if (has_soft) {
            const bool twice = lds.twice;
            for (int j = t; j < entries; j += NT) {
                const int token = lds.token[j];
                if (token < 0)
                    continue;
                float p = exp2_fast(entry(j));
                if (twice) {  // a token listed again: every one of its entries writes the whole sum
                    p = 0.f;
                    for (int i = 0; i < entries; ++i)
                        p += lds.token[i] == token ? exp2_fast(entry(i)) : 0.f;
                }
                const float own = soft_up * (p * over) + (token == label ? hard_up : 0.f);
                dz[token] = T::of_f32(share<T, KIND>(lds.z[j], x, x1, f, f1) - own);
            }
        }
        if (t == 0 && has_label && !(has_soft && lds.label_listed))
            dz[label] = T::of_f32(share<T, KIND>(z_label, x, x1, f, f1) - hard_up);
    }
}

template <typename T, int NT, int NV, int MODE>
__global__ __launch_bounds__(NT) void k_distill(const zero_distill_args_t a, const DistillScalars k,
                                               int64_t first) {
    __shared__ DistillLds<NT> lds;
    const int64_t row = first + blockIdx.x;
    const float weight = a.row_weight ? a.row_weight[row] : 1.f;
    int label = a.labels ? a.labels[row] : -1;
    if (weight == 0.f) {  // the row is not looked at
        if (MODE != kDistillBack && threadIdx.x == 0) {
            a.loss[row] = 0.f;
            if (MODE == kDistillLoss && a.stats)
                a.stats[3 * row] = a.stats[3 * row + 1] = a.stats[3 * row + 2] = 0.f;
        }
        if (MODE != kDistillLoss) {
            typename T::elem* dz = static_cast<typename T::elem*>(a.dlogits) + row * a.ld_dlogits;
            for (int c = threadIdx.x * T::kPer; c < (int)a.vocab; c += NT * T::kPer)
                store_row<T>(dz, c, (int)a.vocab, u32x4{0, 0, 0, 0});
        }
        return;
    }
    if (k.hard == 0.f || label >= a.vocab)
        label = -1;
    // the same for the whole workgroup
    if (label < 0 || k.c == k.c1)
        distill_row<T, NT, NV, MODE, kOneSum>(a, k, lds, row, weight, label);
    else if (2.f * k.c == k.c1)
        distill_row<T, NT, NV, MODE, kSquare>(a, k, lds, row, weight, label);
    else
        distill_row<T, NT, NV, MODE, kTwoSums>(a, k, lds, row, weight, label);
}

}  // namespace zo
