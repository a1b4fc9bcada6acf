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
    float wave_max[NT / 64], wave_sum[NT / 64], wave_sum1[NT / 64];
    float wave_top[NT / 64], wave_teacher[NT / 64], wave_loss[NT / 64];
    int32_t wave_any[NT / 64];
    int32_t twice, label_listed;
    int32_t token[ZERO_DISTILL_MAX_K];
    float z[ZERO_DISTILL_MAX_K], p[ZERO_DISTILL_MAX_K];
    uint32_t marks[kMarkBits / 32];
};

__device__ __forceinline__ float any_f32(const void* p, int64_t i, int dtype) {
    return dtype == ZERO_F32   ? static_cast<const float*>(p)[i]
           : dtype == ZERO_F16 ? F16::to_f32(static_cast<const uint16_t*>(p)[i])
                               : BF16::to_f32(static_cast<const uint16_t*>(p)[i]);
}

// A running maximum and the sums against it.
struct Running {
    float m, s, s1;
};

// The reference that values up to `m` are summed against: finite where m is -inf.
__device__ __forceinline__ float ref(float m) { return m == -__builtin_inff() ? 0.f : m; }

// What turns a sum against `from` into one against m >= from (a sum of nothing stays 0).
__device__ __forceinline__ float rescale(float from, float m, float c) {
    return m == -__builtin_inff() ? 0.f : exp2_fast((from - m) * c);
}

// The exponent c (f - m) - bits.  The difference comes first: c m would lose digits to a large
// maximum, and leaves fp32's range for the lowest value of bf16 and f32.
struct Exponent {
    float c, m, bits;
    __device__ __forceinline__ float operator()(float f) const { return __builtin_fmaf(f - m, c, -bits); }
};

template <typename T, int NT, int NV, int MODE>
__global__ __launch_bounds__(NT) void k_distill(const zero_distill_args_t a, const DistillScalars k,
                                               int64_t first) {
    using elem = typename T::elem;
    constexpr int kPer = T::kPer, kWaves = NT / 64;
    constexpr bool kInRegisters = NV > 0;
    __shared__ DistillLds<NT> lds;
    const int t = threadIdx.x, wave = t / 64, lane = t & 63, vocab = (int)a.vocab, entries = a.k;
    const int64_t row = first + blockIdx.x;
    const float inf = __builtin_inff();
    const elem* z = static_cast<const elem*>(a.logits) + row * a.ld_logits;
    elem* dz = static_cast<elem*>(a.dlogits) + row * a.ld_dlogits;
    const float weight = a.row_weight ? a.row_weight[row] : 1.f;
    const int label = a.labels ? a.labels[row] : -1;

    if (weight == 0.f) {  // the row is not looked at
        if (MODE != kDistillBack && t == 0) {
            a.loss[row] = 0.f;
            if (MODE == kDistillLoss && a.stats)
                a.stats[3 * row] = a.stats[3 * row + 1] = a.stats[3 * row + 2] = 0.f;
        }
        if (MODE != kDistillLoss)
            for (int c = t * kPer; c < vocab; c += NT * kPer)
                store_row<T>(dz, c, vocab, u32x4{0, 0, 0, 0});
        return;
    }
    const bool has_label = k.hard != 0.f && label >= 0 && label < vocab;
    const bool two = has_label && k.c != k.c1;  // the hard term has a sum of its own

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
        lds.p[j] = x;
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
    Running r{-inf, 0.f, 0.f};
    if constexpr (MODE == kDistillBack) {
    } else if constexpr (kInRegisters) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float f[kPer];
            T::unpack(v[i], f);
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                r.m = fmaxf(r.m, f[j]);
        }
        r.m = seg_reduce<64>(r.m, Max());
        const Exponent x{k.c, ref(r.m), 0.f}, x1{k.c1, ref(r.m), 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float f[kPer];
            T::unpack(v[i], f);
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                r.s += exp2_fast(x(f[j]));
            if (two) {
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    r.s1 += exp2_fast(x1(f[j]));
            }
        }
    } else {
        for (int c = t * kPer; c < vocab; c += NT * kPer) {
            float f[kPer];
            T::unpack(load_row<T>(z, c, vocab, T::kLowest), f);
            float m = r.m;
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                m = fmaxf(m, f[j]);
            if (m > r.m) {
                r.s *= rescale(r.m, m, k.c);
                r.s1 *= rescale(r.m, m, k.c1);
                r.m = m;
            }
            const Exponent x{k.c, ref(r.m), 0.f}, x1{k.c1, ref(r.m), 0.f};
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                r.s += exp2_fast(x(f[j]));
            if (two) {
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    r.s1 += exp2_fast(x1(f[j]));
            }
        }
        const float m = seg_reduce<64>(r.m, Max());
        r.s *= rescale(r.m, m, k.c);
        r.s1 *= rescale(r.m, m, k.c1);
        r.m = m;
    }
    r.s = seg_reduce<64>(r.s, Add());
    r.s1 = seg_reduce<64>(r.s1, Add());
    top = seg_reduce<64>(top, Max());
    if (lane == 0) {
        lds.wave_max[wave] = r.m;
        lds.wave_sum[wave] = r.s;
        lds.wave_sum1[wave] = r.s1;
        lds.wave_top[wave] = top;
    }
    const bool wave_any = __ballot(any) != 0;
    if (lane == 0)
        lds.wave_any[wave] = wave_any;
    __syncthreads();

    top = lds.wave_top[0];
    any = lds.wave_any[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
        top = fmaxf(top, lds.wave_top[w]);
        any |= lds.wave_any[w] != 0;
    }
    const bool has_soft = k.soft_grad != 0.f && any;
    float m, bits, bits1;  // the maximum, log2 of the sums
    if constexpr (MODE == kDistillBack) {
        m = a.stats[3 * row];
        bits = a.stats[3 * row + 1];
        bits1 = a.stats[3 * row + 2];
    } else {
        m = lds.wave_max[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w)
            m = fmaxf(m, lds.wave_max[w]);
        float s = 0.f, s1 = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            s += lds.wave_sum[w] * rescale(lds.wave_max[w], m, k.c);
            s1 += lds.wave_sum1[w] * rescale(lds.wave_max[w], m, k.c1);
        }
        bits = log2_fast(s);
        bits1 = two ? log2_fast(s1) : bits;
        if (MODE == kDistillLoss && a.stats && t == 0) {
            a.stats[3 * row] = m;
            a.stats[3 * row + 1] = bits;
            a.stats[3 * row + 2] = bits1;
        }
    }
    // log2 of q_tau and q_1
    const Exponent lq{k.c, m, bits}, lq1{k.c1, m, bits1};

    // the teacher's softmax, and what each entry adds to the loss, in bits
    float sum = 0.f;
    for (int j = t; j < entries; j += NT) {
        const int token = lds.token[j];
        const float e = token >= 0 && has_soft ? exp2_fast((lds.p[j] - top) * k.c) : 0.f;
        sum += e;
    }
    sum = seg_reduce<64>(sum, Add());
    if (lane == 0)
        lds.wave_teacher[wave] = sum;
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
        sum += lds.wave_teacher[w];
    const float over = has_soft ? 1.f / sum : 0.f, bits_teacher = has_soft ? log2_fast(sum) : 0.f;
    float loss = 0.f;
    for (int j = t; j < entries; j += NT) {
        const int token = lds.token[j];
        if (token < 0)
            continue;
        const float x = (lds.p[j] - top) * k.c;
        const float p = has_soft ? exp2_fast(x) * over : 0.f;
        if (p != 0.f)
            loss += p * ((x - bits_teacher) - lq(lds.z[j]));
        lds.p[j] = p;
        if (MODE != kDistillLoss && has_soft) {
            const uint32_t bit = 1u << (token & 31);
            if (atomicOr(&lds.marks[token % kMarkBits / 32], bit) & bit)
                lds.twice = 1;
            if (token == label && has_label)
                lds.label_listed = 1;
        }
    }
    if constexpr (MODE != kDistillBack) {
        loss = seg_reduce<64>(loss, Add());
        if (lane == 0)
            lds.wave_loss[wave] = loss;
    }
    __syncthreads();
    if constexpr (MODE != kDistillBack) {
        if (t == 0) {
            float l = 0.f;
            for (int w = 0; w < kWaves; ++w)
                l += lds.wave_loss[w];
            l = has_soft ? l * k.soft_loss : 0.f;
            if (has_label)
                l += k.hard * 0.6931471805599453f * -lq1(z_label);
            a.loss[row] = weight * l;
        }
    }

    if constexpr (MODE != kDistillLoss) {
        float up = weight * k.scale;
        if (MODE == kDistillBack && a.dloss)
            up *= a.dloss[row];
        // gradient = soft_up q_tau + hard_up q_1 - (the teacher's and the label's own)
        const float soft_up = has_soft ? up * k.soft_grad : 0.f, hard_up = has_label ? up * k.hard : 0.f;
        auto share = [&](float f) {
            float g = 0.f;
            if (has_soft)
                g = soft_up * exp2_fast(lq(f));
            if (has_label)
                g = __builtin_fmaf(hard_up, exp2_fast(lq1(f)), g);
            return g;
        };
        if constexpr (kInRegisters) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * NT) * kPer;
                if (c < vocab) {
                    float f[kPer];
                    T::unpack(v[i], f);
#pragma unroll
                    for (int j = 0; j < kPer; ++j)
                        f[j] = share(f[j]);
                    store_row<T>(dz, c, vocab, T::pack(f));
                }
            }
        } else {
            for (int c = t * kPer; c < vocab; c += NT * kPer) {
                float f[kPer];
                T::unpack(load_row<T>(z, c, vocab, T::kLowest), f);
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    f[j] = share(f[j]);
                store_row<T>(dz, c, vocab, T::pack(f));
            }
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
                float p = lds.p[j];
                if (twice) {  // a token listed again: every one of its entries writes the whole sum
                    p = 0.f;
                    for (int i = 0; i < entries; ++i)
                        p += lds.token[i] == token ? lds.p[i] : 0.f;
                }
                float g = share(lds.z[j]) - soft_up * p;
                if (has_label && token == label)
                    g -= hard_up;
                dz[token] = T::of_f32(g);
            }
        }
        if (t == 0 && has_label && !(has_soft && lds.label_listed))
            dz[label] = T::of_f32(share(z_label) - hard_up);
    }
}

}  // namespace zo
