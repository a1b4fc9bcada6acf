// distill_kernels.hpp -- distillation from a teacher's top logits: a row's loss and the
// gradient of its student logits.
//
// With c = log2(e) / tau and m the row's maximum, q_tau[v] = 2^(c z_v - c m) / S; the
// gradient is q's multiple but at the teacher's few tokens and the label.  So a row
// needs its maximum and one or two sums (of temperature tau for the soft term, of 1 for the hard
// one); then one pass writes multiples of q, less what the few tokens have of their own.
//
// A workgroup takes a row.  In the step it is read once and kept in registers (NV 16-byte
// vectors a thread) until its gradient is written, so HBM sees one read and one write; each
// wave sums against its own maximum, so that maximum and sums cross the workgroup together,
// behind one barrier.  The few tokens' logits are gathered while the row is on its way, and their
// values are written once more, whole, over what the row's pass has stored.  (Putting the vectors that
// hold a listed token aside in LDS and writing each value once takes longer: a look at a mark for
// every vector costs more than the few lines that are written twice; 4096 rows of 50304
// f16 with 64 entries 155 us in place of 144.)
//
// Bound by HBM, with the vector ALU not far behind: 4096 rows of 50257 f16, 64 entries, both terms,
// 143 us, 5.8 TB/s, the ALU busy for 0.69 of it.  With a second exponential an element (temperatures
// other than 1 and 2 with a hard term) 151, and up to 185 in calls that follow one another for longer
// than 1.5 ms, when the clock falls.  1024 of 131072 bf16 109 us, 5.0 TB/s: such a row leaves one
// workgroup a compute unit; 65536 of 2048 f16 114 us, 4.9; 2048 of 50257 f32 148, 5.6; the loss
// alone of 4096 of 50257 f16 72 us, 5.7.
#pragma once

#include "row_ops.hpp"
#include "zero_operators.h"

namespace zo {

enum DistillMode { kDistillStep, kDistillLoss, kDistillBack };

// What a call's rows share, computed on the host.
struct DistillScalars {
    float c, c1;         // log2(e) / temperature, log2(e)
    float bit;           // temperature * ln 2: one bit of a sum in units of the logits
    float soft_in, soft_out;  // factors of soft * temperature: of an entry's term, where below 1, or of their sum
    float soft_grad;     // soft * temperature
    float hard;
    float scale;
};

constexpr int kMaxEdges = zs::kLineBytes / 2 + 8;  // bound of Cut::edges

template <int NT>
struct DistillLds {
    float wave_max[NT / 64], wave_sum[NT / 64], wave_sum1[NT / 64], wave_top[NT / 64];
    int32_t wave_any[NT / 64];
};

// Dynamic LDS of a row of k entries and the label: tokens, both sides' logits, and where a gradient is
// written the chains in which an entry finds those of its own token: links, and `heads`, a power of two.
constexpr int64_t distill_lds_bytes(int k, int heads, int mode) {
    return 12 * (int64_t)(k + 1) + (mode == kDistillLoss ? 0 : 4 * (int64_t)(k + 1 + heads));
}

__device__ __forceinline__ float any_f32(const void* p, int64_t i, int dtype) {
    return dtype == ZERO_F32   ? static_cast<const float*>(p)[i]
           : dtype == ZERO_F16 ? F16::to_f32(static_cast<const uint16_t*>(p)[i])
                               : BF16::to_f32(static_cast<const uint16_t*>(p)[i]);
}

// The exponents x = c (f - m) of terms 2^x summed against a maximum m.  A row or wave of nothing
// but -inf is summed against 0.
//
// The 16-bit types take one fused operation, c f - cm, where cm = c m is rounded once.  That
// shifts every x of a row by the same amount (`shift`), which the quotients of terms and their sum
// do not have; `log_sum` takes it out.  The shift is small while cm is: from 2^20 on (logits
// no model has, but a row may hold nothing but the type's lowest value) neighbouring values
// of the type lie at least 2^9 apart in x, so a term is 1 or 0 whatever the scale, and a
// smaller c keeps cm at 2^20.  fp32 takes the difference first: its bytes leave the time for it.
template <typename T>
struct Against {
    static constexpr bool kFused = sizeof(typename T::elem) == 2;
    float c, m, cm;
    __device__ __forceinline__ Against(float c_, float m_)
        : c(c_), m(m_ == -__builtin_inff() ? 0.f : m_), cm(c * m) {
        if (kFused && fabsf(cm) >= 0x1p20f && fabsf(m) < __builtin_inff()) {
            c = 0x1p20f / fabsf(m);
            cm = c * m;
        }
    }
    __device__ __forceinline__ float operator()(float f) const {
        return kFused ? __builtin_fmaf(f, c, -cm) : (f - m) * c;
    }
    // A sum against `from`, taken against this, which is not less.  A sum of 0 is that of nothing but
    // -inf, which has no maximum to go by.
    __device__ __forceinline__ float moved(float sum, const Against& from) const {
        return sum == 0.f ? 0.f : sum * exp2_fast(kFused && c == from.c ? from.cm - cm : (from.m - m) * c);
    }
    // log2 of the sum of all terms without the shift, that is against m itself.
    __device__ __forceinline__ float log_sum(float sum) const {
        return log2_fast(sum) - (kFused ? (*this)(m) : 0.f);
    }
};

constexpr int kBatch = 4;  // vectors at a time of a row that is read as it is needed

// Whether a row goes past the caches: long ones, which do not come back (4096 of 50304 f16 144 us in place of 154, of
// 32000 96 in place of 104); the tokens' values, written after the rest of a row, find short rows' lines still
// in L2 (16384 of 8192: 110 us, 176 past it; 65536 of 2048: 114, 163).
constexpr bool past_caches(int threads, int vectors) { return vectors == 0 || threads * vectors > 1024; }

// How the soft and the hard term share the exponentials of an element.
enum DistillKind {
    kOneSum,   // one temperature: tau = 1, or one of the terms alone
    kSquare,   // tau = 2: 2^x of temperature 1 is the square of that of temperature 2
    kTwoSums,  // an exponential for each
};

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
__device__ __forceinline__ void add_term(float f, const Against<T>& x, const Against<T>& x1, float& s, float& s1) {
    const float e = exp2_fast(x(f));
    s += e;
    if constexpr (KIND == kSquare)
        s1 = __builtin_fmaf(e, e, s1);
    if constexpr (KIND == kTwoSums)
        s1 += exp2_fast(x1(f));
}

template <typename T, int KIND>
__device__ __forceinline__ void add_terms(u32x4 v, const Against<T>& x, const Against<T>& x1, float& s, float& s1) {
    float f[T::kPer];
    T::unpack(v, f);
#pragma unroll
    for (int j = 0; j < T::kPer; ++j)
        add_term<T, KIND>(f[j], x, x1, s, s1);
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
__device__ __forceinline__ void share_of(u32x4 v, const Against<T>& x, const Against<T>& x1, float a, float a1,
                                         float* g) {
    T::unpack(v, g);
#pragma unroll
    for (int j = 0; j < T::kPer; ++j)
        g[j] = share<T, KIND>(g[j], x, x1, a, a1);
}

// NV > 0: the row lies in the registers, NV vectors a thread; NV = 0: it is read as it is needed.
template <typename T, int NT, int NV, int MODE, int KIND>
__device__ __forceinline__ void distill_row(const zero_distill_args_t& a, const DistillScalars& k, DistillLds<NT>& lds,
                                            int heads, int64_t row, float weight, int label) {
    using elem = typename T::elem;
    constexpr int kPer = T::kPer, kWaves = NT / 64;
    constexpr bool kInRegisters = NV > 0;
    constexpr bool kPast = past_caches(NT, NV);
    static_assert(NT >= kMaxEdges, "a thread for each edge element");
    const int t = threadIdx.x, wave = t / 64, lane = t & 63, vocab = (int)a.vocab, entries = a.k;
    const float inf = __builtin_inff();
    const elem* z = static_cast<const elem*>(a.logits) + row * a.ld_logits;
    elem* dz = static_cast<elem*>(a.dlogits) + row * a.ld_dlogits;
    const bool has_label = label >= 0;
    // entry `entries` is the label
    const int all = entries + 1;
    extern __shared__ int32_t room[];
    int32_t* const token_of = room;  // -1: absent
    float* const teacher_of = reinterpret_cast<float*>(room + all);
    float* const z_of = reinterpret_cast<float*>(room + 2 * all);
    int32_t* const next_of = room + 3 * all;
    int32_t* const head_of = room + 4 * all;
    // vectors begin at a line of the row that is written (or read), so that a wave's accesses are whole
    // lines wherever a row starts (a vocabulary of 50257 has rows at every place of a line)
    const Cut<T> cut(MODE == kDistillLoss ? z : dz, vocab);
    const elem* zv = z + cut.head;

    // the first of the teacher's entries, then the row, so that the list is there before it
    int token = -1;
    float x_teacher = 0.f;
    if (t < entries) {
        token = a.teacher_index[row * entries + t];
        x_teacher = any_f32(a.teacher_logits, row * entries + t, a.teacher_dtype);
    } else if (t == entries) {
        token = label;
    }
    u32x4 v[kInRegisters ? NV : 1];
    if constexpr (kInRegisters) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int n = t + i * NT;
            v[i] = u32x4{T::kLowest, T::kLowest, T::kLowest, T::kLowest};
            if (n < cut.vectors)
                v[i] = load_vec<T, kPast>(zv + n * kPer);
        }
    }
    const bool has_edge = t < cut.edges;
    const int edge_column = cut.edge_column(t);
    const float edge = has_edge ? T::to_f32(z[edge_column]) : -inf;

    if constexpr (MODE != kDistillLoss)
        for (int i = t; i < heads; i += NT)
            head_of[i] = -1;
    float top = -inf;  // the teacher's largest logit
    bool any = false;
    for (int j = t; j < all; j += NT) {
        if (j != t) {
            token = j < entries ? a.teacher_index[row * entries + j] : label;
            x_teacher = j < entries ? any_f32(a.teacher_logits, row * entries + j, a.teacher_dtype) : 0.f;
        }
        const bool present = token >= 0 && token < vocab && x_teacher != -inf;
        token_of[j] = present ? token : -1;
        teacher_of[j] = x_teacher;
        z_of[j] = present ? T::to_f32(z[token]) : 0.f;
        if (present && j < entries) {
            any = true;
            top = fmaxf(top, x_teacher);  // a NaN loses here and counts in the sum
        }
    }

    // the row's maximum and sums, of this thread, then of its wave
    float m = edge, s = 0.f, s1 = 0.f;
    if constexpr (MODE == kDistillBack) {
        // both are in the statistics
    } else if constexpr (kInRegisters) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            m = max_of<T>(v[i], m);
        m = seg_reduce<64>(m, Max());
        const Against<T> x(k.c, m), x1(k.c1, m);
        add_term<T, KIND>(edge, x, x1, s, s1);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            keep_packed(v[i]);
            add_terms<T, KIND>(v[i], x, x1, s, s1);
        }
    } else {
        {
            m = edge == edge ? edge : -inf;
            const Against<T> x(k.c, m), x1(k.c1, m);
            add_term<T, KIND>(edge, x, x1, s, s1);
        }
        for (int n0 = t; n0 < cut.vectors; n0 += kBatch * NT) {
            u32x4 u[kBatch];
            float up = m;
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                u[i] = u32x4{T::kLowest, T::kLowest, T::kLowest, T::kLowest};
                if (n0 + i * NT < cut.vectors)
                    u[i] = load_vec<T, false>(zv + (n0 + i * NT) * kPer);
            }
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                up = max_of<T>(u[i], up);
            const Against<T> x(k.c, up), x1(k.c1, up);
            if (up > m) {
                s = x.moved(s, Against<T>(k.c, m));
                s1 = x1.moved(s1, Against<T>(k.c1, m));
                m = up;
            }
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                keep_packed(u[i]);
                add_terms<T, KIND>(u[i], x, x1, s, s1);
            }
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

    // the teacher's softmax, by every wave for itself: `sum` is of 2^exponent_of
    auto exponent_of = [&](int j) { return (teacher_of[j] - top) * k.c; };
    float sum = 0.f;
    if (has_soft)
        for (int j = lane; j < entries; j += 64)
            sum += token_of[j] >= 0 ? exp2_fast(exponent_of(j)) : 0.f;
    sum = seg_reduce<64>(sum, Add());
    const float over = has_soft ? 1.f / sum : 0.f;

    // log p_j - log q_tau[token_j] = ((t_j - top) - (z_j - m) + tau ln 2 (log2 S - log2 sum)) / tau, so with
    // tau^2 before it a term is a difference of logits (and a few bits of the sums) times tau: nothing in it
    // leaves fp32 before the loss does, whatever the temperature and also where the student holds the
    // type's lowest value.
    if constexpr (MODE != kDistillBack) {
        if (wave == 0) {
            const float bits = k.bit * (x.log_sum(s) - log2_fast(sum));
            // temperature 1; kSquare's sum has twice the exponents of temperature 2, its shift too
            const float shift = Against<T>::kFused && KIND == kSquare ? 2.f * x(m) - x1(m) : 0.f;
            const float nats = 0.6931471805599453f * (x1.log_sum(s1) - shift);
            float soft = 0.f, hard = 0.f;
            for (int j = lane; j < all; j += 64) {
                if (token_of[j] < 0)
                    continue;
                const float below = x.m - z_of[j];
                if (j == entries) {
                    hard = k.hard * (below + nats);
                } else if (has_soft) {
                    const float p = exp2_fast(exponent_of(j)) * over;
                    if (p != 0.f)
                        soft += p * (k.soft_in * ((teacher_of[j] - top) + below + bits));
                }
            }
            soft = seg_reduce<64>(soft, Add());
            hard = seg_reduce<64>(hard, Add());
            if (lane == 0)
                a.loss[row] = weight * ((has_soft ? k.soft_out * soft : 0.f) + hard);
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
        const bool blank = !has_soft && !has_label;  // no term: nothing of the row counts
        for (int j = t; j < all; j += NT)
            if (token_of[j] >= 0)
                next_of[j] = atomicExch(&head_of[token_of[j] & (heads - 1)], j);

        auto write = [&](u32x4 u, int n) __attribute__((always_inline)) {
            float g[kPer] = {};
            if (!blank)
                share_of<T, KIND>(u, x, x1, f, f1, g);
            store_vec<T, kPast>(dz + cut.head + n * kPer, T::pack(g));
        };
        if constexpr (kInRegisters) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                keep_packed(v[i]);
                if (t + i * NT < cut.vectors)
                    write(v[i], t + i * NT);
            }
        } else {
            for (int n0 = t; n0 < cut.vectors; n0 += kBatch * NT) {
                u32x4 u[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; ++i)
                    if (n0 + i * NT < cut.vectors)
                        u[i] = load_vec<T, kPast>(zv + (n0 + i * NT) * kPer);
#pragma unroll
                for (int i = 0; i < kBatch; ++i)
                    if (n0 + i * NT < cut.vectors)
                        write(u[i], n0 + i * NT);
            }
        }
        if (has_edge)
            dz[edge_column] = T::of_f32(blank ? 0.f : share<T, KIND>(edge, x, x1, f, f1));

        // The tokens with a term of their own, over what was just stored: the barrier orders the
        // workgroup's stores before these.  The first entry of a token writes for all of them.
        __syncthreads();
        auto own_of = [&](int j) {
            return j == entries ? hard_up : has_soft ? soft_up * (exp2_fast(exponent_of(j)) * over) : 0.f;
        };
        for (int j = t; j < all && !blank; j += NT) {
            const int mine = token_of[j];
            if (mine < 0)
                continue;
            int n = 0, first = j, last = j;  // the token's entries
            for (int i = head_of[mine & (heads - 1)]; i >= 0; i = next_of[i])
                if (token_of[i] == mine) {
                    ++n;
                    first = i < first ? i : first;
                    last = i > last ? i : last;
                }
            if (first != j)
                continue;
            float g = share<T, KIND>(z_of[j], x, x1, f, f1) - own_of(j);
            if (n == 2)
                g -= own_of(last);
            else if (n > 2)  // in the entries' order, not the chain's
                for (int i = j + 1; i < all; ++i)
                    g -= token_of[i] == mine ? own_of(i) : 0.f;
            dz[mine] = T::of_f32(g);
        }
    }

}

// Waves a SIMD: all eight while the packed row leaves room in 64 registers, six of short workgroups with eight vectors
// a thread (at eight they spill: 8192 rows of 11093 bf16 74 us in place of 72), and one workgroup of 1024 a
// compute unit above that.
template <typename T, int NT, int NV, int MODE>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(NV <= 7 ? 8 : NT < 1024 ? 6 : 4))) void k_distill(
    const zero_distill_args_t a, const DistillScalars k, int heads, int64_t first) {
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
            const Cut<T> cut(dz, (int)a.vocab);
            for (int n = threadIdx.x; n < cut.vectors; n += NT)
                store_vec<T, past_caches(NT, NV)>(dz + cut.head + n * T::kPer, u32x4{0, 0, 0, 0});
            if ((int)threadIdx.x < cut.edges)
                dz[cut.edge_column(threadIdx.x)] = T::of_f32(0.f);
        }
        return;
    }
    if (k.hard == 0.f || label >= a.vocab || label < 0)
        label = -1;
    // the same for the whole workgroup
    if (label < 0 || k.c == k.c1)
        distill_row<T, NT, NV, MODE, kOneSum>(a, k, lds, heads, row, weight, label);
    else if (2.f * k.c == k.c1)
        distill_row<T, NT, NV, MODE, kSquare>(a, k, lds, heads, row, weight, label);
    else
        distill_row<T, NT, NV, MODE, kTwoSums>(a, k, lds, heads, row, weight, label);
}

}  // namespace zo
