// log_prob_kernels.hpp -- log probabilities of given tokens, the entropy and the likeliest tokens of a
// row of logits, and the gradient of the logits.
//
// With x_v = log2(e) (z_v - m) / temperature, m the row's maximum, S = sum of 2^x and U = sum of 2^x x:
//   log p_v = (z_v - m) / temperature - ln S,   entropy = ln 2 (log2 S - U / S),
// both terms of the entropy without cancellation (x <= 0).  The difference is taken before the product, in
// every type: the maximum's own term is then 1 to the bit, so S >= 1, no log probability is above 0 and a
// certain token has 0.
//
// The list: the threads' elements are groups (or their vectors are, for long lists), and the k-th largest of the
// groups' maxima is no more than the k-th largest logit, so only logits from there on can be listed: little more
// than k of them unless they lie close together in the row.  A bound just below it comes from a histogram of the
// maxima's distances from the row's maximum; the threads whose own maximum is above it read their vectors again
// and queue those with such logits, which a thread for each of their elements lists.  An entry's place is the
// number of entries above it.  Where too many are listed for that (rows of equal values), the k-th (logit, token)
// itself is found, eight bits at a time.
#pragma once

#include "row_ops.hpp"
#include "zero_operators.h"

namespace zo {

struct LogProbScalars {
    float c;        // log2(e) / temperature
    float inverse;  // 1 / temperature
    float scale;    // grad_scale / temperature
};

constexpr float kLn2 = 0.6931471805599453f;

// x of a term that counts: 2^x is 0 from -150 on, and a product with x is to be 0 there too.
__device__ __forceinline__ float bounded(float x) { return fmaxf(x, -1000.f); }

// The exponents x = c (f - m) against a maximum m; a row or wave of nothing but -inf is summed against 0.
struct Exponent {
    float c, m;
    __device__ __forceinline__ Exponent(float c_, float m_) : c(c_), m(m_ == -__builtin_inff() ? 0.f : m_) {}
    __device__ __forceinline__ float operator()(float f) const { return (f - m) * c; }
};

__device__ __forceinline__ void add_term(float f, const Exponent& x, float& s, float& u) {
    const float d = x(f), e = exp2_fast(d);
    s += e;
    u = __builtin_fmaf(e, bounded(d), u);
}

// Sums s and u against the maximum `from`, taken against `to`, which is not less.
__device__ __forceinline__ void move_sums(const Exponent& to, float from, float& s, float& u) {
    const float d = bounded(to(Exponent(to.c, from).m)), f = exp2_fast(d);
    u = s == 0.f ? 0.f : f * __builtin_fmaf(d, s, u);
    s = s == 0.f ? 0.f : f * s;
}

// A thread's sums of a long row, in 64 bits: s and u hold those of the latest kVectors vectors, so that a row of any
// length has no more than 512 roundings to 32 bits in turn (without, a row of 2^26 logits of two values 1 apart, 2^16
// terms a thread, had a sum that was off by 3e-4).
struct LongSums {
    static constexpr int kVectors = 64;
    double s = 0.0, u = 0.0;
    int held = 0;
    // As move_sums.
    __device__ __forceinline__ void move(const Exponent& to, float from) {
        if (s == 0.0)
            return;
        const float d = bounded(to(Exponent(to.c, from).m)), f = exp2_fast(d);
        u = (double)f * ((double)d * s + u);
        s = (double)f * s;
    }
    __device__ __forceinline__ void fold(float& s32, float& u32) {
        if (++held == kVectors) {
            s += (double)s32;
            u += (double)u32;
            s32 = u32 = 0.f;
            held = 0;
        }
    }
    __device__ __forceinline__ void join(float& s32, float& u32) const {
        s32 = (float)(s + (double)s32);
        u32 = (float)(u + (double)u32);
    }
};

// (a - b) / temperature without leaving fp32 on the way.
__device__ __forceinline__ float scaled_difference(float a, float b, float inverse) {
    return 2.f * ((0.5f * a - 0.5f * b) * inverse);
}

// A logit as a number of the same order; 0 for what is not listed.  -0 is 0.
__device__ __forceinline__ uint32_t key_of(float f) {
    const uint32_t u = __builtin_bit_cast(uint32_t, f + 0.f);
    return f > -__builtin_inff() ? (u >> 31 ? ~u : u | 0x80000000u) : 0u;
}
__device__ __forceinline__ float of_key(uint32_t k) {
    return __builtin_bit_cast(float, k >> 31 ? k & 0x7FFFFFFFu : ~k);
}

// The order of the list as one number: larger logits first, then lower tokens.
__device__ __forceinline__ uint64_t entry_of(uint32_t key, int token) {
    return (uint64_t)key << 32 | (uint32_t)~token;
}

// A row in a workgroup: NV vectors a thread in registers, or (NV = 0) read as it is needed, and its edges.
template <typename T, int NT, int NV>
struct LogitRow {
    static constexpr int kPer = T::kPer, kBatch = NV > 0 ? NV : 4;
    const typename T::elem* zv;
    Cut<T> cut;
    u32x4 v[NV > 0 ? NV : 1];
    float edge;
    int edge_column;
    __device__ __forceinline__ LogitRow(const typename T::elem* z, int vocab) : zv(z), cut(z, vocab) {
        zv += cut.head;
        if constexpr (NV > 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                v[i] = vector(threadIdx.x + i * NT);
        }
        edge_column = cut.edge_column(threadIdx.x);
        edge = (int)threadIdx.x < cut.edges ? T::to_f32(z[edge_column]) : -__builtin_inff();
    }
    __device__ __forceinline__ u32x4 vector(int n) const {
        u32x4 u = {T::kLowest, T::kLowest, T::kLowest, T::kLowest};
        if (n < cut.vectors)
            u = load_vec<T, false>(zv + n * kPer);
        return u;
    }
    // f(vector, its first column), of all vectors
    template <typename F>
    __device__ __forceinline__ void each(F f) {
        if constexpr (NV > 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                keep_packed(v[i]);
                f(v[i], cut.head + ((int)threadIdx.x + i * NT) * kPer);
            }
        } else {
            for (int n0 = threadIdx.x; n0 < cut.vectors; n0 += kBatch * NT) {
                u32x4 u[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; ++i)
                    u[i] = vector(n0 + i * NT);
#pragma unroll
                for (int i = 0; i < kBatch; ++i)
                    f(u[i], cut.head + (n0 + i * NT) * kPer);
            }
        }
    }
    // the same, from memory
    template <typename F>
    __device__ __forceinline__ void each_again(F f) const {
        constexpr int kAgain = 8;
        for (int n0 = threadIdx.x; n0 < cut.vectors; n0 += kAgain * NT) {
            u32x4 u[kAgain];
#pragma unroll
            for (int i = 0; i < kAgain; ++i)
                u[i] = vector(n0 + i * NT);
#pragma unroll
            for (int i = 0; i < kAgain; ++i)
                f(u[i], cut.head + (n0 + i * NT) * kPer);
        }
    }
};

constexpr int kDistanceBins = 512, kDigitBins = 256;

template <int NT>
struct LogProbLds {
    float wave_max[NT / 64], wave_sum[NT / 64], wave_u[NT / 64];
    __attribute__((aligned(16))) uint32_t bins[kDistanceBins];
    uint32_t listed, queued;
};

// The bin of a distance from the maximum, a sixteenth of an octave from 2^-12 to 2^20, those beyond in the first
// and the last.
constexpr int kFirstBin = (127 - 12) << 4;
__device__ __forceinline__ int distance_bin(float d) {
    const int b = (int)(__builtin_bit_cast(uint32_t, d) >> 19) - kFirstBin;
    return b < 0 ? 0 : b < kDistanceBins ? b : kDistanceBins - 1;
}
// The least distance that lies in no bin up to b.
__device__ __forceinline__ float beyond_bin(int b) {
    return b >= kDistanceBins - 1 ? __builtin_inff() : __builtin_bit_cast(float, (uint32_t)(b + 1 + kFirstBin) << 19);
}

// The first of COUNT bins (in the order of their number, or from the last down) up to which there are at least
// `want` entries, -1: there are fewer.  before: entries in the bins before it, here: in it.  Every wave finds the
// same.
template <int COUNT, bool DOWN>
__device__ __forceinline__ int bin_reaching(const uint32_t* bins, uint32_t want, uint32_t& before, uint32_t& here) {
    constexpr int kPer = COUNT / 64;
    const int lane = threadIdx.x & 63;
    uint32_t n[kPer], all = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        n[j] = bins[DOWN ? COUNT - 1 - (lane * kPer + j) : lane * kPer + j];
        all += n[j];
    }
    uint32_t upto = all;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t o = __shfl_up(upto, d);
        upto += lane >= d ? o : 0;
    }
    const uint64_t reached = __ballot(upto >= want);
    if (!reached)
        return -1;
    uint32_t sum = upto - all, mine = 0;
    int at = -1;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        if (at < 0 && sum + n[j] >= want) {
            at = lane * kPer + j;
            mine = n[j];
        }
        sum += at < 0 ? n[j] : 0;
    }
    const int l = __ffsll((unsigned long long)reached) - 1;
    before = __shfl(sum, l);
    here = __shfl(mine, l);
    at = __shfl(at, l);
    return DOWN ? COUNT - 1 - at : at;
}

// One more in a bin, for the lanes that come here; lanes of a wave that mean the same bin add together.
__device__ __forceinline__ void count_in(uint32_t* bins, int bin) {
    const int first = __builtin_amdgcn_readfirstlane(bin);
    const uint64_t here = __ballot(true);
    if (__ballot(bin == first) == here) {
        if ((threadIdx.x & 63) == __ffsll((unsigned long long)here) - 1)
            atomicAdd(bins + first, (uint32_t)__popcll(here));
    } else {
        atomicAdd(bins + bin, 1u);
    }
}

// The likeliest k tokens of a row, into `entries` in no order; returns how many.  most: the maximum of this
// thread's logits, m: of the row's.  The bins are zero and no entry is listed.
template <typename T, int NT, int NV>
__device__ __forceinline__ int find_top(const LogitRow<T, NT, NV>& row, const typename T::elem* z, float most, float m, int k,
                                        uint64_t* entries, int capacity, LogProbLds<NT>& lds) {
    const int t = threadIdx.x;
    const float inf = __builtin_inff();
    int32_t* const queue = reinterpret_cast<int32_t*>(entries + capacity);  // first columns of vectors
    auto list = [&](float f, int token) __attribute__((always_inline)) {
        const uint32_t at = atomicAdd(&lds.listed, 1u);
        if (at < (uint32_t)capacity)
            entries[at] = entry_of(key_of(f), token);
    };
    if (m == -inf)  // nothing but -inf and NaN
        return 0;
    int n = capacity + 1;
    if (m < inf) {
        auto add = [&](float f) __attribute__((always_inline)) {
            if (f > -inf)
                atomicAdd(lds.bins + distance_bin(m - f), 1u);
        };
        const bool by_thread = k <= NT / 4;
        if (by_thread) {
            add(most);
        } else {
            row.each_again([&](u32x4 u, int) __attribute__((always_inline)) { add(max_of<T>(u, -inf)); });
            if (t < row.cut.edges)
                add(row.edge);
        }
        __syncthreads();
        uint32_t before = 0, here = 0;
        const int bin = bin_reaching<kDistanceBins, false>(lds.bins, (uint32_t)k, before, here);
        const float beyond = beyond_bin(bin < 0 ? kDistanceBins - 1 : bin);
        auto counts = [&](float f) { return beyond < inf ? m - f < beyond : f > -inf; };
        if (counts(most)) {
            row.each_again([&](u32x4 u, int column) __attribute__((always_inline)) {
                if (counts(max_of<T>(u, -inf))) {
                    const uint32_t at = atomicAdd(&lds.queued, 1u);
                    if (at < (uint32_t)capacity)
                        queue[at] = column;
                }
            });
            if (t < row.cut.edges && counts(row.edge))
                list(row.edge, row.edge_column);
        }
        __syncthreads();
        const int queued = (int)lds.queued;
        if (queued <= capacity) {
            for (int i = t; i < queued * T::kPer; i += NT) {
                const int column = queue[i / T::kPer] + i % T::kPer;
                const float f = T::to_f32(z[column]);
                if (counts(f))
                    list(f, column);
            }
            __syncthreads();
            n = (int)lds.listed;
        }
    }
    if (n <= capacity)
        return n;
    // the k-th entry itself, from its highest digit down, or what is left of it where all entries with these
    // digits are listed
    auto each = [&](auto f) __attribute__((always_inline)) {
        row.each_again([&](u32x4 u, int column) __attribute__((always_inline)) {
            float v[T::kPer];
            T::unpack(u, v);
#pragma unroll
            for (int j = 0; j < T::kPer; ++j)
                if (v[j] > -inf)
                    f(v[j], column + j);
        });
        if (t < row.cut.edges && row.edge > -inf)
            f(row.edge, row.edge_column);
    };
    uint64_t bound = 0;
    uint32_t want = (uint32_t)k;
    for (int shift = 56; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = t; i < kDigitBins; i += NT)
            lds.bins[i] = 0;
        __syncthreads();
        each([&](float f, int token) __attribute__((always_inline)) {
            const uint64_t e = entry_of(key_of(f), token) ^ bound;
            if (shift == 56 || e >> (shift + 8 & 63) == 0)
                count_in(lds.bins, (int)(e >> shift & 255));
        });
        __syncthreads();
        uint32_t before = 0, here = 0;
        const int digit = bin_reaching<kDigitBins, true>(lds.bins, want, before, here);
        if (digit < 0)  // fewer than k in all
            break;
        want -= before;
        bound |= (uint64_t)digit << shift;
        if (here == want)
            break;
    }
    __syncthreads();
    if (t == 0)
        lds.listed = 0;
    __syncthreads();
    each([&](float f, int token) __attribute__((always_inline)) {
        if (entry_of(key_of(f), token) >= bound)
            list(f, token);
    });
    __syncthreads();
    return (int)lds.listed;
}

template <typename T, int NT, int NV, bool TOP>
__global__ __launch_bounds__(NT) void k_log_probs(const zero_log_probs_args_t a, const LogProbScalars k, int capacity,
                                                  int64_t first) {
    __shared__ LogProbLds<NT> lds;
    extern __shared__ __attribute__((aligned(16))) uint64_t entries[];
    constexpr int kWaves = NT / 64;
    const int64_t at = first + blockIdx.x;
    const int t = threadIdx.x, wave = t / 64, lane = t & 63, vocab = (int)a.vocab;
    const float inf = __builtin_inff();
    const typename T::elem* const z = static_cast<const typename T::elem*>(a.logits) + at * a.ld_logits;
    if constexpr (TOP) {
        for (int i = t; i < kDistanceBins; i += NT)
            lds.bins[i] = 0;
        if (t == 0)
            lds.listed = lds.queued = 0;
    }
    int token = -1;
    float z_token = 0.f;
    if (a.logp && t == 0) {
        token = a.tokens[at];
        if (token >= 0 && token < vocab)
            z_token = T::to_f32(z[token]);
    }
    LogitRow<T, NT, NV> row(z, vocab);
    float most = row.edge, s = 0.f, u = 0.f, m;
    if constexpr (NV > 0) {
        row.each([&](u32x4 v, int) __attribute__((always_inline)) { most = max_of<T>(v, most); });
        m = seg_reduce<64>(most, Max());
        const Exponent x(k.c, m);
        add_term(row.edge, x, s, u);
        row.each([&](u32x4 v, int) __attribute__((always_inline)) {
            float f[T::kPer];
            T::unpack(v, f);
#pragma unroll
            for (int j = 0; j < T::kPer; ++j)
                add_term(f[j], x, s, u);
        });
    } else {
        m = row.edge == row.edge ? row.edge : -inf;
        add_term(row.edge, Exponent(k.c, m), s, u);
        LongSums sums;
        row.each([&](u32x4 v, int) __attribute__((always_inline)) {
            const float up = max_of<T>(v, m);
            const Exponent x(k.c, up);
            if (up > m) {
                sums.move(x, m);
                move_sums(x, m, s, u);
                m = up;
            }
            float f[T::kPer];
            T::unpack(v, f);
#pragma unroll
            for (int j = 0; j < T::kPer; ++j)
                add_term(f[j], x, s, u);
            sums.fold(s, u);
        });
        sums.join(s, u);
        most = m;
        m = seg_reduce<64>(most, Max());
        move_sums(Exponent(k.c, m), most, s, u);
    }
    s = seg_reduce<64>(s, Add());
    u = seg_reduce<64>(u, Add());
    if (lane == 0) {
        lds.wave_max[wave] = m;
        lds.wave_sum[wave] = s;
        lds.wave_u[wave] = u;
    }
    __syncthreads();
    const int w = lane % kWaves;
    const float wm = lds.wave_max[w];
    s = lds.wave_sum[w];
    u = lds.wave_u[w];
    m = seg_reduce<kWaves>(wm, Max());
    const Exponent x(k.c, m);
    move_sums(x, wm, s, u);
    s = seg_reduce<kWaves>(s, Add());
    u = seg_reduce<kWaves>(u, Add());
    // a row of nothing but -inf; one of nothing but NaN has that maximum too, and a NaN for its sum
    const bool empty = m == -inf && s == 0.f;
    const float log_sum = kLn2 * log2_fast(s);
    auto log_p = [&](float f) { return empty ? -inf : scaled_difference(f, m, k.inverse) - log_sum; };
    if (t == 0) {
        const float entropy = empty ? 0.f : kLn2 * (log2_fast(s) - u / s);
        if (a.logp)
            a.logp[at] = token >= 0 && token < vocab ? log_p(z_token) : 0.f;
        if (a.entropy)
            a.entropy[at] = entropy;
        if (a.stats) {
            a.stats[3 * at] = m;
            a.stats[3 * at + 1] = s;
            a.stats[3 * at + 2] = entropy;
        }
    }
    if constexpr (TOP) {
        const int n = find_top<T, NT, NV>(row, z, most, m, a.k, entries, capacity, lds);
        int32_t* const index = a.top_index + at * a.k;
        float* const lp = a.top_logp + at * a.k;
        // an entry's place is the number of those above it, counted by kShare threads
        constexpr int kShare = 4;
        for (int i0 = 0; i0 < n; i0 += NT / kShare) {
            const int i = i0 + t / kShare, part = t % kShare;
            const uint64_t e = entries[i < n ? i : n - 1];
            int place = 0;
#pragma unroll 8
            for (int j = part; j < n; j += kShare)
                place += entries[j] > e ? 1 : 0;
            place = seg_reduce<kShare>(place, [](int p, int q) { return p + q; });
            if (part == 0 && i < n && place < a.k) {
                index[place] = (int32_t)~(uint32_t)e;
                lp[place] = log_p(of_key((uint32_t)(e >> 32)));
            }
        }
        for (int i = n + t; i < a.k; i += NT) {
            index[i] = -1;
            lp[i] = -inf;
        }
    }
}

// The gradient: dlogits_v = scale (dlogp [v = token] + p_v (b x_v + a)) with the row's numbers folded into a and b,
// a workgroup for a piece of a row, which is cut at the lines of the row written.
constexpr int kLogpBackBlock = 256, kLogpBackVectors = 4;

template <typename T>
__global__ __launch_bounds__(kLogpBackBlock) void k_log_probs_back(const zero_log_probs_backward_args_t a,
                                                                   const LogProbScalars k, int pieces, int64_t first) {
    using elem = typename T::elem;
    constexpr int kPer = T::kPer;
    const int64_t id = first + blockIdx.x, at = id / pieces;
    const int piece = (int)(id - at * pieces), t = threadIdx.x, vocab = (int)a.vocab;
    const elem* const z = static_cast<const elem*>(a.logits) + at * a.ld_logits;
    elem* const dz = static_cast<elem*>(a.dlogits) + at * a.ld_dlogits;
    const Cut<T> cut(dz, vocab);
    const int n0 = piece * kLogpBackBlock * kLogpBackVectors + t;
    u32x4 v[kLogpBackVectors];
#pragma unroll
    for (int i = 0; i < kLogpBackVectors; ++i)
        if (n0 + i * kLogpBackBlock < cut.vectors)
            v[i] = load_vec<T, false>(z + cut.head + (n0 + i * kLogpBackBlock) * kPer);
    const bool has_edge = piece == 0 && t < cut.edges;
    const int edge_column = cut.edge_column(t);
    const float edge = has_edge ? T::to_f32(z[edge_column]) : 0.f;

    const float m = a.stats[3 * at], s = a.stats[3 * at + 1], entropy = a.stats[3 * at + 2];
    int token = a.dlogp ? a.tokens[at] : -1;
    token = token >= 0 && token < vocab ? token : -1;
    const bool empty = m == -__builtin_inff() && s == 0.f;
    const Exponent x(k.c, m);
    const float up = token >= 0 ? k.scale * a.dlogp[at] : 0.f, de = a.dentropy ? k.scale * a.dentropy[at] : 0.f;
    const float over = 1.f / s;
    // log p = ln 2 (x - log2 s)
    const float b = empty ? 0.f : -de * kLn2 * over;
    const float c = empty ? 0.f : (de * (kLn2 * log2_fast(s) - entropy) - up) * over;
    auto gradient = [&](float f, int column) __attribute__((always_inline)) {
        const float d = x(f);
        const float g = exp2_fast(d) * __builtin_fmaf(b, bounded(d), c);
        return empty ? 0.f : column == token ? g + up : g;
    };
#pragma unroll
    for (int i = 0; i < kLogpBackVectors; ++i) {
        const int n = n0 + i * kLogpBackBlock;
        if (n < cut.vectors) {
            float f[kPer];
            T::unpack(v[i], f);
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                f[j] = gradient(f[j], cut.head + n * kPer + j);
            store_vec<T, false>(dz + cut.head + n * kPer, T::pack(f));
        }
    }
    if (has_edge)
        dz[edge_column] = T::of_f32(gradient(edge, edge_column));
}

}  // namespace zo
