// log_prob_kernels.hpp -- log probabilities of given tokens, the entropy and the likeliest tokens of a
// row of logits, and the gradient of the logits.
//
// With x_v = log2(e) (z_v - m) / temperature, m the row's maximum, S = sum of 2^x and U = sum of 2^x x:
//   log p_v = (z_v - m) / temperature - ln S,   entropy = ln 2 (log2 S - U / S),
// both terms of the entropy without cancellation (x <= 0).  The difference is taken before the product, in
// every type: the maximum's own term is then 1 to the bit, so S >= 1, no log probability is above 0 and a
// certain token has 0.
//
// The list: the threads' elements are kM groups, and the k-th largest of the groups' maxima is no more than
// the k-th largest logit, so only logits from there on can be listed: little more than k of them unless
// they lie close together in the row.  They are gathered in LDS and sorted by (logit, token).  Where they are
// too many for that (rows of equal values, sorted rows, long lists), the k-th (logit, token) itself is
// found, bit by bit, by counting.
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
    // f(vector, its first column), of all vectors; f(batch) before each batch's
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
};

template <int NT>
struct LogProbLds {
    float wave_max[NT / 64], wave_sum[NT / 64], wave_u[NT / 64];
    int32_t count[NT / 64];
    uint32_t least;    // candidates' least key
    int32_t listed;
};

// The sum over the workgroup of every wave's count; all threads call it together.
template <int NT>
__device__ __forceinline__ int sum_counts(int mine, LogProbLds<NT>& lds) {
    mine = seg_reduce<64>(mine, [](int a, int b) { return a + b; });
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        lds.count[threadIdx.x / 64] = mine;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w)
        all += lds.count[w];
    return all;
}

// The likeliest k tokens of a row: `entries` ends with the sorted list in its first min(k, capacity) places,
// 0 where there are none.  groups: the maximum of this thread's logits (-inf: none).
template <typename T, int NT, int NV>
__device__ __forceinline__ void find_top(LogitRow<T, NT, NV>& row, float most, int k, int vocab, uint64_t* entries,
                                         int capacity, LogProbLds<NT>& lds) {
    const int t = threadIdx.x, lane = t & 63;
    constexpr int kM = NT;  // groups: one a thread
    uint32_t* const maxima = reinterpret_cast<uint32_t*>(entries);  // of the groups; capacity * 2 >= kM
    uint32_t least = 1;
    if (k <= kM / 2) {
        maxima[t] = key_of(most);
        if (t == 0)
            lds.listed = 0;
        __syncthreads();
        if (t < 64) {
            uint32_t mine[kM / 64];
#pragma unroll
            for (int j = 0; j < kM / 64; ++j)
                mine[j] = maxima[j * 64 + lane];
            uint32_t found = 0;
            for (int b = 31; b >= 0; --b) {
                const uint32_t next = found | 1u << b;
                int n = 0;
#pragma unroll
                for (int j = 0; j < kM / 64; ++j)
                    n += __popcll(__ballot(mine[j] >= next));
                if (n >= k) {
                    found = next;
                    if (n <= k + k / 8 + 4)
                        break;
                }
            }
            if (lane == 0)
                lds.least = found > 1 ? found : 1;
        }
        __syncthreads();
        least = lds.least;
        const float bound = of_key(least);
        auto offer = [&](float f, int column) __attribute__((always_inline)) {
            const uint32_t key = key_of(f);
            if (key >= least && column < vocab) {
                const int at = atomicAdd(&lds.listed, 1);
                if (at < capacity)
                    entries[at] = entry_of(key, column);
            }
        };
        (void)bound;
        row.each([&](u32x4 u, int column) __attribute__((always_inline)) {
            if (key_of(max_of<T>(u, -__builtin_inff())) >= least) {
                float f[T::kPer];
                T::unpack(u, f);
#pragma unroll
                for (int j = 0; j < T::kPer; ++j)
                    offer(f[j], column + j);
            }
        });
        if (t < row.cut.edges)
            offer(row.edge, row.edge_column);
        __syncthreads();
    }
    int n = k <= kM / 2 ? lds.listed : capacity + 1;
    if (n > capacity) {
        // the k-th entry itself: count of keys at least a bound, then of tokens at most one among the equal
        auto count = [&](auto holds) __attribute__((always_inline)) {
            int c = 0;
            row.each([&](u32x4 u, int column) __attribute__((always_inline)) {
                float f[T::kPer];
                T::unpack(u, f);
#pragma unroll
                for (int j = 0; j < T::kPer; ++j)
                    c += holds(key_of(f[j]), column + j) ? 1 : 0;
            });
            if (t < row.cut.edges)
                c += holds(key_of(row.edge), row.edge_column) ? 1 : 0;
            return sum_counts<NT>(c, lds);
        };
        const int there = count([&](uint32_t key, int) { return key >= 1; });
        const int want = there < k ? there : k;
        uint32_t at = 1;  // the want-th largest key
        if (want < there) {
            at = 0;
            for (int b = 31; b >= 0; --b) {
                const uint32_t next = at | 1u << b;
                if (count([&](uint32_t key, int) { return key >= next; }) >= want)
                    at = next;
            }
        }
        int last = vocab;  // tokens below it of the equal ones
        if (want < there) {
            const int above = count([&](uint32_t key, int) { return key > at; });
            int low = 0;
            for (int b = 30; b >= 0; --b) {
                const int next = low | 1 << b;
                if (next <= vocab &&
                    count([&](uint32_t key, int token) { return key == at && token < next; }) < want - above)
                    low = next;
            }
            last = low + 1;
        }
        __syncthreads();
        if (t == 0)
            lds.listed = 0;
        __syncthreads();
        auto take = [&](float f, int token) __attribute__((always_inline)) {
            const uint32_t key = key_of(f);
            if (key > at || (key == at && token < last))
                if (key) {
                    const int to = atomicAdd(&lds.listed, 1);
                    if (to < capacity)
                        entries[to] = entry_of(key, token);
                }
        };
        row.each([&](u32x4 u, int column) __attribute__((always_inline)) {
            float f[T::kPer];
            T::unpack(u, f);
#pragma unroll
            for (int j = 0; j < T::kPer; ++j)
                take(f[j], column + j);
        });
        if (t < row.cut.edges)
            take(row.edge, row.edge_column);
        __syncthreads();
        n = lds.listed;
    }
    // sorted in falling order, 0 behind the last
    int size = 64;
    while (size < n || size < k)
        size *= 2;
    for (int i = n + t; i < size; i += NT)
        entries[i] = 0;
    __syncthreads();
    for (int run = 2; run <= size; run *= 2)
        for (int step = run / 2; step > 0; step /= 2) {
            for (int i = t; i < size / 2; i += NT) {
                const int p = 2 * i - (i & (step - 1)), q = p + step;
                const uint64_t a = entries[p], b = entries[q];
                if ((a < b) == ((p & run) == 0)) {
                    entries[p] = b;
                    entries[q] = a;
                }
            }
            __syncthreads();
        }
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
        row.each([&](u32x4 v, int) __attribute__((always_inline)) {
            const float up = max_of<T>(v, m);
            const Exponent x(k.c, up);
            if (up > m) {
                move_sums(x, m, s, u);
                m = up;
            }
            float f[T::kPer];
            T::unpack(v, f);
#pragma unroll
            for (int j = 0; j < T::kPer; ++j)
                add_term(f[j], x, s, u);
        });
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
        find_top<T, NT, NV>(row, most, a.k, vocab, entries, capacity, lds);
        for (int i = t; i < a.k; i += NT) {
            const uint64_t e = entries[i];
            const uint32_t key = (uint32_t)(e >> 32);
            a.top_index[at * a.k + i] = key ? (int32_t)~(uint32_t)e : -1;
            a.top_logp[at * a.k + i] = key ? log_p(of_key(key)) : -inf;
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
