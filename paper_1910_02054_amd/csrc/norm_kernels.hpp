// norm_kernels.hpp -- root-mean-square norm of rows, with the residual's addition
// and an e4m3 output; its gradients.
//
//   h = x + r (rounded),  rstd = (mean h^2 + eps)^(-1/2),  y = h rstd w
//   dx = rstd (g - n mean(g n)) + dh,  g = dy w,  n = h rstd;  dw = sum over rows of dy n
//
// Both are bound by HBM: an element costs 6 to 18 bytes and 30 to 42 vector instructions (42 with
// e4m3 rows, which keep the vector ALU busy for 0.7 of the time).  A row is read once and stays in
// registers between its reduction and its output: LPR lanes hold a row, NV 16-byte vectors each.
// LPR goes from 16 lanes of a wave to a workgroup of 1024, the smallest for which NV
// stays small, so that short rows share a wave and need no barrier, and long ones are spread over
// enough waves to keep the loads in flight.
//
// Measured: 16384 rows of 8192 bf16 with the residual, both outputs and e4m3 in groups of 128, 212 us,
// 5.7 TB/s; 16384 of 4096 f16 with a scale a row 95 us, 6.4; 8192 of 8192 f32 without e4m3 174 us, 6.2;
// the gradient of 8192 of 4096 f16 49 us, 5.5 TB/s, and 4.6 for the partial sums' kernel; one row of
// 8192 3.8 us.  (The copy kernel reaches 6.7 TB/s.)  The gradient of f32 rows above 16384 columns
// spills 45 registers a lane: 2048 of 25600 195 us, 4.3 TB/s.
#pragma once

#include "row_ops.hpp"
#include "zero_operators.h"

namespace zo {

constexpr float kE4m3Max = 448.0f;
constexpr float kScaleFloor = 0x1p-100f;  // the least magnitude that a scale stands for

constexpr int norm_block(int lpr) { return lpr < 256 ? 256 : lpr; }

// Four e4m3 codes, to nearest even.  The clamp keeps NaN (a comparison with NaN is false).
__device__ __forceinline__ uint32_t pack_e4m3(const float* f) {
    float c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        c[j] = f[j] > kE4m3Max ? kE4m3Max : f[j];
        c[j] = c[j] < -kE4m3Max ? -kE4m3Max : c[j];
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], w, true);
}

template <int PER>
__device__ __forceinline__ void store_e4m3(uint8_t* p, const float* f) {
    typedef uint32_t u32_b __attribute__((aligned(1)));
    typedef u32x2 u32x2_b __attribute__((aligned(1)));
    if constexpr (PER == 8)
        *reinterpret_cast<u32x2_b*>(p) = u32x2{pack_e4m3(f), pack_e4m3(f + 4)};
    else
        *reinterpret_cast<u32_b*>(p) = pack_e4m3(f);
}

// y / scale, rounded once, for many y of one scale t: the product with the rounded reciprocal is off by up
// to two roundings, which puts a quotient beside a midpoint of two codes (bf16 rows have many on one) on the other
// side; the exact remainder of that product corrects it to the nearest fp32.  The remainder has
// bits down to 2^-34 t ulp(1) where the code is not 0, so scales below 1 (least: 2^-100 / 448) are
// raised by 2^24 with their y.  An infinite scale leaves 0 of what is finite, and of -0 stays -0.
struct Quotient {
    float k, t, inv;
    __device__ __forceinline__ explicit Quotient(float scale) : k(scale < 1.f ? 0x1p24f : 1.f) {
        const bool inf = scale == __builtin_inff();
        t = inf ? 0.f : scale * k;
        inv = inf ? 0.f : 1.0f / t;
    }
    __device__ __forceinline__ float operator()(float y) const {
        y *= k;
        const float q = y * inv, excess = __builtin_fmaf(q, t, -y);
        return __builtin_fmaf(-excess, inv, q);
    }
};

// Largest over runs of `lanes` neighbouring lanes (a power of two, 4 to 64, the same in the whole grid).
__device__ __forceinline__ uint32_t run_max(uint32_t x, int lanes) {
    const MaxU op;
    x = seg_reduce<4>(x, op);
    if (lanes >= 8)
        x = op(x, dpp<0x141>(x));
    if (lanes >= 16)
        x = op(x, dpp<0x140>(x));
    if (lanes >= 32)
        x = swap_step<false>(x, op);
    if (lanes >= 64)
        x = swap_step<true>(x, op);
    return x;
}

// A magnitude's bits: they order as the magnitudes, NaN above all.
__device__ __forceinline__ uint32_t mag_bits(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7FFFFFFFu; }

// How LPR lanes hold a row of `cols` elements: the vector at slot i of a lane is number
// lane + i * LPR of `full`, and the elements after the last whole vector lie two a lane on the
// aligned four lanes around the place that a further vector would have, at slot `slot`.  (A run of lanes with
// one scale is four or more, so it has them.)
template <typename T, int LPR>
struct Held {
    int lane, full, slot, tail[2];  // tail: columns of this lane's odd elements, -1: none
    __device__ __forceinline__ Held(int lane_, int cols) : lane(lane_), full(cols / T::kPer), slot(full / LPR) {
        const int from = full * T::kPer, e = lane - (full % LPR & ~3);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int c = from + 2 * e + j;
            tail[j] = e >= 0 && e < 4 && c < cols ? c : -1;
        }
    }
    __device__ __forceinline__ bool has(int i) const { return lane + i * LPR < full; }
    __device__ __forceinline__ int column(int i) const { return (lane + i * LPR) * T::kPer; }
    // calls f(j, column) for this lane's odd elements
    template <typename F>
    __device__ __forceinline__ void odd(F f) const {
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (tail[j] >= 0)
                f(j, tail[j]);
    }
};

// Rows of more than 64 vectors go past the caches: 4096 rows of 1600 f16 10.0 us in place of 11.4, 16384 of
// 4096 with e4m3 95 in place of 108; rows of 512 lose by it (13.3, 14.4).
constexpr bool norm_past(int lpr, int nv) { return lpr * nv > 64; }

// The reciprocal root of a row whose sum of squares, or eps, has left fp32's range (or is so small that
// squares are lost): the squares again, of elements scaled by 2^-80 or 2^80, and the rest in fp64.  A row
// that holds an infinity or a NaN comes out as it went in.  `total` is the mean and eps in fp32, which
// tells such rows: where it lies in [2^-85, inf) all that was lost is below 2^-49 of it.
constexpr float kLeastTotal = 0x1p-85f;

template <int LPR, typename F>
__device__ __forceinline__ float far_rstd(float total, double eps, int cols, float* lds, F sum_of_squares) {
    const float k = total < kLeastTotal ? 0x1p80f : 0x1p-80f;
    const double sum = row_reduce<LPR>(sum_of_squares(k), lds, Add());
    return (float)(1.0 / sqrt(sum / ((double)k * k * cols) + eps));
}

template <typename T, int LPR, int NV>
__global__ __launch_bounds__(norm_block(LPR)) void k_rms_norm(const zero_rms_norm_args_t a, int64_t first) {
    // a run of lanes that shares a scale lies in one slot's lanes, or is all of them
    static_assert(LPR >= 64 || NV == 1, "short rows take one vector a lane");
    using elem = typename T::elem;
    constexpr int kPer = T::kPer, kBlock = norm_block(LPR);
    constexpr bool PAST = norm_past(LPR, NV);
    __shared__ float sums[LPR > 64 ? LPR / 64 : 1];
    __shared__ float far_sums[LPR > 64 ? LPR / 64 : 1];
    __shared__ uint32_t tops[LPR > 64 ? LPR / 64 : 1];
    const int lane = threadIdx.x % LPR, cols = (int)a.cols;
    const int64_t row = first + (int64_t)blockIdx.x * (kBlock / LPR) + threadIdx.x / LPR;
    if (row >= a.rows)
        return;  // whole segments of waves: a workgroup with several rows has no barrier
    const Held<T, LPR> held(lane, cols);
    const elem* x = static_cast<const elem*>(a.x) + row * a.ld_x;
    const elem* r = static_cast<const elem*>(a.residual) + row * a.ld_residual;
    const elem* w = static_cast<const elem*>(a.weight);
    elem* h = static_cast<elem*>(a.h) + row * a.ld_h;
    elem* y = static_cast<elem*>(a.y) + row * a.ld_y;

    // everything the row needs is on its way before any of it is used
    u32x4 v[NV], rv[NV], wv[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        v[i] = rv[i] = wv[i] = u32x4{0, 0, 0, 0};
        if (held.has(i)) {
            v[i] = load_vec<T, PAST>(x + held.column(i));
            if (a.residual)
                rv[i] = load_vec<T, PAST>(r + held.column(i));
        }
    }
    float fo[2] = {}, ro[2] = {}, wo[2] = {};
    held.odd([&](int j, int c) {
        fo[j] = T::to_f32(x[c]);
        if (a.residual)
            ro[j] = T::to_f32(r[c]);
        wo[j] = T::to_f32(w[c]);
    });
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (held.has(i))
            wv[i] = load_vec<T, false>(w + held.column(i));

    float f[NV][kPer];
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        T::unpack(v[i], f[i]);
        if (a.residual) {
            float g[kPer];
            T::unpack(rv[i], g);
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                f[i][j] += g[j];
            v[i] = T::pack(f[i]);
            T::unpack(v[i], f[i]);  // the norm is of the rounded sum, which is what the backward reads
            if (a.h && held.has(i))
                store_vec<T, PAST>(h + held.column(i), v[i]);
        }
#pragma unroll
        for (int j = 0; j < kPer; ++j)
            sum = __builtin_fmaf(f[i][j], f[i][j], sum);
    }
    held.odd([&](int j, int c) {
        if (a.residual) {
            const elem e = T::of_f32(fo[j] + ro[j]);
            fo[j] = T::to_f32(e);
            if (a.h)
                h[c] = e;
        }
        sum = __builtin_fmaf(fo[j], fo[j], sum);
    });
    sum = row_reduce<LPR>(sum, sums, Add());
    const float total = sum / (float)cols + (float)a.eps;
    float rstd = 1.0f / sqrtf(total);
    if (!(total >= kLeastTotal && total < __builtin_inff()))  // the same for all lanes of a row
        rstd = far_rstd<LPR>(total, a.eps, cols, far_sums, [&](float k) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    s = __builtin_fmaf(f[i][j] * k, f[i][j] * k, s);
            held.odd([&](int j, int) { s = __builtin_fmaf(fo[j] * k, fo[j] * k, s); });
            return s;
        });
    if (a.rstd && lane == 0)
        a.rstd[row] = rstd;

    uint32_t top[NV];  // the largest |y| of each slot
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float g[kPer];
        T::unpack(wv[i], g);
        top[i] = 0;
        if (held.has(i)) {  // elsewhere a rstd of inf or NaN would count
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                f[i][j] = f[i][j] * rstd * g[j];
                top[i] = MaxU()(top[i], mag_bits(f[i][j]));
            }
            if (a.y)
                store_vec<T, PAST>(y + held.column(i), T::pack(f[i]));
        }
    }
    uint32_t top_odd = 0;
    held.odd([&](int j, int c) {
        fo[j] = fo[j] * rstd * wo[j];
        top_odd = MaxU()(top_odd, mag_bits(fo[j]));
        if (a.y)
            y[c] = T::of_f32(fo[j]);
    });
    if (!a.q8)
        return;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        top[i] = i == held.slot ? MaxU()(top[i], top_odd) : top[i];
    const int group = a.group;
    if (group == 0) {
        uint32_t m = top[0];
#pragma unroll
        for (int i = 1; i < NV; ++i)
            m = MaxU()(m, top[i]);
        m = row_reduce<LPR>(m, tops, MaxU());
#pragma unroll
        for (int i = 0; i < NV; ++i)
            top[i] = m;
    } else {
        const int run = group / kPer < LPR ? group / kPer : LPR;  // lanes of a group
#pragma unroll
        for (int i = 0; i < NV; ++i)
            top[i] = run_max(top[i], run);
    }
    uint8_t* q = a.q8 + row * a.ld_q8;
    float* scale = a.scale + row * (group ? (cols + group - 1) / group : 1);
    auto scale_of = [](uint32_t m) {
        const float t = __builtin_bit_cast(float, m);
        return (t < kScaleFloor ? kScaleFloor : t) / kE4m3Max;
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = held.column(i);
        const float t = scale_of(top[i]);
        if (c < cols && (group ? (c & (group - 1)) == 0 : c == 0))
            scale[group ? c / group : 0] = t;
        if (held.has(i)) {
            const Quotient over(t);
            float g[kPer];
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                g[j] = over(f[i][j]);
            store_e4m3<kPer>(q + c, g);
        }
        if (i == held.slot) {
            held.odd([&](int j, int at) {
                float g[4] = {Quotient(t)(fo[j])};
                q[at] = (uint8_t)pack_e4m3(g);
            });
        }
    }
}

// Rows are dealt to the grid's workgroups in turn, kRows at a time; each keeps its rows' sum of dy n in
// registers, its lanes' columns being the same in every row, and leaves one row of partial sums
// (`part` [gridDim.x, cols]); where it is the only workgroup it writes dweight itself.
//
// A row's arrays are loaded while the row before it is worked on (kAhead), where the registers are
// enough for that; wider rows read dh and the weight as they are needed.
constexpr int kBackBlock = 1024;

template <typename T, int LPR, int NV>
__global__ __launch_bounds__(kBackBlock) void k_rms_norm_back(const zero_rms_norm_backward_args_t a, float* part) {
    using elem = typename T::elem;
    constexpr int kPer = T::kPer, kBlock = kBackBlock, kRows = kBlock / LPR;
    constexpr bool PAST = norm_past(LPR, NV), kAhead = NV <= 2;
    __shared__ float sums[2][kRows][LPR > 64 ? LPR / 64 : 1];
    __shared__ float join[kRows > 1 ? LPR * NV * kPer : 1];
    const int lane = threadIdx.x % LPR, cols = (int)a.cols;
    const Held<T, LPR> held(lane, cols);
    const elem* w = static_cast<const elem*>(a.weight);
    struct Row {
        u32x4 h[NV], dy[NV], dh[kAhead ? NV : 1];
        float rstd;
    };
    auto load = [&](Row& q, int64_t row) __attribute__((always_inline)) {
        const elem* dy = static_cast<const elem*>(a.dy) + row * a.ld_dy;
        const elem* h = static_cast<const elem*>(a.h) + row * a.ld_h;
        const elem* dh = static_cast<const elem*>(a.dh) + row * a.ld_dh;
        const bool there = row < a.rows;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            q.h[i] = q.dy[i] = u32x4{0, 0, 0, 0};
            if (there && held.has(i)) {
                q.h[i] = load_vec<T, PAST>(h + held.column(i));
                q.dy[i] = load_vec<T, PAST>(dy + held.column(i));
            }
            if constexpr (kAhead) {
                q.dh[i] = u32x4{0, 0, 0, 0};
                if (a.dh && there && held.has(i))
                    q.dh[i] = load_vec<T, PAST>(dh + held.column(i));
            }
        }
        q.rstd = there ? a.rstd[row] : 0.f;
    };
    float dw[NV][kPer] = {}, dwo[2] = {}, wo[2] = {};
    u32x4 wv[kAhead ? NV : 1];
    if constexpr (kAhead) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            wv[i] = u32x4{0, 0, 0, 0};
            if (held.has(i))
                wv[i] = load_vec<T, false>(w + held.column(i));
        }
    }
    held.odd([&](int j, int c) { wo[j] = T::to_f32(w[c]); });
    // all segments of a workgroup take their turns together; one whose row lies past the last has zeros
    const int segment = threadIdx.x / LPR;
    const int64_t step = (int64_t)gridDim.x * kRows;
    Row q;
    load(q, (int64_t)blockIdx.x * kRows + segment);
    int turn = 0;
    for (int64_t base = (int64_t)blockIdx.x * kRows; base < a.rows; base += step, turn ^= 1) {
        const int64_t row = base + segment;
        const bool there = row < a.rows;
        const elem* dy = static_cast<const elem*>(a.dy) + row * a.ld_dy;
        const elem* h = static_cast<const elem*>(a.h) + row * a.ld_h;
        const elem* dh = static_cast<const elem*>(a.dh) + row * a.ld_dh;
        elem* dx = static_cast<elem*>(a.dx) + row * a.ld_dx;
        float no[2] = {}, go[2] = {}, to[2] = {};
        if (there)
            held.odd([&](int j, int c) {
                no[j] = T::to_f32(h[c]);
                go[j] = T::to_f32(dy[c]);
                if (a.dh)
                    to[j] = T::to_f32(dh[c]);
            });
        Row next;
        if constexpr (kAhead)
            load(next, row + step);
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (held.has(i)) {  // elsewhere a rstd of inf or NaN would count
                float n[kPer], g[kPer], k[kPer];
                T::unpack(q.h[i], n);
                T::unpack(q.dy[i], g);
                T::unpack(kAhead ? wv[kAhead ? i : 0] : load_vec<T, false>(w + held.column(i)), k);
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    n[j] *= q.rstd;
                    dw[i][j] = __builtin_fmaf(g[j], n[j], dw[i][j]);
                    dot = __builtin_fmaf(g[j] * k[j], n[j], dot);
                }
            }
        }
        held.odd([&](int j, int) {
            no[j] *= q.rstd;
            dwo[j] = __builtin_fmaf(go[j], no[j], dwo[j]);
            go[j] *= wo[j];
            dot = __builtin_fmaf(go[j], no[j], dot);
        });
        const float mean = row_reduce<LPR>(dot, sums[turn][segment], Add()) / (float)cols;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            keep_packed(q.h[i]);
            keep_packed(q.dy[i]);
            if (there && held.has(i)) {
                float n[kPer], g[kPer], k[kPer], t[kPer] = {};
                T::unpack(q.h[i], n);
                T::unpack(q.dy[i], g);
                T::unpack(kAhead ? wv[kAhead ? i : 0] : load_vec<T, false>(w + held.column(i)), k);
                if (a.dh)
                    T::unpack(kAhead ? q.dh[kAhead ? i : 0] : load_vec<T, PAST>(dh + held.column(i)), t);
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    const float d = q.rstd * (g[j] * k[j] - n[j] * q.rstd * mean);
                    t[j] = a.dh ? d + t[j] : d;
                }
                store_vec<T, PAST>(dx + held.column(i), T::pack(t));
            }
        }
        if (there)
            held.odd([&](int j, int c) {
                const float d = q.rstd * (go[j] - no[j] * mean);
                dx[c] = T::of_f32(a.dh ? d + to[j] : d);
            });
        if constexpr (kAhead)
            q = next;
        else
            load(q, row + step);
    }
    // the workgroup's rows of sums, one after another, in the order of its segments
    elem* out = static_cast<elem*>(a.dweight);
    float* mine = part + (int64_t)blockIdx.x * cols;
    const bool alone = gridDim.x == 1;
    auto put = [&](int c, float d) {
        if (alone)
            out[c] = T::of_f32(d);
        else
            mine[c] = d;
    };
    if constexpr (kRows > 1) {
        for (int s = 0; s < kRows; ++s) {
            if (segment == s) {
                auto add = [&](int c, float d) { join[c] = s ? join[c] + d : d; };
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (held.has(i))
#pragma unroll
                        for (int j = 0; j < kPer; ++j)
                            add(held.column(i) + j, dw[i][j]);
                held.odd([&](int j, int c) { add(c, dwo[j]); });
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < cols; c += kBlock)
            put(c, join[c]);
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (held.has(i))
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    put(held.column(i) + j, dw[i][j]);
        held.odd([&](int j, int c) { put(c, dwo[j]); });
    }
}

// dweight from the workgroups' partial sums: 32 columns a workgroup, 32 runs of partial rows
// side by side, joined in a fixed order.
constexpr int kSumCols = 32, kSumRuns = 32;

template <typename T>
__global__ __launch_bounds__(kSumCols* kSumRuns) void k_column_sums(const float* part, int parts, int cols,
                                                                    typename T::elem* out) {
    __shared__ float run[kSumRuns][kSumCols];
    const int k = threadIdx.x / kSumCols, l = threadIdx.x % kSumCols, c = blockIdx.x * kSumCols + l;
    float s = 0.f;
    if (c < cols) {
#pragma unroll 4
        for (int p = k; p < parts; p += kSumRuns)
            s += part[(int64_t)p * cols + c];
    }
    run[k][l] = s;
    __syncthreads();
    if (k == 0 && c < cols) {
        for (int i = 1; i < kSumRuns; ++i)
            s += run[i][l];
        out[c] = T::of_f32(s);
    }
}

}  // namespace zo
