// norm_kernels.hpp -- root-mean-square norm of rows, with the residual's addition
// and an e4m3 output; its gradients.
//
//   h = x + r (rounded),  rstd = (mean h^2 + eps)^(-1/2),  y = h rstd w
//   dx = rstd (g - n mean(g n)) + dh,  g = dy w,  n = h rstd;  dw = sum over rows of dy n
//
// Both are bound by HBM: an element costs 6 to 18 bytes and about ten operations.  A
// row is read once and stays in registers between its reduction and its output:
// LPR lanes hold a row, NV 16-byte vectors each.  LPR is a sixteenth of a wave's
// row of lanes up to a workgroup of 1024, the smallest for which NV stays small, so that short
// rows share a wave and need no barrier, and long ones are spread over enough
// waves to keep the loads in flight.
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
__device__ __forceinline__ void store_e4m3(uint8_t* p, int col, int cols, const float* f) {
    typedef uint32_t u32_b __attribute__((aligned(1)));
    typedef u32x2 u32x2_b __attribute__((aligned(1)));
    uint32_t w[PER / 4];
#pragma unroll
    for (int j = 0; j < PER / 4; ++j)
        w[j] = pack_e4m3(f + 4 * j);
    if (col + PER <= cols) {
        if constexpr (PER == 8)
            *reinterpret_cast<u32x2_b*>(p + col) = u32x2{w[0], w[1]};
        else
            *reinterpret_cast<u32_b*>(p + col) = w[0];
    } else {
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (col + j < cols)
                p[col + j] = (uint8_t)(w[j / 4] >> 8 * (j % 4));
    }
}

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

template <typename T, int LPR, int NV>
__global__ __launch_bounds__(norm_block(LPR)) void k_rms_norm(const zero_rms_norm_args_t a, int64_t first) {
    // a run of lanes that shares a scale lies in one vector's lanes, or is all of them
    static_assert(LPR >= 64 || NV == 1, "short rows take one vector a lane");
    using elem = typename T::elem;
    constexpr int kPer = T::kPer, kBlock = norm_block(LPR);
    __shared__ float sums[LPR > 64 ? LPR / 64 : 1];
    __shared__ uint32_t tops[LPR > 64 ? LPR / 64 : 1];
    const int lane = threadIdx.x % LPR, cols = (int)a.cols;
    const int64_t row = first + (int64_t)blockIdx.x * (kBlock / LPR) + threadIdx.x / LPR;
    if (row >= a.rows)
        return;  // whole segments of waves: a workgroup with several rows has no barrier
    const elem* x = static_cast<const elem*>(a.x) + row * a.ld_x;
    const elem* r = static_cast<const elem*>(a.residual) + row * a.ld_residual;
    const elem* w = static_cast<const elem*>(a.weight);
    elem* h = static_cast<elem*>(a.h) + row * a.ld_h;
    elem* y = static_cast<elem*>(a.y) + row * a.ld_y;

    float f[NV][kPer];
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (lane + i * LPR) * kPer;
        u32x4 v = {0, 0, 0, 0};
        if (c < cols) {
            v = load_row<T>(x, c, cols, 0);
            if (a.residual) {
                float p[kPer], g[kPer];
                T::unpack(v, p);
                T::unpack(load_row<T>(r, c, cols, 0), g);
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    p[j] += g[j];
                v = T::pack(p);
                if (a.h)
                    store_row<T>(h, c, cols, v);
            }
        }
        T::unpack(v, f[i]);  // the norm is of the rounded sum, which is what the backward reads
#pragma unroll
        for (int j = 0; j < kPer; ++j)
            sum = __builtin_fmaf(f[i][j], f[i][j], sum);
    }
    sum = row_reduce<LPR>(sum, sums, Add());
    const float rstd = 1.0f / sqrtf(sum / (float)cols + (float)a.eps);
    if (a.rstd && lane == 0)
        a.rstd[row] = rstd;

    uint32_t top[NV];  // the largest |y| of each vector
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (lane + i * LPR) * kPer;
        top[i] = 0;
        if (c < cols) {
            float g[kPer];
            T::unpack(load_row<T>(w, c, cols, 0), g);
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                f[i][j] = f[i][j] * rstd * g[j];
                if (c + j < cols)  // past the row a rstd of inf or NaN would count
                    top[i] = MaxU()(top[i], mag_bits(f[i][j]));
            }
            if (a.y)
                store_row<T>(y, c, cols, T::pack(f[i]));
        }
    }
    if (!a.q8)
        return;
    uint8_t* q = a.q8 + row * a.ld_q8;
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
    float* scale = a.scale + row * (group ? (cols + group - 1) / group : 1);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (lane + i * LPR) * kPer;
        if (c < cols) {
            float t = __builtin_bit_cast(float, top[i]);
            t = (t < kScaleFloor ? kScaleFloor : t) / kE4m3Max;
            if (group ? c % group == 0 : c == 0)
                scale[group ? c / group : 0] = t;
            const float inv = 1.0f / t;
            float g[kPer];
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                g[j] = f[i][j] * inv;
            store_e4m3<kPer>(q, c, cols, g);
        }
    }
}

// Rows are dealt to the grid's workgroups in turn (a workgroup takes kBlock / LPR at a time); each
// keeps its rows' sum of dy n in registers, its lanes' columns being the same in every row, and
// leaves one row of partial sums (`part` [gridDim.x, cols]); where it is the only workgroup it
// writes dweight itself.
template <typename T, int LPR, int NV>
__global__ __launch_bounds__(norm_block(LPR)) void k_rms_norm_back(const zero_rms_norm_backward_args_t a,
                                                                   float* part) {
    using elem = typename T::elem;
    constexpr int kPer = T::kPer, kBlock = norm_block(LPR), kRows = kBlock / LPR;
    __shared__ float sums[2][LPR > 64 ? LPR / 64 : 1];
    __shared__ float join[kRows > 1 ? LPR * NV * kPer : 1];
    const int lane = threadIdx.x % LPR, cols = (int)a.cols;
    const elem* w = static_cast<const elem*>(a.weight);
    float dw[NV][kPer] = {};
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LPR; row < a.rows;
         row += (int64_t)gridDim.x * kRows, turn ^= 1) {
        const elem* dy = static_cast<const elem*>(a.dy) + row * a.ld_dy;
        const elem* h = static_cast<const elem*>(a.h) + row * a.ld_h;
        const elem* dh = static_cast<const elem*>(a.dh) + row * a.ld_dh;
        elem* dx = static_cast<elem*>(a.dx) + row * a.ld_dx;
        const float rstd = a.rstd[row];
        u32x4 hv[NV], gv[NV], tv[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (lane + i * LPR) * kPer;
            hv[i] = gv[i] = tv[i] = u32x4{0, 0, 0, 0};
            if (c < cols) {
                hv[i] = load_row<T>(h, c, cols, 0);
                gv[i] = load_row<T>(dy, c, cols, 0);
                if (a.dh)
                    tv[i] = load_row<T>(dh, c, cols, 0);
            }
        }
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (lane + i * LPR) * kPer;
            if (c < cols) {
                float n[kPer], g[kPer], k[kPer];
                T::unpack(hv[i], n);
                T::unpack(gv[i], g);
                T::unpack(load_row<T>(w, c, cols, 0), k);
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    n[j] *= rstd;
                    dw[i][j] = __builtin_fmaf(g[j], n[j], dw[i][j]);
                    if (c + j < cols)  // past the row a rstd of inf or NaN would count
                        dot = __builtin_fmaf(g[j] * k[j], n[j], dot);
                }
            }
        }
        const float mean = row_reduce<LPR>(dot, sums[turn], Add()) / (float)cols;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (lane + i * LPR) * kPer;
            if (c < cols) {
                float n[kPer], g[kPer], k[kPer], t[kPer];
                T::unpack(hv[i], n);
                T::unpack(gv[i], g);
                T::unpack(load_row<T>(w, c, cols, 0), k);
                T::unpack(tv[i], t);
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    const float d = rstd * (g[j] * k[j] - n[j] * rstd * mean);
                    t[j] = a.dh ? d + t[j] : d;
                }
                store_row<T>(dx, c, cols, T::pack(t));
            }
        }
    }
    // the workgroup's rows of sums, one after another, in the order of its segments
    elem* dwo = static_cast<elem*>(a.dweight);
    float* mine = part + (int64_t)blockIdx.x * cols;
    const bool alone = gridDim.x == 1;
    if constexpr (kRows > 1) {
        for (int s = 0; s < kRows; ++s) {
            if ((int)threadIdx.x / LPR == s) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int j = 0; j < kPer; ++j) {
                        const int c = (lane + i * LPR) * kPer + j;
                        join[c] = s ? join[c] + dw[i][j] : dw[i][j];
                    }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < cols; c += kBlock) {
            if (alone)
                dwo[c] = T::of_f32(join[c]);
            else
                mine[c] = join[c];
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (lane + i * LPR) * kPer;
            if (c < cols) {
                if (alone) {
                    store_row<T>(dwo, c, cols, T::pack(dw[i]));
                } else {
#pragma unroll
                    for (int j = 0; j < kPer; ++j)
                        if (c + j < cols)
                            mine[c + j] = dw[i][j];
                }
            }
        }
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
