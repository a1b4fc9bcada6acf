// row_ops.hpp -- what the row operators' kernels share (norm_kernels.hpp, route_kernels.hpp,
// distill_kernels.hpp, expert_kernels.hpp, log_prob_kernels.hpp): 16-byte vectors of the three element types at any
// element alignment, and reductions over segments of a wave and over a workgroup
// in the vector ALU.
//
// All arithmetic is in fp32; a store rounds once, to nearest even.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "shard_kernels.hpp"

namespace zo {

using zs::u32x2;
using zs::u32x4;

// 16 bytes at the alignment of an element (gfx950 runs in unaligned access mode: one
// instruction whatever the address).
typedef u32x4 u32x4_e2 __attribute__((aligned(2)));
typedef u32x4 u32x4_e4 __attribute__((aligned(4)));

struct F32 {
    using elem = float;
    using vec = u32x4_e4;
    static constexpr int kPer = 4;  // elements of 16 bytes
    static constexpr uint32_t kLowest = 0xFF800000u;  // -inf in every element of a word
    static __device__ __forceinline__ float to_f32(float x) { return x; }
    static __device__ __forceinline__ float of_f32(float x) { return x; }
    static __device__ __forceinline__ void unpack(u32x4 v, float* f) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            f[j] = __builtin_bit_cast(float, (uint32_t)v[j]);
    }
    static __device__ __forceinline__ u32x4 pack(const float* f) {
        u32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[j] = __builtin_bit_cast(uint32_t, f[j]);
        return v;
    }
};

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

struct F16 {
    using elem = uint16_t;
    using vec = u32x4_e2;
    static constexpr int kPer = 8;
    static constexpr uint32_t kLowest = 0xFC00FC00u;
    static __device__ __forceinline__ float to_f32(uint16_t x) { return (float)__builtin_bit_cast(_Float16, x); }
    static __device__ __forceinline__ uint16_t of_f32(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
    static __device__ __forceinline__ void unpack(u32x4 v, float* f) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f16x2 h = __builtin_bit_cast(f16x2, (uint32_t)v[j]);
            f[2 * j] = (float)h.x;
            f[2 * j + 1] = (float)h.y;
        }
    }
    static __device__ __forceinline__ u32x4 pack(const float* f) {
        u32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{f[2 * j], f[2 * j + 1]}), f16x2));
        return v;
    }
};

struct BF16 {
    using elem = uint16_t;
    using vec = u32x4_e2;
    static constexpr int kPer = 8;
    static constexpr uint32_t kLowest = 0xFF80FF80u;
    static __device__ __forceinline__ float to_f32(uint16_t x) {
        return __builtin_bit_cast(float, (uint32_t)x << 16);
    }
    static __device__ __forceinline__ uint16_t of_f32(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
    static __device__ __forceinline__ void unpack(u32x4 v, float* f) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f[2 * j] = __builtin_bit_cast(float, (uint32_t)v[j] << 16);
            f[2 * j + 1] = __builtin_bit_cast(float, (uint32_t)v[j] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ u32x4 pack(const float* f) {
        u32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{f[2 * j], f[2 * j + 1]}), bf16x2));
        return v;
    }
};

// NT: past the caches, for rows that are read or written once and do not come back.
template <typename T, bool NT>
__device__ __forceinline__ u32x4 load_vec(const typename T::elem* p) {
    const typename T::vec* q = reinterpret_cast<const typename T::vec*>(p);
    if constexpr (NT)
        return __builtin_nontemporal_load(q);
    else
        return *q;
}

template <typename T, bool NT>
__device__ __forceinline__ void store_vec(typename T::elem* p, u32x4 v) {
    typename T::vec* q = reinterpret_cast<typename T::vec*>(p);
    if constexpr (NT)
        __builtin_nontemporal_store(v, q);
    else
        *q = v;
}

// The 16 bytes of row `p` from column `col`, elements at or past `cols` filled from
// `fill` (a word of two or one of them).
template <typename T>
__device__ __forceinline__ u32x4 load_row(const typename T::elem* p, int col, int cols, uint32_t fill) {
    if (col + T::kPer <= cols)
        return load_vec<T, false>(p + col);
    u32x4 v = {fill, fill, fill, fill};
    if constexpr (T::kPer == 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (col + j < cols)
                v[j] = __builtin_bit_cast(uint32_t, p[col + j]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t lo = fill & 0xFFFFu, hi = fill >> 16;
            if (col + 2 * j < cols)
                lo = p[col + 2 * j];
            if (col + 2 * j + 1 < cols)
                hi = p[col + 2 * j + 1];
            v[j] = lo | hi << 16;
        }
    }
    return v;
}

// Stores the 16 bytes at column `col` of row `p`, but for elements at or past `cols`.
template <typename T>
__device__ __forceinline__ void store_row(typename T::elem* p, int col, int cols, u32x4 v) {
    if (col + T::kPer <= cols) {
        store_vec<T, false>(p + col, v);
        return;
    }
    if constexpr (T::kPer == 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (col + j < cols)
                p[col + j] = __builtin_bit_cast(float, (uint32_t)v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (col + 2 * j < cols)
                p[col + 2 * j] = (uint16_t)v[j];
            if (col + 2 * j + 1 < cols)
                p[col + 2 * j + 1] = (uint16_t)(v[j] >> 16);
        }
    }
}

// A row cut at 128-byte lines: its elements before the first line that starts in it, its whole vectors
// from there, and the elements after them.  Those before and after are its edges, fewer than
// kLineBytes / sizeof(elem) + kPer: a thread each.
template <typename T>
struct Cut {
    int head, vectors, edges, tail;  // tail: column of the first element after the vectors
    __device__ __forceinline__ Cut(const typename T::elem* p, int cols) {
        constexpr int kLine = zs::kLineBytes / (int)sizeof(typename T::elem);
        const int into = (int)(reinterpret_cast<uintptr_t>(p) / sizeof(typename T::elem)) & (kLine - 1);
        head = (kLine - into) & (kLine - 1);
        head = head < cols ? head : cols;
        vectors = (cols - head) / T::kPer;
        tail = head + vectors * T::kPer;
        edges = head + cols - tail;
    }
    __device__ __forceinline__ int edge_column(int e) const { return e < head ? e : tail + e - head; }
};

// The maximum of m and a packed vector's values; a NaN loses.
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

// Keeps a packed vector in its registers between two passes over it: without it the compiler holds
// the first pass's fp32 values for the second, at twice the registers or more.
__device__ __forceinline__ void keep_packed(u32x4& v) { asm volatile("" : "+v"(v)); }

// ---------------------------------------------------------------------------
// Reductions.  Steps within rows of 16 lanes by DPP, across them by gfx950's row and
// half-wave swaps (as zs::wave_sum); every lane of a segment ends with the same bits.
// ---------------------------------------------------------------------------
template <int CTRL, typename V>
__device__ __forceinline__ V dpp(V x) {
    return __builtin_bit_cast(
        V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}

template <bool HALF, typename V, typename OP>
__device__ __forceinline__ V swap_step(V x, OP op) {
    const uint32_t w = __builtin_bit_cast(uint32_t, x);
    const auto r = HALF ? __builtin_amdgcn_permlane32_swap(w, w, false, false)
                        : __builtin_amdgcn_permlane16_swap(w, w, false, false);
    return op(__builtin_bit_cast(V, (uint32_t)r[0]), __builtin_bit_cast(V, (uint32_t)r[1]));
}

// op over segments of L lanes (2, 4, 8, 16, 32 or 64).
template <int L, typename V, typename OP>
__device__ __forceinline__ V seg_reduce(V x, OP op) {
    static_assert(L == 2 || L == 4 || L == 8 || L == 16 || L == 32 || L == 64, "segment of a wave");
    x = op(x, dpp<0xB1>(x));  // the neighbour
    if constexpr (L >= 4)
        x = op(x, dpp<0x4E>(x));  // the other pair
    if constexpr (L >= 8)
        x = op(x, dpp<0x141>(x));  // the other quad (row_half_mirror)
    if constexpr (L >= 16)
        x = op(x, dpp<0x140>(x));  // the other half row (row_mirror)
    if constexpr (L >= 32)
        x = swap_step<false>(x, op);
    if constexpr (L >= 64)
        x = swap_step<true>(x, op);
    return x;
}

struct Add {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct Max {  // a NaN loses
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct MaxU {
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};

// op over the LANES lanes that share a row.  Where they are more than a wave, `lds` (LANES / 64 words,
// the row's own, last read before the workgroup's latest barrier) carries the waves' values and
// all of the workgroup's threads call this together.
template <int LANES, typename V, typename OP>
__device__ __forceinline__ V row_reduce(V x, V* lds, OP op) {
    if constexpr (LANES <= 64) {
        return seg_reduce<LANES>(x, op);
    } else {
        constexpr int kWaves = LANES / 64;
        x = seg_reduce<64>(x, op);
        if ((threadIdx.x & 63) == 0)
            lds[threadIdx.x % LANES / 64] = x;
        __syncthreads();
        return seg_reduce<kWaves>(lds[threadIdx.x % kWaves], op);
    }
}

// 2^x and log2 by the hardware's instructions (about 1 ulp; results below the normal
// range are 0, which for the terms of a softmax is what they round to beside its sum).
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_fast(float x) { return __builtin_amdgcn_logf(x); }

}  // namespace zo
