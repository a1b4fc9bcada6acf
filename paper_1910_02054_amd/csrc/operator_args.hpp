// operator_args.hpp -- host side shared by the operators' translation units
// (zero_operators.hip, zero_experts.hip, zero_log_probs.hip): the checks of a call's arrays and the dispatch
// on its type.  Not part of the C ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <utility>

#include "host_common.hpp"
#include "row_ops.hpp"
#include "zero_operators.h"

namespace zsh {
namespace {

constexpr int64_t kMaxLaunch = 1 << 20;  // workgroups of one launch; more rows take several

inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline int pow2_up(int64_t x) {
    int p = 1;
    while (p < x)
        p *= 2;
    return p;
}

// ---------------------------------------------------------------------------
// Arguments.  Every array of a call goes through one table: presence, stride, extent and
// alignment first, then overlaps, then (eager calls) the allocations.
// ---------------------------------------------------------------------------
struct Matrix {
    const char* name;
    const void* p;
    int64_t rows, cols, ld;
    size_t elem;
    bool out;
    size_t pitch() const { return (size_t)ld * elem; }
    size_t width() const { return (size_t)cols * elem; }
    size_t bytes() const { return rows > 0 ? (size_t)(rows - 1) * pitch() + width() : 0; }
};

inline size_t elem_size(int dtype) { return dtype == ZERO_F32 ? 4 : 2; }

// Whether x is finite as the kernels have it.
inline bool is_fin32(double x) { return std::fabs(x) <= FLT_MAX; }

inline bool known_type(int dtype) { return dtype == ZERO_F32 || dtype == ZERO_F16 || dtype == ZERO_BF16; }

struct Arrays {
    static constexpr int kMost = 12;
    const char* fn;
    Matrix m[kMost];
    int n = 0;

    explicit Arrays(const char* f) : fn(f) {}

    // Rows x cols elements, rows ld apart.  NULL is refused unless `optional` (the array is then left out).
    int add(const char* name, const void* p, int64_t rows, int64_t cols, int64_t ld, size_t elem, bool out,
            bool optional = false) {
        if (!p)
            return optional || rows == 0 || cols == 0 ? ZERO_OK : fail(ZERO_EINVAL, "%s: %s is NULL", fn, name);
        if (ld < cols)
            return fail(ZERO_EINVAL, "%s: %s has rows %lld elements apart, %lld columns", fn, name, (long long)ld,
                        (long long)cols);
        if (rows > 0 && ld > kMaxNumel / rows)
            return fail(ZERO_EINVAL, "%s: %s is larger than 2^40 elements", fn, name);
        if (reinterpret_cast<uintptr_t>(p) % elem)
            return fail(ZERO_EINVAL, "%s: %s is not aligned to its elements", fn, name);
        if (rows > 0 && cols > 0)
            m[n++] = Matrix{name, p, rows, cols, ld, elem, out};
        return ZERO_OK;
    }

    static bool same_place(const Matrix& a, const Matrix& b) {
        return a.p == b.p && a.elem == b.elem && a.cols == b.cols && a.rows == b.rows && (a.ld == b.ld || a.rows == 1);
    }

    static bool meet(const Matrix& a, const Matrix& b) {
        const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
        if (!overlaps(pa, a.bytes(), pb, b.bytes()))
            return false;
        if (a.pitch() != b.pitch() || a.rows == 1 || b.rows == 1)
            return true;
        // columns of one buffer: b's start within a's row
        const size_t pitch = a.pitch(), d = pb >= pa ? (pb - pa) % pitch : (pitch - (pa - pb) % pitch) % pitch;
        return d < a.width() || d + b.width() > pitch;
    }

    // `in_place` lists the outputs (pairs of names) that may lie exactly on an input.
    int check_overlaps(std::initializer_list<std::pair<const void*, const void*>> in_place) const {
        for (int i = 0; i < n; ++i)
            for (int j = i + 1; j < n; ++j) {
                if ((!m[i].out && !m[j].out) || !meet(m[i], m[j]))
                    continue;
                bool allowed = false;
                for (const auto& pr : in_place)
                    allowed |= same_place(m[i], m[j]) && ((pr.first == m[i].name && pr.second == m[j].name) ||
                                                          (pr.first == m[j].name && pr.second == m[i].name));
                if (!allowed)
                    return fail(ZERO_EINVAL, "%s: %s and %s overlap", fn, m[i].name, m[j].name);
            }
        return ZERO_OK;
    }

    // The stream's device, and (unless the stream is being captured) the arrays' allocations.
    int check_memory(hipStream_t stream) const {
        int dev = 0;
        int rc = current_device(stream, &dev);
        if (rc)
            return rc;
        hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
        HIP_TRY(hipStreamIsCapturing(stream, &cap));
        if (cap != hipStreamCaptureStatusNone)
            return ZERO_OK;
        // an allocation that one array has been found in is not looked up again for the next
        uintptr_t base[kMost], end[kMost];
        int found = 0;
        for (int i = 0; i < n; ++i) {
            const uintptr_t p = reinterpret_cast<uintptr_t>(m[i].p), e = p + m[i].bytes();
            int k = 0;
            while (k < found && !(p >= base[k] && e <= end[k]))
                ++k;
            if (k < found)
                continue;
            hipDeviceptr_t b = nullptr;
            size_t size = 0;
            if (hipMemGetAddressRange(&b, &size, const_cast<void*>(m[i].p)) != hipSuccess || !b) {
                (void)hipGetLastError();
                return fail(ZERO_EINVAL, "%s: %s is not in GPU-accessible memory", fn, m[i].name);
            }
            base[found] = reinterpret_cast<uintptr_t>(b);
            end[found] = base[found] + size;
            if (p < base[found] || e > end[found])
                return fail(ZERO_EINVAL, "%s: %s ([%p, +%zu B)) overruns its allocation ([%p, +%zu B))", fn, m[i].name,
                            m[i].p, m[i].bytes(), b, size);
            ++found;
        }
        return ZERO_OK;
    }
};

#define TRY(expr)        \
    do {                 \
        int rc_ = (expr); \
        if (rc_)         \
            return rc_;  \
    } while (0)

inline int check_sizes(const char* fn, int dtype, int64_t rows) {
    if (!known_type(dtype))
        return fail(ZERO_EINVAL, "%s: dtype %d is none of ZERO_F32, ZERO_F16, ZERO_BF16", fn, dtype);
    if (rows < 0 || rows > kMaxNumel)
        return fail(ZERO_EINVAL, "%s: rows = %lld is outside [0, 2^40]", fn, (long long)rows);
    return ZERO_OK;
}

// Calls f(T{}) with the kernels' type of `dtype`.
template <typename F>
inline int with_type(int dtype, F f) {
    switch (dtype) {
        case ZERO_F32: return f(zo::F32{});
        case ZERO_F16: return f(zo::F16{});
        default: return f(zo::BF16{});
    }
}

}  // namespace
}  // namespace zsh
