// zero_log_probs.hip -- host side of zero_log_probs and its gradient, declared in
// include/zero_operators.h: argument checks, choice of the kernels' shapes, launches.
#include <hip/hip_runtime.h>

#include "operator_args.hpp"
#include "log_prob_kernels.hpp"

namespace zsh {
namespace {

template <int NT_, int NV_>
struct LogitShape {
    static constexpr int NT = NT_, NV = NV_;
};

// Threads and vectors a thread, (NT, NV), of a row of so many vectors: the least that hold it, as more leave threads
// without work.  Full rows at the last size of each, f16, and the next shape's time: 131072 x 1024 80 us and 171, 32768 x
// 4096 51 and 87, 16384 x 8192 52 and 152, 4096 x 32768 54 and 71, 2340 x 57344 51 and 108.  Longer rows are read as
// they are needed, two workgroups to a compute unit; 16 vectors a thread leave room for one, which is faster only where
// there are few rows and long ones (bf16, without a list: 64 x 131072 11.3 us and 12.5, 64 x 100352 10.8 and 10.7, 256 x
// 131072 18.7 and 16.3, 1024 x 131072 58.3 and 50.8, 1024 x 64000 46.0 and 28.1).
template <typename F>
int with_logit_shape(int64_t vectors, int64_t rows, bool list, F f) {
    if (vectors <= 128) return f(LogitShape<128, 1>{});
    if (vectors <= 512) return f(LogitShape<128, 4>{});
    if (vectors <= 1024) return f(LogitShape<256, 4>{});
    if (vectors <= 4 * 1024) return f(LogitShape<512, 8>{});
    if (vectors <= 7 * 1024) return f(LogitShape<1024, 7>{});
    if (rows <= 64 && vectors > 12 * 1024 && vectors <= 16 * 1024 && !list) return f(LogitShape<1024, 16>{});
    return f(LogitShape<1024, 0>{});
}

int check_log_probs(const char* fn, int dtype, int64_t rows, int64_t vocab, double temperature) {
    TRY(check_sizes(fn, dtype, rows));
    if (vocab < 1 || vocab > (int64_t)1 << 30)
        return fail(ZERO_EINVAL, "%s: vocab = %lld is outside [1, 2^30]", fn, (long long)vocab);
    if (!(temperature >= 1e-30 && temperature <= 1e30))  // its reciprocal is held in fp32
        return fail(ZERO_EINVAL, "%s: temperature must lie in [1e-30, 1e30]", fn);
    return ZERO_OK;
}

zo::LogProbScalars scalars(double temperature, double grad_scale) {
    return zo::LogProbScalars{(float)(1.4426950408889634074 / temperature), (float)(1.0 / temperature),
                              (float)(grad_scale / temperature)};
}

}  // namespace
}  // namespace zsh

using namespace zsh;

extern "C" {

int zero_log_probs(const zero_log_probs_args_t* args, void* stream_) {
    const char* fn = "zero_log_probs";
    if (!args)
        return fail(ZERO_EINVAL, "%s: NULL args", fn);
    const zero_log_probs_args_t a = *args;
    TRY(check_log_probs(fn, a.dtype, a.rows, a.vocab, a.temperature));
    if (a.k < 0 || a.k > ZERO_LOG_PROBS_MAX_K)
        return fail(ZERO_EINVAL, "%s: k = %d is outside [0, %d]", fn, a.k, ZERO_LOG_PROBS_MAX_K);
    if (a.rows > 0 && !a.logp != !a.tokens)
        return fail(ZERO_EINVAL, "%s: tokens and logp come together", fn);
    Arrays t(fn);
    TRY(t.add("logits", a.logits, a.rows, a.vocab, a.ld_logits, elem_size(a.dtype), false));
    TRY(t.add("tokens", a.tokens, a.rows, 1, 1, 4, false, true));
    TRY(t.add("logp", a.logp, a.rows, 1, 1, 4, true, true));
    TRY(t.add("entropy", a.entropy, a.rows, 1, 1, 4, true, true));
    TRY(t.add("top_index", a.top_index, a.rows, a.k, a.k, 4, true));
    TRY(t.add("top_logp", a.top_logp, a.rows, a.k, a.k, 4, true));
    TRY(t.add("stats", a.stats, a.rows, 3, 3, 4, true, true));
    TRY(t.check_overlaps({}));
    if (a.rows == 0)
        return ZERO_OK;
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    TRY(t.check_memory(stream));
    const zo::LogProbScalars k = scalars(a.temperature, 1.0);
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        return with_logit_shape(a.vocab / T::kPer, a.rows, a.k > 0, [&](auto shape) {
            using S = decltype(shape);
            const int capacity = 3 * a.k + 64;  // entries of the list's room, vectors of its queue
            const size_t room = a.k ? (size_t)capacity * 12 : 0;
            auto* const kernel = a.k ? zo::k_log_probs<T, S::NT, S::NV, true> : zo::k_log_probs<T, S::NT, S::NV, false>;
            for (int64_t first = 0; first < a.rows; first += kMaxLaunch)
                kernel<<<(unsigned)std::min(kMaxLaunch, a.rows - first), S::NT, room, stream>>>(a, k, capacity, first);
            HIP_TRY(hipGetLastError());
            return ZERO_OK;
        });
    });
}

int zero_log_probs_backward(const zero_log_probs_backward_args_t* args, void* stream_) {
    const char* fn = "zero_log_probs_backward";
    if (!args)
        return fail(ZERO_EINVAL, "%s: NULL args", fn);
    const zero_log_probs_backward_args_t a = *args;
    TRY(check_log_probs(fn, a.dtype, a.rows, a.vocab, a.temperature));
    if (!is_fin32(a.grad_scale) || !is_fin32(a.grad_scale / a.temperature))
        return fail(ZERO_EINVAL, "%s: grad_scale and grad_scale / temperature must be finite in fp32", fn);
    if (a.rows > 0 && !a.dlogp != !a.tokens)
        return fail(ZERO_EINVAL, "%s: tokens and dlogp come together", fn);
    const size_t e = elem_size(a.dtype);
    static const char *const kLogits = "logits", *const kGrad = "dlogits";
    Arrays t(fn);
    TRY(t.add(kLogits, a.logits, a.rows, a.vocab, a.ld_logits, e, false));
    TRY(t.add("tokens", a.tokens, a.rows, 1, 1, 4, false, true));
    TRY(t.add("stats", a.stats, a.rows, 3, 3, 4, false));
    TRY(t.add("dlogp", a.dlogp, a.rows, 1, 1, 4, false, true));
    TRY(t.add("dentropy", a.dentropy, a.rows, 1, 1, 4, false, true));
    TRY(t.add(kGrad, a.dlogits, a.rows, a.vocab, a.ld_dlogits, e, true));
    TRY(t.check_overlaps({{kLogits, kGrad}}));
    if (a.rows == 0)
        return ZERO_OK;
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    TRY(t.check_memory(stream));
    const zo::LogProbScalars k = scalars(a.temperature, a.grad_scale);
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        const int64_t piece = zo::kLogpBackBlock * zo::kLogpBackVectors;
        const int64_t pieces = std::max<int64_t>(1, div_up(a.vocab / T::kPer, piece)), all = a.rows * pieces;
        for (int64_t first = 0; first < all; first += kMaxLaunch)
            zo::k_log_probs_back<T><<<(unsigned)std::min(kMaxLaunch, all - first), zo::kLogpBackBlock, 0, stream>>>(
                a, k, (int)pieces, first);
        HIP_TRY(hipGetLastError());
        return ZERO_OK;
    });
}

}  // extern "C"
