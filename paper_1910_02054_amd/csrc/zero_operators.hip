// zero_operators.hip -- host side of the training operators declared in
// include/zero_operators.h: argument checks, choice of the kernels' shapes, launches.
//
// The operators feed ZeRO's mixed-precision step (arXiv 1910.02054, Sec. 3.1): their fp16
// gradients carry the loss scale and overflow to inf, which the shard step finds.
#include <hip/hip_runtime.h>

#include "operator_args.hpp"
#include "norm_kernels.hpp"
#include "route_kernels.hpp"
#include "distill_kernels.hpp"

namespace zsh {
namespace {

// ---------------------------------------------------------------------------
// Norm.  The lanes of a row and its vectors a lane, from the row's 16-byte vectors: lanes of one
// wave while they hold the row in four vectors, then a workgroup, and of 1024 where that leaves a lane
// one vector or the rows are too few to fill the device otherwise (one row of 8192 f16 3.8 us, 5.2 with 256 lanes of
// four vectors).
// ---------------------------------------------------------------------------
template <int LPR_, int NV_>
struct RowShape {
    static constexpr int LPR = LPR_, NV = NV_;
};

template <typename T, typename F>
int with_wide_shape(int64_t vectors, F f) {
    if (vectors <= 1024) return f(RowShape<1024, 1>{});
    if (vectors <= 2048) return f(RowShape<1024, 2>{});
    if (T::kPer > 4 || vectors <= 4096) return f(RowShape<1024, 4>{});
    if constexpr (T::kPer == 4)
        return f(RowShape<1024, 8>{});
    return ZERO_EINVAL;  // more than ZERO_NORM_MAX_COLS
}

template <typename T, typename F>
int with_row_shape(int64_t vectors, int64_t rows, F f) {
    const bool few = rows <= 256;
    if (vectors <= 16) return f(RowShape<16, 1>{});
    if (vectors <= 64) return f(RowShape<64, 1>{});
    if (vectors <= 128) return f(RowShape<64, 2>{});
    if (vectors <= 256 && !few) return f(RowShape<64, 4>{});
    if (vectors <= 512 && !few) return f(RowShape<256, 2>{});
    return with_wide_shape<T>(vectors, f);
}

// The backward's workgroup has 1024 threads whatever the row, and a lane's registers hold two
// rows' arrays and a sum for each of its columns, so a lane has one vector up to rows of 1024.
template <typename T, typename F>
int with_back_shape(int64_t vectors, F f) {
    if (vectors <= 16) return f(RowShape<16, 1>{});
    if (vectors <= 64) return f(RowShape<64, 1>{});
    if (vectors <= 128) return f(RowShape<128, 1>{});
    if (vectors <= 256) return f(RowShape<256, 1>{});
    if (vectors <= 512) return f(RowShape<512, 1>{});
    return with_wide_shape<T>(vectors, f);
}

// Workgroups of the backward's grid, one a compute unit, each of which leaves one row of partial sums.
constexpr int64_t kBackBlocks = 256;

int64_t back_blocks(int64_t rows) { return std::max<int64_t>(1, std::min<int64_t>(rows, kBackBlocks)); }

int check_norm_sizes(const char* fn, int64_t rows, int64_t cols) {
    if (rows < 0 || rows > kMaxNumel)
        return fail(ZERO_EINVAL, "%s: rows = %lld is outside [0, 2^40]", fn, (long long)rows);
    if (cols < 1 || cols > ZERO_NORM_MAX_COLS)
        return fail(ZERO_EINVAL, "%s: cols = %lld is outside [1, %d]", fn, (long long)cols, ZERO_NORM_MAX_COLS);
    return ZERO_OK;
}

// ---------------------------------------------------------------------------
// Route.
// ---------------------------------------------------------------------------
template <int LPT_, int VPL_>
struct TokenShape {
    static constexpr int LPT = LPT_, VPL = VPL_;
};

// Keys a lane; what token_lanes leaves to each number of lanes.
template <int LPT, typename F>
int with_keys(int64_t need, F f) {
    if constexpr (LPT == 64)
        if (need > 16) return f(TokenShape<LPT, 32>{});
    if constexpr (LPT >= 32)
        if (need > 8) return f(TokenShape<LPT, 16>{});
    if (need > 4) return f(TokenShape<LPT, 8>{});
    return f(TokenShape<LPT, 4>{});
}

int log2_of(int pow2) { return __builtin_ctz((unsigned)pow2); }

// Lanes of a token: at least one a group and one a slot, and few enough keys a lane.  A round of the
// choice costs a few steps across the lanes and an operation for each key of a lane, and the
// tokens of a wave share them: up to 8 keys a lane (16384 tokens of 256 experts, 8 of them: 15.9 us, 19.8
// with 4 keys), up to 16 where a token would take a whole wave otherwise (32768 of 384, 10 of them: 45
// us, 50 with 8).
int token_lanes(int experts, int k, int groups) {
    const int g = pow2_up(groups), size = experts / groups;
    int lanes = std::max({8, pow2_up(k), g});
    while (lanes < 64 && div_up(size, lanes / g) > (lanes < 32 ? 8 : 16))
        lanes *= 2;
    return lanes;
}

// Slots that a workgroup of the ordering aims at: with fewer, every workgroup has more counts to read (the second
// kernel of 131072 slots of 256 experts 7.9 us, 9.5 with 1024; 24594 of 60: 5.7 either way).
constexpr int64_t kOrderRun = 2048, kOrderMaxBlocks = 256;

struct OrderPlan {
    int64_t blocks, run;
};

OrderPlan order_plan(int64_t slots) {
    int64_t blocks = std::max<int64_t>(1, std::min(kOrderMaxBlocks, div_up(slots, kOrderRun)));
    const int64_t run = std::max<int64_t>(1, div_up(div_up(slots, blocks), zo::kOrderBlock)) * zo::kOrderBlock;
    blocks = std::max<int64_t>(1, div_up(slots, run));
    return OrderPlan{blocks, run};
}

int check_order_sizes(const char* fn, int64_t slots, int experts) {
    if (slots < 0 || slots > INT32_MAX)
        return fail(ZERO_EINVAL, "%s: slots = %lld is outside [0, 2^31)", fn, (long long)slots);
    if (experts < 1 || experts > ZERO_ROUTE_MAX_EXPERTS)
        return fail(ZERO_EINVAL, "%s: experts = %d is outside [1, %d]", fn, experts, ZERO_ROUTE_MAX_EXPERTS);
    return ZERO_OK;
}

int check_choice(const char* fn, int dtype, int score, int64_t rows, int experts, int k, double scale) {
    TRY(check_sizes(fn, dtype, rows));
    if (score != ZERO_SCORE_SOFTMAX && score != ZERO_SCORE_SIGMOID)
        return fail(ZERO_EINVAL, "%s: score %d is neither softmax nor sigmoid", fn, score);
    if (experts < 1 || experts > ZERO_ROUTE_MAX_EXPERTS)
        return fail(ZERO_EINVAL, "%s: experts = %d is outside [1, %d]", fn, experts, ZERO_ROUTE_MAX_EXPERTS);
    if (k < 1 || k > ZERO_ROUTE_MAX_K || k > experts)
        return fail(ZERO_EINVAL, "%s: k = %d is outside [1, %d] or above experts = %d", fn, k, ZERO_ROUTE_MAX_K,
                    experts);
    if (rows > INT32_MAX / k)
        return fail(ZERO_EINVAL, "%s: rows * k = %lld * %d is not below 2^31", fn, (long long)rows, k);
    if (!is_fin32(scale))
        return fail(ZERO_EINVAL, "%s: scale must be finite in fp32", fn);
    return ZERO_OK;
}

// ---------------------------------------------------------------------------
// Distillation.  Threads of a row's workgroup and vectors a thread: in registers while a
// thread of 1024 needs at most 16, re-read above that (NV = 0).  Short rows take few threads with many
// vectors each, so that more rows are under way on a compute unit: 8192 rows of 11093 bf16, soft term alone, 72 us with
// 256 threads of 8 vectors, 110 with 1024 of 2 (the loss alone 37 and 74); 65536 of 2048 f16 114 us with 128 of 2,
// 164 with 256 of 1.
// ---------------------------------------------------------------------------
template <int NT_, int NV_>
struct DistillShape {
    static constexpr int NT = NT_, NV = NV_;
};

template <typename F>
int with_distill_shape(int64_t vectors, F f) {
    if (vectors <= 128) return f(DistillShape<128, 1>{});
    if (vectors <= 256) return f(DistillShape<128, 2>{});
    if (vectors <= 512) return f(DistillShape<128, 4>{});
    if (vectors <= 1024) return f(DistillShape<256, 4>{});
    if (vectors <= 2 * 1024) return f(DistillShape<256, 8>{});
    if (vectors <= 4 * 1024) return f(DistillShape<512, 8>{});
    if (vectors <= 7 * 1024) return f(DistillShape<1024, 7>{});
    if (vectors <= 10 * 1024) return f(DistillShape<1024, 10>{});
    if (vectors <= 13 * 1024) return f(DistillShape<1024, 13>{});
    if (vectors <= 16 * 1024) return f(DistillShape<1024, 16>{});
    return f(DistillShape<1024, 0>{});
}

template <int MODE>
int distill(const char* fn, const zero_distill_args_t* args, void* stream_) {
    if (!args)
        return fail(ZERO_EINVAL, "%s: NULL args", fn);
    const zero_distill_args_t a = *args;
    TRY(check_sizes(fn, a.dtype, a.rows));
    if (a.k > 0 && !known_type(a.teacher_dtype))
        return fail(ZERO_EINVAL, "%s: teacher_dtype %d is none of ZERO_F32, ZERO_F16, ZERO_BF16", fn, a.teacher_dtype);
    if (a.vocab < 1 || a.vocab > (int64_t)1 << 30)
        return fail(ZERO_EINVAL, "%s: vocab = %lld is outside [1, 2^30]", fn, (long long)a.vocab);
    if (a.k < 0 || a.k > ZERO_DISTILL_MAX_K)
        return fail(ZERO_EINVAL, "%s: k = %d is outside [0, %d]", fn, a.k, ZERO_DISTILL_MAX_K);
    if (!(a.temperature >= 1e-30 && a.temperature <= 1e30))  // its reciprocal is held in fp32
        return fail(ZERO_EINVAL, "%s: temperature must lie in [1e-30, 1e30]", fn);
    if (!is_fin32(a.soft * a.temperature) || !is_fin32(a.hard) || !is_fin32(a.grad_scale))
        return fail(ZERO_EINVAL, "%s: soft * temperature, hard and grad_scale must be finite in fp32", fn);
    const bool back = MODE == zo::kDistillBack;
    if (back ? a.loss != nullptr : a.dloss != nullptr)
        return fail(ZERO_EINVAL, "%s: %s must be NULL", fn, back ? "loss" : "dloss");
    if (MODE == zo::kDistillStep && a.stats)
        return fail(ZERO_EINVAL, "%s: stats must be NULL", fn);
    if (MODE == zo::kDistillLoss && a.dlogits)
        return fail(ZERO_EINVAL, "%s: dlogits must be NULL", fn);
    const size_t e = elem_size(a.dtype);
    Arrays t(fn);
    static const char *const kLogits = "logits", *const kGrad = "dlogits";
    TRY(t.add(kLogits, a.logits, a.rows, a.vocab, a.ld_logits, e, false));
    TRY(t.add("teacher_index", a.teacher_index, a.rows, a.k, a.k, 4, false));
    TRY(t.add("teacher_logits", a.teacher_logits, a.rows, a.k, a.k, a.k ? elem_size(a.teacher_dtype) : 1, false));
    TRY(t.add("labels", a.labels, a.rows, 1, 1, 4, false, true));
    TRY(t.add("row_weight", a.row_weight, a.rows, 1, 1, 4, false, true));
    if (!back)
        TRY(t.add("loss", a.loss, a.rows, 1, 1, 4, true));
    if (MODE != zo::kDistillStep)
        TRY(t.add("stats", a.stats, a.rows, 3, 3, 4, !back, !back));
    TRY(t.add("dloss", a.dloss, a.rows, 1, 1, 4, false, true));
    if (MODE != zo::kDistillLoss)
        TRY(t.add(kGrad, a.dlogits, a.rows, a.vocab, a.ld_dlogits, e, true));
    TRY(t.check_overlaps({{kLogits, kGrad}}));
    if (a.rows == 0)
        return ZERO_OK;
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    TRY(t.check_memory(stream));

    const double log2e = 1.4426950408889634074, ln2 = 0.69314718055994530942;
    zo::DistillScalars k;
    k.c = (float)(log2e / (a.soft != 0.0 ? a.temperature : 1.0));  // the hard term alone is of temperature 1
    k.c1 = (float)log2e;
    k.bit = (float)(a.temperature * ln2);
    k.soft_grad = (float)(a.soft * a.temperature);
    k.soft_in = std::fabs(k.soft_grad) < 1.f ? k.soft_grad : 1.f;
    k.soft_out = std::fabs(k.soft_grad) < 1.f ? 1.f : k.soft_grad;
    k.hard = a.labels ? (float)a.hard : 0.f;
    k.scale = (float)a.grad_scale;
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        const int64_t vectors = a.vocab / T::kPer;
        const int heads = pow2_up(2 * (a.k + 1));
        auto launch = [&](auto shape) {
            using S = decltype(shape);
            for (int64_t first = 0; first < a.rows; first += kMaxLaunch)
                zo::k_distill<T, S::NT, S::NV, MODE>
                    <<<(unsigned)std::min(kMaxLaunch, a.rows - first), S::NT,
                       zo::distill_lds_bytes(a.k, heads, MODE), stream>>>(a, k, heads, first);
            HIP_TRY(hipGetLastError());
            return ZERO_OK;
        };
        return with_distill_shape(vectors, launch);
    });
}

}  // namespace
}  // namespace zsh

using namespace zsh;

extern "C" {

int zero_rms_norm(const zero_rms_norm_args_t* args, void* stream_) {
    const char* fn = "zero_rms_norm";
    if (!args)
        return fail(ZERO_EINVAL, "%s: NULL args", fn);
    const zero_rms_norm_args_t a = *args;
    TRY(check_sizes(fn, a.dtype, a.rows));
    TRY(check_norm_sizes(fn, a.rows, a.cols));
    if (!is_fin(a.eps) || a.eps < 0.0)
        return fail(ZERO_EINVAL, "%s: eps must be finite and >= 0", fn);
    if (a.group != 0 && a.group != 32 && a.group != 64 && a.group != 128 && a.group != 256)
        return fail(ZERO_EINVAL, "%s: group = %d is none of 0, 32, 64, 128, 256", fn, a.group);
    if (!a.q8 != !a.scale)
        return fail(ZERO_EINVAL, "%s: q8 and scale come together", fn);
    if (a.h && !a.residual)
        return fail(ZERO_EINVAL, "%s: h is x where there is no residual", fn);
    const size_t e = elem_size(a.dtype);
    static const char *const kX = "x", *const kRes = "residual", *const kH = "h", *const kY = "y";
    Arrays t(fn);
    TRY(t.add(kX, a.x, a.rows, a.cols, a.ld_x, e, false));
    TRY(t.add(kRes, a.residual, a.rows, a.cols, a.ld_residual, e, false, true));
    TRY(t.add("weight", a.weight, 1, a.cols, a.cols, e, false));
    TRY(t.add(kH, a.h, a.rows, a.cols, a.ld_h, e, true, true));
    TRY(t.add(kY, a.y, a.rows, a.cols, a.ld_y, e, true, true));
    TRY(t.add("q8", a.q8, a.rows, a.cols, a.ld_q8, 1, true, true));
    const int64_t groups = a.group ? div_up(a.cols, a.group) : 1;
    TRY(t.add("scale", a.scale, a.rows, groups, groups, 4, true, true));
    TRY(t.add("rstd", a.rstd, a.rows, 1, 1, 4, true, true));
    TRY(t.check_overlaps({{kH, kX}, {kH, kRes}, {kY, kX}, {kY, kRes}}));
    if (a.rows == 0)
        return ZERO_OK;
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    TRY(t.check_memory(stream));
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        return with_row_shape<T>(div_up(a.cols, T::kPer), a.rows, [&](auto shape) {
            using S = decltype(shape);
            constexpr int kRows = zo::norm_block(S::LPR) / S::LPR;
            for (int64_t first = 0; first < a.rows; first += kMaxLaunch * kRows)
                zo::k_rms_norm<T, S::LPR, S::NV>
                    <<<(unsigned)std::min(kMaxLaunch, div_up(a.rows - first, kRows)), zo::norm_block(S::LPR), 0,
                       stream>>>(a, first);
            HIP_TRY(hipGetLastError());
            return ZERO_OK;
        });
    });
}

int zero_rms_norm_workspace(int64_t rows, int64_t cols, int64_t* floats) {
    const char* fn = "zero_rms_norm_workspace";
    if (!floats)
        return fail(ZERO_EINVAL, "%s: NULL floats", fn);
    TRY(check_norm_sizes(fn, rows, cols));
    const int64_t blocks = back_blocks(rows);
    *floats = blocks > 1 ? blocks * cols : 0;
    return ZERO_OK;
}

int zero_rms_norm_backward(const zero_rms_norm_backward_args_t* args, void* stream_) {
    const char* fn = "zero_rms_norm_backward";
    if (!args)
        return fail(ZERO_EINVAL, "%s: NULL args", fn);
    const zero_rms_norm_backward_args_t a = *args;
    TRY(check_sizes(fn, a.dtype, a.rows));
    TRY(check_norm_sizes(fn, a.rows, a.cols));
    const size_t e = elem_size(a.dtype);
    static const char *const kDy = "dy", *const kH = "h", *const kDh = "dh", *const kDx = "dx";
    int64_t floats = 0;
    TRY(zero_rms_norm_workspace(a.rows, a.cols, &floats));
    if (a.workspace_floats < floats)
        return fail(ZERO_EINVAL, "%s: the workspace has %lld floats, %lld are needed", fn,
                    (long long)a.workspace_floats, (long long)floats);
    Arrays t(fn);
    TRY(t.add(kDy, a.dy, a.rows, a.cols, a.ld_dy, e, false));
    TRY(t.add(kH, a.h, a.rows, a.cols, a.ld_h, e, false));
    TRY(t.add("weight", a.weight, 1, a.cols, a.cols, e, false));
    TRY(t.add("rstd", a.rstd, a.rows, 1, 1, 4, false));
    TRY(t.add(kDh, a.dh, a.rows, a.cols, a.ld_dh, e, false, true));
    TRY(t.add(kDx, a.dx, a.rows, a.cols, a.ld_dx, e, true));
    TRY(t.add("dweight", a.dweight, 1, a.cols, a.cols, e, true));
    TRY(t.add("workspace", a.workspace, 1, floats, floats, 4, true));
    TRY(t.check_overlaps({{kDx, kDy}, {kDx, kH}, {kDx, kDh}}));
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    TRY(t.check_memory(stream));
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        using elem = typename T::elem;
        return with_back_shape<T>(div_up(a.cols, T::kPer), [&](auto shape) {
            using S = decltype(shape);
            constexpr int kRows = zo::kBackBlock / S::LPR;
            const int64_t grid = std::max<int64_t>(1, std::min(back_blocks(a.rows), div_up(a.rows, kRows)));
            zo::k_rms_norm_back<T, S::LPR, S::NV>
                <<<(unsigned)grid, zo::kBackBlock, 0, stream>>>(a, a.workspace);
            HIP_TRY(hipGetLastError());
            if (grid > 1) {
                zo::k_column_sums<T><<<(unsigned)div_up(a.cols, zo::kSumCols), zo::kSumCols * zo::kSumRuns, 0, stream>>>(
                    a.workspace, (int)grid, (int)a.cols, static_cast<elem*>(a.dweight));
                HIP_TRY(hipGetLastError());
            }
            return ZERO_OK;
        });
    });
}

int zero_route(const zero_route_args_t* args, void* stream_) {
    const char* fn = "zero_route";
    if (!args)
        return fail(ZERO_EINVAL, "%s: NULL args", fn);
    const zero_route_args_t a = *args;
    TRY(check_choice(fn, a.dtype, a.score, a.rows, a.experts, a.k, a.scale));
    if (a.groups < 1 || a.groups > 64 || a.experts % a.groups)
        return fail(ZERO_EINVAL, "%s: groups = %d is outside [1, 64] or does not divide experts = %d", fn, a.groups,
                    a.experts);
    if (a.top_groups < 1 || a.top_groups > a.groups)
        return fail(ZERO_EINVAL, "%s: top_groups = %d is outside [1, %d]", fn, a.top_groups, a.groups);
    if (a.group_top != 1 && a.group_top != 2)
        return fail(ZERO_EINVAL, "%s: group_top = %d is neither 1 nor 2", fn, a.group_top);
    if (a.groups > 1 && a.group_top == 2 && a.experts / a.groups < 2)
        return fail(ZERO_EINVAL, "%s: group_top = 2 needs groups of two experts or more", fn);
    Arrays t(fn);
    TRY(t.add("logits", a.logits, a.rows, a.experts, a.ld_logits, elem_size(a.dtype), false));
    TRY(t.add("bias", a.bias, 1, a.experts, a.experts, 4, false, true));
    TRY(t.add("index", a.index, a.rows, a.k, a.k, 4, true));
    TRY(t.add("weight", a.weight, a.rows, a.k, a.k, 4, true));
    TRY(t.check_overlaps({}));
    if (a.rows == 0)
        return ZERO_OK;
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    TRY(t.check_memory(stream));
    const int lanes = token_lanes(a.experts, a.k, a.groups), size = a.experts / a.groups;
    const int per_group = lanes / pow2_up(a.groups);
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        auto launch = [&](auto shape) {
            using S = decltype(shape);
            constexpr int kTokens = zo::kRouteBlock / S::LPT;
            for (int64_t first = 0; first < a.rows; first += kMaxLaunch * kTokens)
                zo::k_route<T, S::LPT, S::VPL>
                    <<<(unsigned)std::min(kMaxLaunch, div_up(a.rows - first, kTokens)), zo::kRouteBlock, 0, stream>>>(
                        a, size, log2_of(per_group), first);
            HIP_TRY(hipGetLastError());
            return ZERO_OK;
        };
        const int64_t need = div_up(size, per_group);
        switch (lanes) {
            case 8: return with_keys<8>(need, launch);
            case 16: return with_keys<16>(need, launch);
            case 32: return with_keys<32>(need, launch);
            default: return with_keys<64>(need, launch);
        }
    });
}

int zero_route_workspace(int64_t slots, int32_t experts, int64_t* ints) {
    const char* fn = "zero_route_workspace";
    if (!ints)
        return fail(ZERO_EINVAL, "%s: NULL ints", fn);
    TRY(check_order_sizes(fn, slots, experts));
    const OrderPlan p = order_plan(slots);
    *ints = p.blocks > 1 ? p.blocks * (experts + 1) : 0;
    return ZERO_OK;
}

int zero_route_order(const zero_route_order_args_t* args, void* stream_) {
    const char* fn = "zero_route_order";
    if (!args)
        return fail(ZERO_EINVAL, "%s: NULL args", fn);
    const zero_route_order_args_t a = *args;
    int64_t ints = 0;
    TRY(check_order_sizes(fn, a.slots, a.experts));
    TRY(zero_route_workspace(a.slots, a.experts, &ints));
    if (a.workspace_ints < ints)
        return fail(ZERO_EINVAL, "%s: the workspace has %lld ints, %lld are needed", fn, (long long)a.workspace_ints,
                    (long long)ints);
    Arrays t(fn);
    TRY(t.add("index", a.index, 1, a.slots, a.slots, 4, false));
    TRY(t.add("offsets", a.offsets, 1, a.experts + 1, a.experts + 1, 4, true));
    TRY(t.add("order", a.order, 1, a.slots, a.slots, 4, true));
    TRY(t.add("workspace", a.workspace, 1, ints, ints, 4, true));
    TRY(t.check_overlaps({}));
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    TRY(t.check_memory(stream));
    const OrderPlan p = order_plan(a.slots);
    if (p.blocks > 1) {
        zo::k_route_count<<<(unsigned)p.blocks, zo::kOrderBlock, 0, stream>>>(a.index, a.slots, a.experts, p.run,
                                                                             a.workspace);
        HIP_TRY(hipGetLastError());
    }
    // a thread looks after one key, or with more experts than that after a few
    auto* const kernel = a.experts < zo::kOrderBlock ? zo::k_route_order<1> : zo::k_route_order<zo::kOrderOwn>;
    kernel<<<(unsigned)p.blocks, zo::kOrderBlock, 0, stream>>>(
        a.index, a.slots, a.experts, p.run, p.blocks > 1 ? a.workspace : nullptr, a.offsets, a.order);
    HIP_TRY(hipGetLastError());
    return ZERO_OK;
}

int zero_route_backward(const zero_route_backward_args_t* args, void* stream_) {
    const char* fn = "zero_route_backward";
    if (!args)
        return fail(ZERO_EINVAL, "%s: NULL args", fn);
    const zero_route_backward_args_t a = *args;
    TRY(check_choice(fn, a.dtype, a.score, a.rows, a.experts, a.k, a.scale));
    const size_t e = elem_size(a.dtype);
    static const char *const kLogits = "logits", *const kGrad = "dlogits";
    Arrays t(fn);
    TRY(t.add(kLogits, a.logits, a.rows, a.experts, a.ld_logits, e, false));
    TRY(t.add("bias", a.bias, 1, a.experts, a.experts, 4, false, true));
    TRY(t.add("index", a.index, a.rows, a.k, a.k, 4, false));
    TRY(t.add("dweight", a.dweight, a.rows, a.k, a.k, 4, false));
    TRY(t.add(kGrad, a.dlogits, a.rows, a.experts, a.ld_dlogits, e, true));
    TRY(t.check_overlaps({{kLogits, kGrad}}));
    if (a.rows == 0)
        return ZERO_OK;
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    TRY(t.check_memory(stream));
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        auto launch = [&](auto lanes) {
            constexpr int kLanes = decltype(lanes)::value, kTokens = zo::kRouteBlock / kLanes;
            for (int64_t first = 0; first < a.rows; first += kMaxLaunch * kTokens)
                zo::k_route_back<T, kLanes>
                    <<<(unsigned)std::min(kMaxLaunch, div_up(a.rows - first, kTokens)), zo::kRouteBlock,
                       sizeof(float) * kTokens * a.experts, stream>>>(a, first);
            HIP_TRY(hipGetLastError());
            return ZERO_OK;
        };
        const int lanes = std::min(64, std::max({8, pow2_up(a.k), pow2_up(div_up(a.experts, T::kPer))}));
        switch (lanes) {
            case 8: return launch(std::integral_constant<int, 8>{});
            case 16: return launch(std::integral_constant<int, 16>{});
            case 32: return launch(std::integral_constant<int, 32>{});
            default: return launch(std::integral_constant<int, 64>{});
        }
    });
}

int zero_distill_step(const zero_distill_args_t* args, void* stream) {
    return distill<zo::kDistillStep>("zero_distill_step", args, stream);
}

int zero_distill_loss(const zero_distill_args_t* args, void* stream) {
    return distill<zo::kDistillLoss>("zero_distill_loss", args, stream);
}

int zero_distill_backward(const zero_distill_args_t* args, void* stream) {
    return distill<zo::kDistillBack>("zero_distill_backward", args, stream);
}

}  // extern "C"
