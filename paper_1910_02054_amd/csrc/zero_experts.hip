// zero_experts.hip -- host side of the experts' operators declared in include/zero_operators.h
// (zero_expert_*): argument checks, choice of the kernels' shapes, launches.
#include <hip/hip_runtime.h>

#include <cmath>

#include "operator_args.hpp"
#include "expert_kernels.hpp"

namespace zsh {
namespace {

int check_expert_sizes(const char* fn, int64_t slots, int experts, int64_t cols_in, int64_t cols_out) {
    if (slots < 0 || slots > INT32_MAX)
        return fail(ZERO_EINVAL, "%s: slots = %lld is outside [0, 2^31)", fn, (long long)slots);
    if (experts < 1 || experts > ZERO_ROUTE_MAX_EXPERTS)
        return fail(ZERO_EINVAL, "%s: experts = %d is outside [1, %d]", fn, experts, ZERO_ROUTE_MAX_EXPERTS);
    if (cols_in < 1 || cols_in > ZERO_EXPERT_MAX_COLS || cols_out < 1 || cols_out > ZERO_EXPERT_MAX_COLS)
        return fail(ZERO_EINVAL, "%s: cols_in = %lld or cols_out = %lld is outside [1, %d]", fn, (long long)cols_in,
                    (long long)cols_out, ZERO_EXPERT_MAX_COLS);
    return ZERO_OK;
}

// `per`: slots that share a row.
int check_slots(const char* fn, const char* name, int per, int most, int64_t slots, const void* order) {
    if (per < 0 || per > most)
        return fail(ZERO_EINVAL, "%s: %s = %d is outside [0, %d]", fn, name, per, most);
    if (per > 1 && slots % per)
        return fail(ZERO_EINVAL, "%s: %s = %d does not divide slots = %lld", fn, name, per, (long long)slots);
    if (per > 0 && slots > 0 && !order)
        return fail(ZERO_EINVAL, "%s: order is NULL with %s = %d", fn, name, per);
    return ZERO_OK;
}

int64_t matrix_rows(int64_t slots, int per) { return per > 1 ? slots / per : slots; }

// The quotient of a slot below 2^31 by `per` as (slot * mul) >> shift: with L bits in per - 1 and
// mul = floor(2^(31 + L) / per) + 1 the excess of the product is below 2^(31 + L) / per.
zo::SlotMap slot_map(int per) {
    zo::SlotMap m{per, 0, 0};
    if (per > 1) {
        int bits = 0;
        while ((int64_t)1 << bits < per)
            ++bits;
        m.shift = 31 + bits;
        m.mul = (uint32_t)(((uint64_t)1 << m.shift) / (uint64_t)per + 1);
    }
    return m;
}

// Whether a matrix's rows are made of aligned 16-byte chunks.
bool whole_chunks(const void* p, int64_t ld, int64_t cols, size_t elem) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * elem % 16 == 0 && cols * elem % 16 == 0;
}

constexpr int64_t kCus = 256;  // MI355X

// The kernel that takes tiles in a run, in tiles of 256 or 128 rows by 256 columns: the shape whose rounds of
// tiles over the compute units cost less.  A round of 128 rows is 0.58 of one of 256 (8192 slots of 16 experts
// 4096 to 1600 f16, 280 tiles in 2 rounds of 256 or 504 in 2 of 128: 210 and 150 us; 4096 of 8 experts 1600 to
// 6400, 500 in 2 or 900 in 4: 107 and 124; 131072 of 64, 1024 to 4096 bf16: 1157 and 1338).
template <typename F>
int with_run_shape(int64_t slots, int experts, int64_t cols_out, F f) {
    auto rounds = [&](int64_t rows) {
        return (double)div_up((slots / rows + experts / 2) * div_up(cols_out, 256), kCus);
    };
    if (0.58 * rounds(128) < rounds(256)) return f(zo::TileShape<128, 256, 2, 4, 3>{});
    return f(zo::TileShape<256, 256, 2, 4, 2>{});
}

// Rows of a part of the weights' gradient's sums, 0: an expert's rows are one.  A longer part takes longer (1.5 us
// for 64 rows), a shorter one leaves more sums to be written and read again (at 4.5 TB/s): slots / part matrices
// of `size` floats.  The length at which both are the same, 256 at least, if the workspace's bound allows it.  Half and
// twice that: 65536 slots of 8, 512 by 512 bf16: 68.2 us, 68.7 and 96.3; 16384 of 8, 128 by 256 f16: 23.0, 23.0 and 24.8;
// 16384 of one of 8, 256 by 256 f16: 44.4, 46.3 and 43.2; 65536 of 64, 512 by 256 bf16: 61.4, 61.4 and 53.2.  128 or 512 at
// least: 16384 of 16, 128 by 128 fp32: 38.3, 33.5 and 61.1; 16384 of 8, 128 by 256 f16: 23.0, 23.0 and 26.0.
int64_t part_rows(int64_t slots, int experts, int64_t size) {
    const int64_t room = ZERO_EXPERT_WORKSPACE_MAX / size - experts;  // parts behind each expert's first
    if (room < 1)
        return 0;
    const double even = std::sqrt(8.0 * (double)size * (double)slots / 4.5e6 * 64 / 1.5);
    const int64_t rows = std::max({(int64_t)256, (int64_t)even, div_up(slots, room)});
    return rows < slots ? div_up(rows, 64) * 64 : 0;
}

// Slots to an expert on average up to which its rows go in tiles of 32 by 128, a workgroup each, instead of in runs of
// large tiles: many more workgroups where the experts or columns are few, but every 32 rows copy the weights to LDS
// again.  Small tiles and large, bf16, 48 rows an expert: 8 experts 4096 to 1024 33.5 us and 67.5, 1024 to 4096 21.3
// and 24.1; 64 experts 134 and 104, 152 and 119.  8 rows: 31.8 and 66.9, 17.8 and 22.9; 64 experts 99.9 and 98.9, 118 and
// 109.  128 rows: 50.3 and 69.7, 33.9 and 25.9; 64 experts 211 and 140, 226 and 153.  The host knows the average alone: 2048
// slots of 64 experts 1024 to 4096 that all chose one take 40.5 us, in large tiles 24.3.
constexpr int64_t kFewRows = 48;
constexpr uint32_t kMaxTiles = 1 << 20;  // workgroups of one launch

}  // namespace
}  // namespace zsh

using namespace zsh;

extern "C" {

int zero_expert_product(const zero_expert_product_args_t* args, void* stream_) {
    const char* fn = "zero_expert_product";
    if (!args)
        return fail(ZERO_EINVAL, "%s: NULL args", fn);
    const zero_expert_product_args_t a = *args;
    TRY(check_sizes(fn, a.dtype, a.slots));
    TRY(check_expert_sizes(fn, a.slots, a.experts, a.cols_in, a.cols_out));
    TRY(check_slots(fn, "x_slots", a.x_slots, INT32_MAX, a.slots, a.order));
    TRY(check_slots(fn, "y_slots", a.y_slots, 1, a.slots, a.order));
    const size_t e = elem_size(a.dtype);
    const int64_t w_rows = a.experts * (a.transposed ? a.cols_out : a.cols_in), w_cols = a.transposed ? a.cols_in : a.cols_out;
    Arrays t(fn);
    TRY(t.add("offsets", a.offsets, 1, a.experts + 1, a.experts + 1, 4, false));
    TRY(t.add("order", a.order, 1, a.slots, a.slots, 4, false, true));
    TRY(t.add("x", a.x, matrix_rows(a.slots, a.x_slots), a.cols_in, a.ld_x, e, false));
    TRY(t.add("weight", a.weight, w_rows, w_cols, a.ld_weight, e, false));
    TRY(t.add("y", a.y, a.slots, a.cols_out, a.ld_y, e, true));
    TRY(t.check_overlaps({}));
    if (a.slots == 0)
        return ZERO_OK;
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    TRY(t.check_memory(stream));
    zo::ExpertCall c{};
    c.offsets = a.offsets;
    c.order = a.order;
    c.x = a.x;
    c.ld_x = a.ld_x;
    c.w = a.weight;
    c.ld_w = a.ld_weight;
    c.out = a.y;
    c.ld_out = a.ld_y;
    c.slots = a.slots;
    c.experts = a.experts;
    c.cols_in = (int)a.cols_in;
    c.cols_out = (int)a.cols_out;
    c.x_map = slot_map(a.x_slots);
    c.out_map = slot_map(a.y_slots);
    const bool dma = whole_chunks(a.x, a.ld_x, a.cols_in, e) && whole_chunks(a.weight, a.ld_weight, w_cols, e);
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        auto by_tile = [&](auto shape, auto* kernel) {  // a workgroup a tile
            using S = decltype(shape);
            // every expert's last tile may hold one row
            const int64_t rows = std::min<int64_t>(a.slots, a.slots / S::BM + a.experts);
            const int64_t tiles = rows * div_up(a.cols_out, S::BN);
            for (int64_t first = 0; first < tiles; first += kMaxTiles) {
                const uint32_t n = (uint32_t)std::min<int64_t>(kMaxTiles, tiles - first);
                kernel<<<(n + 7) / 8 * 8, S::kThreads, 0, stream>>>(c, (uint32_t)first, n);
            }
            HIP_TRY(hipGetLastError());
            return (int)ZERO_OK;
        };
        if (a.slots / a.experts <= kFewRows) {
            using S = zo::TileShape<32, 128, 1, 4, 4>;
            return by_tile(S{}, a.transposed ? (dma ? zo::k_expert_product<T, S, true, true>
                                                    : zo::k_expert_product<T, S, true, false>)
                                             : (dma ? zo::k_expert_product<T, S, false, true>
                                                    : zo::k_expert_product<T, S, false, false>));
        }
        auto in_runs = [&](auto shape, auto* kernel) {
            using S = decltype(shape);
            kernel<<<kCus * S::kPerCu, S::kThreads, 0, stream>>>(c);
            HIP_TRY(hipGetLastError());
            return (int)ZERO_OK;
        };
        // fp32: the products take most of the time whatever the tile (a sixteenth of bf16's rate), so small tiles,
        // evenly over the compute units, three workgroups to each (3063 slots of 12 experts 803 to 1203: 102 us, 116
        // in tiles of 64 by 128, 201 of 128 by 128; 1065 of 8 experts 6943 to 3769: 957 and 1401 of 64 by 128)
        if constexpr (T::kPer == 4) {
            using S = zo::TileShape<64, 64, 2, 2, 2>;
            return in_runs(S{}, a.transposed ? (dma ? zo::k_expert_product_run<T, S, true, true>
                                                    : zo::k_expert_product_run<T, S, true, false>)
                                             : (dma ? zo::k_expert_product_run<T, S, false, true>
                                                    : zo::k_expert_product_run<T, S, false, false>));
        } else {
            if (!dma) {
                using S = zo::TileShape<128, 256, 2, 4, 2>;
                return in_runs(S{}, a.transposed ? zo::k_expert_product_run<T, S, true, false>
                                                 : zo::k_expert_product_run<T, S, false, false>);
            }
            return with_run_shape(a.slots, a.experts, a.cols_out, [&](auto shape) {
                using S = decltype(shape);
                return in_runs(shape, a.transposed ? zo::k_expert_product_run<T, S, true, true>
                                                   : zo::k_expert_product_run<T, S, false, true>);
            });
        }
    });
}

int zero_expert_workspace(int64_t slots, int32_t experts, int64_t cols_in, int64_t cols_out, int64_t* floats) {
    const char* fn = "zero_expert_workspace";
    if (!floats)
        return fail(ZERO_EINVAL, "%s: NULL floats", fn);
    TRY(check_expert_sizes(fn, slots, experts, cols_in, cols_out));
    const int64_t rows = part_rows(slots, experts, cols_in * cols_out);
    *floats = rows ? (slots / rows + experts) * cols_in * cols_out : 0;
    return ZERO_OK;
}

int zero_expert_weight_backward(const zero_expert_weight_backward_args_t* args, void* stream_) {
    const char* fn = "zero_expert_weight_backward";
    if (!args)
        return fail(ZERO_EINVAL, "%s: NULL args", fn);
    const zero_expert_weight_backward_args_t a = *args;
    TRY(check_sizes(fn, a.dtype, a.slots));
    TRY(check_expert_sizes(fn, a.slots, a.experts, a.cols_in, a.cols_out));
    TRY(check_slots(fn, "x_slots", a.x_slots, INT32_MAX, a.slots, a.order));
    TRY(check_slots(fn, "dy_slots", a.dy_slots, INT32_MAX, a.slots, a.order));
    int64_t floats = 0;
    TRY(zero_expert_workspace(a.slots, a.experts, a.cols_in, a.cols_out, &floats));
    if (a.workspace_floats < floats)
        return fail(ZERO_EINVAL, "%s: the workspace has %lld floats, %lld are needed", fn,
                    (long long)a.workspace_floats, (long long)floats);
    const size_t e = elem_size(a.dtype);
    Arrays t(fn);
    TRY(t.add("offsets", a.offsets, 1, a.experts + 1, a.experts + 1, 4, false));
    TRY(t.add("order", a.order, 1, a.slots, a.slots, 4, false, true));
    TRY(t.add("x", a.x, matrix_rows(a.slots, a.x_slots), a.cols_in, a.ld_x, e, false));
    TRY(t.add("dy", a.dy, matrix_rows(a.slots, a.dy_slots), a.cols_out, a.ld_dy, e, false));
    TRY(t.add("dweight", a.dweight, a.experts * a.cols_in, a.cols_out, a.ld_dweight, e, true));
    TRY(t.add("workspace", a.workspace, 1, floats, floats, 4, true));
    TRY(t.check_overlaps({}));
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    TRY(t.check_memory(stream));
    zo::ExpertCall c{};
    c.offsets = a.offsets;
    c.order = a.order;
    c.x = a.x;
    c.ld_x = a.ld_x;
    c.w = a.dy;
    c.ld_w = a.ld_dy;
    c.out = a.dweight;
    c.ld_out = a.ld_dweight;
    c.partial = a.workspace;
    c.slots = a.slots;
    c.experts = a.experts;
    c.cols_in = (int)a.cols_in;
    c.cols_out = (int)a.cols_out;
    c.part = (int)part_rows(a.slots, a.experts, a.cols_in * a.cols_out);
    c.x_map = slot_map(a.x_slots);
    c.out_map = slot_map(a.dy_slots);
    const bool dma = whole_chunks(a.x, a.ld_x, a.cols_in, e) && whole_chunks(a.dy, a.ld_dy, a.cols_out, e);
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        // Tiles of 256 by 256, but where they would be half empty (16384 slots of 64 experts, 128 by 128 f16: 19
        // us, 24 in tiles of 256; 65536 of 64, 512 by 256 bf16: 80 and 61) and for fp32, bound by the products
        // (8192 of 8, 1024 by 4096: 720 and 830).
        using Wide = zo::TileShape<256, 256, 2, 4, 2>;
        using Small = zo::TileShape<128, 128, 2, 2, 2>;  // two workgroups to a compute unit
        if (!dma)
            zo::k_expert_weight_back<T, Small, false><<<kCus * Small::kPerCu, Small::kThreads, 0, stream>>>(c);
        else if (T::kPer == 4 || std::min(a.cols_in, a.cols_out) <= 128)
            zo::k_expert_weight_back<T, Small, true><<<kCus * Small::kPerCu, Small::kThreads, 0, stream>>>(c);
        else if constexpr (T::kPer == 8)
            zo::k_expert_weight_back<T, Wide, true><<<kCus * Wide::kPerCu, Wide::kThreads, 0, stream>>>(c);
        HIP_TRY(hipGetLastError());
        if (c.part) {
            const dim3 grid((unsigned)div_up(a.cols_in * a.cols_out, 4 * zo::kJoinBlock), (unsigned)a.experts);
            zo::k_expert_join<T><<<grid, zo::kJoinBlock, 0, stream>>>(c);
            HIP_TRY(hipGetLastError());
        }
        return (int)ZERO_OK;
    });
}

static int check_mix(const char* fn, int dtype, int64_t tokens, int64_t cols, int k, int experts) {
    TRY(check_sizes(fn, dtype, tokens));
    if (k < 1 || k > ZERO_ROUTE_MAX_K)
        return fail(ZERO_EINVAL, "%s: k = %d is outside [1, %d]", fn, k, ZERO_ROUTE_MAX_K);
    if (tokens > INT32_MAX / k)
        return fail(ZERO_EINVAL, "%s: tokens * k = %lld * %d is not below 2^31", fn, (long long)tokens, k);
    if (cols < 1 || cols > ZERO_EXPERT_MAX_COLS)
        return fail(ZERO_EINVAL, "%s: cols = %lld is outside [1, %d]", fn, (long long)cols, ZERO_EXPERT_MAX_COLS);
    if (experts < 0)
        return fail(ZERO_EINVAL, "%s: experts = %d is below 0", fn, experts);
    return ZERO_OK;
}

int zero_expert_mix(const zero_expert_mix_args_t* args, void* stream_) {
    const char* fn = "zero_expert_mix";
    if (!args)
        return fail(ZERO_EINVAL, "%s: NULL args", fn);
    const zero_expert_mix_args_t a = *args;
    TRY(check_mix(fn, a.dtype, a.tokens, a.cols, a.k, a.experts));
    const size_t e = elem_size(a.dtype);
    static const char *const kBase = "base", *const kOut = "out";
    Arrays t(fn);
    TRY(t.add("index", a.index, a.tokens, a.k, a.k, 4, false, true));
    TRY(t.add("weight", a.weight, a.tokens, a.k, a.k, 4, false, true));
    TRY(t.add("y", a.y, a.tokens * a.k, a.cols, a.ld_y, e, false));
    TRY(t.add(kBase, a.base, a.tokens, a.cols, a.ld_base, e, false, true));
    TRY(t.add(kOut, a.out, a.tokens, a.cols, a.ld_out, e, true));
    TRY(t.check_overlaps({{kBase, kOut}}));
    if (a.tokens == 0)
        return ZERO_OK;
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    TRY(t.check_memory(stream));
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        const int64_t lanes = div_up(a.cols, T::kPer), all = a.tokens * lanes, most = kMaxLaunch * zo::kMixBlock;
        for (int64_t first = 0; first < all; first += most)
            zo::k_expert_mix<T><<<(unsigned)div_up(std::min(most, all - first), zo::kMixBlock), zo::kMixBlock, 0,
                                  stream>>>(a, (int)lanes, first);
        HIP_TRY(hipGetLastError());
        return ZERO_OK;
    });
}

int zero_expert_mix_backward(const zero_expert_mix_backward_args_t* args, void* stream_) {
    const char* fn = "zero_expert_mix_backward";
    if (!args)
        return fail(ZERO_EINVAL, "%s: NULL args", fn);
    const zero_expert_mix_backward_args_t a = *args;
    TRY(check_mix(fn, a.dtype, a.tokens, a.cols, a.k, a.experts));
    if (!a.dweight != !a.y)
        return fail(ZERO_EINVAL, "%s: y and dweight come together", fn);
    const size_t e = elem_size(a.dtype);
    static const char *const kY = "y", *const kDy = "dy";
    Arrays t(fn);
    TRY(t.add("index", a.index, a.tokens, a.k, a.k, 4, false, true));
    TRY(t.add("weight", a.weight, a.tokens, a.k, a.k, 4, false, true));
    TRY(t.add("dout", a.dout, a.tokens, a.cols, a.ld_dout, e, false));
    TRY(t.add(kY, a.y, a.tokens * a.k, a.cols, a.ld_y, e, false, true));
    TRY(t.add(kDy, a.dy, a.tokens * a.k, a.cols, a.ld_dy, e, true, true));
    TRY(t.add("dweight", a.dweight, a.tokens, a.k, a.k, 4, true, true));
    TRY(t.check_overlaps({{kY, kDy}}));
    if (a.tokens == 0)
        return ZERO_OK;
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    TRY(t.check_memory(stream));
    return with_type(a.dtype, [&](auto type) {
        using T = decltype(type);
        constexpr int kWaves = zo::kMixBlock / 64;
        const int64_t slots = a.tokens * a.k;
        for (int64_t first = 0; first < slots; first += kMaxLaunch * kWaves)
            zo::k_expert_mix_back<T><<<(unsigned)std::min(kMaxLaunch, div_up(slots - first, kWaves)), zo::kMixBlock, 0,
                                       stream>>>(a, first);
        HIP_TRY(hipGetLastError());
        return ZERO_OK;
    });
}

}  // extern "C"
