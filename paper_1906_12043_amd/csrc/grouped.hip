// Grouped products of ragged batches: argument checks, choice of the tile, and the three directions of a layer.
#include "operator_call.hpp"
#include "product_finish.hpp"

#include <cmath>

namespace cocod {
namespace {

// The splits' sums, in order, and what a block without splits does with them.
template <class T, bool WEIGHTS> __global__ __launch_bounds__(256) void join_kernel(const ProductParams p)
{
    const uint32_t quads = (p.n + 3) / 4;
    const uint64_t all = WEIGHTS ? static_cast<uint64_t>(p.groups) * p.m : p.rows;
    const uint64_t first = WEIGHTS ? 0 : bound_at(p, 0), end = WEIGHTS ? all : bound_at(p, p.groups);
    const uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x;
    const uint64_t row = first + i / quads;
    if (row >= end) return;
    const uint32_t col = static_cast<uint32_t>(i % quads) * 4;
    f4 v = *reinterpret_cast<const f4 *>(p.part + row * p.ld_part + col);
    for (uint32_t s = 1; s < p.splits; ++s) v += *reinterpret_cast<const f4 *>(p.part + (s * all + row) * p.ld_part + col);
    const uint32_t group = WEIGHTS ? static_cast<uint32_t>(row / p.m) : 0;
    finish_quad<T, WEIGHTS>(p, group, row, WEIGHTS ? static_cast<uint32_t>(row % p.m) : 0, col, v, WEIGHTS ? group_factor(p, group) : p.scale);
}

template <class T> hipError_t launch_join_of(hipStream_t stream, bool weights, uint32_t blocks, const ProductParams &p)
{
    if (weights) hipLaunchKernelGGL((join_kernel<T, true>), dim3(blocks), dim3(256), 0, stream, p);
    else         hipLaunchKernelGGL((join_kernel<T, false>), dim3(blocks), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_join(hipStream_t stream, Dtype type, Layout layout, const ProductParams &p)
{
    const bool weights = layout == Layout::Weights;
    const uint64_t blocks = ((weights ? static_cast<uint64_t>(p.groups) * p.m : p.rows) * ((p.n + 3) / 4) + 255) / 256;
    if (blocks * 256 >= (1ull << 32)) return hipErrorInvalidConfiguration;
    const uint32_t n = static_cast<uint32_t>(blocks);
    return type == Dtype::BF16 ? launch_join_of<Bf16>(stream, weights, n, p)
           : type == Dtype::F16 ? launch_join_of<F16>(stream, weights, n, p) : launch_join_of<F32>(stream, weights, n, p);
}

// The tile and the number of splits that are expected to take least time.  A compute unit takes ceil(blocks / 256) blocks one after the other (where it
// holds several at a time they share it), each `per_slice` for every slice of its sum (`alone` times that if the unit has no other block) and `per_tile`
// once, in us; a launch costs 5, joining splits 4 and their traffic at 4 TB/s.  Fitted to 111 products of 1 to 64 groups, 1 to 8192 rows and widths 300
// to 32000, every tile with 1 to 16 splits (the 16-bit large tile, that of four slices in LDS and the tall one again to 90, fp32 to 24, operands through
// registers to 39): the choice costs 2 % more time than the best one in the mean.  For instance, us (large / medium / small tile, best splits in brackets):
// bf16 16 groups of one row, 1024 x 1024: 16 (4) / 12 (4) / 8 (1); 4 of 64 rows, 2048 x 2048: 22 (4) / 18 (4) / 14 (1); 16 of 512 rows, 1024 x
// 1024: 33 (1) / 26 (1) / 50 (1); 16 of 500 rows, 2048 x 1024, input gradient: 40 (1) / 47 (1) / 93 (1); 4 of 768 rows, 32000 x 1024: 239 (4) / 266 (8) /
// 468 (4), weight gradient 283 (1) / 342 (1) / 701 (1); through registers one row, 4095 x 2047: - / 18 (8) / 14 (8), 2048 rows, 2047 x 2047: - / 46 (1) /
// 77 (1); fp32 16 of 250 rows, 1024 x 1024: - / 56 (1) / 97 (1), 8 of 8 rows, 2048 x 2048: - / 58 (4) / 31 (2).
struct TileCost { uint32_t bm, bn, bk; double per_slice, per_tile, alone; Tile tile; uint32_t most_turns; };
constexpr TileCost kCostDirect[] = {{256, 256, 64, 1.05, 7.0, 1.0, Tile::Large, ~0u}, {128, 128, 64, 0.40, 1.4, 1.75, Tile::Medium, ~0u},
                                    {32, 64, 128, 0.25, 0.5, 1.0, Tile::Small, ~0u}, {128, 128, 64, 0.50, 1.6, 1.0, Tile::Deep, 1},
                                    {192, 128, 64, 0.63, 4.0, 1.0, Tile::Tall, ~0u}};
constexpr TileCost kCostRegs[] = {{128, 128, 64, 0.70, 3.4, 1.6, Tile::Medium, ~0u}, {32, 64, 128, 0.45, 0.65, 1.4, Tile::Small, ~0u}};
constexpr TileCost kCost32[] = {{128, 128, 32, 1.25, 3.7, 1.0, Tile::Medium, ~0u}, {32, 64, 64, 0.57, 1.3, 1.4, Tile::Small, ~0u},
                                {64, 64, 32, 0.48, 1.5, 1.75, Tile::Square, ~0u}};
constexpr uint32_t kMaxSplits = 16;

ProductPlan plan_product(Layout layout, Dtype type, bool direct, uint64_t rows, uint32_t groups, uint32_t m, uint32_t n, uint32_t k, bool may_split, bool stored)
{
    const bool weights = layout == Layout::Weights;
    const double mean_rows = static_cast<double>(rows) / groups, terms = weights ? mean_rows : k;
    const double cells = weights ? static_cast<double>(groups) * m * n : static_cast<double>(rows) * n;
    const TileCost *const costs = type == Dtype::F32 ? kCost32 : direct ? kCostDirect : kCostRegs;
    const uint32_t n_costs = type == Dtype::F32 ? 3 : !direct ? 2 : stored && !weights ? 5 : 4;
    ProductPlan best{Tile::Medium, 1};
    double least = 1e300;
    for (uint32_t i = 0; i < n_costs; ++i) {
        const TileCost &c = costs[i];
        // ragged groups end half a tile short, in the mean
        const double high = weights || groups == 1 ? std::ceil((weights ? m : mean_rows) / c.bm) : std::fmax(1.0, mean_rows / c.bm + 0.5);
        const double tiles = groups * high * std::ceil(static_cast<double>(n) / c.bn);
        for (uint32_t splits = 1; splits <= (may_split ? kMaxSplits : 1u); splits *= 2) {
            const double turns = std::fmax(1.0, std::ceil(tiles * splits / 256.0 - 1e-9)), slices = std::fmax(1.0, std::ceil(terms / c.bk / splits));
            if (turns > c.most_turns) continue;
            const double us = 5.0 + turns * (slices * c.per_slice * (turns == 1.0 ? c.alone : 1.0) + c.per_tile) + (splits > 1 ? 4.0 + cells * 4.0 * (splits + 1) / 4.0e6 : 0.0);
            if (us < least) { least = us; best = {c.tile, splits}; }
        }
    }
    return best;
}

uint64_t part_bytes(const ProductPlan &plan, Layout layout, uint64_t rows, uint32_t groups, uint32_t m, uint32_t n)
{
    if (plan.splits <= 1) return 0;
    return plan.splits * (layout == Layout::Weights ? static_cast<uint64_t>(groups) * m : rows) * part_pitch(n) * sizeof(float);
}

namespace {

const Dtype kTypes[] = {Dtype::F32, Dtype::BF16, Dtype::F16};

int check_shape(const cocod_grouped *g)
{
    if (!g) return set_error(COCOD_ERR_INVALID, "the description is NULL");
    if (g->struct_size != sizeof(cocod_grouped))
        return set_error(COCOD_ERR_INVALID, "struct_size %u does not match this library (%zu)", g->struct_size, sizeof(cocod_grouped));
    if (int rc = check_dtype(g->dtype)) return rc;
    if (g->flags & ~(COCOD_GROUPED_RELU_OUT | COCOD_GROUPED_RELU_IN)) return set_error(COCOD_ERR_INVALID, "unknown flag bits 0x%x", g->flags);
    if (g->groups < 1 || g->groups > kMaxGroups) return set_error(COCOD_ERR_INVALID, "groups must be in 1..65535");
    if (g->rows > kMaxRows) return set_error(COCOD_ERR_INVALID, "rows must be below 2^31");
    if (g->inner < 1 || g->inner > kMaxWidth || g->outer < 1 || g->outer > kMaxWidth) return set_error(COCOD_ERR_INVALID, "inner and outer must be in 1..2^30");
    if (!g->offsets || (reinterpret_cast<uintptr_t>(g->offsets) & 7)) return set_error(COCOD_ERR_INVALID, "offsets is NULL or not 8-byte aligned");
    return COCOD_OK;
}

ProductPlan plan_of(const cocod_grouped *g, Layout layout, bool may_split)
{
    const Dtype t = kTypes[g->dtype];
    const bool k8 = g->inner % 8 == 0, n8 = g->outer % 8 == 0;       // as dense arrays
    if (layout == Layout::Rows_KN) return plan_product(layout, t, k8 && n8, g->rows, g->groups, 0, g->outer, g->inner, may_split);
    if (layout == Layout::Rows_NK) return plan_product(layout, t, n8, g->rows, g->groups, 0, g->inner, g->outer, may_split);
    return plan_product(layout, t, k8 && n8, g->rows, g->groups, g->inner, g->outer, 0, may_split);
}
uint64_t workspace_of(const cocod_grouped *g, Layout layout, const ProductPlan &plan)
{
    return part_bytes(plan, layout, g->rows, g->groups, g->inner, layout == Layout::Rows_NK ? g->inner : g->outer);
}

int check_codes(const cocod_grouped *g)
{
    if (int rc = check_matrix("x_codes", g->x_codes, g->inner, g->ld_codes, 1, g->rows)) return rc;
    return check_matrix("x_scales", g->x_scales, (static_cast<uint64_t>(g->inner) + 31) / 32, g->ld_scales, 1, g->rows);
}

// The parameters that all directions share, the split sums' memory, and the launch.
int start(const cocod_grouped *g, Layout layout, ProductParams &p, ProductPlan &plan, const Extent &out, const Extent *in, int n_in)
{
    const Dtype t = kTypes[g->dtype];
    plan = plan_of(g, layout, true);
    const uint64_t need = workspace_of(g, layout, plan);
    const bool own = g->workspace && need;
    if (own && (reinterpret_cast<uintptr_t>(g->workspace) & 15)) return set_error(COCOD_ERR_INVALID, "workspace is not 16-byte aligned");
    if (own && g->workspace_bytes < need)
        return set_error(COCOD_ERR_INVALID, "workspace holds %llu bytes, %llu are needed", (unsigned long long)g->workspace_bytes, (unsigned long long)need);
    if (!own) plan = plan_of(g, layout, false);    // the sums are then formed by one block each
    const Extent ws = {"workspace", own ? g->workspace : nullptr, need};
    const Extent offsets = {"offsets", g->offsets, (static_cast<uint64_t>(g->groups) + 1) * 8};
    if (int rc = check_apart(out, in, n_in)) return rc;
    if (int rc = check_apart(out, &offsets, 1)) return rc;
    if (int rc = check_apart(ws, &out, 1)) return rc;
    if (int rc = check_apart(ws, in, n_in)) return rc;
    if (int rc = check_apart(ws, &offsets, 1)) return rc;
    p.offsets = g->offsets;
    p.groups = g->groups;
    p.rows = g->rows;
    p.scale = 1.0f;
    p.part = own ? static_cast<float *>(g->workspace) : nullptr;
    p.splits = plan.splits;
    p.ld_part = part_pitch(p.n);
    plan.tile = settle_tile(t, layout, plan.tile, p);
    return COCOD_OK;
}

int prepare_forward(const cocod_grouped *g, ProductParams &p, ProductPlan &plan)
{
    const uint64_t s = dtype_bytes(kTypes[g->dtype]);
    if (int rc = check_matrix("x", g->x, g->inner, g->ldx, s, g->rows)) return rc;
    if (int rc = check_matrix("w", g->w, g->outer, g->ldw, s)) return rc;
    if (int rc = check_stride("w", g->w_stride, g->groups, g->inner, g->outer, g->ldw, true)) return rc;
    if (int rc = check_matrix("y", g->y, g->outer, g->ldy, s, g->rows)) return rc;
    p.a = g->x; p.lda = g->ldx;
    p.b = g->w; p.ldb = g->ldw; p.b_group = g->groups > 1 ? g->w_stride : 0;
    p.n = g->outer; p.k = g->inner;
    p.out = g->y; p.ldc = g->ldy;
    p.relu = (g->flags & COCOD_GROUPED_RELU_OUT) != 0;
    const Extent in[] = {{"x", g->x, matrix_bytes(g->rows, g->inner, g->ldx, s)}, {"w", g->w, stack_bytes(g->groups, g->w_stride, g->inner, g->outer, g->ldw, s)}};
    return start(g, Layout::Rows_KN, p, plan, {"y", g->y, matrix_bytes(g->rows, g->outer, g->ldy, s)}, in, 2);
}

int prepare_input_grad(const cocod_grouped *g, ProductParams &p, ProductPlan &plan)
{
    const uint64_t s = dtype_bytes(kTypes[g->dtype]);
    if (int rc = check_matrix("dy", g->dy, g->outer, g->lddy, s, g->rows)) return rc;
    if (int rc = check_matrix("w", g->w, g->outer, g->ldw, s)) return rc;
    if (int rc = check_stride("w", g->w_stride, g->groups, g->inner, g->outer, g->ldw, true)) return rc;
    if (int rc = check_matrix("dx", g->dx, g->inner, g->lddx, s, g->rows)) return rc;
    p.a = g->dy; p.lda = g->lddy;
    p.b = g->w; p.ldb = g->ldw; p.b_group = g->groups > 1 ? g->w_stride : 0;
    p.n = g->inner; p.k = g->outer;
    p.out = g->dx; p.ldc = g->lddx;
    Extent in[4] = {{"dy", g->dy, matrix_bytes(g->rows, g->outer, g->lddy, s)}, {"w", g->w, stack_bytes(g->groups, g->w_stride, g->inner, g->outer, g->ldw, s)}};
    if (g->flags & COCOD_GROUPED_RELU_IN) {
        if (g->x) {
            if (int rc = check_matrix("x", g->x, g->inner, g->ldx, s, g->rows)) return rc;
            p.mask = g->x; p.ld_mask = g->ldx;
            in[2] = {"x", g->x, matrix_bytes(g->rows, g->inner, g->ldx, s)};
        } else {
            if (int rc = check_matrix("x_codes", g->x_codes, g->inner, g->ld_codes, 1, g->rows)) return rc;
            p.mask_codes = g->x_codes; p.ld_mask = g->ld_codes;
            in[2] = {"x_codes", g->x_codes, matrix_bytes(g->rows, g->inner, g->ld_codes, 1)};
        }
    }
    return start(g, Layout::Rows_NK, p, plan, {"dx", g->dx, matrix_bytes(g->rows, g->inner, g->lddx, s)}, in, 3);
}

int prepare_weight_grad(const cocod_grouped *g, ProductParams &p, ProductPlan &plan)
{
    const uint64_t s = dtype_bytes(kTypes[g->dtype]);
    if (g->dw_dtype != g->dtype && g->dw_dtype != COCOD_F32) return set_error(COCOD_ERR_INVALID, "dw_dtype must be the element type or COCOD_F32");
    const uint64_t so = dtype_bytes(kTypes[g->dw_dtype]);
    Extent in[3];
    int n_in = 1;
    if (g->x) {
        if (int rc = check_matrix("x", g->x, g->inner, g->ldx, s, g->rows)) return rc;
        p.a = g->x; p.lda = g->ldx;
        in[0] = {"x", g->x, matrix_bytes(g->rows, g->inner, g->ldx, s)};
    } else {
        if (int rc = check_codes(g)) return rc;
        p.a_codes = g->x_codes; p.ld_codes = g->ld_codes;
        p.a_scales = g->x_scales; p.ld_scales = g->ld_scales;
        in[0] = {"x_codes", g->x_codes, matrix_bytes(g->rows, g->inner, g->ld_codes, 1)};
        in[1] = {"x_scales", g->x_scales, matrix_bytes(g->rows, (static_cast<uint64_t>(g->inner) + 31) / 32, g->ld_scales, 1)};
        n_in = 2;
    }
    if (int rc = check_matrix("dy", g->dy, g->outer, g->lddy, s, g->rows)) return rc;
    if (int rc = check_matrix("dw", g->dw, g->outer, g->lddw, so)) return rc;
    if (int rc = check_stride("dw", g->dw_stride, g->groups, g->inner, g->outer, g->lddw, false)) return rc;
    in[n_in++] = {"dy", g->dy, matrix_bytes(g->rows, g->outer, g->lddy, s)};
    p.b = g->dy; p.ldb = g->lddy;
    p.m = g->inner; p.n = g->outer;
    p.out = g->dw; p.ldc = g->lddw; p.out_group = g->dw_stride;
    p.out_f32 = g->dw_dtype == COCOD_F32;
    return start(g, Layout::Weights, p, plan, {"dw", g->dw, stack_bytes(g->groups, g->dw_stride, g->inner, g->outer, g->lddw, so)}, in, n_in);
}

// Checks of a direction's arguments, its parameters and plan.
int prepare(const cocod_grouped *g, Layout layout, ProductParams &p, ProductPlan &plan)
{
    if (int rc = check_shape(g)) return rc;
    return layout == Layout::Rows_KN ? prepare_forward(g, p, plan) : layout == Layout::Rows_NK ? prepare_input_grad(g, p, plan) : prepare_weight_grad(g, p, plan);
}

int run(void *stream, const cocod_grouped *g, Layout layout, const char *what)
{
    ProductParams p{};
    ProductPlan plan;
    if (int rc = prepare(g, layout, p, plan)) return rc;
    if (!g->rows && layout != Layout::Weights) return COCOD_OK;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const OnStreamDevice device(s);
    if (device.status() != hipSuccess) return launch_status(device.status(), what);
    return launch_status(launch_store(s, kTypes[g->dtype], layout, plan.tile, p), what);
}

int layout_of(int direction, Layout &layout)
{
    if (direction < COCOD_GROUPED_FORWARD || direction > COCOD_GROUPED_WEIGHT_GRAD) return set_error(COCOD_ERR_INVALID, "unknown direction %d", direction);
    layout = direction == COCOD_GROUPED_FORWARD ? Layout::Rows_KN : direction == COCOD_GROUPED_INPUT_GRAD ? Layout::Rows_NK : Layout::Weights;
    return COCOD_OK;
}

}  // namespace
}  // namespace cocod

using namespace cocod;

extern "C" {

int cocod_grouped_workspace(const cocod_grouped *g, int direction, uint64_t *bytes)
{
    if (!bytes) return set_error(COCOD_ERR_INVALID, "bytes is NULL");
    if (int rc = check_shape(g)) return rc;
    Layout layout;
    if (int rc = layout_of(direction, layout)) return rc;
    *bytes = workspace_of(g, layout, plan_of(g, layout, true));
    return COCOD_OK;
}

int cocod_grouped_forward(void *stream, const cocod_grouped *g) { return run(stream, g, Layout::Rows_KN, "cocod_grouped_forward"); }
int cocod_grouped_input_grad(void *stream, const cocod_grouped *g) { return run(stream, g, Layout::Rows_NK, "cocod_grouped_input_grad"); }
int cocod_grouped_weight_grad(void *stream, const cocod_grouped *g) { return run(stream, g, Layout::Weights, "cocod_grouped_weight_grad"); }

int cocod_debug_grouped_plan(const cocod_grouped *g, int direction, cocod_product_plan *out)
{
    if (!out) return set_error(COCOD_ERR_INVALID, "out is NULL");
    Layout layout;
    if (int rc = layout_of(direction, layout)) return rc;
    ProductParams p{};
    ProductPlan plan;
    if (int rc = prepare(g, layout, p, plan)) return rc;
    *out = plan_as_run(kTypes[g->dtype], layout, plan.tile, plan.splits, p);
    return COCOD_OK;
}

}  // extern "C"
