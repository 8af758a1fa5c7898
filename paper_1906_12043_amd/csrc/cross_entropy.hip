// Mean softmax cross-entropy of ragged batches over a large vocabulary, and its gradient, without the logits in memory.
//
//   z = h E_g^T,  loss_r = log sum_v exp z_rv - z_r,t(r),  L_g = sum_r loss_r / n_g,
//   dL/dz_rv = (exp z_rv / sum_u exp z_ru - [v = t(r)]) / n_g,  dh = dz E_g,  dE_g = dz^T h
//
// Rows without a target take no part: the others are gathered to the front of their group, so that no product sees a row that is
// masked (whatever its values are) and masked rows cost nothing.  The vocabulary is gone through twice: once for maximum and sum
// of exponentials of every row, tile by tile in the products' epilogue, and once more, piece by piece, for dz, of which one piece
// at a time is in memory in the element type, for the two products that follow it.  The logits are formed twice, 8 instead of 6
// products' worth of work; kept in 16 bits they would be rows x vocab x 2 bytes (2 GiB at 8192 x 131072).
//
// dz is rounded to the element type before the products (fp32: not), because the matrix cores take both operands of a product in one type and a
// second plane would double the work of two of the three products.  Each of its values is off by at most half a step, 2^-8 of itself (fp16: 2^-11, not
// below steps of 2^-38), and in bf16 where its exponential was kept in fp16 between the passes by 2^-11 more.  An entry of dh or dE is thus off by up to
// that part of its sum of MAGNITUDES, beside its own last rounding.  Far from a minimum that is hidden by the last rounding; where the slopes cancel it is
// not: 8192 rows, 256 entries, 64 columns in bf16, relative error of dE 1.6e-3 with a table of zeros (its last rounding alone: as much), 2.5e-3 / 7.6e-3
// after 20 / 60 optimiser steps (magnitudes 13 / 45 times the entries), 0.2 after 400 (1200 times); 2^-12.5 of the magnitudes in all three.
#include "vocabulary.hpp"

#include <cmath>

namespace cocod {
namespace {

constexpr uint64_t kMaxLossRows = 1ull << 26;        // a wave a row in one launch

// A row's gathered copy (pitch a multiple of 8, zeros behind dim) by the lanes of a wave.
template <class E> struct Hidden {
    const E *h;
    uint64_t ldh;
    uint32_t dim;
    E *out;
    uint64_t pitch;
    float *loss;
    E *dh;                            // may be null
    uint64_t lddh;
};
template <class E> __device__ __forceinline__ void gather_row(const Hidden<E> &p, uint64_t r, uint32_t from, uint32_t lane)
{
    copy_row(p.h + from * p.ldh, p.dim, p.out + r * p.pitch, p.pitch, lane);
}
// A row without a target: loss 0, gradient 0.
template <class E> __device__ __forceinline__ void clear_row(const Hidden<E> &p, uint64_t r, uint32_t lane)
{
    if (lane == 0) p.loss[r] = 0.0f;
    if (p.dh) for (uint32_t j = lane; j < p.dim; j += 64) p.dh[r * p.lddh + j] = 0;
}

// One block per group: the rows with a target, in order, to the front of the group's part of `index`; kNoRow behind them.  And every such row's
// gradient factor.  GATHER: the rows themselves, too (a launch less where there is little to copy).
constexpr int kCompactThreads = 1024;
template <class E, bool GATHER>
__global__ __launch_bounds__(kCompactThreads) void compact_kernel(const Rows p, uint32_t *index, int32_t *target, int64_t *ends, int sum_only, float scale,
                                                                  float *row_scale, const Hidden<E> hidden)
{
    __shared__ uint32_t counts[kCompactThreads / 64];
    const uint32_t g = blockIdx.x, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint64_t begin = clamped(p, g), next = clamped(p, g + 1), end = next > begin ? next : begin;
    uint64_t at = begin;
    for (uint64_t r0 = begin; r0 < end; r0 += kCompactThreads) {
        const uint64_t r = r0 + threadIdx.x;
        const bool in = r < end && has_target(p, r);
        const unsigned long long votes = __ballot(in);
        if (lane == 0) counts[wave] = __popcll(votes);
        __syncthreads();
        uint32_t before = 0, all = 0;
        for (int w = 0; w < kCompactThreads / 64; ++w) { if (w < static_cast<int>(wave)) before += counts[w]; all += counts[w]; }
        if (in) {
            const uint64_t to = at + before + __popcll(votes & ((1ull << lane) - 1));
            index[to] = static_cast<uint32_t>(r);
            target[to] = p.target[r];
        }
        at += all;
        __syncthreads();
    }
    for (uint64_t r = at + threadIdx.x; r < end; r += kCompactThreads) index[r] = kNoRow;
    const float factor = sum_only ? scale : scale / static_cast<float>(at - begin);
    for (uint64_t r = begin + threadIdx.x; r < at; r += kCompactThreads) row_scale[r] = factor;
    if (threadIdx.x == 0) ends[g] = static_cast<int64_t>(at);
    if constexpr (GATHER) {                                    // (the barrier that ended the loop ordered the block's own writes of index)
        for (uint64_t r = begin + wave; r < end; r += kCompactThreads / 64) {
            if (r < at) {
                // Groups whose offsets do not ascend share rows, and the block of another one may have left kNoRow in this place since.
                const uint32_t from = index[r];
                if (from != kNoRow) gather_row(hidden, r, from, lane);
            }
            if (!has_target(p, r)) clear_row(hidden, r, lane);
        }
    }
}

// The gathered rows by a launch of their own, a wave a row (a block's waves take further rows where that would be more threads than a launch holds).
constexpr uint32_t kMostGatherBlocks = 1u << 23;
template <class E> __global__ __launch_bounds__(256) void gather_kernel(const Rows p, const uint32_t *index, const Hidden<E> hidden)
{
    const uint32_t lane = threadIdx.x % 64;
    for (uint64_t r = static_cast<uint64_t>(blockIdx.x) * 4 + threadIdx.x / 64; r < p.rows; r += static_cast<uint64_t>(gridDim.x) * 4) {
        if (r < clamped(p, 0) || r >= clamped(p, p.groups)) continue;
        if (index[r] != kNoRow) gather_row(hidden, r, index[r], lane);
        if (!has_target(p, r)) clear_row(hidden, r, lane);
    }
}

// What a row's slopes need, from the column tiles' maxima and sums, and its loss, also in the place of the target's logit.  The target is not among
// those sums: with s the sum of the other exponentials, all below the larger one m of the others' maximum and the target's logit z,
//   loss = (m - z) + log(s + exp(z - m)), log1p(s) where z = m;   slope of the target = -s / (s + exp(z - m)),
// so that both keep their digits where the target is almost certain, however large the logits are (a logarithm of the whole sum, rounded at the
// size of m, left none of a loss of 1e-6 at logits of 40, and the target's slope with steps of |m| 2^-24).
// ROWS rows per pass of a block, THREADS threads a row.
constexpr int kNormThreads = 16, kNormAhead = 4, kFewThreads = 4;
struct Norms {
    const uint32_t *index;
    const float2 *stats;              // [tiles][rows]
    uint32_t tiles;
    float *target_logit, *top, *inverse, *target_slope, *loss;
};
__device__ __forceinline__ void add_part(float &top, float &sum, float2 s)
{
    const float m = fmaxf(top, s.x), base = m == -INFINITY ? 0.0f : m;
    sum = sum * expf(top - base) + s.y * expf(s.x - base);
    top = m;
}
// the loss of row r in the threads with y == 0 (others: 0); GATHERED: it comes from another row of the caller's
template <int ROWS, bool GATHERED, int THREADS> __device__ __forceinline__ float norm_rows(const Rows &p, const Norms &n, uint64_t r, bool in, float2 (&part)[THREADS][ROWS])
{
    const uint32_t x = threadIdx.x % ROWS, y = threadIdx.x / ROWS;
    float top = -INFINITY, sum = 0.0f;
    if (in) {
        for (uint32_t t = y; t < n.tiles; t += THREADS * kNormAhead) {
            float2 s[kNormAhead];
            #pragma unroll
            for (int i = 0; i < kNormAhead; ++i) {
                const uint32_t u = t + i * THREADS;
                s[i] = u < n.tiles ? n.stats[u * p.rows + r] : make_float2(-INFINITY, 0.0f);
            }
            #pragma unroll
            for (int i = 0; i < kNormAhead; ++i) add_part(top, sum, s[i]);
        }
    }
    part[y][x] = make_float2(top, sum);
    __syncthreads();
    float l = 0.0f;
    if (y == 0 && in) {
        #pragma unroll
        for (int w = 1; w < THREADS; ++w) add_part(top, sum, part[w][x]);
        const float z = n.target_logit[r], m = fmaxf(top, z), others = sum * expf(top - m), all = others + expf(z - m);
        n.top[r] = m;
        n.inverse[r] = 1.0f / all;
        n.target_slope[r] = -others / all;
        l = (m - z) + (z >= top ? log1pf(others) : logf(all));
        n.target_logit[r] = l;
        n.loss[GATHERED ? n.index[r] : r] = l;
    }
    __syncthreads();
    return l;
}

constexpr int kNormRows = 16;
__global__ __launch_bounds__(kNormRows * kNormThreads) void norm_kernel(const Rows p, const Norms n)
{
    __shared__ float2 part[kNormThreads][kNormRows];
    const uint64_t r = static_cast<uint64_t>(blockIdx.x) * kNormRows + threadIdx.x % kNormRows;
    norm_rows<kNormRows, true>(p, n, r, r >= clamped(p, 0) && r < clamped(p, p.groups) && n.index[r] != kNoRow, part);
}

// One block per group: the mean (or sum) of its rows' losses, summed in a fixed order in 64 bits.  NORMS: the rows' losses, too (a launch less where a
// block has little to do).  Not GATHERED: rows without a target lie between the others.
constexpr int kMeanThreads = 1024;
template <bool NORMS, bool GATHERED = true, int THREADS = kNormThreads> __global__ __launch_bounds__(kMeanThreads) void mean_kernel(const Rows p, const Norms n, const int64_t *ends, float *group_loss, int sum_only)
{
    constexpr int ROWS = kMeanThreads / THREADS;
    __shared__ double part[kMeanThreads];
    __shared__ float2 parts[THREADS][NORMS ? ROWS : 1];
    const uint32_t g = blockIdx.x;
    const uint64_t begin = clamped(p, g), end = GATHERED ? static_cast<uint64_t>(ends[g]) : clamped(p, g + 1);
    uint64_t count = end > begin ? end - begin : 0;
    double s = 0.0;
    static_assert(NORMS || GATHERED, "statistics of rows where they lie are summed up here");
    if constexpr (!GATHERED) {
        count = 0;
        for (uint64_t r0 = begin; r0 < end; r0 += ROWS) {
            const uint64_t r = r0 + threadIdx.x % ROWS;
            const bool first = threadIdx.x < ROWS && r < end, in = r < end && has_target(p, r);
            if (first && !in) n.loss[r] = 0.0f;
            count += __syncthreads_count(first && in);
            s += norm_rows<ROWS, false>(p, n, r, in, parts);
        }
    } else if constexpr (NORMS) {
        for (uint64_t r0 = begin; r0 < end; r0 += ROWS) {
            const uint64_t r = r0 + threadIdx.x % ROWS;
            s += norm_rows<ROWS, true>(p, n, r, r < end && n.index[r] != kNoRow, parts);         // (offsets that do not ascend may leave holes)
        }
    } else {
        for (uint64_t r = begin + threadIdx.x; r < end; r += kMeanThreads) s += n.target_logit[r];
    }
    part[threadIdx.x] = s;
    __syncthreads();
    for (int d = kMeanThreads / 2; d > 0; d >>= 1) {
        if (static_cast<int>(threadIdx.x) < d) part[threadIdx.x] += part[threadIdx.x + d];
        __syncthreads();
    }
    if (threadIdx.x == 0 && group_loss) group_loss[g] = static_cast<float>(count ? (sum_only ? part[0] : part[0] / static_cast<double>(count)) : 0.0);
}

// Slopes from kept exponentials, in their place: exp(z - top) exp(top - m) / sum, top the tile's maximum; the target's is there.  Eight columns a thread.
template <class T> __global__ __launch_bounds__(256) void slope_kernel(const Rows p, const Norms n, const int32_t *target, void *slopes, uint64_t pitch, uint32_t v0,
                                                                       uint32_t columns, uint32_t columns_end, uint32_t tile_cols, uint32_t parts)
{
    typedef typename T::elem elem;
    const uint64_t r = blockIdx.x / parts;
    const uint32_t c = (blockIdx.x % parts * 256 + threadIdx.x) * 8;
    if (c >= columns_end || r < clamped(p, 0) || r >= clamped(p, p.groups) || n.index[r] == kNoRow) return;
    const float factor = expf(n.stats[static_cast<uint64_t>(c / tile_cols) * p.rows + r].x - n.top[r]) * n.inverse[r];
    const uint32_t number = static_cast<uint32_t>(target[r]) - v0 - c;
    elem *at = static_cast<elem *>(slopes) + r * pitch + c;
    float v[8];
    if constexpr (sizeof(elem) == 4) {
        #pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = at[j] * factor;
    } else {
        const u4 w = *reinterpret_cast<const u4 *>(at);
        #pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(w[j / 2] >> (16 * (j % 2))))) * (kKeepUnscale * factor);
    }
    #pragma unroll
    for (uint32_t j = 0; j < 8; ++j) {
        if (number == j) v[j] = n.target_slope[r];
        if (c + j >= columns) v[j] = 0.0f;
    }
    if constexpr (sizeof(elem) == 4) {
        *reinterpret_cast<f4 *>(at) = f4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f4 *>(at + 4) = f4{v[4], v[5], v[6], v[7]};
    } else {
        *reinterpret_cast<u4 *>(at) = u4{T::pack(v[0], v[1]), T::pack(v[2], v[3]), T::pack(v[4], v[5]), T::pack(v[6], v[7])};
    }
}

// Up to so many bytes of hidden states per group, and so many statistics per thread of a group's block, one block of 1024 threads does the small work of a group
// together with what precedes or follows it; beyond, kernels of their own spread it over the chip (with gradients, us together / apart: 64 rows of 256
// 31 / 31, 256 rows 39 / 32, 512 rows 51 / 36).  And so many bytes up to which rows stay where they are if only their losses are wanted.
constexpr uint64_t kGatherHere = 32u << 10, kStatsHere = 8, kLeaveHere = 1u << 20;

// The caller's memory, carved up.
struct Workspace {
    uint64_t index, target, ends, top, inverse, target_slope, target_logit, row_scale, hidden, stats, slope, sum, part, bytes;
    uint64_t pitch, piece, sum_pitch;
    uint32_t pieces;
    bool keep;                        // the last piece's exponentials stay from the first pass, as slopes to be
    ProductPlan logits, slopes, to_hidden, to_table;
};

Workspace carve(const cocod_cross_entropy_call *c)
{
    Workspace w{};
    const Dtype t = kTypes[c->dtype];
    const uint64_t s = dtype_bytes(t), rows = c->rows;
    const bool grads = c->dh || c->de;
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) { const uint64_t o = at; at += (bytes + 255) / 256 * 256; return o; };
    w.pitch = (static_cast<uint64_t>(c->dim) + 7) / 8 * 8;
    const Pieces pieces = pieces_of(c->piece, rows, c->vocab);
    w.piece = pieces.size;
    w.pieces = pieces.count;
    const uint32_t n = static_cast<uint32_t>(w.piece < c->vocab ? w.piece : c->vocab);
    const bool dim8 = c->dim % 8 == 0;                         // a dense table's rows then start on 16 bytes
    w.logits = plan_product(Layout::Rows_NK, t, dim8, rows, c->groups, 0, c->vocab, c->dim, false, false);
    w.slopes = plan_product(Layout::Rows_NK, t, dim8, rows, c->groups, 0, n, c->dim, false, false);             // (exponentials need the whole sum)
    w.to_hidden = plan_product(Layout::Rows_KN, t, dim8, rows, c->groups, 0, c->dim, n, true);
    w.to_table = plan_product(Layout::Weights, t, true, rows, c->groups, n, c->dim, 0, true);
    w.index = take(rows * 4);
    w.target = take(rows * 4);
    w.ends = take(c->groups * 8ull);
    w.top = take(rows * 4);
    w.inverse = take(rows * 4);
    w.target_slope = take(rows * 4);
    w.target_logit = take(rows * 4);
    w.row_scale = take(rows * 4);
    w.hidden = take(rows * w.pitch * s);
    const uint32_t planned = tile_cols(t, w.logits.tile), narrow = planned < 128 ? planned : 128;        // the large tile may have to give way to the medium one
    w.stats = take((static_cast<uint64_t>(c->vocab) + narrow - 1) / narrow * rows * 8);
    if (grads) {
        w.slope = take(rows * w.piece * s);
        w.sum_pitch = part_pitch(c->dim);
        if (c->dh && w.pieces > 1) w.sum = take(rows * w.sum_pitch * 4);
        uint64_t part = 0;
        if (c->dh) part = part_bytes(w.to_hidden, Layout::Rows_KN, rows, c->groups, 0, c->dim);
        if (c->de) { const uint64_t q = part_bytes(w.to_table, Layout::Weights, rows, c->groups, n, c->dim); part = part > q ? part : q; }
        w.part = take(part);
    }
    w.keep = grads && rows != 0 && t != Dtype::F16 && rows * ((w.piece / 8 + 255) / 256) * 256 < (1ull << 32);
    w.bytes = at;
    return w;
}

int check(const cocod_cross_entropy_call *c)
{
    if (!c) return set_error(COCOD_ERR_INVALID, "the description is NULL");
    if (c->struct_size != sizeof(cocod_cross_entropy_call))
        return set_error(COCOD_ERR_INVALID, "struct_size %u does not match this library (%zu)", c->struct_size, sizeof(cocod_cross_entropy_call));
    if (int rc = check_dtype(c->dtype)) return rc;
    if (c->flags & ~(COCOD_CROSS_ENTROPY_SUM | COCOD_CROSS_ENTROPY_RELU_IN)) return set_error(COCOD_ERR_INVALID, "unknown flag bits 0x%x", c->flags);
    if (c->groups < 1 || c->groups > kMaxGroups) return set_error(COCOD_ERR_INVALID, "groups must be in 1..65535");
    if (c->rows >= kMaxLossRows) return set_error(COCOD_ERR_INVALID, "rows must be below 2^26");
    if (c->dim < 1 || c->dim > kMaxWidth || c->vocab < 1 || c->vocab > kMaxWidth) return set_error(COCOD_ERR_INVALID, "dim and vocab must be in 1..2^30");
    if (!std::isfinite(c->grad_scale)) return set_error(COCOD_ERR_INVALID, "grad_scale is not finite");
    return COCOD_OK;
}

template <class E> hipError_t launch_gather(hipStream_t s, const Rows &rows, const cocod_cross_entropy_call *c, const Workspace &w, uint8_t *ws, float scale)
{
    const Hidden<E> hidden = {static_cast<const E *>(c->h), c->ldh, c->dim, reinterpret_cast<E *>(ws + w.hidden), w.pitch, c->loss, static_cast<E *>(c->dh), c->lddh};
    uint32_t *index = reinterpret_cast<uint32_t *>(ws + w.index);
    int32_t *target = reinterpret_cast<int32_t *>(ws + w.target);
    int64_t *ends = reinterpret_cast<int64_t *>(ws + w.ends);
    float *row_scale = reinterpret_cast<float *>(ws + w.row_scale);
    const int sum_only = (c->flags & COCOD_CROSS_ENTROPY_SUM) != 0;
    if (c->rows * w.pitch * sizeof(E) <= kGatherHere * c->groups) {
        hipLaunchKernelGGL((compact_kernel<E, true>), dim3(c->groups), dim3(kCompactThreads), 0, s, rows, index, target, ends, sum_only, scale, row_scale, hidden);
    } else {
        hipLaunchKernelGGL((compact_kernel<E, false>), dim3(c->groups), dim3(kCompactThreads), 0, s, rows, index, target, ends, sum_only, scale, row_scale, hidden);
        const uint32_t blocks = static_cast<uint32_t>((rows.rows + 3) / 4);
        hipLaunchKernelGGL(gather_kernel<E>, dim3(blocks < kMostGatherBlocks ? blocks : kMostGatherBlocks), dim3(256), 0, s, rows, index, hidden);
    }
    return hipGetLastError();
}

// The operands of the call's products (the rest of the parameters is the call's): logits of the gathered rows, and of a piece that begins at entry v0 the
// gradients of the hidden states and of the table.
ProductParams logits_operands(const cocod_cross_entropy_call *c, const Workspace &w, const uint8_t *ws)
{
    ProductParams p{};
    p.a = ws + w.hidden; p.lda = w.pitch;
    p.b = c->e; p.ldb = c->lde; p.b_group = c->groups > 1 ? c->e_stride : 0;
    p.k = c->dim;
    return p;
}
ProductParams hidden_operands(const cocod_cross_entropy_call *c, const Workspace &w, const uint8_t *ws, uint64_t v0, uint32_t n)
{
    ProductParams p{};
    p.a = ws + w.slope; p.lda = w.piece; p.a_zero_padded = 1;
    p.b = static_cast<const uint8_t *>(c->e) + v0 * c->lde * dtype_bytes(kTypes[c->dtype]); p.ldb = c->lde; p.b_group = c->groups > 1 ? c->e_stride : 0;
    p.k = n;
    return p;
}
ProductParams table_operands(const Workspace &w, const uint8_t *ws)
{
    ProductParams p{};
    p.a = ws + w.slope; p.lda = w.piece;
    p.b = ws + w.hidden; p.ldb = w.pitch;
    return p;
}

// Every launch that the call makes holds its product, or nothing is begun.
int check_launches(const cocod_cross_entropy_call *c, const Workspace &w, const uint8_t *ws, const char *what)
{
    const Dtype t = kTypes[c->dtype];
    const uint32_t n = static_cast<uint32_t>(w.piece < c->vocab ? w.piece : c->vocab);
    auto fits = [&](Layout layout, const ProductPlan &plan, const ProductParams &p, uint32_t m, uint32_t cols, uint32_t splits) {
        const TileSize size = tile_size(t, settle_tile(t, layout, plan.tile, p));
        return fits_a_launch(size, blocks_of(size, layout == Layout::Weights, c->rows, c->groups, m, cols, splits));
    };
    const ProductParams z = logits_operands(c, w, ws);
    const bool rows = c->rows != 0, formed_again = (c->dh || c->de) && (w.pieces > 1 || !w.keep);
    const uint32_t kept = w.keep ? static_cast<uint32_t>(c->vocab - (w.pieces - 1) * w.piece) : 0;      // columns of a launch of their own
    const bool all = (!rows || (fits(Layout::Rows_NK, w.logits, z, 0, c->vocab - kept, 1) && fits(Layout::Rows_NK, w.logits, z, 0, kept, 1))) &&
                     (!rows || !formed_again || fits(Layout::Rows_NK, w.slopes, z, 0, n, 1)) &&
                     (!rows || !c->dh || fits(Layout::Rows_KN, w.to_hidden, hidden_operands(c, w, ws, 0, n), 0, c->dim, w.to_hidden.splits)) &&
                     (!c->de || fits(Layout::Weights, w.to_table, table_operands(w, ws), n, c->dim, w.to_table.splits));
    return all ? COCOD_OK : launch_status(hipErrorInvalidConfiguration, what);
}

}  // namespace
}  // namespace cocod

using namespace cocod;

extern "C" {

int cocod_cross_entropy_workspace(const cocod_cross_entropy_call *c, uint64_t *bytes)
{
    if (!bytes) return set_error(COCOD_ERR_INVALID, "bytes is NULL");
    if (int rc = check(c)) return rc;
    *bytes = carve(c).bytes;
    return COCOD_OK;
}

int cocod_cross_entropy(void *stream, const cocod_cross_entropy_call *c)
{
    if (int rc = check(c)) return rc;
    const Dtype t = kTypes[c->dtype];
    const uint64_t s = dtype_bytes(t);
    if (!c->offsets || (reinterpret_cast<uintptr_t>(c->offsets) & 7)) return set_error(COCOD_ERR_INVALID, "offsets is NULL or not 8-byte aligned");
    if (int rc = check_matrix("h", c->h, c->dim, c->ldh, s, c->rows)) return rc;
    if (int rc = check_matrix("e", c->e, c->dim, c->lde, s)) return rc;
    if (int rc = check_stride("e", c->e_stride, c->groups, c->vocab, c->dim, c->lde, true)) return rc;
    if (int rc = check_matrix("targets", c->targets, 1, 1, 4, c->rows)) return rc;
    if (int rc = check_matrix("loss", c->loss, 1, 1, 4, c->rows)) return rc;
    if (c->group_loss) if (int rc = check_matrix("group_loss", c->group_loss, 1, 1, 4)) return rc;
    if (c->dh) if (int rc = check_matrix("dh", c->dh, c->dim, c->lddh, s)) return rc;
    if (c->de) {
        if (int rc = check_matrix("de", c->de, c->dim, c->ldde, s)) return rc;
        if (int rc = check_stride("de", c->de_stride, c->groups, c->vocab, c->dim, c->ldde, false)) return rc;
    }
    const Workspace w = carve(c);
    if (!c->workspace || (reinterpret_cast<uintptr_t>(c->workspace) & 255)) return set_error(COCOD_ERR_INVALID, "workspace is NULL or not 256-byte aligned");
    if (c->workspace_bytes < w.bytes)
        return set_error(COCOD_ERR_INVALID, "workspace holds %llu bytes, %llu are needed", (unsigned long long)c->workspace_bytes, (unsigned long long)w.bytes);
    const Extent all[] = {
        {"workspace", c->workspace, w.bytes}, {"loss", c->loss, c->rows * 4}, {"group_loss", c->group_loss, c->groups * 4ull},
        {"dh", c->dh, matrix_bytes(c->rows, c->dim, c->lddh, s)},
        {"de", c->de, c->de ? stack_bytes(c->groups, c->de_stride, c->vocab, c->dim, c->ldde, s) : 0},
        {"h", c->h, matrix_bytes(c->rows, c->dim, c->ldh, s)}, {"e", c->e, stack_bytes(c->groups, c->e_stride, c->vocab, c->dim, c->lde, s)},
        {"targets", c->targets, c->rows * 4}, {"offsets", c->offsets, (c->groups + 1ull) * 8},
    };
    for (int i = 0; i < 5; ++i)
        if (int rc = check_apart(all[i], all + i + 1, 9 - i - 1)) return rc;

    const hipStream_t q = static_cast<hipStream_t>(stream);
    const OnStreamDevice device(q);
    const char *const what = "cocod_cross_entropy";
    if (device.status() != hipSuccess) return launch_status(device.status(), what);
    uint8_t *ws = static_cast<uint8_t *>(c->workspace);
    if (int rc = check_launches(c, w, ws, what)) return rc;
    uint32_t *index = reinterpret_cast<uint32_t *>(ws + w.index);
    int64_t *ends = reinterpret_cast<int64_t *>(ws + w.ends);
    float *const top = reinterpret_cast<float *>(ws + w.top), *const inverse = reinterpret_cast<float *>(ws + w.inverse);
    float *const target_slope = reinterpret_cast<float *>(ws + w.target_slope), *const row_scale = reinterpret_cast<float *>(ws + w.row_scale);
    int32_t *target = reinterpret_cast<int32_t *>(ws + w.target);
    const Rows rows = {c->offsets, c->groups, c->rows, c->targets, c->vocab};
    const float unslope = t == Dtype::F16 ? 0x1p-14f : 1.0f;   // fp16 slopes are kept times 2^14
    const int sum_only = (c->flags & COCOD_CROSS_ENTROPY_SUM) != 0;

    const float scale = c->grad_scale * unslope;
    const ProductParams gathered_rows = logits_operands(c, w, ws);
    ProductParams z = gathered_rows;
    z.a = c->h; z.lda = c->ldh;
    z.offsets = c->offsets; z.ends = ends; z.groups = c->groups; z.rows = c->rows;
    z.splits = 1; z.target = target;
    // The loss alone of a few rows that the product can take where they are: those without a target go through it, too, and are left out of the
    // sums (64 rows, 1000 x 256: 11 us instead of 16; 512 rows 14 instead of 18; 16 rows, 16000 x 1024: 17 instead of 21).  Not in fp32, where a
    // row that is not finite has its whole tile formed again.
    const bool few = t != Dtype::F32 && !c->dh && !c->de && direct_a(Layout::Rows_NK, z) && c->rows * w.pitch * s <= kLeaveHere * c->groups;
    if (!few) { z.a = gathered_rows.a; z.lda = gathered_rows.lda; }
    const Tile tile = settle_tile(t, Layout::Rows_NK, w.logits.tile, z);
    const uint32_t cols = tile_cols(t, tile);
    Norms norms = {index, reinterpret_cast<const float2 *>(ws + w.stats), (c->vocab + cols - 1) / cols, reinterpret_cast<float *>(ws + w.target_logit), top, inverse,
                   target_slope, c->loss};
    const bool here = c->rows * norms.tiles <= kStatsHere * kMeanThreads * c->groups, gathered = !(few && here && c->rows);
    if (gathered) {
        z.a = gathered_rows.a; z.lda = gathered_rows.lda;
        if (int rc = launch_status(t == Dtype::F32 ? launch_gather<float>(q, rows, c, w, ws, scale) : launch_gather<uint16_t>(q, rows, c, w, ws, scale), what)) return rc;
    } else {
        z.ends = nullptr; z.target = c->targets;
    }
    const uint32_t kept_v0 = static_cast<uint32_t>((w.pieces - 1) * w.piece);
    const uint64_t kept_tile0 = kept_v0 / cols;                // (pieces are whole tiles)
    if (c->rows) {
        ProductParams p = z;
        p.n = c->vocab;
        p.stats = reinterpret_cast<float2 *>(ws + w.stats);
        p.target_logit = norms.target_logit;
        p.n = w.keep ? kept_v0 : c->vocab;
        if (p.n) if (int rc = launch_status(launch_logits(q, t, Finish::Stats, tile, p), what)) return rc;
        if (w.keep) {
            p.b = static_cast<const uint8_t *>(c->e) + static_cast<uint64_t>(kept_v0) * c->lde * s;
            p.n = c->vocab - kept_v0;
            p.v0 = kept_v0;
            p.stats += kept_tile0 * c->rows;
            p.out = ws + w.slope;
            p.ldc = w.piece;
            if (int rc = launch_status(launch_logits(q, t, Finish::Keep, tile, p), what)) return rc;
        }
        if (!here) hipLaunchKernelGGL(norm_kernel, dim3(static_cast<uint32_t>((c->rows + kNormRows - 1) / kNormRows)), dim3(kNormRows * kNormThreads), 0, q, rows, norms);
    }
    if (here || c->group_loss) {
        // a few statistics a row: more rows at a time (256 rows, 1000 x 256: 11 us instead of 22, half of 512 rows, 512 x 256: 13.5 instead of 33)
        const bool wide = norms.tiles <= kFewThreads * kNormAhead;
        const auto mean = !here      ? mean_kernel<false>
                          : gathered ? (wide ? mean_kernel<true, true, kFewThreads> : mean_kernel<true, true>)
                                     : (wide ? mean_kernel<true, false, kFewThreads> : mean_kernel<true, false>);
        hipLaunchKernelGGL(mean, dim3(c->groups), dim3(kMeanThreads), 0, q, rows, norms, ends, c->group_loss, sum_only);
    }
    if (int rc = launch_status(hipGetLastError(), what)) return rc;
    if (!c->dh && !c->de) return COCOD_OK;

    for (uint32_t i = 0; i < w.pieces; ++i) {                  // the last piece first: its exponentials are there
        const uint64_t v0 = (w.pieces - 1 - i) * w.piece;
        const uint32_t n = static_cast<uint32_t>(c->vocab - v0 < w.piece ? c->vocab - v0 : w.piece);
        const uint8_t *e = static_cast<const uint8_t *>(c->e) + v0 * c->lde * s;
        if (w.keep && i == 0) {
            const uint32_t end = (n + 7) / 8 * 8, parts = (end / 8 + 255) / 256;
            const dim3 grid(static_cast<uint32_t>(c->rows * parts));
            Norms kept = norms;
            kept.stats += kept_tile0 * c->rows;
            if (t == Dtype::F32) hipLaunchKernelGGL(slope_kernel<F32>, grid, dim3(256), 0, q, rows, kept, target, ws + w.slope, w.piece, kept_v0, n, end, cols, parts);
            else                 hipLaunchKernelGGL(slope_kernel<Bf16>, grid, dim3(256), 0, q, rows, kept, target, ws + w.slope, w.piece, kept_v0, n, end, cols, parts);
            if (int rc = launch_status(hipGetLastError(), what)) return rc;
        } else if (c->rows) {
            ProductParams p = z;
            p.b = e; p.n = n; p.v0 = static_cast<uint32_t>(v0);
            p.top = top; p.inverse = inverse; p.target_slope = target_slope;
            p.out = ws + w.slope; p.ldc = w.piece; p.ldc_zero = (n + 7) / 8 * 8;
            if (int rc = launch_status(launch_logits(q, t, Finish::Slope, settle_tile(t, Layout::Rows_NK, w.slopes.tile, p), p), what)) return rc;
        }
        auto common = [&](ProductParams &d) {
            d.offsets = c->offsets; d.ends = ends; d.groups = c->groups; d.rows = c->rows;
            d.n = c->dim;
            d.part = reinterpret_cast<float *>(ws + w.part); d.ld_part = part_pitch(c->dim);
        };
        if (c->dh && c->rows) {
            ProductParams d = hidden_operands(c, w, ws, v0, n);
            common(d);
            d.out = c->dh; d.ldc = c->lddh; d.out_row = index; d.row_scale = row_scale;
            if (c->flags & COCOD_CROSS_ENTROPY_RELU_IN) { d.mask = ws + w.hidden; d.ld_mask = w.pitch; }       // (rows of C are gathered ones)
            if (w.pieces > 1) { d.sum = reinterpret_cast<float *>(ws + w.sum); d.ld_sum = w.sum_pitch; d.sum_read = i > 0; d.sum_write = i + 1 < w.pieces; }
            d.splits = w.to_hidden.splits;
            if (int rc = launch_status(launch_store(q, t, Layout::Rows_KN, settle_tile(t, Layout::Rows_KN, w.to_hidden.tile, d), d), what)) return rc;
        }
        if (c->de) {
            ProductParams d = table_operands(w, ws);
            common(d);
            d.m = n;
            d.out = static_cast<uint8_t *>(c->de) + v0 * c->ldde * s; d.ldc = c->ldde; d.out_group = c->de_stride;
            d.scale = scale; d.mean = !sum_only;
            d.splits = w.to_table.splits;
            if (int rc = launch_status(launch_store(q, t, Layout::Weights, settle_tile(t, Layout::Weights, w.to_table.tile, d), d), what)) return rc;
        }
    }
    return COCOD_OK;
}

int cocod_debug_cross_entropy_plan(const cocod_cross_entropy_call *c, cocod_product_plan out[4], uint32_t *pieces)
{
    if (!out || !pieces) return set_error(COCOD_ERR_INVALID, "out or pieces is NULL");
    if (int rc = check(c)) return rc;
    const Dtype t = kTypes[c->dtype];
    const Workspace w = carve(c);
    const uint8_t *ws = static_cast<const uint8_t *>(c->workspace);
    const ProductParams z = logits_operands(c, w, ws), h = hidden_operands(c, w, ws, 0, static_cast<uint32_t>(w.piece < c->vocab ? w.piece : c->vocab)),
                        e = table_operands(w, ws);
    auto plan = [&](Layout layout, const ProductPlan &planned, const ProductParams &p) {
        return plan_as_run(t, layout, settle_tile(t, layout, planned.tile, p), planned.splits, p);
    };
    const cocod_product_plan none = {0, 0, 0};
    out[0] = plan(Layout::Rows_NK, w.logits, z);
    out[1] = (c->dh || c->de) && (w.pieces > 1 || !w.keep) ? plan(Layout::Rows_NK, w.slopes, z) : none;
    out[2] = c->dh ? plan(Layout::Rows_KN, w.to_hidden, h) : none;
    out[3] = c->de ? plan(Layout::Weights, w.to_table, e) : none;
    *pieces = w.pieces;
    return COCOD_OK;
}

}  // extern "C"
