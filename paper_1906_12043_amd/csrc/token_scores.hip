// Log probability of given tokens, entropy and the most probable alternatives at a vocabulary, and the gradients of the first two, without the logits
// in memory.
//
//   z = scale h E_g^T,  m = max z,  d = z - m,  1 + rest = sum exp d,  D = sum d exp d / (1 + rest)
//   log p_t = d_t - log(1 + rest),  H = -sum p log p = log(1 + rest) - D,  alternatives: the largest z, of equal ones those in front, z - m - log(1 + rest)
//   slopes a of log p_t and b of H:  dz_v = a ([v = t] - p_v) - b p_v (d_v - D),  dh = scale dz E_g,  dE_g = scale dz^T h
//
// In `rest` one of the largest entries is left out, so that log1p(rest), and 1 - p_t = rest / (1 + rest) where the target is the largest, keep their digits where a row is
// sure of its token; elsewhere p_t is at most one half.  D comes from distances, so nothing cancels in H (both parts are positive) nor in d_v - D.
//
// Forward: one product, whose epilogue leaves m, rest and sum d exp d of every row and column tile and, where alternatives are wanted, the largest of every
// four columns (1/4 of the logits: 1 GiB at 8192 x 131072).  Then a wave per row joins them and finds the tiles with the `top` largest maxima, and in these the
// quads (any of the `top` largest entries lies in one of them, and of equal ones those in front); a block per row forms the quads' logits again, four dot
// products each, and sorts.  A quad's largest entry keeps the product's bits, so that the alternatives agree with log p_t; the others may
// differ from the product's in the order of their sums.  No atomics: results do not depend on the order of blocks.
//
// Backward: the logits are formed again, piece by piece, as slopes in the element type, for the two products that follow, as the loss does; in 16 bits a
// slope is off by half a step of itself.  The largest slope of most rows is the target's, and its rounding would be that of the row's whole gradient; so the mantissa
// of the target's slope is taken out of the row's slopes, which leaves a power of two there: dh is multiplied by it in fp32, and the product for dE
// takes rows of h times it (a row whose entry no other row has for its target is then rounded once, as its last rounding would; 4096 rows, 32003 entries of 1024,
// error against 64 bits: dh 1.00 and dE 1.23 times that of a plain form in fp32, both 1.41 times without).  fp16 slopes are also taken times a power of two per
// group that brings their bound below 2^14: p |d - D| is below 22 for any vocabulary up to 2^30, so |a| + 32 |b| bounds a slope; and the rows of h for dE times one that brings the
// group's largest number to 2^14.  Rows whose slopes a and b are both zero take no part.
#include "vocabulary.hpp"
#include "row_access.hpp"

#include <cmath>

namespace cocod {
namespace {

constexpr uint64_t kMaxScoreRows = 1ull << 26;
constexpr uint32_t kMostTop = 32;
// Up to so many rows four waves take a row's statistics instead of one (32000 entries: 300 rows with 20 alternatives 11.8 us instead of 17.6, 2000 with 8 20 against
// 14.5), and sixteen its alternatives instead of four (16 rows with 20 of 512: 7.5 us instead of 12.1, 300 rows 14.2 against 12.8).
constexpr uint32_t kFewRows = 512, kVeryFewRows = 64;
constexpr float kEntropyBound = 32.0f, kSlopeScale16 = 0x1p14f;
// Up to so many bytes of hidden states per group rows stay where they are, those without a target among them (509 rows of 512 in fp32, forward and backward: 143 us instead of 149).
constexpr uint64_t kLeaveHere = 1u << 20;
// Up to so many bytes per group, and of so many groups in all, the block that finds the rows also copies them (9 rows of 1728 in fp16, gradient: 6 us instead of 3 and 5 in two launches;
// 16 groups of 16 rows of 1024 in bf16 would take 24 instead of 27).  All rows may lie in one group, whose block then copies alone: gradients of 8000 rows of 1024 in one of 512 groups
// 270 us instead of 1690 without the second bound, 256 rows in one of 16 27 instead of 57.
constexpr uint64_t kGatherHere = 32u << 10;
constexpr uint32_t kGatherGroups = 4;

// Which rows take part, and with what slopes.
struct Taking {
    Rows rows;                        // target may be null: every row takes part
    int grad;
    const float *d_logp, *d_entropy;  // may be null: 0
};
__device__ __forceinline__ float slope_of_logp(const Taking &p, uint64_t r) { return p.rows.target && p.d_logp ? p.d_logp[r] : 0.0f; }
__device__ __forceinline__ float slope_of_entropy(const Taking &p, uint64_t r) { return p.d_entropy ? p.d_entropy[r] : 0.0f; }
__device__ __forceinline__ bool takes_part(const Taking &p, uint64_t r)
{
    if (p.rows.target && !has_target(p.rows, r)) return false;
    return !p.grad || slope_of_logp(p, r) != 0.0f || slope_of_entropy(p, r) != 0.0f;
}
__device__ __forceinline__ bool in_groups(const Rows &p, uint64_t r) { return r >= clamped(p, 0) && r < clamped(p, p.groups); }

// Copies of the rows that take part, and what their slopes are made of.
template <class E> struct Gather {
    const uint32_t *index;
    const E *h;
    uint64_t ldh;
    uint32_t dim;
    E *out;
    uint64_t pitch;
    E *scaled;                        // non-null: rows times the mantissa of their target's slope
    float *lift;                      // non-null (fp16, with scaled): [rows] power of two that the rows of `scaled` are taken times
    // gradient
    E *dh;                            // may be null
    uint64_t lddh;
    const float4 *norms;
    float scale;
    int normal;                       // row_scale holds the group's factor
    float *row_scale;                 // may be null (fp32: nothing is taken out)
    float *top, *none, *one, *target_slope;
};
// A row times a factor, rounded to the type.
template <class T> __device__ __forceinline__ void scaled_row(const typename T::elem *src, uint32_t dim, typename T::elem *dst, uint64_t pitch, float factor, uint32_t lane)
{
    typedef Piece<T> V;
    for (uint32_t j = lane * V::N; j < pitch; j += 64 * V::N) {
        const u4 raw = j < dim ? V::load(src + j, dim - j) : u4{0, 0, 0, 0};
        float v[V::N];
        #pragma unroll
        for (uint32_t i = 0; i < V::N; ++i) v[i] = V::value(raw, i) * factor;
        V::store(dst + j, V::pack(v));
    }
}
// The largest magnitude of a row that is finite, in all lanes of a wave.
template <class T> __device__ __forceinline__ float largest_of_row(const typename T::elem *src, uint32_t dim, uint32_t lane)
{
    typedef Piece<T> V;
    float most = 0.0f;
    for (uint32_t j = lane * V::N; j < dim; j += 64 * V::N) {
        const u4 raw = V::load(src + j, dim - j);
        #pragma unroll
        for (uint32_t i = 0; i < V::N; ++i) {
            const float v = fabsf(V::value(raw, i));
            if (v < INFINITY) most = fmaxf(most, v);
        }
    }
    #pragma unroll
    for (int d = 1; d < 64; d <<= 1) most = fmaxf(most, __shfl_xor(most, d, 64));
    return most;
}
// Row r of the copies, from row `from` of the caller's, by a wave.
template <class T> __device__ __forceinline__ void gather_row(const Taking &p, const Gather<typename T::elem> &q, uint64_t r, uint32_t from, uint32_t lane)
{
    const typename T::elem *h = q.h + from * q.ldh;
    copy_row(h, q.dim, q.out + r * q.pitch, q.pitch, lane);
    if (!p.grad) return;
    const float4 n = q.norms[from];                            // top, rest, D, distance of the target
    const float a = slope_of_logp(p, from), b = slope_of_entropy(p, from), inverse = 1.0f / (1.0f + n.y);
    const float back = q.normal ? q.row_scale[r] : 1.0f, k = q.scale / back;
    const float pt = expf(n.w) * inverse, others = n.w == 0.0f ? n.y * inverse : 1.0f - pt;
    // (a target at minus infinity has no part in the entropy's slope; a NaN is in pt as well)
    float target = (a * others + b * pt * (n.z - fmaxf(n.w, kFarBelow))) * k, mantissa = 1.0f;
    if (q.row_scale && p.rows.target && fabsf(target) > 0x1p-126f && fabsf(target) < 0x1p126f) {
        mantissa = __builtin_amdgcn_frexp_mantf(fabsf(target));       // in 1/2 .. 1
        target = copysignf(ldexpf(1.0f, __builtin_amdgcn_frexp_expf(target)), target);
    }
    if (q.scaled) scaled_row<T>(h, q.dim, q.scaled + r * q.pitch, q.pitch, q.lift ? mantissa * q.lift[r] : mantissa, lane);
    if (lane == 0) {
        const float even = inverse * k / mantissa;
        q.top[r] = n.x;
        q.none[r] = (b * n.z - a) * even;
        q.one[r] = -b * even;
        q.target_slope[r] = target;
        if (q.row_scale) q.row_scale[r] = back * mantissa;
    }
}
// Row r of the caller's: no gradient where it takes no part.
template <class T> __device__ __forceinline__ void clear_row(const Taking &p, const Gather<typename T::elem> &q, uint64_t r, uint32_t lane)
{
    if (p.grad && q.dh && !takes_part(p, r))
        for (uint32_t j = lane; j < q.dim; j += 64) q.dh[r * q.lddh + j] = 0;
}

// By row of the caller's that takes part, its largest magnitude; a wave a row.
constexpr uint32_t kMostRowBlocks = 1u << 23, kMostAlternativeBlocks = 1u << 21;
template <class T> __global__ __launch_bounds__(256) void scores_reach_kernel(const Taking p, const Gather<typename T::elem> q)
{
    const uint32_t lane = threadIdx.x % 64;
    for (uint64_t r = static_cast<uint64_t>(blockIdx.x) * 4 + threadIdx.x / 64; r < p.rows.rows; r += static_cast<uint64_t>(gridDim.x) * 4) {
        if (!in_groups(p.rows, r) || !takes_part(p, r)) continue;
        const float most = largest_of_row<T>(q.h + r * q.ldh, q.dim, lane);
        if (lane == 0) q.lift[r] = most;
    }
}

// One block per group: the rows that take part, in order, to the front of the group's part of `index`; kNoRow behind them.  NORMAL: the group's power of
// two, for the table's gradient and row by row, and where h gets a second copy the power of two that brings the largest magnitude of the group's rows to 2^14 .. 2^15 there: 16-bit
// floats below 2^-14 have fewer digits, and h times a mantissa would be rounded by up to a third of itself.  HERE: the copies as well (a launch less where there is little to copy).
constexpr int kTakeThreads = 1024;
template <class T, bool NORMAL, bool HERE>
__global__ __launch_bounds__(kTakeThreads) void take_kernel(const Taking p, float scale, uint32_t *index, int32_t *target, int64_t *ends, float *group_scale, float *row_scale,
                                                            const Gather<typename T::elem> gather)
{
    __shared__ uint32_t counts[kTakeThreads / 64];
    __shared__ float most[kTakeThreads / 64], furthest[kTakeThreads / 64];
    const uint32_t g = blockIdx.x, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint64_t begin = clamped(p.rows, g), next = clamped(p.rows, g + 1), end = next > begin ? next : begin;
    uint64_t at = begin;
    float bound = 0.0f, reach = 0.0f;
    for (uint64_t r0 = begin; r0 < end; r0 += kTakeThreads) {
        const uint64_t r = r0 + threadIdx.x;
        const bool in = r < end && takes_part(p, r);
        const unsigned long long votes = __ballot(in);
        if (lane == 0) counts[wave] = __popcll(votes);
        __syncthreads();
        uint32_t before = 0, all = 0;
        for (int w = 0; w < kTakeThreads / 64; ++w) { if (w < static_cast<int>(wave)) before += counts[w]; all += counts[w]; }
        if (in) {
            const uint64_t to = at + before + __popcll(votes & ((1ull << lane) - 1));
            index[to] = static_cast<uint32_t>(r);
            target[to] = p.rows.target ? p.rows.target[r] : -1;
            if (NORMAL) bound = fmaxf(bound, fabsf(slope_of_logp(p, r)) + kEntropyBound * fabsf(slope_of_entropy(p, r)));
            if (NORMAL && !HERE && gather.lift) reach = fmaxf(reach, gather.lift[r]);
        }
        at += all;
        __syncthreads();
    }
    for (uint64_t r = at + threadIdx.x; r < end; r += kTakeThreads) index[r] = kNoRow;
    if (threadIdx.x == 0) ends[g] = static_cast<int64_t>(at);
    if constexpr (NORMAL) {
        if (HERE && gather.lift) {
            for (uint64_t r = begin + wave; r < end; r += kTakeThreads / 64)
                if (takes_part(p, r)) reach = fmaxf(reach, largest_of_row<T>(gather.h + r * gather.ldh, gather.dim, lane));
        }
        #pragma unroll
        for (int d = 1; d < 64; d <<= 1) { bound = fmaxf(bound, __shfl_xor(bound, d, 64)); reach = fmaxf(reach, __shfl_xor(reach, d, 64)); }
        if (lane == 0) { most[wave] = bound; furthest[wave] = reach; }
        __syncthreads();
        for (int w = 0; w < kTakeThreads / 64; ++w) { bound = fmaxf(bound, most[w]); reach = fmaxf(reach, furthest[w]); }
        bound *= scale;
        int e = bound > 0.0f && bound < INFINITY ? __builtin_amdgcn_frexp_expf(bound) : 0;
        e = e < -100 ? -100 : e > 100 ? 100 : e;
        const float back = ldexpf(1.0f / kSlopeScale16, e);    // what the products are multiplied by
        const float lift = reach > 0.0f && reach < 0x1p14f ? ldexpf(1.0f, 15 - __builtin_amdgcn_frexp_expf(reach)) : 1.0f;       // (no row to lift: 1)
        if (threadIdx.x == 0) group_scale[g] = back / lift;
        for (uint64_t r = begin + threadIdx.x; r < at; r += kTakeThreads) {
            row_scale[r] = back;
            if (gather.lift) gather.lift[r] = lift;            // (from here on by gathered row)
        }
    }
    if constexpr (HERE) {
        __syncthreads();                                       // (also the block's writes of index and row_scale)
        for (uint64_t r = begin + wave; r < end; r += kTakeThreads / 64) {
            if (r < at) {
                // Groups whose offsets do not ascend share rows, and the block of another one may have left kNoRow in this place since.
                const uint32_t from = index[r];
                if (from != kNoRow) gather_row<T>(p, gather, r, from, lane);
            }
            clear_row<T>(p, gather, r, lane);
        }
    }
}

// The copies by a launch of their own, a wave a row.
template <class T> __global__ __launch_bounds__(256) void scores_gather_kernel(const Taking p, const Gather<typename T::elem> q)
{
    const uint32_t lane = threadIdx.x % 64;
    for (uint64_t r = static_cast<uint64_t>(blockIdx.x) * 4 + threadIdx.x / 64; r < p.rows.rows; r += static_cast<uint64_t>(gridDim.x) * 4) {
        if (!in_groups(p.rows, r)) continue;
        const uint32_t from = q.index[r];
        if (from != kNoRow) gather_row<T>(p, q, r, from, lane);
        clear_row<T>(p, q, r, lane);
    }
}

// ---- a row's scores --------------------------------------------------------------------------------------

struct Joined { float top, rest, far; };
__device__ __forceinline__ Joined join(const Joined &a, const Joined &b)
{
    const bool first = a.top >= b.top;
    const Joined hi = first ? a : b, lo = first ? b : a;
    const float d = lo.top - (hi.top == -INFINITY ? 0.0f : hi.top), e = expf(d), w = (1.0f + lo.rest) * e;
    return {hi.top, hi.rest + w, hi.far + fmaf(e, lo.far, fmaxf(d, kFarBelow) * w)};
}
__device__ __forceinline__ Joined join_lane(const Joined &a, int d) { return join(a, {__shfl_xor(a.top, d, 64), __shfl_xor(a.rest, d, 64), __shfl_xor(a.far, d, 64)}); }

// A number that is larger for larger values, and for smaller places of equal values; NaN counts as minus infinity; 0 is none.
__device__ __forceinline__ unsigned long long rank_of(float v, uint32_t place)
{
    const uint32_t bits = __float_as_uint(v == v ? v + 0.0f : -INFINITY);
    return static_cast<unsigned long long>(bits >> 31 ? ~bits : bits | 0x80000000u) << 32 | ~place;
}
__device__ __forceinline__ uint32_t place_of(unsigned long long rank) { return ~static_cast<uint32_t>(rank); }
__device__ __forceinline__ float value_of(unsigned long long rank)
{
    const uint32_t u = static_cast<uint32_t>(rank >> 32);
    return __uint_as_float(u >> 31 ? u & 0x7fffffffu : ~u);
}
// The largest of the lanes' numbers, by lane moves within rows of 16 and broadcasts of their last lanes.
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t larger_moved(uint32_t v)
{
    const uint32_t u = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(static_cast<int>(v), static_cast<int>(v), CTRL, ROWS, 0xf, false));
    return u > v ? u : v;
}
__device__ __forceinline__ uint32_t wave_largest(uint32_t v)
{
    v = larger_moved<0x111, 0xf>(v);                           // from 1, 2, 4 and 8 lanes below
    v = larger_moved<0x112, 0xf>(v);
    v = larger_moved<0x114, 0xf>(v);
    v = larger_moved<0x118, 0xf>(v);
    v = larger_moved<0x142, 0xa>(v);                           // rows 1 and 3 from the last lane of the row below
    v = larger_moved<0x143, 0xc>(v);                           // rows 2 and 3 from lane 31
    return __builtin_amdgcn_readlane(v, 63);
}

// All threads that work on a row: a wave, or a block.
template <int THREADS> __device__ __forceinline__ void together()
{
    if constexpr (THREADS == 64) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    } else {
        __syncthreads();
    }
}

// How many of the wave's first `count` ranks are above this lane's.
__device__ __forceinline__ uint32_t above(unsigned long long mine, uint32_t count, unsigned long long *scratch, uint32_t lane)
{
    together<64>();
    scratch[lane] = mine;
    together<64>();
    uint32_t n = 0;
    for (uint32_t i = 0; i < count; i += 4) {
        #pragma unroll
        for (uint32_t j = 0; j < 4; ++j) n += scratch[i + j] > mine ? 1 : 0;       // (behind `count` there are zeros)
    }
    return n;
}

// The k largest of the `all` ranks in `list` (all different, but for 0), in order, by one wave: lane j returns the j-th, 0 where there are fewer.  A lane's best is the best of every
// 64th; what is not below the k-th of the lanes' bests, k ranks and hardly more, is put together and each one's place counted.  (Where that is
// more than a wave, one after the other: a lane keeps its best two and looks for more when both are taken.  300 rows, 20 of 32000 entries: the kernel takes 15 us instead of 23.)
__device__ __forceinline__ unsigned long long pick(const unsigned long long *list, uint32_t all, uint32_t k, unsigned long long *scratch, uint32_t lane)
{
    unsigned long long best = 0, next = 0;
    #pragma unroll 2
    for (uint32_t i = lane; i < all; i += 64) {
        const unsigned long long v = list[i];
        next = v > best ? best : v > next ? v : next;
        best = v > best ? v : best;
    }
    unsigned long long candidate = best;
    uint32_t count = 64;
    if (all > 64) {
        const unsigned long long last = __ballot(above(best, 64, scratch, lane) == k - 1 && best != 0);
        unsigned long long least = 1;                          // fewer lanes than k hold any: every rank is a candidate
        if (last) {
            const int who = __ffsll(last) - 1;
            least = static_cast<unsigned long long>(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<uint32_t>(best >> 32), who))) << 32 |
                    static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<uint32_t>(best), who));
        }
        count = 0;
        unsigned long long kept = 0;
        together<64>();
        scratch[lane] = 0;
        together<64>();
        for (uint32_t i0 = 0; i0 < all; i0 += 64) {
            const unsigned long long v = i0 + lane < all ? list[i0 + lane] : 0;
            const bool in = v >= least;
            const unsigned long long votes = __ballot(in);
            const uint32_t at = count + __popcll(votes & ((1ull << lane) - 1));
            if (in && at < 64) scratch[at] = v;
            count += __popcll(votes);
        }
        together<64>();
        kept = scratch[lane];
        candidate = kept;
        if (count > 64) {
            unsigned long long mine = 0;
            bool known = true;                                 // `next` is the lane's second best
            for (uint32_t j = 0; j < k; ++j) {
                const uint32_t high = wave_largest(static_cast<uint32_t>(best >> 32));
                const uint32_t low = wave_largest(static_cast<uint32_t>(best >> 32) == high ? static_cast<uint32_t>(best) : 0);
                const unsigned long long taken = static_cast<unsigned long long>(high) << 32 | low;
                if (lane == j) mine = taken;
                if (taken == 0) break;
                if (best == taken) {
                    if (known) {
                        best = next;
                        known = false;
                    } else {
                        best = next = 0;
                        known = true;
                        for (uint32_t i = lane; i < all; i += 64) {
                            const unsigned long long v = list[i] < taken ? list[i] : 0;
                            next = v > best ? best : v > next ? v : next;
                            best = v > best ? v : best;
                        }
                    }
                }
            }
            return mine;
        }
    }
    const uint32_t place = above(candidate, count, scratch, lane);
    together<64>();
    scratch[lane] = 0;
    together<64>();
    if (candidate != 0 && place < k) scratch[place] = candidate;
    together<64>();
    return lane < k ? scratch[lane] : 0;
}

// The k largest of rank(0) .. rank(n - 1), in order, to list[0 .. k - 1]; 0 behind them.  THREADS threads fetch `kRanks` of them at a time into LDS, behind the list so far.
template <int THREADS> constexpr uint32_t kRanks = THREADS == 64 ? 512 : 2048;
template <int THREADS> struct Picking { unsigned long long list[kMostTop + kRanks<THREADS>], scratch[64]; };
template <int THREADS, class Rank> __device__ __forceinline__ void largest(uint32_t n, uint32_t k, const Rank &rank, Picking<THREADS> &p, uint32_t tid)
{
    if (tid < k) p.list[tid] = 0;
    for (uint32_t base = 0; base < n; base += kRanks<THREADS>) {
        const uint32_t count = n - base < kRanks<THREADS> ? n - base : kRanks<THREADS>;
        #pragma unroll 4
        for (uint32_t i = tid; i < count; i += THREADS) p.list[k + i] = rank(base + i);
        together<THREADS>();
        if (tid < 64) {
            const unsigned long long mine = pick(p.list, k + count, k, p.scratch, tid);
            together<64>();
            if (tid < k) p.list[tid] = mine;
        }
        together<THREADS>();
    }
}

struct Scores {
    Taking taking;
    const uint32_t *index;            // null: rows lie where the caller has them
    const float4 *moments;
    uint32_t tiles, tile_quads;
    const float *target_logit;        // null: no targets
    float *logp, *entropy;            // may be null
    float4 *norms;                    // may be null
    // alternatives
    uint32_t top;
    int32_t *top_ids;
    float *top_logp;
    uint64_t ld_top;
    const float *quads;
    uint64_t ld_quads;
    QuadOrder order;
    unsigned long long *quad_rank;    // [rows][top]
    float2 *row_norm;                 // [rows]: largest logit, log(1 + rest)
    const int32_t *target;            // by row of the product; null: none
    const void *h, *e;                // h: rows of the product
    uint64_t ldh, lde, e_stride;
    uint32_t dim;
    float scale;
};

// Log probability and entropy of a row, and the quads of its alternatives.  WAVES waves a row: four where rows are few and have alternatives.
template <int WAVES, bool TOP> __global__ __launch_bounds__(256) void scores_kernel(const Scores p)
{
    constexpr int ROWS = 4 / WAVES, THREADS = 64 * WAVES;
    __shared__ Joined parts[WAVES];
    __shared__ unsigned long long tile_rank[ROWS][TOP ? kMostTop : 1];
    __shared__ typename std::conditional<TOP, Picking<THREADS>, char>::type picking[ROWS];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, tid = threadIdx.x % THREADS, mine = threadIdx.x / THREADS;
    const Rows &rows = p.taking.rows;
    // (all threads of a row leave a turn together)
    for (uint64_t r = static_cast<uint64_t>(blockIdx.x) * ROWS + mine; r < rows.rows; r += static_cast<uint64_t>(gridDim.x) * ROWS) {
        if (!in_groups(rows, r)) continue;
        if (!takes_part(p.taking, r)) {
            if (tid == 0) {
                if (p.logp) p.logp[r] = 0.0f;
                if (p.entropy) p.entropy[r] = 0.0f;
                if (p.norms) p.norms[r] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
            if (TOP && tid < p.top) { p.top_ids[r * p.ld_top + tid] = -1; p.top_logp[r * p.ld_top + tid] = -INFINITY; }
            if (!p.index) continue;
        }
        const uint32_t to = p.index ? p.index[r] : static_cast<uint32_t>(r);
        if (to == kNoRow) continue;

        Joined sum = {-INFINITY, -1.0f, 0.0f};
        const float4 *moments = p.moments + r * p.tiles;
        constexpr int AHEAD = 4;
        for (uint32_t t = tid; t < p.tiles; t += THREADS * AHEAD) {
            float4 m[AHEAD];
            #pragma unroll
            for (int a = 0; a < AHEAD; ++a) m[a] = t + a * THREADS < p.tiles ? moments[t + a * THREADS] : make_float4(-INFINITY, -1.0f, 0.0f, 0.0f);
            #pragma unroll
            for (int a = 0; a < AHEAD; ++a) sum = join(sum, {m[a].x, m[a].y, m[a].z});
        }
        #pragma unroll
        for (int d = 1; d < 64; d <<= 1) sum = join_lane(sum, d);
        if constexpr (WAVES > 1) {
            if (lane == 0) parts[wave] = sum;
            __syncthreads();
            sum = parts[0];
            #pragma unroll
            for (int w = 1; w < WAVES; ++w) sum = join(sum, parts[w]);
        }
        if (tid == 0) {
            const float norm = log1pf(sum.rest), far = sum.far / (1.0f + sum.rest), distance = p.target_logit ? p.target_logit[r] - sum.top : 0.0f;
            if (p.logp) p.logp[to] = distance - norm;
            if (p.entropy) p.entropy[to] = norm - far;
            if (p.norms) p.norms[to] = make_float4(sum.top, sum.rest, far, distance);
            if (TOP) p.row_norm[r] = make_float2(sum.top, norm);
        }
        if constexpr (TOP) {
            // the tiles, the quads in them
            unsigned long long *const list = picking[mine].list, *const tiles = tile_rank[mine];
            const float *quads = p.quads + r * p.ld_quads;
            largest<THREADS>(p.tiles, p.top, [&](uint32_t t) { return rank_of(moments[t].x, t); }, picking[mine], tid);
            if (tid < p.top) tiles[tid] = list[tid];
            together<THREADS>();
            const uint32_t others = p.order.width / p.order.each, all = (rows.vocab + 3) / 4;
            largest<THREADS>(p.top * p.tile_quads, p.top, [&](uint32_t i) -> unsigned long long {
                const unsigned long long tile = tiles[i / p.tile_quads];
                if (!tile) return 0;
                const uint32_t at = place_of(tile) * p.tile_quads + i % p.tile_quads, in = at % p.order.width;
                const uint32_t quad = at - in + in % p.order.each * others + in / p.order.each;
                return quad < all ? rank_of(quads[at], quad) : 0;
            }, picking[mine], tid);
            if (tid < p.top) p.quad_rank[r * p.top + tid] = list[tid];
            together<THREADS>();                               // the next row's
        }
    }
}

// A row's alternatives from its quads: their logits, a quad a wave at a time, and the largest of these.  A block a row.
template <class T> __global__ __launch_bounds__(1024) void alternatives_kernel(const Scores p)
{
    typedef Piece<T> V;
    typedef typename T::elem elem;
    __shared__ unsigned long long entries[4 * kMostTop], scratch[64];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, waves = blockDim.x / 64;
    const Rows &rows = p.taking.rows;
    for (uint64_t r = blockIdx.x; r < rows.rows; r += gridDim.x) {
        if (!in_groups(rows, r) || (!p.index && !takes_part(p.taking, r))) continue;
        const uint32_t to = p.index ? p.index[r] : static_cast<uint32_t>(r);
        if (to == kNoRow) continue;
        uint32_t g = 0;
        for (uint32_t lo = 0, hi = rows.groups; hi - lo > 1;) {      // group of the row: the last one that begins at it or in front, if it is not empty
            const uint32_t mid = (lo + hi) / 2;
            if (clamped(rows, mid) <= r) lo = mid; else hi = mid;
            g = lo;
        }
        const elem *h = static_cast<const elem *>(p.h) + r * p.ldh, *e = static_cast<const elem *>(p.e) + g * p.e_stride;
        const uint32_t target = p.target ? static_cast<uint32_t>(p.target[r]) : ~0u;
        for (uint32_t j = wave; j < p.top; j += waves) {
            const unsigned long long rank = p.quad_rank[r * p.top + j];
            if (!rank) { if (lane < 4) entries[4 * j + lane] = 0; continue; }
            const uint32_t v0 = __builtin_amdgcn_readfirstlane(place_of(rank)) * 4, count = rows.vocab - v0 < 4 ? rows.vocab - v0 : 4;
            float dot[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            const elem *row[4];
            #pragma unroll
            for (uint32_t k = 0; k < 4; ++k) row[k] = e + static_cast<uint64_t>(v0 + (k < count ? k : 0)) * p.lde;
            uint32_t c = lane * V::N;
            #pragma unroll 2
            for (; c + V::N <= p.dim; c += 64 * V::N) {
                const u4 a = V::load(h + c);
                u4 b[4];
                #pragma unroll
                for (uint32_t k = 0; k < 4; ++k) b[k] = V::load(row[k] + c);
                #pragma unroll
                for (uint32_t k = 0; k < 4; ++k)
                    #pragma unroll
                    for (uint32_t i = 0; i < V::N; ++i) dot[k] = fmaf(V::value(a, i), V::value(b[k], i), dot[k]);
            }
            #pragma unroll 1
            for (; c < p.dim; ++c) {                           // the last columns of one lane
                const float a = widen<T>(h[c]);
                #pragma unroll
                for (uint32_t k = 0; k < 4; ++k) dot[k] = fmaf(a, widen<T>(row[k][c]), dot[k]);
            }
            #pragma unroll
            for (int d = 1; d < 64; d <<= 1)
                #pragma unroll
                for (int k = 0; k < 4; ++k) dot[k] += __shfl_xor(dot[k], d, 64);
            const float most = value_of(rank);
            uint32_t first = 0;
            #pragma unroll
            for (uint32_t k = 0; k < 4; ++k) {
                dot[k] = k < count ? dot[k] * p.scale : -INFINITY;
                if (dot[k] != dot[k]) dot[k] = -INFINITY;
                if (k > 0 && dot[k] > dot[first]) first = k;
            }
            if (lane < 4) {
                float v = lane == 0 ? dot[0] : lane == 1 ? dot[1] : lane == 2 ? dot[2] : dot[3];
                v = lane == first ? most : fminf(v, most);
                if (v0 + lane == target) v = p.target_logit[r];
                entries[4 * j + lane] = lane < count ? rank_of(v, v0 + lane) : 0;
            }
        }
        __syncthreads();
        if (wave == 0) {
            const unsigned long long rank = pick(entries, 4 * p.top, p.top, scratch, lane);
            const float2 norm = p.row_norm[r];
            if (lane < p.top) {
                p.top_ids[to * p.ld_top + lane] = rank ? static_cast<int32_t>(place_of(rank)) : -1;
                p.top_logp[to * p.ld_top + lane] = rank ? (value_of(rank) - norm.x) - norm.y : -INFINITY;
            }
        }
        __syncthreads();                                       // the next row's
    }
}

// ---- the calls -------------------------------------------------------------------------------------------

struct Workspace {
    uint64_t index, target, ends, hidden, target_logit, moments, quads, ld_quads, quad_rank, row_norm;
    uint64_t scaled, lift, row_scale, group_scale, top, none, one, target_slope, slope, sum, part;
    uint64_t pitch, piece, sum_pitch, bytes;
    uint32_t pieces;
    ProductPlan logits, to_hidden, to_table;
};

Workspace carve(const cocod_token_scores_call *c, bool grad)
{
    Workspace w{};
    const Dtype t = kTypes[c->dtype];
    const uint64_t s = dtype_bytes(t), rows = c->rows;
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) { const uint64_t o = at; at += (bytes + 255) / 256 * 256; return o; };
    const bool dim8 = c->dim % 8 == 0;                         // a dense table's rows then start on 16 bytes
    w.pitch = (static_cast<uint64_t>(c->dim) + 7) / 8 * 8;
    w.index = take(rows * 4);
    w.target = take(rows * 4);
    w.ends = take(c->groups * 8ull);
    w.hidden = take(rows * w.pitch * s);
    if (!grad) {
        w.logits = plan_product(Layout::Rows_NK, t, dim8, rows, c->groups, 0, c->vocab, c->dim, false, false);
        w.target_logit = take(rows * 4);
        const uint32_t planned = tile_cols(t, w.logits.tile), narrow = planned < 128 ? planned : 128;        // the large tile may have to give way to the medium one
        w.moments = take((static_cast<uint64_t>(c->vocab) + narrow - 1) / narrow * rows * 16);
        w.ld_quads = (static_cast<uint64_t>(c->vocab) + 255) / 256 * 64;
        if (c->top) {
            w.quads = take(rows * w.ld_quads * 4);
            w.quad_rank = take(rows * c->top * 8);
            w.row_norm = take(rows * 8);
        }
    } else {
        const Pieces pieces = pieces_of(c->piece, rows, c->vocab);
        w.piece = pieces.size;
        w.pieces = pieces.count;
        const uint32_t n = static_cast<uint32_t>(w.piece < c->vocab ? w.piece : c->vocab);
        w.logits = plan_product(Layout::Rows_NK, t, dim8, rows, c->groups, 0, n, c->dim, false, false);
        w.to_hidden = plan_product(Layout::Rows_KN, t, dim8, rows, c->groups, 0, c->dim, n, true);
        w.to_table = plan_product(Layout::Weights, t, true, rows, c->groups, n, c->dim, 0, true);
        w.scaled = c->de && t != Dtype::F32 ? take(rows * w.pitch * s) : w.hidden;
        w.lift = c->de && t == Dtype::F16 ? take(rows * 4) : 0;
        w.row_scale = take(rows * 4);
        w.group_scale = take(c->groups * 4ull);
        w.top = take(rows * 4);
        w.none = take(rows * 4);
        w.one = take(rows * 4);
        w.target_slope = take(rows * 4);
        w.slope = take(rows * w.piece * s);
        w.sum_pitch = part_pitch(c->dim);
        if (c->dh && w.pieces > 1) w.sum = take(rows * w.sum_pitch * 4);
        uint64_t part = 0;
        if (c->dh) part = part_bytes(w.to_hidden, Layout::Rows_KN, rows, c->groups, 0, c->dim);
        if (c->de) { const uint64_t q = part_bytes(w.to_table, Layout::Weights, rows, c->groups, n, c->dim); part = part > q ? part : q; }
        w.part = take(part);
    }
    w.bytes = at;
    return w;
}

int check(const cocod_token_scores_call *c)
{
    if (!c) return set_error(COCOD_ERR_INVALID, "the description is NULL");
    if (c->struct_size != sizeof(cocod_token_scores_call))
        return set_error(COCOD_ERR_INVALID, "struct_size %u does not match this library (%zu)", c->struct_size, sizeof(cocod_token_scores_call));
    if (int rc = check_dtype(c->dtype)) return rc;
    if (c->flags & ~COCOD_TOKEN_SCORES_RELU_IN) return set_error(COCOD_ERR_INVALID, "unknown flag bits 0x%x", c->flags);
    if (c->groups < 1 || c->groups > kMaxGroups) return set_error(COCOD_ERR_INVALID, "groups must be in 1..65535");
    if (c->rows >= kMaxScoreRows) return set_error(COCOD_ERR_INVALID, "rows must be below 2^26");
    if (c->dim < 1 || c->dim > kMaxWidth || c->vocab < 1 || c->vocab > kMaxWidth) return set_error(COCOD_ERR_INVALID, "dim and vocab must be in 1..2^30");
    if (c->top > kMostTop) return set_error(COCOD_ERR_INVALID, "top must be in 0..32");
    if (!std::isfinite(c->scale) || !(c->scale > 0.0f)) return set_error(COCOD_ERR_INVALID, "scale must be finite and above 0");
    return COCOD_OK;
}

// What both directions read, and the workspace.
int check_inputs(const cocod_token_scores_call *c, const Workspace &w)
{
    const uint64_t s = dtype_bytes(kTypes[c->dtype]);
    if (!c->offsets || (reinterpret_cast<uintptr_t>(c->offsets) & 7)) return set_error(COCOD_ERR_INVALID, "offsets is NULL or not 8-byte aligned");
    if (int rc = check_matrix("h", c->h, c->dim, c->ldh, s, c->rows)) return rc;
    if (int rc = check_matrix("e", c->e, c->dim, c->lde, s)) return rc;
    if (int rc = check_stride("e", c->e_stride, c->groups, c->vocab, c->dim, c->lde, true)) return rc;
    if (c->targets) if (int rc = check_matrix("targets", c->targets, 1, 1, 4)) return rc;
    if (c->norms && (reinterpret_cast<uintptr_t>(c->norms) & 15)) return set_error(COCOD_ERR_INVALID, "norms is not 16-byte aligned");
    if (!c->workspace || (reinterpret_cast<uintptr_t>(c->workspace) & 255)) return set_error(COCOD_ERR_INVALID, "workspace is NULL or not 256-byte aligned");
    if (c->workspace_bytes < w.bytes)
        return set_error(COCOD_ERR_INVALID, "workspace holds %llu bytes, %llu are needed", (unsigned long long)c->workspace_bytes, (unsigned long long)w.bytes);
    return COCOD_OK;
}

ProductParams logits_operands(const cocod_token_scores_call *c, const Workspace &w, const uint8_t *ws, bool gathered)
{
    ProductParams p{};
    p.a = gathered ? ws + w.hidden : c->h; p.lda = gathered ? w.pitch : c->ldh;
    p.b = c->e; p.ldb = c->lde; p.b_group = c->groups > 1 ? c->e_stride : 0;
    p.k = c->dim;
    return p;
}
ProductParams hidden_operands(const cocod_token_scores_call *c, const Workspace &w, const uint8_t *ws, uint64_t v0, uint32_t n)
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
    p.b = ws + w.scaled; p.ldb = w.pitch;
    return p;
}
// Operands of the forward call.  Rows stay where they are if all of them take part or they are few, and the product can take them there.
ProductParams forward_operands(const cocod_token_scores_call *c, const Workspace &w, const uint8_t *ws, bool &gathered)
{
    const Dtype t = kTypes[c->dtype];
    const uint64_t s = dtype_bytes(t);
    ProductParams z = logits_operands(c, w, ws, false);
    gathered = (c->targets && c->rows * w.pitch * s > kLeaveHere * c->groups) || (t != Dtype::F32 && direct_b(Layout::Rows_NK, z) && !direct_a(Layout::Rows_NK, z));
    if (gathered) z = logits_operands(c, w, ws, true);
    // (one table for 16 groups of a row, 32000 entries of 1024: 113 us instead of 128 past the caches; 4 groups of two rows, 131072 of 2048: 213 against 209)
    z.b_once = c->rows <= tile_size(t, Tile::Small).bm && static_cast<uint64_t>(z.b_group ? c->groups : 1) * c->vocab * c->dim * s > kLastLevelCache;
    return z;
}
bool fits(const cocod_token_scores_call *c, Layout layout, const ProductPlan &plan, const ProductParams &p, uint32_t m, uint32_t n, uint32_t splits)
{
    const Dtype t = kTypes[c->dtype];
    const TileSize size = tile_size(t, settle_tile(t, layout, plan.tile, p));
    return fits_a_launch(size, blocks_of(size, layout == Layout::Weights, c->rows, c->groups, m, n, splits));
}

template <class T> hipError_t launch_gather(hipStream_t q, const Taking &taking, const cocod_token_scores_call *c, const Workspace &w, uint8_t *ws)
{
    typedef typename T::elem E;
    const bool normal = taking.grad && kTypes[c->dtype] == Dtype::F16;
    uint32_t *index = reinterpret_cast<uint32_t *>(ws + w.index);
    float *row_scale = reinterpret_cast<float *>(ws + w.row_scale);
    Gather<E> g{};
    g.index = index;
    g.h = static_cast<const E *>(c->h); g.ldh = c->ldh; g.dim = c->dim;
    g.out = reinterpret_cast<E *>(ws + w.hidden); g.pitch = w.pitch;
    if (taking.grad) {
        g.dh = static_cast<E *>(c->dh); g.lddh = c->lddh;
        g.norms = reinterpret_cast<const float4 *>(c->norms);
        g.scale = c->scale;
        g.normal = normal;
        g.row_scale = sizeof(E) == 2 ? row_scale : nullptr;
        g.scaled = w.scaled != w.hidden ? reinterpret_cast<E *>(ws + w.scaled) : nullptr;
        g.lift = g.scaled && normal ? reinterpret_cast<float *>(ws + w.lift) : nullptr;
        g.top = reinterpret_cast<float *>(ws + w.top); g.none = reinterpret_cast<float *>(ws + w.none);
        g.one = reinterpret_cast<float *>(ws + w.one); g.target_slope = reinterpret_cast<float *>(ws + w.target_slope);
    }
    const bool here = c->rows * w.pitch * sizeof(E) <= kGatherHere * (c->groups < kGatherGroups ? c->groups : kGatherGroups);
    const uint64_t blocks = (c->rows + 3) / 4;
    const dim3 by_rows(static_cast<uint32_t>(blocks < kMostRowBlocks ? blocks : kMostRowBlocks));
    if (g.lift && !here) hipLaunchKernelGGL(scores_reach_kernel<T>, by_rows, dim3(256), 0, q, taking, g);
    const auto take = normal ? (here ? take_kernel<T, true, true> : take_kernel<T, true, false>) : (here ? take_kernel<T, false, true> : take_kernel<T, false, false>);
    hipLaunchKernelGGL(take, dim3(c->groups), dim3(kTakeThreads), 0, q, taking, c->scale, index, reinterpret_cast<int32_t *>(ws + w.target), reinterpret_cast<int64_t *>(ws + w.ends),
                       reinterpret_cast<float *>(ws + w.group_scale), row_scale, g);
    if (here) return hipGetLastError();
    hipLaunchKernelGGL(scores_gather_kernel<T>, by_rows, dim3(256), 0, q, taking, g);
    return hipGetLastError();
}

void launch_scores(hipStream_t q, const Scores &p)
{
    const bool few = p.top && p.taking.rows.rows <= kFewRows;
    const uint64_t blocks = few ? p.taking.rows.rows : (p.taking.rows.rows + 3) / 4;
    const dim3 grid(static_cast<uint32_t>(blocks < kMostRowBlocks ? blocks : kMostRowBlocks));
    if (few)        hipLaunchKernelGGL((scores_kernel<4, true>), grid, dim3(256), 0, q, p);
    else if (p.top) hipLaunchKernelGGL((scores_kernel<1, true>), grid, dim3(256), 0, q, p);
    else            hipLaunchKernelGGL((scores_kernel<1, false>), grid, dim3(256), 0, q, p);
}
template <class T> hipError_t launch_scores(hipStream_t q, const Scores &p)
{
    launch_scores(q, p);
    if (!p.top) return hipGetLastError();
    const uint64_t rows = p.taking.rows.rows;
    const uint32_t most = rows <= kVeryFewRows ? 16 : 4, waves = p.top < most ? p.top : most;
    hipLaunchKernelGGL(alternatives_kernel<T>, dim3(static_cast<uint32_t>(rows < kMostAlternativeBlocks ? rows : kMostAlternativeBlocks)), dim3(64 * waves), 0, q, p);
    return hipGetLastError();
}

}  // namespace
}  // namespace cocod

using namespace cocod;

extern "C" {

int cocod_token_scores_workspace(const cocod_token_scores_call *c, int direction, uint64_t *bytes)
{
    if (!bytes) return set_error(COCOD_ERR_INVALID, "bytes is NULL");
    if (int rc = check(c)) return rc;
    if (direction != COCOD_TOKEN_SCORES_FORWARD && direction != COCOD_TOKEN_SCORES_GRAD) return set_error(COCOD_ERR_INVALID, "unknown direction %d", direction);
    *bytes = carve(c, direction == COCOD_TOKEN_SCORES_GRAD).bytes;
    return COCOD_OK;
}

int cocod_token_scores(void *stream, const cocod_token_scores_call *c)
{
    if (int rc = check(c)) return rc;
    const Dtype t = kTypes[c->dtype];
    const uint64_t s = dtype_bytes(t);
    const Workspace w = carve(c, false);
    if (int rc = check_inputs(c, w)) return rc;
    if (!c->logp && !c->entropy && !c->norms && !c->top) return set_error(COCOD_ERR_INVALID, "no output is asked for");
    if (c->logp && !c->targets && c->rows) return set_error(COCOD_ERR_INVALID, "logp is asked for, but targets is NULL");
    if (c->logp) if (int rc = check_matrix("logp", c->logp, 1, 1, 4)) return rc;
    if (c->entropy) if (int rc = check_matrix("entropy", c->entropy, 1, 1, 4)) return rc;
    if (c->top) {
        if (int rc = check_matrix("top_ids", c->top_ids, c->top, c->ld_top, 4, c->rows)) return rc;
        if (int rc = check_matrix("top_logp", c->top_logp, c->top, c->ld_top, 4, c->rows)) return rc;
    }
    const Extent all[] = {
        {"workspace", c->workspace, w.bytes}, {"logp", c->logp, c->rows * 4}, {"entropy", c->entropy, c->rows * 4}, {"norms", c->norms, c->rows * 16},
        {"top_ids", c->top ? c->top_ids : nullptr, matrix_bytes(c->rows, c->top, c->ld_top, 4)}, {"top_logp", c->top ? c->top_logp : nullptr, matrix_bytes(c->rows, c->top, c->ld_top, 4)},
        {"h", c->h, matrix_bytes(c->rows, c->dim, c->ldh, s)}, {"e", c->e, stack_bytes(c->groups, c->e_stride, c->vocab, c->dim, c->lde, s)},
        {"targets", c->targets, c->rows * 4}, {"offsets", c->offsets, (c->groups + 1ull) * 8},
    };
    for (int i = 0; i < 6; ++i)
        if (int rc = check_apart(all[i], all + i + 1, 10 - i - 1)) return rc;
    if (c->rows == 0) return COCOD_OK;

    const hipStream_t q = static_cast<hipStream_t>(stream);
    const OnStreamDevice device(q);
    const char *const what = "cocod_token_scores";
    if (device.status() != hipSuccess) return launch_status(device.status(), what);
    uint8_t *ws = static_cast<uint8_t *>(c->workspace);
    Taking taking{};
    taking.rows = {c->offsets, c->groups, c->rows, c->targets, c->vocab};
    bool gathered;
    ProductParams z = forward_operands(c, w, ws, gathered);
    if (!fits(c, Layout::Rows_NK, w.logits, z, 0, c->vocab, 1)) return launch_status(hipErrorInvalidConfiguration, what);
    if (gathered)
        if (int rc = launch_status(t == Dtype::F32 ? launch_gather<F32>(q, taking, c, w, ws) : t == Dtype::BF16 ? launch_gather<Bf16>(q, taking, c, w, ws) : launch_gather<F16>(q, taking, c, w, ws), what)) return rc;
    const Tile tile = settle_tile(t, Layout::Rows_NK, w.logits.tile, z);
    const uint32_t cols = tile_cols(t, tile);
    z.offsets = c->offsets; z.ends = gathered ? reinterpret_cast<const int64_t *>(ws + w.ends) : nullptr; z.groups = c->groups; z.rows = c->rows;
    z.n = c->vocab;
    z.splits = 1;
    z.target = !c->targets ? nullptr : gathered ? reinterpret_cast<const int32_t *>(ws + w.target) : c->targets;
    z.target_logit = reinterpret_cast<float *>(ws + w.target_logit);
    z.logit_scale = c->scale;
    z.moments = reinterpret_cast<float4 *>(ws + w.moments);
    z.moment_tiles = (c->vocab + cols - 1) / cols;
    z.quads = c->top ? reinterpret_cast<float *>(ws + w.quads) : nullptr;
    z.ld_quads = w.ld_quads;
    if (int rc = launch_status(launch_logits(q, t, Finish::Moments, tile, z), what)) return rc;

    Scores p{};
    p.taking = taking;
    p.index = gathered ? reinterpret_cast<const uint32_t *>(ws + w.index) : nullptr;
    p.moments = z.moments; p.tiles = z.moment_tiles; p.tile_quads = cols / 4;
    p.target_logit = c->targets ? z.target_logit : nullptr;
    p.logp = c->logp; p.entropy = c->entropy; p.norms = reinterpret_cast<float4 *>(c->norms);
    p.top = c->top; p.top_ids = c->top_ids; p.top_logp = c->top_logp; p.ld_top = c->ld_top;
    p.quads = z.quads; p.ld_quads = z.ld_quads; p.order = quad_order(t, tile);
    p.quad_rank = reinterpret_cast<unsigned long long *>(ws + w.quad_rank); p.row_norm = reinterpret_cast<float2 *>(ws + w.row_norm);
    p.target = z.target;
    p.h = z.a; p.ldh = z.lda; p.e = c->e; p.lde = c->lde; p.e_stride = z.b_group;
    p.dim = c->dim; p.scale = c->scale;
    return launch_status(t == Dtype::F32 ? launch_scores<F32>(q, p) : t == Dtype::BF16 ? launch_scores<Bf16>(q, p) : launch_scores<F16>(q, p), what);
}

int cocod_token_scores_grad(void *stream, const cocod_token_scores_call *c)
{
    if (int rc = check(c)) return rc;
    const Dtype t = kTypes[c->dtype];
    const uint64_t s = dtype_bytes(t);
    const Workspace w = carve(c, true);
    if (int rc = check_inputs(c, w)) return rc;
    if (!c->dh && !c->de) return set_error(COCOD_ERR_INVALID, "dh and de are NULL");
    if (!c->norms && c->rows) return set_error(COCOD_ERR_INVALID, "norms is NULL");
    if (c->d_logp) if (int rc = check_matrix("d_logp", c->d_logp, 1, 1, 4)) return rc;
    if (c->d_entropy) if (int rc = check_matrix("d_entropy", c->d_entropy, 1, 1, 4)) return rc;
    if (c->dh) if (int rc = check_matrix("dh", c->dh, c->dim, c->lddh, s)) return rc;
    if (c->de) {
        if (int rc = check_matrix("de", c->de, c->dim, c->ldde, s)) return rc;
        if (int rc = check_stride("de", c->de_stride, c->groups, c->vocab, c->dim, c->ldde, false)) return rc;
    }
    const Extent all[] = {
        {"workspace", c->workspace, w.bytes}, {"dh", c->dh, matrix_bytes(c->rows, c->dim, c->lddh, s)},
        {"de", c->de, c->de ? stack_bytes(c->groups, c->de_stride, c->vocab, c->dim, c->ldde, s) : 0},
        {"h", c->h, matrix_bytes(c->rows, c->dim, c->ldh, s)}, {"e", c->e, stack_bytes(c->groups, c->e_stride, c->vocab, c->dim, c->lde, s)},
        {"targets", c->targets, c->rows * 4}, {"offsets", c->offsets, (c->groups + 1ull) * 8}, {"norms", c->norms, c->rows * 16},
        {"d_logp", c->d_logp, c->rows * 4}, {"d_entropy", c->d_entropy, c->rows * 4},
    };
    for (int i = 0; i < 3; ++i)
        if (int rc = check_apart(all[i], all + i + 1, 10 - i - 1)) return rc;

    const hipStream_t q = static_cast<hipStream_t>(stream);
    const OnStreamDevice device(q);
    const char *const what = "cocod_token_scores_grad";
    if (device.status() != hipSuccess) return launch_status(device.status(), what);
    uint8_t *ws = static_cast<uint8_t *>(c->workspace);
    const uint32_t widest = static_cast<uint32_t>(w.piece < c->vocab ? w.piece : c->vocab);
    if ((c->rows && !fits(c, Layout::Rows_NK, w.logits, logits_operands(c, w, ws, true), 0, widest, 1)) ||
        (c->rows && c->dh && !fits(c, Layout::Rows_KN, w.to_hidden, hidden_operands(c, w, ws, 0, widest), 0, c->dim, w.to_hidden.splits)) ||
        (c->de && !fits(c, Layout::Weights, w.to_table, table_operands(w, ws), widest, c->dim, w.to_table.splits)))
        return launch_status(hipErrorInvalidConfiguration, what);

    Taking taking{};
    taking.rows = {c->offsets, c->groups, c->rows, c->targets, c->vocab};
    taking.grad = 1;
    taking.d_logp = c->d_logp; taking.d_entropy = c->d_entropy;
    if (int rc = launch_status(t == Dtype::F32 ? launch_gather<F32>(q, taking, c, w, ws) : t == Dtype::BF16 ? launch_gather<Bf16>(q, taking, c, w, ws) : launch_gather<F16>(q, taking, c, w, ws), what)) return rc;
    const uint32_t *index = reinterpret_cast<const uint32_t *>(ws + w.index);
    const int64_t *ends = reinterpret_cast<const int64_t *>(ws + w.ends);
    const float *row_scale = t != Dtype::F32 ? reinterpret_cast<const float *>(ws + w.row_scale) : nullptr;
    for (uint32_t i = 0; i < w.pieces; ++i) {
        const uint64_t v0 = i * w.piece;
        const uint32_t n = static_cast<uint32_t>(c->vocab - v0 < w.piece ? c->vocab - v0 : w.piece);
        auto common = [&](ProductParams &d) { d.offsets = c->offsets; d.ends = ends; d.groups = c->groups; d.rows = c->rows; };
        if (c->rows) {
            ProductParams p = logits_operands(c, w, ws, true);
            common(p);
            p.b = static_cast<const uint8_t *>(c->e) + v0 * c->lde * s;
            p.n = n; p.v0 = static_cast<uint32_t>(v0); p.splits = 1;
            p.target = reinterpret_cast<const int32_t *>(ws + w.target);
            p.top = reinterpret_cast<const float *>(ws + w.top); p.inverse = reinterpret_cast<const float *>(ws + w.none);
            p.slope_one = reinterpret_cast<const float *>(ws + w.one); p.target_slope = reinterpret_cast<const float *>(ws + w.target_slope);
            p.logit_scale = c->scale;
            p.out = ws + w.slope; p.ldc = w.piece; p.ldc_zero = (n + 7) / 8 * 8;
            if (int rc = launch_status(launch_logits(q, t, Finish::Score, settle_tile(t, Layout::Rows_NK, w.logits.tile, p), p), what)) return rc;
        }
        auto product = [&](ProductParams &d, const ProductPlan &plan) {
            common(d);
            d.n = c->dim;
            d.scale = 1.0f;
            d.part = reinterpret_cast<float *>(ws + w.part); d.ld_part = part_pitch(c->dim);
            d.splits = plan.splits;
        };
        if (c->dh && c->rows) {
            ProductParams d = hidden_operands(c, w, ws, v0, n);
            product(d, w.to_hidden);
            d.out = c->dh; d.ldc = c->lddh; d.out_row = index; d.row_scale = row_scale;
            if (c->flags & COCOD_TOKEN_SCORES_RELU_IN) { d.mask = ws + w.hidden; d.ld_mask = w.pitch; }       // (rows of C are gathered ones)
            if (w.pieces > 1) { d.sum = reinterpret_cast<float *>(ws + w.sum); d.ld_sum = w.sum_pitch; d.sum_read = i > 0; d.sum_write = i + 1 < w.pieces; }
            if (int rc = launch_status(launch_store(q, t, Layout::Rows_KN, settle_tile(t, Layout::Rows_KN, w.to_hidden.tile, d), d), what)) return rc;
        }
        if (c->de) {
            ProductParams d = table_operands(w, ws);
            product(d, w.to_table);
            d.m = n;
            d.out = static_cast<uint8_t *>(c->de) + v0 * c->ldde * s; d.ldc = c->ldde; d.out_group = c->de_stride;
            if (t == Dtype::F16) d.group_scale = reinterpret_cast<const float *>(ws + w.group_scale);
            if (int rc = launch_status(launch_store(q, t, Layout::Weights, settle_tile(t, Layout::Weights, w.to_table.tile, d), d), what)) return rc;
        }
    }
    return COCOD_OK;
}

int cocod_debug_token_scores_plan(const cocod_token_scores_call *c, int direction, cocod_product_plan out[3], uint32_t *pieces)
{
    if (!out || !pieces) return set_error(COCOD_ERR_INVALID, "out or pieces is NULL");
    if (int rc = check(c)) return rc;
    if (direction != COCOD_TOKEN_SCORES_FORWARD && direction != COCOD_TOKEN_SCORES_GRAD) return set_error(COCOD_ERR_INVALID, "unknown direction %d", direction);
    const Dtype t = kTypes[c->dtype];
    const bool grad = direction == COCOD_TOKEN_SCORES_GRAD;
    const Workspace w = carve(c, grad);
    const uint8_t *ws = static_cast<const uint8_t *>(c->workspace);
    auto plan = [&](Layout layout, const ProductPlan &planned, const ProductParams &p) {
        return plan_as_run(t, layout, settle_tile(t, layout, planned.tile, p), planned.splits, p);
    };
    const cocod_product_plan none = {0, 0, 0};
    if (!grad) {
        bool gathered;
        const ProductParams z = forward_operands(c, w, ws, gathered);
        out[0] = plan(Layout::Rows_NK, w.logits, z);
        if (z.b_once && out[0].tile == static_cast<uint32_t>(Tile::Small) && out[0].operands == 0) out[0].operands = 3;
        out[1] = out[2] = none;
        *pieces = 1;
        return COCOD_OK;
    }
    out[0] = plan(Layout::Rows_NK, w.logits, logits_operands(c, w, ws, true));
    out[1] = c->dh ? plan(Layout::Rows_KN, w.to_hidden, hidden_operands(c, w, ws, 0, static_cast<uint32_t>(w.piece < c->vocab ? w.piece : c->vocab))) : none;
    out[2] = c->de ? plan(Layout::Weights, w.to_table, table_operands(w, ws)) : none;
    *pieces = w.pieces;
    return COCOD_OK;
}

}  // extern "C"
