// Tokens to the rows of the groups that own them, and back.
//
// A pair (t, j) is token t's j-th choice of a group.  Sorting gives every pair its row: pairs in the order of group, token, choice.
//   place[t][j] = offsets[g] + number of pairs of group g in front of (t, j),  offsets[g] = number of rows of the groups in front of g
//   xs[place[t][j]] = x[t]                              dx[t] = sum_j dxs[place[t][j]]
//   y[t] = sum_j w[t][j] ys[place[t][j]]                dys[place[t][j]] = w[t][j] dy[t],  dw[t][j] = <dy[t], ys[place[t][j]]>
//
// Everything but the sort goes from token to rows, never from row to token: a token's row is read once for all its choices, sums over
// choices stay in registers, in the order of the choices, and no two writes meet, so there are no atomics on results.  Bound by memory.
//
// The sort counts: every wave numbers a run of pairs in order (lanes with the same group find each other by ballots over the bits of the
// group's number), on top of what the runs in front of it hold.
#include "operator_call.hpp"
#include "row_access.hpp"

namespace cocod {
namespace {

constexpr uint32_t kMostChoices = 64;
constexpr uint32_t kRunPairs = 256;                  // pairs of a run at least (16384 x 8 to 128 groups: 12.5 us, with 512 13.7, 1024 19.4)
constexpr uint32_t kMostRuns = 1024;
constexpr uint32_t kCountRange = 8192, kPlaceRange = 4096;       // groups that a block counts / places (32 KiB of LDS each)
constexpr uint32_t kOffsetsHere = 512;               // groups up to which every run sums up the groups in front for itself
// One block does it all up to so many pairs and groups (us, one block / three launches: 2048 pairs to 8 groups 4.4 / 8.1, 8192 8.4 / 9.3, to 512 groups 11.8 / 13.9).
constexpr uint32_t kSmallPairs = 8192, kSmallGroups = 512, kSmallWaves = 16;

struct SortParams {
    const int32_t *experts;
    uint64_t ld_experts;
    int32_t *place;
    uint64_t ld_place;
    int64_t *offsets;
    uint32_t pairs, choices, groups, capacity;       // capacity: ~0 where there is none
    uint32_t per_run, runs;
    uint32_t bits;                                   // of the largest number within a range of groups
    uint32_t *before;                                // [runs][groups]: pairs of the run by group, then those of the runs in front
    uint32_t *taken;                                 // [groups]: rows of the group
};

__device__ __forceinline__ uint64_t at_pair(uint32_t i, uint32_t choices, uint64_t ld)
{
    return ld == choices ? i : static_cast<uint64_t>(i / choices) * ld + i % choices;
}
__device__ __forceinline__ uint32_t group_at(const SortParams &p, uint32_t i) { return static_cast<uint32_t>(p.experts[at_pair(i, p.choices, p.ld_experts)]); }

__device__ __forceinline__ uint32_t wave_scan(uint32_t v, uint32_t lane)        // sum of the lanes up to this one
{
    #pragma unroll
    for (int d = 1; d < 64; d <<= 1) { const uint32_t u = __shfl_up(v, d, 64); if (lane >= static_cast<uint32_t>(d)) v += u; }
    return v;
}

// A wave's pairs begin .. end - 1 in order; rank[g]: pairs of group first + g in front of them.
template <class Offset>
__device__ __forceinline__ void place_run(const SortParams &p, uint32_t begin, uint32_t end, uint32_t first, uint32_t count, uint32_t *rank, const Offset &offset, uint32_t lane)
{
    constexpr int AHEAD = 8;
    for (uint32_t i0 = begin; i0 < end; i0 += 64 * AHEAD) {
        uint32_t group[AHEAD];
        #pragma unroll
        for (int a = 0; a < AHEAD; ++a) { const uint32_t i = i0 + a * 64 + lane; group[a] = i < end ? group_at(p, i) : ~0u; }
        #pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const uint32_t i = i0 + a * 64 + lane, g = group[a] - first;
            if (i0 + a * 64 >= end) break;
            const bool in = i < end && group[a] >= first && g < count;
            unsigned long long same = __ballot(in);
            for (uint32_t b = 0; b < p.bits; ++b) {
                const unsigned long long set = __ballot(in && (g >> b & 1));
                same &= g >> b & 1 ? set : ~set;
            }
            const uint32_t mine = __popcll(same & ((1ull << lane) - 1));
            const uint32_t r = in ? rank[g] + mine : 0;
            __builtin_amdgcn_wave_barrier();
            if (in && mine == 0) rank[g] = r + __popcll(same);
            __builtin_amdgcn_wave_barrier();
            if (in) p.place[at_pair(i, p.choices, p.ld_place)] = r < p.capacity ? static_cast<int32_t>(offset(g) + r) : -1;
            else if (first == 0 && i < end && group[a] >= p.groups) p.place[at_pair(i, p.choices, p.ld_place)] = -1;
        }
    }
}

__global__ __launch_bounds__(64 * kSmallWaves) void sort_small_kernel(const SortParams p)
{
    __shared__ uint32_t rank[kSmallWaves][kSmallGroups];
    __shared__ uint32_t offset[kSmallGroups];
    __shared__ uint32_t part[kSmallWaves];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint32_t begin = wave * p.per_run, end = begin + p.per_run < p.pairs ? begin + p.per_run : p.pairs;
    for (uint32_t g = lane; g < p.groups; g += 64) rank[wave][g] = 0;
    __builtin_amdgcn_wave_barrier();
    for (uint32_t i = begin + lane; i < end; i += 64) { const uint32_t g = group_at(p, i); if (g < p.groups) atomicAdd(&rank[wave][g], 1u); }
    __syncthreads();
    const uint32_t g = threadIdx.x;
    uint32_t taken = 0;
    if (g < p.groups) {
        for (uint32_t w = 0; w < kSmallWaves; ++w) { const uint32_t n = rank[w][g]; rank[w][g] = taken; taken += n; }
        taken = taken < p.capacity ? taken : p.capacity;
    }
    const uint32_t incl = wave_scan(taken, lane);
    if (lane == 63) part[wave] = incl;
    __syncthreads();
    uint32_t in_front = 0;
    for (uint32_t w = 0; w < wave; ++w) in_front += part[w];
    if (g < p.groups) {
        offset[g] = in_front + incl - taken;
        p.offsets[g + 1] = in_front + incl;
        if (g == 0) p.offsets[0] = 0;
    }
    __syncthreads();
    place_run(p, begin, end, 0, p.groups, rank[wave], [&](uint32_t i) { return offset[i]; }, lane);
}

__global__ __launch_bounds__(256) void count_kernel(const SortParams p)
{
    __shared__ uint32_t counts[kCountRange];
    const uint32_t first = blockIdx.y * kCountRange, count = p.groups - first < kCountRange ? p.groups - first : kCountRange;
    const uint32_t begin = blockIdx.x * p.per_run, end = p.pairs - begin < p.per_run ? p.pairs : begin + p.per_run;
    for (uint32_t i = threadIdx.x; i < count; i += 256) counts[i] = 0;
    __syncthreads();
    for (uint32_t i = begin + threadIdx.x; i < end; i += 256) { const uint32_t g = group_at(p, i); if (g >= first && g - first < count) atomicAdd(&counts[g - first], 1u); }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < count; i += 256) p.before[static_cast<uint64_t>(blockIdx.x) * p.groups + first + i] = counts[i];
}

// 32 groups of a block, 32 threads a group, each with a part of the runs: what every run has in front of it, and what the group takes.
__global__ __launch_bounds__(1024) void scan_kernel(const SortParams p)
{
    __shared__ uint32_t part[32][33];
    const uint32_t x = threadIdx.x % 32, y = threadIdx.x / 32, g = blockIdx.x * 32 + x;
    const uint32_t per = (p.runs + 31) / 32, r0 = y * per, r1 = r0 + per < p.runs ? r0 + per : p.runs;
    uint32_t sum = 0;
    if (g < p.groups)
        #pragma unroll 8
        for (uint32_t r = r0; r < r1; ++r) sum += p.before[static_cast<uint64_t>(r) * p.groups + g];
    part[y][x] = sum;
    __syncthreads();
    uint32_t at = 0, all = 0;
    #pragma unroll
    for (uint32_t k = 0; k < 32; ++k) { const uint32_t n = part[k][x]; if (k < y) at += n; all += n; }
    if (g >= p.groups) return;
    if (y == 0) p.taken[g] = all < p.capacity ? all : p.capacity;
    #pragma unroll 8
    for (uint32_t r = r0; r < r1; ++r) {
        uint32_t *n = p.before + static_cast<uint64_t>(r) * p.groups + g;
        const uint32_t own = *n;
        *n = at;
        at += own;
    }
}

// The groups' offsets where there are many of them; a thread sums a run of groups.
__global__ __launch_bounds__(1024) void offsets_kernel(const SortParams p)
{
    __shared__ uint32_t part[16];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, per = (p.groups + 1023) / 1024;
    const uint32_t g0 = threadIdx.x * per, g1 = g0 + per < p.groups ? g0 + per : p.groups;
    uint32_t sum = 0;
    for (uint32_t g = g0; g < g1; ++g) sum += p.taken[g];
    const uint32_t incl = wave_scan(sum, lane);
    if (lane == 63) part[wave] = incl;
    __syncthreads();
    uint32_t at = incl - sum;
    for (uint32_t w = 0; w < wave; ++w) at += part[w];
    if (threadIdx.x == 0) p.offsets[0] = 0;
    for (uint32_t g = g0; g < g1; ++g) { at += p.taken[g]; p.offsets[g + 1] = at; }
}

// One wave a run.  HERE: the offsets of the groups are summed up here (and written down by the first run).
template <bool HERE> __global__ __launch_bounds__(64) void place_kernel(const SortParams p)
{
    extern __shared__ uint32_t lds[];
    const uint32_t lane = threadIdx.x, first = blockIdx.y * kPlaceRange, count = p.groups - first < kPlaceRange ? p.groups - first : kPlaceRange;
    uint32_t *rank = lds, *offset = lds + count;
    const uint32_t begin = blockIdx.x * p.per_run, end = p.pairs - begin < p.per_run ? p.pairs : begin + p.per_run;
    for (uint32_t i = lane; i < count; i += 64) rank[i] = p.before[static_cast<uint64_t>(blockIdx.x) * p.groups + first + i];
    if constexpr (HERE) {
        uint32_t at = 0, taken[kOffsetsHere / 64];
        #pragma unroll
        for (uint32_t k = 0; k < kOffsetsHere / 64; ++k) taken[k] = k * 64 + lane < p.groups ? p.taken[k * 64 + lane] : 0;
        #pragma unroll
        for (uint32_t k = 0; k < kOffsetsHere / 64; ++k) {
            if (k * 64 >= p.groups) break;
            const uint32_t incl = wave_scan(taken[k], lane), g = k * 64 + lane;
            if (g < p.groups) {
                offset[g] = at + incl - taken[k];
                if (blockIdx.x == 0) p.offsets[g + 1] = at + incl;
            }
            at += __shfl(incl, 63, 64);
        }
        if (blockIdx.x == 0 && lane == 0) p.offsets[0] = 0;
    } else {
        for (uint32_t i = lane; i < count; i += 64) offset[i] = static_cast<uint32_t>(p.offsets[first + i]);
    }
    __builtin_amdgcn_wave_barrier();
    place_run(p, begin, end, first, count, rank, [&](uint32_t i) { return offset[i]; }, lane);
}

struct SortPlan { uint32_t per_run, runs; bool small; uint64_t before, taken, bytes; };
SortPlan plan_sort(const cocod_route *r)
{
    SortPlan s{};
    const uint32_t pairs = static_cast<uint32_t>(r->tokens * r->choices);
    s.small = pairs <= kSmallPairs && r->groups <= kSmallGroups;
    if (s.small) {
        s.per_run = ((pairs + kSmallWaves - 1) / kSmallWaves + 63) / 64 * 64;
        s.runs = kSmallWaves;
        return s;
    }
    // at most 2^24 counts in memory
    uint32_t runs = (1u << 24) / r->groups;
    runs = runs < kMostRuns ? runs : kMostRuns;
    const uint64_t per = (static_cast<uint64_t>(pairs) + runs - 1) / runs;
    s.per_run = static_cast<uint32_t>((per < kRunPairs ? kRunPairs : per) + 63) / 64 * 64;
    s.runs = (pairs + s.per_run - 1) / s.per_run;
    s.taken = (static_cast<uint64_t>(s.runs) * r->groups * 4 + 255) / 256 * 256;
    s.bytes = s.taken + r->groups * 4ull;
    return s;
}

hipError_t launch_sort(hipStream_t q, const cocod_route *r, const SortPlan &plan)
{
    SortParams p{};
    p.experts = r->experts; p.ld_experts = r->ld_experts;
    p.place = r->place; p.ld_place = r->ld_place;
    p.offsets = r->offsets;
    p.pairs = static_cast<uint32_t>(r->tokens * r->choices);
    p.choices = r->choices; p.groups = r->groups;
    p.capacity = r->capacity && r->capacity < ~0u ? static_cast<uint32_t>(r->capacity) : ~0u;
    p.per_run = plan.per_run; p.runs = plan.runs;
    const uint32_t range = !plan.small && r->groups > kPlaceRange ? kPlaceRange : r->groups;
    while (p.bits < 32 && (range - 1) >> p.bits) ++p.bits;
    if (plan.small) {
        hipLaunchKernelGGL(sort_small_kernel, dim3(1), dim3(64 * kSmallWaves), 0, q, p);
        return hipGetLastError();
    }
    p.before = static_cast<uint32_t *>(r->workspace);
    p.taken = reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(r->workspace) + plan.taken);
    const bool here = r->groups <= kOffsetsHere;
    if (plan.runs) hipLaunchKernelGGL(count_kernel, dim3(plan.runs, (r->groups + kCountRange - 1) / kCountRange), dim3(256), 0, q, p);
    hipLaunchKernelGGL(scan_kernel, dim3((r->groups + 31) / 32), dim3(1024), 0, q, p);
    if (!here) hipLaunchKernelGGL(offsets_kernel, dim3(1), dim3(1024), 0, q, p);
    const dim3 grid(plan.runs, (r->groups + kPlaceRange - 1) / kPlaceRange);
    if (plan.runs && here) hipLaunchKernelGGL(place_kernel<true>, grid, dim3(64), range * 8, q, p);
    else if (plan.runs)    hipLaunchKernelGGL(place_kernel<false>, grid, dim3(64), range * 8, q, p);
    return hipGetLastError();
}

// ---- rows ------------------------------------------------------------------------------------------------

// `lanes` lanes (a power of two) take a token's row, or a segment of it of U pieces a lane.
struct RowsParams {
    const int32_t *place;
    uint64_t ld_place;
    const float *weights;             // may be null: 1
    uint64_t ld_weights;
    const void *from;                 // dispatch: x;  combine: ys or dxs;  its gradient: ys
    uint64_t ld_from;
    void *to;                         // dispatch: xs;  combine: y or dx;  its gradient: dys
    uint64_t ld_to;
    const void *dy;
    uint64_t lddy;
    float *dweights;
    uint64_t ld_dweights;
    uint64_t tokens;
    uint32_t choices, width, rows;    // rows: of xs, ys
    uint32_t lanes, segments;
};

// Of this thread: lane among those of its token, and the first task; tasks further on lie stride() apart.
struct Task {
    uint32_t lane;
    uint64_t at, step;
    __device__ __forceinline__ explicit Task(uint32_t lanes)
    {
        lane = threadIdx.x & (lanes - 1);
        at = (static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x) / lanes;
        step = static_cast<uint64_t>(gridDim.x) * 256 / lanes;
    }
};
__device__ __forceinline__ uint64_t quotient(uint64_t a, uint32_t b) { return a >> 32 ? a / b : static_cast<uint32_t>(a) / b; }

// Where a piece that begins at column c < width is taken: the last one of a row as far back as it has to be to be whole, so that some columns are taken twice, with the same values
// (rows shorter than a piece are taken element by element).  5768 tokens with 4 rows of 2815 columns each back: 36 us instead of 49.
template <uint32_t N> __device__ __forceinline__ uint32_t whole_piece(uint32_t c, uint32_t width) { return c + N > width && width >= N ? width - N : c; }

template <class T, int U, bool STREAM> __global__ __launch_bounds__(256) void dispatch_kernel(const RowsParams p)
{
    typedef Piece<T> V;
    typedef typename T::elem elem;
    const uint32_t span = p.lanes * V::N;
    for (Task task(p.lanes); task.at < p.tokens * p.segments; task.at += task.step) {
        const uint64_t token = quotient(task.at, p.segments);
        const uint32_t c0 = static_cast<uint32_t>(task.at - token * p.segments) * span * U + task.lane * V::N;
        const elem *x = static_cast<const elem *>(p.from) + token * p.ld_from;
        u4 raw[U];
        #pragma unroll
        for (int u = 0; u < U; ++u) if (c0 + u * span < p.width) { const uint32_t c = whole_piece<V::N>(c0 + u * span, p.width); raw[u] = V::load(x + c, p.width - c); }
        for (uint32_t j = 0; j < p.choices; ++j) {
            const uint32_t row = static_cast<uint32_t>(p.place[token * p.ld_place + j]);
            if (row >= p.rows) continue;
            elem *to = static_cast<elem *>(p.to) + row * p.ld_to;
            #pragma unroll
            for (int u = 0; u < U; ++u) if (c0 + u * span < p.width) { const uint32_t c = whole_piece<V::N>(c0 + u * span, p.width); V::template store<STREAM>(to + c, raw[u], p.width - c); }
        }
    }
}

// Sums over the choices in fp32, in their order, rounded once.
template <class T, int U, bool STREAM> __global__ __launch_bounds__(256) void combine_kernel(const RowsParams p)
{
    typedef Piece<T> V;
    typedef typename T::elem elem;
    constexpr int AHEAD = 2;                                   // choices whose rows are on their way at a time
    const uint32_t span = p.lanes * V::N;
    for (Task task(p.lanes); task.at < p.tokens * p.segments; task.at += task.step) {
        const uint64_t token = quotient(task.at, p.segments);
        const uint32_t c0 = static_cast<uint32_t>(task.at - token * p.segments) * span * U + task.lane * V::N;
        float sum[U][V::N];
        #pragma unroll
        for (int u = 0; u < U; ++u)
            #pragma unroll
            for (uint32_t e = 0; e < V::N; ++e) sum[u][e] = 0.0f;
        for (uint32_t j0 = 0; j0 < p.choices; j0 += AHEAD) {
            u4 raw[AHEAD][U];
            float weight[AHEAD];
            bool has[AHEAD];
            #pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                const uint32_t j = j0 + a, row = j < p.choices ? static_cast<uint32_t>(p.place[token * p.ld_place + j]) : ~0u;
                has[a] = row < p.rows;
                weight[a] = has[a] && p.weights ? p.weights[token * p.ld_weights + j] : 1.0f;
                const elem *from = static_cast<const elem *>(p.from) + row * p.ld_from;
                #pragma unroll
                for (int u = 0; u < U; ++u)
                    if (has[a] && c0 + u * span < p.width) { const uint32_t c = whole_piece<V::N>(c0 + u * span, p.width); raw[a][u] = V::template load<STREAM>(from + c, p.width - c); }
            }
            #pragma unroll
            for (int a = 0; a < AHEAD; ++a)
                if (has[a])
                    #pragma unroll
                    for (int u = 0; u < U; ++u)
                        #pragma unroll
                        for (uint32_t e = 0; e < V::N; ++e) sum[u][e] = fmaf(weight[a], V::value(raw[a][u], e), sum[u][e]);
        }
        elem *y = static_cast<elem *>(p.to) + token * p.ld_to;
        #pragma unroll
        for (int u = 0; u < U; ++u) if (c0 + u * span < p.width) { const uint32_t c = whole_piece<V::N>(c0 + u * span, p.width); V::store(y + c, V::pack(sum[u]), p.width - c); }
    }
}

// The lanes of a task take one pair; pairs of a token run beside each other, so that its dy comes from the caches but once.
template <class T, int U, bool STREAM> __global__ __launch_bounds__(256) void combine_grad_kernel(const RowsParams p)
{
    typedef Piece<T> V;
    typedef typename T::elem elem;
    const uint32_t span = p.lanes * V::N;
    const uint64_t pairs = p.tokens * p.choices;
    for (Task task(p.lanes); task.at < pairs; task.at += task.step) {
        const uint64_t token = quotient(task.at, p.choices);
        const uint32_t j = static_cast<uint32_t>(task.at - token * p.choices);
        const uint32_t row = static_cast<uint32_t>(p.place[token * p.ld_place + j]);
        float dot = 0.0f;
        if (row < p.rows) {
            const float weight = p.weights ? p.weights[token * p.ld_weights + j] : 1.0f;
            const elem *dy = static_cast<const elem *>(p.dy) + token * p.lddy, *ys = static_cast<const elem *>(p.from) + row * p.ld_from;
            elem *dys = static_cast<elem *>(p.to) + row * p.ld_to;
            for (uint32_t c0 = task.lane * V::N; c0 < p.width; c0 += span * U) {
                u4 g[U], v[U];
                #pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (c0 + u * span >= p.width) continue;
                    const uint32_t c = whole_piece<V::N>(c0 + u * span, p.width);
                    g[u] = V::load(dy + c, p.width - c);
                    if (p.dweights) v[u] = V::template load<STREAM>(ys + c, p.width - c);
                }
                #pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (c0 + u * span >= p.width) continue;
                    const uint32_t c = whole_piece<V::N>(c0 + u * span, p.width), again = c0 + u * span - c;       // columns that another lane has as well
                    float out[V::N];
                    #pragma unroll
                    for (uint32_t e = 0; e < V::N; ++e) {
                        const float d = V::value(g[u], e);
                        out[e] = weight * d;
                        if (p.dweights && e >= again) dot = fmaf(d, V::value(v[u], e), dot);
                    }
                    if (p.to) V::template store<STREAM>(dys + c, V::pack(out), p.width - c);
                }
            }
        }
        if (!p.dweights) continue;
        for (uint32_t d = 1; d < p.lanes; d <<= 1) dot += __shfl_xor(dot, d, 64);
        if (task.lane == 0) p.dweights[token * p.ld_dweights + j] = dot;
    }
}

enum class RowsCall { Dispatch, Combine, CombineGrad };

template <class T, int U, bool STREAM> void launch_rows(hipStream_t q, RowsCall call, uint32_t grid, const RowsParams &p)
{
    if (call == RowsCall::Dispatch)     hipLaunchKernelGGL((dispatch_kernel<T, U, STREAM>), dim3(grid), dim3(256), 0, q, p);
    else if (call == RowsCall::Combine) hipLaunchKernelGGL((combine_kernel<T, U, STREAM>), dim3(grid), dim3(256), 0, q, p);
    else                                hipLaunchKernelGGL((combine_grad_kernel<T, U, STREAM>), dim3(grid), dim3(256), 0, q, p);
}
template <class T, bool STREAM> void launch_rows(hipStream_t q, RowsCall call, uint32_t u, uint32_t grid, const RowsParams &p)
{
    if (u == 1)      launch_rows<T, 1, STREAM>(q, call, grid, p);
    else if (u == 2) launch_rows<T, 2, STREAM>(q, call, grid, p);
    else             launch_rows<T, 4, STREAM>(q, call, grid, p);
}

template <class T> hipError_t launch_rows(hipStream_t q, RowsCall call, RowsParams p)
{
    constexpr uint32_t N = Piece<T>::N;
    constexpr uint64_t kMostBlocks = 1u << 22, kFewWaves = 1024;
    const uint32_t pieces = (p.width + N - 1) / N;
    p.lanes = 64;
    while (p.lanes > 1 && p.lanes / 2 >= pieces) p.lanes /= 2;
    // pieces a lane: as many as the row has, up to four; one where that leaves the chip too few waves
    uint32_t u = pieces <= p.lanes ? 1 : pieces <= 2 * p.lanes ? 2 : 4;
    if (call != RowsCall::CombineGrad && p.tokens * ((pieces + u * p.lanes - 1) / (u * p.lanes)) < kFewWaves) u = 1;
    p.segments = (pieces + u * p.lanes - 1) / (u * p.lanes);
    const uint64_t tasks = call == RowsCall::CombineGrad ? p.tokens * p.choices : p.tokens * p.segments;
    const uint64_t blocks = (tasks * p.lanes + 255) / 256;
    const uint32_t grid = static_cast<uint32_t>(blocks < kMostBlocks ? blocks : kMostBlocks);
    // the groups' rows past the caches (16384 tokens to 8 of 128 groups, 2048 columns in bf16: out 122 -> 110 us, the weighted way back's gradient 203 -> 186)
    const bool past = p.tokens * p.choices * p.width * sizeof(typename T::elem) * (call == RowsCall::CombineGrad ? 2 : 1) > kLastLevelCache;
    if (past) launch_rows<T, true>(q, call, u, grid, p);
    else      launch_rows<T, false>(q, call, u, grid, p);
    return hipGetLastError();
}

int check_shape(const cocod_route *r, bool rows = true)
{
    if (!r) return set_error(COCOD_ERR_INVALID, "the description is NULL");
    if (r->struct_size != sizeof(cocod_route)) return set_error(COCOD_ERR_INVALID, "struct_size %u does not match this library (%zu)", r->struct_size, sizeof(cocod_route));
    if (int rc = check_dtype(r->dtype)) return rc;
    if (r->flags) return set_error(COCOD_ERR_INVALID, "unknown flag bits 0x%x", r->flags);
    if (r->groups < 1 || r->groups > kMaxGroups) return set_error(COCOD_ERR_INVALID, "groups must be in 1..65535");
    if (r->choices < 1 || r->choices > kMostChoices) return set_error(COCOD_ERR_INVALID, "choices must be in 1..64");
    if (r->tokens > kMaxRows / r->choices) return set_error(COCOD_ERR_INVALID, "tokens * choices must be below 2^31");
    if (rows && (r->width < 1 || r->width > kMaxWidth)) return set_error(COCOD_ERR_INVALID, "width must be in 1..2^30");
    return COCOD_OK;
}

// What the four calls that move rows have in common: `from` is read, `to` (and dweights) written.
struct Matrix { const char *name; const void *ptr; uint64_t rows, cols, ld, size; };
int check_rows(const Matrix *all, int outputs, int n)
{
    Extent extents[8];
    for (int i = 0; i < n; ++i) {
        const Matrix &m = all[i];
        if (int rc = check_matrix(m.name, m.ptr, m.cols, m.ld, m.size, m.rows)) return rc;
        extents[i] = {m.name, m.ptr, matrix_bytes(m.rows, m.cols, m.ld, m.size)};
    }
    for (int i = 0; i < outputs; ++i)
        if (int rc = check_apart(extents[i], extents + i + 1, n - i - 1)) return rc;
    return COCOD_OK;
}

int run_rows(void *stream, const cocod_route *r, RowsCall call, RowsParams &p, const char *what)
{
    if (r->tokens == 0) return COCOD_OK;
    p.place = r->place; p.ld_place = r->ld_place;
    p.tokens = r->tokens;
    p.choices = r->choices; p.width = r->width;
    p.rows = static_cast<uint32_t>(r->tokens * r->choices);
    const hipStream_t q = static_cast<hipStream_t>(stream);
    const OnStreamDevice device(q);
    if (device.status() != hipSuccess) return launch_status(device.status(), what);
    const Dtype t = static_cast<Dtype>(r->dtype);
    return launch_status(t == Dtype::F32 ? launch_rows<F32>(q, call, p) : t == Dtype::BF16 ? launch_rows<Bf16>(q, call, p) : launch_rows<F16>(q, call, p), what);
}

}  // namespace
}  // namespace cocod

using namespace cocod;

extern "C" {

int cocod_route_workspace(const cocod_route *r, uint64_t *bytes)
{
    if (!bytes) return set_error(COCOD_ERR_INVALID, "bytes is NULL");
    if (int rc = check_shape(r, false)) return rc;
    *bytes = plan_sort(r).bytes;
    return COCOD_OK;
}

int cocod_route_sort(void *stream, const cocod_route *r)
{
    if (int rc = check_shape(r, false)) return rc;
    if (!r->offsets || (reinterpret_cast<uintptr_t>(r->offsets) & 7)) return set_error(COCOD_ERR_INVALID, "offsets is NULL or not 8-byte aligned");
    const SortPlan plan = plan_sort(r);
    const Matrix all[] = {{"place", r->place, r->tokens, r->choices, r->ld_place, 4}, {"experts", r->experts, r->tokens, r->choices, r->ld_experts, 4}};
    if (int rc = check_rows(all, 1, 2)) return rc;
    if (plan.bytes && (!r->workspace || (reinterpret_cast<uintptr_t>(r->workspace) & 15))) return set_error(COCOD_ERR_INVALID, "workspace is NULL or not 16-byte aligned");
    if (r->workspace_bytes < plan.bytes && plan.bytes)
        return set_error(COCOD_ERR_INVALID, "workspace holds %llu bytes, %llu are needed", (unsigned long long)r->workspace_bytes, (unsigned long long)plan.bytes);
    const Extent extents[] = {{"offsets", r->offsets, (r->groups + 1ull) * 8}, {"workspace", r->workspace, plan.bytes},
                              {"place", r->place, matrix_bytes(r->tokens, r->choices, r->ld_place, 4)},
                              {"experts", r->experts, matrix_bytes(r->tokens, r->choices, r->ld_experts, 4)}};
    for (int i = 0; i < 2; ++i)
        if (int rc = check_apart(extents[i], extents + i + 1, 3 - i)) return rc;
    const hipStream_t q = static_cast<hipStream_t>(stream);
    const OnStreamDevice device(q);
    if (device.status() != hipSuccess) return launch_status(device.status(), "cocod_route_sort");
    return launch_status(launch_sort(q, r, plan), "cocod_route_sort");
}

int cocod_route_dispatch(void *stream, const cocod_route *r)
{
    if (int rc = check_shape(r)) return rc;
    const uint64_t s = dtype_bytes(static_cast<Dtype>(r->dtype)), pairs = r->tokens * r->choices;
    const Matrix all[] = {{"xs", r->xs, pairs, r->width, r->ldxs, s}, {"x", r->x, r->tokens, r->width, r->ldx, s}, {"place", r->place, r->tokens, r->choices, r->ld_place, 4}};
    if (int rc = check_rows(all, 1, 3)) return rc;
    RowsParams p{};
    p.from = r->x; p.ld_from = r->ldx; p.to = r->xs; p.ld_to = r->ldxs;
    return run_rows(stream, r, RowsCall::Dispatch, p, "cocod_route_dispatch");
}

int cocod_route_dispatch_grad(void *stream, const cocod_route *r)
{
    if (int rc = check_shape(r)) return rc;
    const uint64_t s = dtype_bytes(static_cast<Dtype>(r->dtype)), pairs = r->tokens * r->choices;
    const Matrix all[] = {{"dx", r->dx, r->tokens, r->width, r->lddx, s}, {"dxs", r->dxs, pairs, r->width, r->lddxs, s}, {"place", r->place, r->tokens, r->choices, r->ld_place, 4}};
    if (int rc = check_rows(all, 1, 3)) return rc;
    RowsParams p{};
    p.from = r->dxs; p.ld_from = r->lddxs; p.to = r->dx; p.ld_to = r->lddx;
    return run_rows(stream, r, RowsCall::Combine, p, "cocod_route_dispatch_grad");
}

int cocod_route_combine(void *stream, const cocod_route *r)
{
    if (int rc = check_shape(r)) return rc;
    const uint64_t s = dtype_bytes(static_cast<Dtype>(r->dtype)), pairs = r->tokens * r->choices;
    const Matrix all[] = {{"y", r->y, r->tokens, r->width, r->ldy, s}, {"ys", r->ys, pairs, r->width, r->ldys, s}, {"place", r->place, r->tokens, r->choices, r->ld_place, 4},
                          {"weights", r->weights, r->tokens, r->choices, r->ld_weights, 4}};
    if (int rc = check_rows(all, 1, r->weights ? 4 : 3)) return rc;
    RowsParams p{};
    p.from = r->ys; p.ld_from = r->ldys; p.to = r->y; p.ld_to = r->ldy;
    p.weights = r->weights; p.ld_weights = r->ld_weights;
    return run_rows(stream, r, RowsCall::Combine, p, "cocod_route_combine");
}

int cocod_route_combine_grad(void *stream, const cocod_route *r)
{
    if (int rc = check_shape(r)) return rc;
    const uint64_t s = dtype_bytes(static_cast<Dtype>(r->dtype)), pairs = r->tokens * r->choices;
    if (!r->dys && !r->dweights && r->tokens) return set_error(COCOD_ERR_INVALID, "dys and dweights are NULL");
    Matrix all[6];
    int n = 0;
    if (r->dys) all[n++] = {"dys", r->dys, pairs, r->width, r->lddys, s};
    if (r->dweights) all[n++] = {"dweights", r->dweights, r->tokens, r->choices, r->ld_dweights, 4};
    const int outputs = n;
    all[n++] = {"dy", r->dy, r->tokens, r->width, r->lddy, s};
    all[n++] = {"place", r->place, r->tokens, r->choices, r->ld_place, 4};
    if (r->dweights) all[n++] = {"ys", r->ys, pairs, r->width, r->ldys, s};
    if (r->weights) all[n++] = {"weights", r->weights, r->tokens, r->choices, r->ld_weights, 4};
    if (int rc = check_rows(all, outputs, n)) return rc;
    RowsParams p{};
    p.from = r->ys; p.ld_from = r->ldys; p.to = r->dys; p.ld_to = r->lddys;
    p.dy = r->dy; p.lddy = r->lddy;
    p.weights = r->weights; p.ld_weights = r->ld_weights;
    p.dweights = r->dweights; p.ld_dweights = r->ld_dweights;
    return run_rows(stream, r, RowsCall::CombineGrad, p, "cocod_route_combine_grad");
}

}  // extern "C"
