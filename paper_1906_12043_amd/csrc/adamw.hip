// One AdamW step over the tensors of a model, for all workers, in one pass over memory.
//
//   g' = grad_scale g,  m' = b1 m + (1 - b1) g',  v' = b2 v + ((1 - b2) g') g'   (fp32, rounded after every product and sum)
//   p' = p (1 - lr wd) - (lr / c1) m' / (sqrt(v' / c2) + eps),  c = 1 - b^step
//
// States of 8 bits: 32 consecutive elements of a tensor share a scale 2^e, m is held as an e4m3 code of m / 2^e, v as the code of sqrt(v) / 2^e
// (the format of the 8-bit activations), whose range of 2^18 within a block would be 2^9 of v's roots if it held v.  A step changes v by a
// thousandth of itself, a code's step is a sixteenth to an eighth: rounded to the nearest, v would stand still.  So a code is rounded up or down by chance,
// with 16 random bits each, so that the stored m, and the SQUARE of the stored root of v, are m' and v' in the mean (to 2^-16 of a step).  The random bits are
// a function of (seed, tensor, worker, element): a multiply-and-shift mixer of 32 bits, three multiplications an element, where a
// ten-round counter generator would cost more time than the memory leaves.  p' comes from m' and v' before they are rounded.
//
// Bound by memory: fp32 with 16-bit gradients and copies 28 bytes an element, with 8-bit states 16.1.  A thread takes eight elements, four threads a
// scale.  Tensors travel in the kernel's arguments, a launch for every kMostTensors of them, so nothing has to be laid out on the device and a captured
// launch holds all it needs.
#include "operator_call.hpp"
#include "row_access.hpp"

#include <cmath>

namespace cocod {
namespace {

constexpr uint32_t kStateBlock = 32;                 // elements that share a scale
constexpr int kThreads = 256;
constexpr uint32_t kEach = 8;                        // elements of a thread
constexpr uint32_t kTile = kThreads * kEach;         // of a block
constexpr uint32_t kMostTensors = 40;                // of a launch: its arguments stay below 4 KiB
constexpr uint32_t kMostBlocks = 1u << 20;
constexpr uint64_t kMostElements = 1ull << 40;       // of a tensor

struct Tensor {
    void *p;
    const void *g;
    void *m, *v;
    uint8_t *m_scales, *v_scales;
    void *copy;
    uint64_t n;
    float weight_decay, lr_scale;
};
struct AdamWParams {
    Tensor tensor[kMostTensors];
    uint32_t first_tile[kMostTensors + 1];           // of every tensor, in tiles of a worker
    uint32_t count, number;                          // tensors of this launch; number of the first one in the call
    uint64_t tiles;                                  // of all workers
    uint32_t workers, copy_dtype;
    uint64_t stride;
    float beta1, beta2, rest1, rest2, eps;
    cocod_adamw_now now;
    const cocod_adamw_now *now_device;
};
static_assert(sizeof(AdamWParams) <= 4096, "arguments of a kernel");

__device__ __forceinline__ float power(int e) { return __uint_as_float(static_cast<unsigned>(e + 127) << 23); }      // 2^e, e in -126 .. 127
__device__ __forceinline__ float larger_of_block(float v)      // over the four threads of a block of 32
{
    v = fmaxf(v, __shfl_xor(v, 1, 64));
    return fmaxf(v, __shfl_xor(v, 2, 64));
}
// Smallest e, not below low, for which the block's largest finite magnitude is at most 448 2^e.
__device__ __forceinline__ int block_scale(float most, int low)
{
    if (!(most > 0.0f)) return low;
    const int exp = __builtin_amdgcn_frexp_expf(most);
    const int e = exp - (__builtin_amdgcn_frexp_mantf(most) <= 0.875f ? 9 : 8);
    return e > low ? e : low;
}

// y >= 0 in units of the smallest code.  The code not above y, what it stands for and the step to the next one.
struct Below { uint32_t code; float low, step; };
__device__ __forceinline__ Below code_below(float y)
{
    const uint32_t bits = __float_as_uint(y);
    Below b;
    if (y < 8.0f) {
        b.code = static_cast<uint32_t>(y);
        b.low = static_cast<float>(b.code);
        b.step = 1.0f;
    } else {
        b.code = (bits >> 20) - (130u << 3) + 8;
        b.low = __uint_as_float(bits & 0xfff00000u);
        b.step = __uint_as_float((bits & 0x7f800000u) - (3u << 23));
    }
    return b;
}
// What a code stands for, times `unit` (the smallest code's value).
__device__ __forceinline__ float value_of(uint32_t code, float unit)
{
    const uint32_t mag = code & 0x7f;
    if (mag == 0x7f) return __uint_as_float(0x7fc00000u);
    const float v = mag < 8 ? static_cast<float>(mag) : __uint_as_float((mag - 8 + (130u << 3)) << 20);
    return (code & 0x80 ? -v : v) * unit;
}
__device__ __forceinline__ float unit_of(uint8_t scale)        // 2^(scale - 127 - 9), split where it leaves the normal range
{
    const int e = static_cast<int>(scale) - 136;
    return power(e / 2) * power(e - e / 2);
}

__device__ __forceinline__ uint32_t random_bits(uint64_t at, uint32_t stream)
{
    uint32_t x = static_cast<uint32_t>(at) * 0x9E3779B1u + static_cast<uint32_t>(at >> 32) * 0x85EBCA6Bu + stream;
    x = (x ^ (x >> 16)) * 0x7FEB352Du;
    x = (x ^ (x >> 15)) * 0x846CA68Bu;
    return x ^ (x >> 16);
}

// Eight consecutive elements in fp32, and back; count < 8 at a tensor's end.
template <class T> __device__ __forceinline__ void load_eight(const void *base, uint64_t at, uint32_t count, float (&v)[kEach])
{
    typedef Piece<T> V;
    const typename T::elem *from = static_cast<const typename T::elem *>(base) + at;
    #pragma unroll
    for (uint32_t h = 0; h < kEach; h += V::N) {
        const u4 raw = count > h ? V::load(from + h, count - h) : u4{0, 0, 0, 0};
        #pragma unroll
        for (uint32_t j = 0; j < V::N; ++j) v[h + j] = V::value(raw, j);
    }
}
template <class T> __device__ __forceinline__ void store_eight(void *base, uint64_t at, uint32_t count, const float (&v)[kEach])
{
    typedef Piece<T> V;
    typename T::elem *to = static_cast<typename T::elem *>(base) + at;
    #pragma unroll
    for (uint32_t h = 0; h < kEach; h += V::N) {
        float part[V::N];
        #pragma unroll
        for (uint32_t j = 0; j < V::N; ++j) part[j] = v[h + j];
        if (count > h) V::store(to + h, V::pack(part), count - h);
    }
}
__device__ __forceinline__ u2 load_codes(const void *base, uint64_t at, uint32_t count)
{
    const uint8_t *from = static_cast<const uint8_t *>(base) + at;
    if (count >= kEach) return *reinterpret_cast<const u2_any *>(from);
    u2 w = {0, 0};
    #pragma unroll
    for (uint32_t j = 0; j < kEach; ++j) if (j < count) w[j / 4] |= static_cast<unsigned>(from[j]) << (8 * (j % 4));
    return w;
}
__device__ __forceinline__ void store_codes(void *base, uint64_t at, uint32_t count, u2 w)
{
    uint8_t *to = static_cast<uint8_t *>(base) + at;
    if (count >= kEach) { *reinterpret_cast<u2_any *>(to) = w; return; }
    #pragma unroll
    for (uint32_t j = 0; j < kEach; ++j) if (j < count) to[j] = static_cast<uint8_t>(w[j / 4] >> (8 * (j % 4)));
}

template <class TP, class TG, bool EIGHT> __global__ __launch_bounds__(kThreads) void adamw_kernel(const AdamWParams s)
{
    #pragma clang fp contract(off)
    const cocod_adamw_now now = s.now_device ? *s.now_device : s.now;
    if (now.skip) return;
    const float root_bias2 = 1.0f / sqrtf(now.bias2);
    for (uint64_t tile = blockIdx.x; tile < s.tiles; tile += gridDim.x) {
        const uint32_t per_worker = s.first_tile[s.count];
        const uint32_t worker = static_cast<uint32_t>(tile / per_worker), in = static_cast<uint32_t>(tile - static_cast<uint64_t>(worker) * per_worker);
        uint32_t lo = 0, hi = s.count;                         // first_tile[lo] <= in < first_tile[hi]
        while (hi - lo > 1) { const uint32_t mid = (lo + hi) / 2; if (s.first_tile[mid] <= in) lo = mid; else hi = mid; }
        const Tensor &t = s.tensor[lo];
        const uint64_t at = static_cast<uint64_t>(in - s.first_tile[lo]) * kTile + threadIdx.x * kEach;       // of the tensor
        const uint64_t base = worker * s.stride + at;
        const uint32_t count = at >= t.n ? 0 : t.n - at < kEach ? static_cast<uint32_t>(t.n - at) : kEach;
        const float lr = now.lr * t.lr_scale, keep = 1.0f - lr * t.weight_decay, step = lr / now.bias1;

        float p[kEach], g[kEach], m[kEach], v[kEach];
        load_eight<TP>(t.p, base, count, p);
        load_eight<TG>(t.g, base, count, g);
        uint64_t scale_at = 0;
        if constexpr (EIGHT) {
            const u2 cm = load_codes(t.m, base, count), cv = load_codes(t.v, base, count);
            scale_at = worker * (s.stride / kStateBlock) + at / kStateBlock;
            const float um = count ? unit_of(t.m_scales[scale_at]) : 0.0f, uv = count ? unit_of(t.v_scales[scale_at]) : 0.0f;
            #pragma unroll
            for (uint32_t j = 0; j < kEach; ++j) {
                m[j] = value_of(cm[j / 4] >> (8 * (j % 4)), um);
                const float root = value_of(cv[j / 4] >> (8 * (j % 4)), uv);
                v[j] = root * root;
            }
        } else {
            load_eight<F32>(t.m, base, count, m);
            load_eight<F32>(t.v, base, count, v);
        }
        #pragma unroll
        for (uint32_t j = 0; j < kEach; ++j) {
            const float d = g[j] * now.grad_scale;
            m[j] = m[j] * s.beta1 + d * s.rest1;
            v[j] = v[j] * s.beta2 + (d * s.rest2) * d;
            g[j] = sqrtf(v[j]);
            p[j] = p[j] * keep - step * (m[j] * __builtin_amdgcn_rcpf(g[j] * root_bias2 + s.eps));
        }
        store_eight<TP>(t.p, base, count, p);
        if constexpr (sizeof(typename TP::elem) == 4) {
            if (t.copy && s.copy_dtype == COCOD_BF16) store_eight<Bf16>(t.copy, base, count, p);
            else if (t.copy)                          store_eight<F16>(t.copy, base, count, p);
        }
        if constexpr (!EIGHT) {
            store_eight<F32>(t.m, base, count, m);
            store_eight<F32>(t.v, base, count, v);
        } else {
            float most_m = 0.0f, most_r = 0.0f;
            #pragma unroll
            for (uint32_t j = 0; j < kEach; ++j) {
                if (j >= count) { m[j] = 0.0f; v[j] = 0.0f; g[j] = 0.0f; }
                if (__builtin_isfinite(m[j])) most_m = fmaxf(most_m, fabsf(m[j]));
                if (__builtin_isfinite(g[j])) most_r = fmaxf(most_r, g[j]);
            }
            const int em = block_scale(larger_of_block(most_m), -117), er = block_scale(larger_of_block(most_r), -51);
            const float um1 = power((9 - em) / 2), um2 = power((9 - em) - (9 - em) / 2), ur = power(9 - er);
            const uint32_t stream = now.seed + (s.number + lo) * 0x632BE5ABu + worker * 0x85157AF5u;
            u2 cm = {0, 0}, cv = {0, 0};
            #pragma unroll
            for (uint32_t j = 0; j < kEach; ++j) {
                const uint32_t bits = random_bits(at + j, stream);
                const bool fine_m = __builtin_isfinite(m[j]), fine_r = __builtin_isfinite(g[j]);
                const float y = fine_m ? fabsf(m[j]) * um1 * um2 : 0.0f;
                const Below a = code_below(y);
                uint32_t code = a.code + (y - a.low > static_cast<float>(bits >> 16) * 0x1p-16f * a.step ? 1u : 0u);
                code = (fine_m ? code : 0x7fu) | (__float_as_uint(m[j]) >> 31 << 7);
                cm[j / 4] |= code << (8 * (j % 4));
                const float r = fine_r ? g[j] * ur : 0.0f, w = fine_r ? v[j] * ur * ur : 0.0f;
                const Below b = code_below(r);
                code = b.code + (w - b.low * b.low > static_cast<float>(bits & 0xffffu) * 0x1p-16f * (b.step * (2.0f * b.low + b.step)) ? 1u : 0u);
                if (code == 0 && g[j] > 0.0f) code = 1;
                cv[j / 4] |= (fine_r ? code : 0x7fu) << (8 * (j % 4));
            }
            store_codes(t.m, base, count, cm);
            store_codes(t.v, base, count, cv);
            if (count && threadIdx.x % 4 == 0) {
                t.m_scales[scale_at] = static_cast<uint8_t>(em + 127);
                t.v_scales[scale_at] = static_cast<uint8_t>(er + 127);
            }
        }
    }
}

template <class TP, class TG> void launch(hipStream_t q, bool eight, uint32_t grid, const AdamWParams &s)
{
    if (eight) hipLaunchKernelGGL((adamw_kernel<TP, TG, true>), dim3(grid), dim3(kThreads), 0, q, s);
    else       hipLaunchKernelGGL((adamw_kernel<TP, TG, false>), dim3(grid), dim3(kThreads), 0, q, s);
}
template <class TP> void launch(hipStream_t q, uint32_t grad, bool eight, uint32_t grid, const AdamWParams &s)
{
    if (grad == COCOD_F32)       launch<TP, F32>(q, eight, grid, s);
    else if (grad == COCOD_BF16) launch<TP, Bf16>(q, eight, grid, s);
    else                         launch<TP, F16>(q, eight, grid, s);
}

bool finite_in(float v, float low, float high) { return std::isfinite(v) && v >= low && v < high; }

int check_call(const cocod_adamw_call *c)
{
    if (!c) return set_error(COCOD_ERR_INVALID, "the description is NULL");
    if (c->struct_size != sizeof(cocod_adamw_call)) return set_error(COCOD_ERR_INVALID, "struct_size %u does not match this library (%zu)", c->struct_size, sizeof(cocod_adamw_call));
    if (int rc = check_dtype(c->dtype)) return rc;
    if (int rc = check_dtype(c->grad_dtype)) return rc;
    if (int rc = check_dtype(c->copy_dtype)) return rc;
    if (c->state != COCOD_ADAMW_STATE_F32 && c->state != COCOD_ADAMW_STATE_8BIT) return set_error(COCOD_ERR_INVALID, "unknown state %u", c->state);
    if (c->flags) return set_error(COCOD_ERR_INVALID, "unknown flag bits 0x%x", c->flags);
    if (c->workers < 1 || c->workers > kMaxGroups) return set_error(COCOD_ERR_INVALID, "workers must be in 1..65535");
    if (c->workers > 1 && c->stride > kMaxGroupStride) return set_error(COCOD_ERR_INVALID, "more than 2^44 elements between workers");
    if (c->workers > 1 && c->state == COCOD_ADAMW_STATE_8BIT && c->stride % kStateBlock) return set_error(COCOD_ERR_INVALID, "stride must be a multiple of 32 where states have 8 bits");
    if (!c->tensors && c->count) return set_error(COCOD_ERR_INVALID, "tensors is NULL");
    if (c->count > (1u << 20)) return set_error(COCOD_ERR_INVALID, "at most 2^20 tensors");
    if (!finite_in(c->beta1, 0.0f, 1.0f) || !finite_in(c->beta2, 0.0f, 1.0f)) return set_error(COCOD_ERR_INVALID, "beta1 and beta2 must be in 0 .. 1, 1 excluded");
    if (!finite_in(c->eps, 0.0f, INFINITY)) return set_error(COCOD_ERR_INVALID, "eps must be finite and not negative");
    if (c->now && (reinterpret_cast<uintptr_t>(c->now) & 3)) return set_error(COCOD_ERR_INVALID, "now is not 4-byte aligned");
    if (!c->now) {
        if (!std::isfinite(c->lr)) return set_error(COCOD_ERR_INVALID, "lr is not finite");
        if (!std::isfinite(c->grad_scale)) return set_error(COCOD_ERR_INVALID, "grad_scale is not finite");
        if (c->step < 1) return set_error(COCOD_ERR_INVALID, "step counts from 1");
    }
    return COCOD_OK;
}

// An array of every worker, `size` bytes an element.
int check_array(uint64_t i, const char *name, const void *ptr, uint64_t size)
{
    if (!ptr) return set_error(COCOD_ERR_INVALID, "tensor %llu: %s is NULL", (unsigned long long)i, name);
    if (reinterpret_cast<uintptr_t>(ptr) % size) return set_error(COCOD_ERR_INVALID, "tensor %llu: %s is not aligned to its elements", (unsigned long long)i, name);
    return COCOD_OK;
}

int check_tensor(const cocod_adamw_call *c, uint64_t i)
{
    const cocod_adamw_tensor &t = c->tensors[i];
    const unsigned long long number = i;
    if (t.n == 0) return COCOD_OK;
    if (t.n > kMostElements) return set_error(COCOD_ERR_INVALID, "tensor %llu: more than 2^40 elements", number);
    if (c->workers > 1 && c->stride < t.n) return set_error(COCOD_ERR_INVALID, "tensor %llu: %llu elements between workers, the tensors overlap", number, (unsigned long long)c->stride);
    if (!std::isfinite(t.weight_decay) || !std::isfinite(t.lr_scale)) return set_error(COCOD_ERR_INVALID, "tensor %llu: weight_decay or lr_scale is not finite", number);
    const uint64_t sp = dtype_bytes(static_cast<Dtype>(c->dtype)), sg = dtype_bytes(static_cast<Dtype>(c->grad_dtype)), sc = dtype_bytes(static_cast<Dtype>(c->copy_dtype));
    const bool eight = c->state == COCOD_ADAMW_STATE_8BIT;
    const uint64_t ss = eight ? 1 : 4, blocks = (t.n + kStateBlock - 1) / kStateBlock;
    if (int rc = check_array(i, "p", t.p, sp)) return rc;
    if (int rc = check_array(i, "g", t.g, sg)) return rc;
    if (int rc = check_array(i, "m", t.m, ss)) return rc;
    if (int rc = check_array(i, "v", t.v, ss)) return rc;
    if (eight) {
        if (int rc = check_array(i, "m_scales", t.m_scales, 1)) return rc;
        if (int rc = check_array(i, "v_scales", t.v_scales, 1)) return rc;
    }
    if (t.copy) {
        if (c->dtype != COCOD_F32 || c->copy_dtype == COCOD_F32) return set_error(COCOD_ERR_INVALID, "tensor %llu: a copy in 16 bits goes with parameters in 32", number);
        if (int rc = check_array(i, "copy", t.copy, sc)) return rc;
    }
    // A worker's arrays lie apart (those of several workers may be interleaved, [workers][stride], so whole extents say nothing).
    const Extent all[] = {{"p", t.p, t.n * sp}, {"m", t.m, t.n * ss}, {"v", t.v, t.n * ss}, {"copy", t.copy, t.copy ? t.n * sc : 0},
                          {"m_scales", t.m_scales, eight ? blocks : 0}, {"v_scales", t.v_scales, eight ? blocks : 0}, {"g", t.g, t.n * sg},
                          {"now", c->now, c->now ? sizeof(cocod_adamw_now) : 0}};
    for (int k = 0; k < 6; ++k)
        if (int rc = check_apart(all[k], all + k + 1, 8 - k - 1)) return rc;
    return COCOD_OK;
}

// 1 - beta^step
float bias(float beta, uint64_t step) { return beta > 0.0f ? static_cast<float>(-std::expm1(static_cast<double>(step) * std::log(static_cast<double>(beta)))) : 1.0f; }

}  // namespace
}  // namespace cocod

using namespace cocod;

extern "C" {

int cocod_adamw_now_of(const cocod_adamw_call *c, cocod_adamw_now *now)
{
    if (!now) return set_error(COCOD_ERR_INVALID, "now is NULL");
    if (!c) return set_error(COCOD_ERR_INVALID, "the description is NULL");
    cocod_adamw_call host = *c;
    host.now = nullptr;
    host.count = 0;
    if (int rc = check_call(&host)) return rc;
    *now = {c->lr, c->grad_scale, bias(c->beta1, c->step), bias(c->beta2, c->step), c->seed, 0, {0, 0}};
    return COCOD_OK;
}

int cocod_adamw(void *stream, const cocod_adamw_call *c)
{
    if (int rc = check_call(c)) return rc;
    for (uint64_t i = 0; i < c->count; ++i)
        if (int rc = check_tensor(c, i)) return rc;
    const hipStream_t q = static_cast<hipStream_t>(stream);
    const char *const what = "cocod_adamw";
    AdamWParams s{};
    s.workers = c->workers;
    s.stride = c->workers > 1 ? c->stride : 0;
    s.copy_dtype = c->copy_dtype;
    s.beta1 = c->beta1; s.beta2 = c->beta2; s.eps = c->eps;
    s.rest1 = static_cast<float>(1.0 - static_cast<double>(c->beta1));
    s.rest2 = static_cast<float>(1.0 - static_cast<double>(c->beta2));
    s.now_device = c->now;
    if (!c->now) s.now = {c->lr, c->grad_scale, bias(c->beta1, c->step), bias(c->beta2, c->step), c->seed, 0, {0, 0}};
    const OnStreamDevice device(q);
    bool begun = false;
    auto flush = [&]() -> int {
        if (!s.count) return COCOD_OK;
        if (!begun && device.status() != hipSuccess) return launch_status(device.status(), what);
        begun = true;
        s.tiles = static_cast<uint64_t>(s.first_tile[s.count]) * s.workers;
        const uint32_t grid = static_cast<uint32_t>(s.tiles < kMostBlocks ? s.tiles : kMostBlocks);
        const bool eight = c->state == COCOD_ADAMW_STATE_8BIT;
        if (c->dtype == COCOD_F32)       launch<F32>(q, c->grad_dtype, eight, grid, s);
        else if (c->dtype == COCOD_BF16) launch<Bf16>(q, c->grad_dtype, eight, grid, s);
        else                             launch<F16>(q, c->grad_dtype, eight, grid, s);
        s.count = 0;
        return launch_status(hipGetLastError(), what);
    };
    for (uint64_t i = 0; i < c->count; ++i) {
        const cocod_adamw_tensor &t = c->tensors[i];
        const uint64_t tiles = (t.n + kTile - 1) / kTile;
        if (!tiles) continue;
        // (the tensors of a launch have consecutive numbers)
        if (s.count && (s.count == kMostTensors || s.number + s.count != i || s.first_tile[s.count] + tiles > ~0u))
            if (int rc = flush()) return rc;
        if (!s.count) s.number = static_cast<uint32_t>(i);
        s.tensor[s.count] = {t.p, t.g, t.m, t.v, t.m_scales, t.v_scales, t.copy, t.n, t.weight_decay, t.lr_scale};
        s.first_tile[s.count + 1] = s.first_tile[s.count] + static_cast<uint32_t>(tiles);
        ++s.count;
    }
    return flush();
}

}  // extern "C"
