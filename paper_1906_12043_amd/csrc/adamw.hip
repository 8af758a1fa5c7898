// One AdamW step over the tensors of a model, for all workers, in one pass over memory.
//
//   g' = grad_scale g,  m' = b1 m + (1 - b1) g',  v' = b2 v + ((1 - b2) g') g'   (fp32, rounded after every product and sum)
//   p' = p (1 - lr wd) - (lr / c1) m' / (sqrt(v' / c2) + eps),  c = 1 - b^step
//
// States of 8 bits: 32 consecutive elements of a tensor share a scale 2^e, m is held as an e4m3 code of m / 2^e, v as the code of sqrt(v) / 2^e
// (the format of the 8-bit activations), whose range of 2^18 within a block would be 2^9 of v's roots if it held v.  A step changes v by a
// thousandth of itself, a code's step is a sixteenth to an eighth: rounded to the nearest, v would stand still.  So a code is rounded up or down by chance,
// with 16 random bits each, so that the stored m, and the SQUARE of the stored root of v, are m' and v' in the mean (to 2^-16 of a step).  The random bits are
// a function of (seed, tensor, worker, element): the published mixer of 32 bits lowbias32 (C. Wellons, public domain), three multiplications an element, where a
// ten-round counter generator would cost more time than the memory leaves.  p' comes from m' and v' before they are rounded.
//
// Bound by memory: fp32 with 16-bit gradients and copies 28 bytes an element (16 workers of 11.2 M: 842 us, 6.0 TB/s), with 8-bit states 16.1 (138 M: 404 us,
// 5.5 TB/s; four streams read and five written, a copy reaches 6.6).  A thread takes four elements, eight lanes a scale.  What it took, us for these two: four elements side by
// side instead of eight in a thread, past the caches where the states are larger than those (1000 -> 903 / 501 -> 480), tiles within a tensor without a decision between their
// loads, a wait behind each, and 8-bit states that find out once a wave whether every code is a normal one and every number finite (480 -> 413), seven waves a SIMD instead of six (413
// -> 404), four for fp32 states
// out of memory (907 -> 842).  Twice and four times the tile, 512 or 1024 threads, runs of tiles per die, blocks that stay for several tiles: no better.
// Tensors travel in the kernel's arguments, 4 KiB, a launch for 55 to 64 of them, so nothing has to be laid out on the device and a captured
// launch holds all it needs (61 000 parameters in 150 tensors: 18 us, 22 M in 400 with 8-bit states 130).
#include "operator_call.hpp"
#include "row_access.hpp"

#include <cmath>

namespace cocod {
namespace {

constexpr uint32_t kStateBlock = 32;                 // elements that share a scale
constexpr int kThreads = 256;
constexpr uint32_t kSpan = kThreads * 4;             // elements of a block's threads side by side, four each
constexpr uint32_t kSpans = 1;                       // of them a tile has
constexpr uint32_t kTile = kSpan * kSpans;
constexpr uint32_t kMostBlocks = 1u << 20;
constexpr uint64_t kMostElements = 1ull << 40;       // of a tensor

// A tensor in the kernel's arguments: p, g, m, v, the scales where states have 8 bits, the copy where there is one, and the elements with the number of its pair of
// weight decay and factor of the learning rate above them.
constexpr uint32_t kMostTensors = 64, kMostPairs = 16, kWords = 440, kPairShift = 48;
struct Pair { float weight_decay, lr_scale; };
struct AdamWParams {
    uint64_t words[kWords];
    Pair pairs[kMostPairs];
    uint32_t first_tile[kMostTensors + 1];           // of every tensor, in tiles of a worker
    uint32_t count, number;                          // tensors of this launch; number of the first one in the call
    uint32_t words_each;
    uint64_t tiles;                                  // of all workers
    uint32_t workers, copy_dtype;                    // copy_dtype: COCOD_F32 where there is none
    uint64_t stride;
    float beta1, beta2, rest1, rest2, eps;
    cocod_adamw_now now;
    const cocod_adamw_now *now_device;
};
struct Tensor {
    char *p;
    const char *g;
    char *m, *v;
    uint8_t *m_scales, *v_scales;
    char *copy;
    uint64_t n;
};
static_assert(sizeof(AdamWParams) <= 4096, "arguments of a kernel");

// Four consecutive elements in fp32, and back; count < 4 at a tensor's end.
// STREAM: past the caches.
template <class T, bool STREAM> struct Four {
    typedef typename T::elem elem;
    static __device__ __forceinline__ f4 load(const void *base, uint64_t at, uint32_t count)
    {
        const elem *from = static_cast<const elem *>(base) + at;
        f4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        if (count >= 4) {
            if constexpr (sizeof(elem) == 4) return __builtin_bit_cast(f4, fetch16<STREAM>(from));
            else {
                const u2 w = fetch8<STREAM>(from);
                #pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = widen<T>(static_cast<elem>(w[j / 2] >> (16 * (j % 2))));
                return v;
            }
        }
        #pragma unroll
        for (uint32_t j = 0; j < 4; ++j) if (j < count) v[j] = widen<T>(from[j]);
        return v;
    }
    static __device__ __forceinline__ void store(void *base, uint64_t at, uint32_t count, f4 v)
    {
        elem *to = static_cast<elem *>(base) + at;
        if constexpr (sizeof(elem) == 4) {
            if (count >= 4) { put16<STREAM>(to, __builtin_bit_cast(u4, v)); return; }
            #pragma unroll
            for (uint32_t j = 0; j < 4; ++j) if (j < count) to[j] = v[j];
        } else {
            const u2 w = {T::pack(v[0], v[1]), T::pack(v[2], v[3])};
            if (count >= 4) { put8<STREAM>(to, w); return; }
            #pragma unroll
            for (uint32_t j = 0; j < 4; ++j) if (j < count) to[j] = static_cast<elem>(w[j / 2] >> (16 * (j % 2)));
        }
    }
};
template <bool STREAM> __device__ __forceinline__ uint32_t load_codes(const void *base, uint64_t at, uint32_t count)
{
    const uint8_t *from = static_cast<const uint8_t *>(base) + at;
    if (count >= 4) return fetch4<STREAM>(from);
    uint32_t w = 0;
    #pragma unroll
    for (uint32_t j = 0; j < 4; ++j) if (j < count) w |= static_cast<uint32_t>(from[j]) << (8 * j);
    return w;
}
template <bool STREAM> __device__ __forceinline__ void store_codes(void *base, uint64_t at, uint32_t count, uint32_t w)
{
    uint8_t *to = static_cast<uint8_t *>(base) + at;
    if (count >= 4) { put4<STREAM>(to, w); return; }
    #pragma unroll
    for (uint32_t j = 0; j < 4; ++j) if (j < count) to[j] = static_cast<uint8_t>(w >> (8 * j));
}

// ---- states of 8 bits: a block of 32 lies in eight neighbouring lanes, four elements each --------------------------------

__device__ __forceinline__ float power(int e) { return __uint_as_float(static_cast<unsigned>(e + 127) << 23); }      // 2^e, e in -126 .. 127
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }
template <int CTRL> __device__ __forceinline__ uint32_t larger_moved(uint32_t v)
{
    return larger(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xf, 0xf, false)));
}
__device__ __forceinline__ uint32_t larger_of_block(uint32_t v)
{
    return larger_moved<0x141>(larger_moved<0x4e>(larger_moved<0xb1>(v)));      // lanes 1 and 2 apart, eight lanes mirrored
}
// Smallest e, not below `low`, for which the magnitude with these bits is at most 448 2^e (448 = 1.75 * 2^8).
__device__ __forceinline__ int block_scale(uint32_t bits, int low)
{
    const int e = static_cast<int>((bits + 0x1fffffu) >> 23) - 135;
    return e > low ? e : low;
}
__device__ __forceinline__ void decode(uint32_t codes, uint8_t scale, f4 &v)
{
    const float unit = __uint_as_float(static_cast<unsigned>(scale) << 23);
    const v2 low = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, unit, false), high = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, unit, true);
    v = f4{low.x, low.y, high.x, high.y};
}

// Random bits of element `at` of a tensor; those of the elements behind it follow by adding kNextElement to x.
constexpr uint32_t kNextElement = 0x9E3779B1u;
__device__ __forceinline__ uint32_t random_seed(uint64_t at, uint32_t stream) { return static_cast<uint32_t>(at) * kNextElement + static_cast<uint32_t>(at >> 32) * 0x85EBCA6Bu + stream; }
__device__ __forceinline__ uint32_t mixed(uint32_t x)        // lowbias32: its shifts and multipliers are the published ones
{
    x = (x ^ (x >> 16)) * 0x7FEB352Du;
    x = (x ^ (x >> 15)) * 0x846CA68Bu;
    return x ^ (x >> 16);
}

// y in units of the smallest code.  A code is its neighbour below, plus one where the way from there to y, in 65536ths of the step, is above the random number.
// Normal codes (y >= 8) are the upper bits of y's: adding 2^20 - 1 - 16 * random to the lower twenty carries where they are above 16 * random.
constexpr uint32_t kCodeOfBits = 1032;               // y's upper bits less its code: 8 is code 8
__device__ __forceinline__ uint32_t normal_code(float y, uint32_t random_up) { return (__float_as_uint(y) + (0xfffffu - 16u * random_up - (kCodeOfBits << 20))) >> 20; }
__device__ __forceinline__ uint32_t any_code(float y, uint32_t random_up)
{
    if (y >= 8.0f) return normal_code(y, random_up);
    const uint32_t code = static_cast<uint32_t>(y);
    return code + ((y - static_cast<float>(code)) * 65536.0f > static_cast<float>(random_up) ? 1u : 0u);
}
// The same for the root y of w, by the way of the squares; what is not zero gets a code that is not.
__device__ __forceinline__ uint32_t normal_root(float y, float w, uint32_t random_up)
{
    const uint32_t bits = __float_as_uint(y) & 0xfff00000u;
    const float low = __uint_as_float(bits), high = __uint_as_float(bits + 0x100000u), low2 = low * low, way = w - low2;
    return (bits >> 20) - kCodeOfBits + (way * 65536.0f > static_cast<float>(random_up) * fmaf(high, high, -low2) ? 1u : 0u);
}
__device__ __forceinline__ uint32_t any_root(float y, float w, uint32_t random_up, bool some)
{
    if (y >= 8.0f) return normal_root(y, w, random_up);
    const float low = floorf(y), high = low + 1.0f;
    const uint32_t code = static_cast<uint32_t>(low) + ((w - low * low) * 65536.0f > static_cast<float>(random_up) * (high * high - low * low) ? 1u : 0u);
    return code == 0 && some ? 1u : code;
}

// Codes of four elements and the scales of their block.  Where every element of a wave is finite and has a normal code, nothing else is looked at.
struct Stored { uint32_t m, v; uint8_t m_scale, v_scale; };
__device__ __forceinline__ Stored store_states(const f4 &m, const f4 &v, const f4 &root, uint32_t x)
{
    #pragma clang fp contract(off)
    constexpr uint32_t kInfinity = 0x7f800000u;
    uint32_t bm[4], bv[4], most_m = 0, most_v = 0;
    #pragma unroll
    for (int j = 0; j < 4; ++j) {
        bm[j] = __float_as_uint(m[j]) & 0x7fffffffu;
        bv[j] = __float_as_uint(v[j]);                         // (never negative; a NaN's sign is left out)
        most_m = larger(most_m, bm[j]);
        most_v = larger(most_v, bv[j] & 0x7fffffffu);
    }
    most_m = larger_of_block(most_m);
    most_v = larger_of_block(most_v);
    bool plain = most_m < kInfinity && most_v < kInfinity;
    if (!plain) {                                              // what is not finite does not count
        most_m = most_v = 0;
        #pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (bm[j] < kInfinity) most_m = larger(most_m, bm[j]);
            if ((bv[j] & 0x7fffffffu) < kInfinity) most_v = larger(most_v, bv[j]);
        }
        most_m = larger_of_block(most_m);
        most_v = larger_of_block(most_v);
    }
    const int em = block_scale(most_m, -117), er = block_scale(__float_as_uint(sqrtf(__uint_as_float(most_v))), -51);
    const float um = power(9 - em), ur = power(9 - er), ur2 = ur * ur;
    float ym[4], yr[4], w[4];
    #pragma unroll
    for (int j = 0; j < 4; ++j) {
        ym[j] = fabsf(m[j]) * um;
        yr[j] = root[j] * ur;
        w[j] = v[j] * ur2;
        plain = plain && ym[j] >= 8.0f && yr[j] >= 8.0f;
    }
    Stored out = {0, 0, static_cast<uint8_t>(em + 127), static_cast<uint8_t>(er + 127)};
    if (__all(plain)) {
        #pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t random = mixed(x + j * kNextElement);
            out.m |= (normal_code(ym[j], random >> 16) | (__float_as_uint(m[j]) >> 24 & 0x80u)) << (8 * j);
            out.v |= normal_root(yr[j], w[j], random & 0xffffu) << (8 * j);
        }
    } else {
        #pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t random = mixed(x + j * kNextElement);
            const bool fine_m = bm[j] < kInfinity, fine_v = (bv[j] & 0x7fffffffu) < kInfinity;
            out.m |= ((fine_m ? any_code(ym[j], random >> 16) : 0x7fu) | (__float_as_uint(m[j]) >> 24 & 0x80u)) << (8 * j);
            out.v |= (fine_v ? any_root(yr[j], w[j], random & 0xffffu, bv[j] != 0) : 0x7fu) << (8 * j);
        }
    }
    return out;
}

// An address in device memory from its number (said so, as accesses that might also go to LDS wait for it).
__device__ __forceinline__ char *in_memory(uint64_t address) { return (char *)(__attribute__((address_space(1))) char *)address; }

constexpr uint32_t kLeastNormal = 0x00800000u;       // bits of 2^-126

// A tile of a tensor.  WHOLE: it lies within the tensor, so that nothing is decided between the loads, which are then all on their way at a time.
struct Terms { float grad_scale, keep, step, root_bias2; uint32_t stream; };
template <class TP, class TG, bool EIGHT, bool STREAM, bool WHOLE>
__device__ __forceinline__ void update(const AdamWParams &s, const Tensor &t, const Terms &now, uint32_t worker, uint64_t first)
{
    #pragma clang fp contract(off)
    f4 p[kSpans], g[kSpans], m[kSpans], v[kSpans];
    uint32_t codes_m[kSpans], codes_v[kSpans], count[kSpans];
    uint8_t scale_m[kSpans], scale_v[kSpans];
    #pragma unroll
    for (uint32_t u = 0; u < kSpans; ++u) {
        const uint64_t at = first + u * kSpan, base = worker * s.stride + at;
        count[u] = WHOLE ? 4 : at >= t.n ? 0 : t.n - at < 4 ? static_cast<uint32_t>(t.n - at) : 4;
        p[u] = Four<TP, STREAM>::load(t.p, base, count[u]);
        g[u] = Four<TG, STREAM>::load(t.g, base, count[u]);
        if constexpr (EIGHT) {
            const uint64_t scale_at = worker * (s.stride / kStateBlock) + at / kStateBlock;
            codes_m[u] = load_codes<STREAM>(t.m, base, count[u]);
            codes_v[u] = load_codes<STREAM>(t.v, base, count[u]);
            scale_m[u] = count[u] ? t.m_scales[scale_at] : 0;
            scale_v[u] = count[u] ? t.v_scales[scale_at] : 0;
        } else {
            m[u] = Four<F32, STREAM>::load(t.m, base, count[u]);
            v[u] = Four<F32, STREAM>::load(t.v, base, count[u]);
        }
    }
    #pragma unroll
    for (uint32_t u = 0; u < kSpans; ++u) {
        const uint64_t at = first + u * kSpan, base = worker * s.stride + at;
        if constexpr (EIGHT) {
            decode(codes_m[u], scale_m[u], m[u]);
            decode(codes_v[u], scale_v[u], v[u]);
            v[u] *= v[u];
        }
        f4 root;
        uint32_t least = ~0u;
        #pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            const float d = g[u][j] * now.grad_scale;
            m[u][j] = m[u][j] * s.beta1 + d * s.rest1;
            v[u][j] = v[u][j] * s.beta2 + (d * s.rest2) * d;
            // (a code hangs on the last bit of the root only through its block's largest, of which store_states takes an exact one)
            root[j] = EIGHT ? __builtin_amdgcn_sqrtf(v[u][j]) : sqrtf(v[u][j]);
            const uint32_t bits = __float_as_uint(v[u][j]) - 1;          // (zero, whose root is right, is far above)
            least = least < bits ? least : bits;
        }
        // the instruction takes what is below the normal numbers for zero: with an eps of zero the step would be infinite
        if (EIGHT && __any(least < kLeastNormal - 1)) {
            #pragma unroll
            for (uint32_t j = 0; j < 4; ++j) root[j] = sqrtf(v[u][j]);
        }
        #pragma unroll
        for (uint32_t j = 0; j < 4; ++j) p[u][j] = fmaf(-now.step, m[u][j] * __builtin_amdgcn_rcpf(fmaf(root[j], now.root_bias2, s.eps)), p[u][j] * now.keep);
        Four<TP, STREAM>::store(t.p, base, count[u], p[u]);
        if constexpr (sizeof(typename TP::elem) == 4) {
            if (t.copy && s.copy_dtype == COCOD_BF16) Four<Bf16, STREAM>::store(t.copy, base, count[u], p[u]);
            else if (t.copy)                          Four<F16, STREAM>::store(t.copy, base, count[u], p[u]);
        }
        if constexpr (!EIGHT) {
            Four<F32, STREAM>::store(t.m, base, count[u], m[u]);
            Four<F32, STREAM>::store(t.v, base, count[u], v[u]);
        } else {
            #pragma unroll
            for (uint32_t j = 0; j < 4; ++j) if (j >= count[u]) { m[u][j] = 0.0f; v[u][j] = 0.0f; root[j] = 0.0f; }
            const Stored stored = store_states(m[u], v[u], root, random_seed(at, now.stream));
            store_codes<STREAM>(t.m, base, count[u], stored.m);
            store_codes<STREAM>(t.v, base, count[u], stored.v);
            if (count[u] && threadIdx.x % 8 == 0) {
                const uint64_t scale_at = worker * (s.stride / kStateBlock) + at / kStateBlock;
                t.m_scales[scale_at] = stored.m_scale;
                t.v_scales[scale_at] = stored.v_scale;
            }
        }
    }
}

// Waves of a SIMD: 8-bit states take the most there are registers for; fp32 states out of memory stream faster with four, whose requests lie closer together (16 workers of 11.2 M, us
// with 8 / 5 / 4 / 3 / 2 waves: 907 / 878 / 842 / 830 / 976; 400 tensors of 80 000 for 16 workers 161 / - / 167 / 185 / -; 138 M with 8-bit states 405 with 7, 416 / 435 / 485 with 6 / 5 / 4).
constexpr int waves_of(bool eight, bool stream) { return eight ? 7 : stream ? 4 : 8; }
template <class TP, class TG, bool EIGHT, bool STREAM>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(waves_of(EIGHT, STREAM), waves_of(EIGHT, STREAM)))) void adamw_kernel(const AdamWParams s)
{
    cocod_adamw_now now = s.now;
    if (s.now_device) {
        now = *s.now_device;
        if (now.skip) return;
    }
    const uint32_t lane = threadIdx.x % 64, per_worker = s.first_tile[s.count];
    const uint32_t mine = lane < s.count ? s.first_tile[lane] : ~0u;       // (a tile's number is below that)
    static_assert(kMostTensors <= 64, "a lane a tensor");
    for (uint64_t tile = blockIdx.x; tile < s.tiles; tile += gridDim.x) {
        const uint32_t worker = s.workers == 1 ? 0 : static_cast<uint32_t>(tile / per_worker), in = static_cast<uint32_t>(tile - static_cast<uint64_t>(worker) * per_worker);
        const uint32_t which = __builtin_amdgcn_readfirstlane(__popcll(__ballot(mine <= in)) - 1);
        const uint64_t *const w = s.words + which * s.words_each;
        Tensor t = {in_memory(w[0]), in_memory(w[1]), in_memory(w[2]), in_memory(w[3]), nullptr, nullptr, nullptr, 0};
        uint32_t at = 4;
        if constexpr (EIGHT) { t.m_scales = reinterpret_cast<uint8_t *>(in_memory(w[4])); t.v_scales = reinterpret_cast<uint8_t *>(in_memory(w[5])); at = 6; }
        if (sizeof(typename TP::elem) == 4 && s.copy_dtype != COCOD_F32) t.copy = in_memory(w[at++]);
        const uint64_t last = w[at];
        t.n = last & ((1ull << kPairShift) - 1);
        const Pair pair = s.pairs[last >> kPairShift];
        const uint64_t begin = static_cast<uint64_t>(in - s.first_tile[which]) * kTile, first = begin + threadIdx.x * 4;
        const float lr = now.lr * pair.lr_scale;
        const Terms terms = {now.grad_scale, 1.0f - lr * pair.weight_decay, lr / now.bias1, 1.0f / sqrtf(now.bias2),
                             now.seed + (s.number + which) * 0x632BE5ABu + worker * 0x85157AF5u};
        if (t.n - begin >= kTile) update<TP, TG, EIGHT, STREAM, true>(s, t, terms, worker, first);
        else                      update<TP, TG, EIGHT, STREAM, false>(s, t, terms, worker, first);
    }
}

template <class TP, class TG> void launch(hipStream_t q, bool eight, bool stream, uint32_t grid, const AdamWParams &s)
{
    const auto kernel = eight ? (stream ? adamw_kernel<TP, TG, true, true> : adamw_kernel<TP, TG, true, false>)
                              : (stream ? adamw_kernel<TP, TG, false, true> : adamw_kernel<TP, TG, false, false>);
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(kThreads), 0, q, s);
}
template <class TP> void launch(hipStream_t q, uint32_t grad, bool eight, bool stream, uint32_t grid, const AdamWParams &s)
{
    if (grad == COCOD_F32)       launch<TP, F32>(q, eight, stream, grid, s);
    else if (grad == COCOD_BF16) launch<TP, Bf16>(q, eight, stream, grid, s);
    else                         launch<TP, F16>(q, eight, stream, grid, s);
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
    // (the reciprocal's instruction takes what is below the normal numbers for zero, and a parameter without gradients would become NaN)
    if (c->eps > 0.0f && c->eps < 0x1p-126f) return set_error(COCOD_ERR_INVALID, "eps must be 0 or at least 2^-126");
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
    s.beta1 = c->beta1; s.beta2 = c->beta2; s.eps = c->eps;
    s.rest1 = static_cast<float>(1.0 - static_cast<double>(c->beta1));
    s.rest2 = static_cast<float>(1.0 - static_cast<double>(c->beta2));
    s.now_device = c->now;
    if (!c->now) s.now = {c->lr, c->grad_scale, bias(c->beta1, c->step), bias(c->beta2, c->step), c->seed, 0, {0, 0}};
    const bool eight = c->state == COCOD_ADAMW_STATE_8BIT;
    uint64_t elements = 0;
    for (uint64_t i = 0; i < c->count; ++i) elements += c->tensors[i].n;
    const uint64_t each = dtype_bytes(static_cast<Dtype>(c->dtype)) + dtype_bytes(static_cast<Dtype>(c->grad_dtype)) + (eight ? 2 : 8);
    // (16 workers of 11.2 M, fp32: 852 us instead of 1001; 3 M in 16 and 8 bits: 17.1 instead of 16.1)
    const bool stream_past = elements * each * c->workers > kLastLevelCache;
    const OnStreamDevice device(q);
    bool begun = false;
    auto flush = [&]() -> int {
        if (!s.count) return COCOD_OK;
        if (!begun && device.status() != hipSuccess) return launch_status(device.status(), what);
        begun = true;
        s.tiles = static_cast<uint64_t>(s.first_tile[s.count]) * s.workers;
        const uint32_t grid = static_cast<uint32_t>(s.tiles < kMostBlocks ? s.tiles : kMostBlocks);
        if (c->dtype == COCOD_F32)       launch<F32>(q, c->grad_dtype, eight, stream_past, grid, s);
        else if (c->dtype == COCOD_BF16) launch<Bf16>(q, c->grad_dtype, eight, stream_past, grid, s);
        else                             launch<F16>(q, c->grad_dtype, eight, stream_past, grid, s);
        s.count = 0;
        return launch_status(hipGetLastError(), what);
    };
    bool copies = false;
    for (uint64_t i = 0; i < c->count; ++i) copies = copies || (c->tensors[i].n && c->tensors[i].copy);
    s.copy_dtype = copies ? c->copy_dtype : COCOD_F32;
    s.words_each = 5 + (eight ? 2 : 0) + (copies ? 1 : 0);
    const uint32_t most = kWords / s.words_each < kMostTensors ? kWords / s.words_each : kMostTensors;
    uint32_t pairs = 0;
    for (uint64_t i = 0; i < c->count; ++i) {
        const cocod_adamw_tensor &t = c->tensors[i];
        const uint64_t tiles = (t.n + kTile - 1) / kTile;
        if (!tiles) continue;
        const auto pair_of = [&] {
            uint32_t k = 0;
            while (k < pairs && (s.pairs[k].weight_decay != t.weight_decay || s.pairs[k].lr_scale != t.lr_scale)) ++k;
            return k;
        };
        uint32_t pair = pair_of();
        // (the tensors of a launch have consecutive numbers)
        if (s.count && (s.count == most || s.number + s.count != i || s.first_tile[s.count] + tiles > ~0u || pair == kMostPairs)) {
            if (int rc = flush()) return rc;
            pairs = pair = 0;
        }
        if (pair == pairs) s.pairs[pairs++] = {t.weight_decay, t.lr_scale};
        if (!s.count) s.number = static_cast<uint32_t>(i);
        uint64_t *w = s.words + s.count * s.words_each;
        for (const void *array : {static_cast<const void *>(t.p), t.g, static_cast<const void *>(t.m), static_cast<const void *>(t.v)}) *w++ = reinterpret_cast<uintptr_t>(array);
        if (eight) { *w++ = reinterpret_cast<uintptr_t>(t.m_scales); *w++ = reinterpret_cast<uintptr_t>(t.v_scales); }
        if (copies) *w++ = reinterpret_cast<uintptr_t>(t.copy);
        *w = t.n | static_cast<uint64_t>(pair) << kPairShift;
        s.first_tile[s.count + 1] = s.first_tile[s.count] + static_cast<uint32_t>(tiles);
        ++s.count;
    }
    return flush();
}

}  // extern "C"
