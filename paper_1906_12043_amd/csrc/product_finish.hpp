// What the kernels of the products share: element types, the groups' rows, and what becomes of a value of C.
#pragma once
#include "product.hpp"

#include <type_traits>

namespace cocod {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef unsigned int u4 __attribute__((ext_vector_type(4)));
typedef unsigned int u2 __attribute__((ext_vector_type(2)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 hf2 __attribute__((ext_vector_type(2)));
typedef _Float16 hf8 __attribute__((ext_vector_type(8)));
typedef float v2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) s4 lds_s4;
typedef u4 __attribute__((aligned(2))) u4_any;       // 16 bytes at any element's address
typedef u2 __attribute__((aligned(1))) u2_any;
typedef u4 __attribute__((aligned(1))) u4_bytes;

// fp32 operands go in as three bf16 planes, exactly (8 + 8 + 8 bits), times 2^24 so that the last bit of the smallest numbers is
// a normal bf16 too; sums come out times 2^48.  Where that leaves the range, or an operand is not finite, the sum is not finite,
// and the tile is formed again with fp32 products.
constexpr float kPlaneScale = 0x1p24f, kPlaneUnscale = 0x1p-48f;

// exp(x, base): e^(x - base); in 16 bits the instruction for powers of two, off by 2^-23 of |x - base| beside its own last bit
constexpr float kLog2e = 1.44269504f;
constexpr float kKeepScale = 0x1p14f, kKeepUnscale = 0x1p-14f;   // of exponentials, at most 1, kept in fp16: exact to 2^-11 down to 2^-28 of the largest

struct Bf16 {
    typedef uint16_t elem;
    static constexpr Dtype dtype = Dtype::BF16;
    static constexpr int planes = 1;
    static __device__ __forceinline__ f16v mfma(u4 a, u4 b, f16v c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f4 mfma(u4 a, u4 b, f4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ unsigned pack(float a, float b) { return __builtin_bit_cast(unsigned, __builtin_convertvector(v2{a, b}, bf2)); }
    static __device__ __forceinline__ float exp(float x, float base) { return __builtin_amdgcn_exp2f((x - base) * kLog2e); }
    static __device__ __forceinline__ unsigned codes(unsigned four, float scale, bool high)
    {
        return high ? __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, scale, true))
                    : __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, scale, false));
    }
};
struct F16 {
    typedef uint16_t elem;
    static constexpr Dtype dtype = Dtype::F16;
    static constexpr int planes = 1;
    static __device__ __forceinline__ f16v mfma(u4 a, u4 b, f16v c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(hf8, a), __builtin_bit_cast(hf8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f4 mfma(u4 a, u4 b, f4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(hf8, a), __builtin_bit_cast(hf8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ unsigned pack(float a, float b) { return __builtin_bit_cast(unsigned, __builtin_convertvector(v2{a, b}, hf2)); }
    static __device__ __forceinline__ float exp(float x, float base) { return __builtin_amdgcn_exp2f((x - base) * kLog2e); }
    static __device__ __forceinline__ unsigned codes(unsigned four, float scale, bool high)
    {
        return high ? __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(four, scale, true))
                    : __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(four, scale, false));
    }
};
struct F32 : Bf16 {
    typedef float elem;
    static constexpr Dtype dtype = Dtype::F32;
    static constexpr int planes = 3;
    static __device__ __forceinline__ float exp(float x, float base) { return expf(x - base); }
};

// Slope of an entry with the logit z, d below the row's largest, from the row's two factors (Finish::Score).  Below -200 the exponential is zero, and so is
// the slope, also where d is minus infinity.  z is a product, rounded as `top` was: unrounded, the largest entry of a sure row would lie a rounding of `top`, not zero, from
// itself, far more than its slope of the entropy.
constexpr float kFarBelow = -200.0f;
template <class T> __device__ __forceinline__ float score_slope(float z, float top, float none, float one)
{
    #pragma clang fp contract(off)
    const float d = fmaxf(z - top, kFarBelow);
    return T::exp(d, 0.0f) * fmaf(one, d, none);
}

__device__ __forceinline__ uint64_t bound_at(const ProductParams &p, uint32_t i)
{
    const int64_t v = p.offsets[i];
    return v < 0 ? 0 : static_cast<uint64_t>(v) > p.rows ? p.rows : static_cast<uint64_t>(v);
}
__device__ __forceinline__ uint64_t length_at(const ProductParams &p, uint32_t g)
{
    const uint64_t a = bound_at(p, g), next = bound_at(p, g + 1);
    uint64_t b = next;
    if (p.ends) { const int64_t e = p.ends[g]; b = e < 0 ? 0 : static_cast<uint64_t>(e) < next ? static_cast<uint64_t>(e) : next; }
    return b > a ? b - a : 0;
}

// ---- what happens to four consecutive columns of a row of C ----------------------------------------------

template <class T> __device__ __forceinline__ void store_values(void *out, uint64_t at, f4 v, uint32_t count, bool f32)
{
    if (f32 || sizeof(typename T::elem) == 4) {
        float *o = static_cast<float *>(out) + at;
        if (count == 4 && (reinterpret_cast<uintptr_t>(o) & 15) == 0) { *reinterpret_cast<f4 *>(o) = v; return; }
        #pragma unroll
        for (uint32_t j = 0; j < 4; ++j) if (j < count) o[j] = v[j];
    } else {
        uint16_t *o = static_cast<uint16_t *>(out) + at;
        const unsigned lo = T::pack(v.x, v.y), hi = T::pack(v.z, v.w);
        if (count == 4 && (reinterpret_cast<uintptr_t>(o) & 7) == 0) { *reinterpret_cast<u2 *>(o) = u2{lo, hi}; return; }
        #pragma unroll
        for (uint32_t j = 0; j < 4; ++j) if (j < count) o[j] = static_cast<uint16_t>((j < 2 ? lo : hi) >> (16 * (j % 2)));
    }
}

// Exponentials between the two passes over the vocabulary: fp32 as they are, for bf16 slopes in fp16, whose eleven bits leave the rounding to eight alone.
template <class T> __device__ __forceinline__ void keep_values(void *out, uint64_t at, f4 v)
{
    if constexpr (sizeof(typename T::elem) == 4) *reinterpret_cast<f4 *>(static_cast<float *>(out) + at) = v;
    else *reinterpret_cast<u2 *>(static_cast<uint16_t *>(out) + at) = u2{F16::pack(v.x * kKeepScale, v.y * kKeepScale), F16::pack(v.z * kKeepScale, v.w * kKeepScale)};
}

template <class T> __device__ __forceinline__ bool above_zero(const ProductParams &p, uint64_t row, uint32_t col)
{
    if (p.mask_codes) { const uint8_t c = p.mask_codes[row * p.ld_mask + col]; return c != 0 && c < 0x7f; }
    if constexpr (sizeof(typename T::elem) == 4) return static_cast<const float *>(p.mask)[row * p.ld_mask + col] > 0.0f;
    else {
        // sign clear, not zero, not NaN
        const uint16_t b = static_cast<const uint16_t *>(p.mask)[row * p.ld_mask + col];
        return b != 0 && b <= (std::is_same<T, F16>::value ? 0x7c00 : 0x7f80);
    }
}

// row: of all groups (Weights: group * m + row of C_g); local: row of C_g
template <class T, bool WEIGHTS>
__device__ __forceinline__ void finish_quad(const ProductParams &p, uint32_t group, uint64_t row, uint32_t local, uint32_t col, f4 v, float factor)
{
    const uint32_t count = p.n - col < 4 ? p.n - col : 4;
    if (!WEIGHTS && p.out_row && p.out_row[row] == kNoRow) return;
    if (p.sum) {
        float *s = p.sum + row * p.ld_sum + col;               // ld_sum is a multiple of 4, the columns behind n are its own
        if (p.sum_read) v += *reinterpret_cast<const f4 *>(s);
        if (p.sum_write) { *reinterpret_cast<f4 *>(s) = v; return; }
    }
    if (!WEIGHTS && p.row_scale) factor = p.row_scale[row];
    v *= factor;
    if (p.relu) {
        #pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = v[j] < 0.0f ? 0.0f : v[j];
    }
    if (p.mask || p.mask_codes) {
        #pragma unroll
        for (uint32_t j = 0; j < 4; ++j) if (j < count && !above_zero<T>(p, row, col + j)) v[j] = 0.0f;
    }
    const uint64_t at = WEIGHTS ? group * p.out_group + static_cast<uint64_t>(local) * p.ldc + col
                                : (p.out_row ? static_cast<uint64_t>(p.out_row[row]) : row) * p.ldc + col;
    store_values<T>(p.out, at, v, count, p.out_f32 != 0);
}

__device__ __forceinline__ float group_factor(const ProductParams &p, uint32_t group)
{
    if (p.group_scale) return p.group_scale[group];
    if (!p.mean) return p.scale;
    const uint64_t len = length_at(p, group);
    return len ? p.scale / static_cast<float>(len) : 0.0f;
}

}  // namespace
}  // namespace cocod
