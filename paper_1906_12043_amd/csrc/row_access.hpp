// Rows of elements in pieces of 16 bytes, at any element's address.
#pragma once
#include "product_finish.hpp"

namespace cocod {
namespace {

// What a launch moves beyond this goes past the caches (STREAM below): it would only displace itself.
constexpr uint64_t kLastLevelCache = 256ull << 20;

// 16, 8 or 4 bytes at any address.  (An alignment is lost where a template deduces a type, so these name theirs.)
typedef u4 __attribute__((aligned(1))) u4_at;
typedef u2 __attribute__((aligned(1))) u2_at;
typedef uint32_t __attribute__((aligned(1))) u1_at;
template <bool STREAM> __device__ __forceinline__ u4 fetch16(const void *from)
{
    if constexpr (STREAM) return __builtin_nontemporal_load(static_cast<const u4_at *>(from)); else return *static_cast<const u4_at *>(from);
}
template <bool STREAM> __device__ __forceinline__ u2 fetch8(const void *from)
{
    if constexpr (STREAM) return __builtin_nontemporal_load(static_cast<const u2_at *>(from)); else return *static_cast<const u2_at *>(from);
}
template <bool STREAM> __device__ __forceinline__ uint32_t fetch4(const void *from)
{
    if constexpr (STREAM) return __builtin_nontemporal_load(static_cast<const u1_at *>(from)); else return *static_cast<const u1_at *>(from);
}
template <bool STREAM> __device__ __forceinline__ void put16(void *to, u4 v)
{
    if constexpr (STREAM) __builtin_nontemporal_store(v, static_cast<u4_at *>(to)); else *static_cast<u4_at *>(to) = v;
}
template <bool STREAM> __device__ __forceinline__ void put8(void *to, u2 v)
{
    if constexpr (STREAM) __builtin_nontemporal_store(v, static_cast<u2_at *>(to)); else *static_cast<u2_at *>(to) = v;
}
template <bool STREAM> __device__ __forceinline__ void put4(void *to, uint32_t v)
{
    if constexpr (STREAM) __builtin_nontemporal_store(v, static_cast<u1_at *>(to)); else *static_cast<u1_at *>(to) = v;
}

template <class T> __device__ __forceinline__ float widen(typename T::elem v)
{
    if constexpr (sizeof(v) == 4) return v;
    else if constexpr (std::is_same<T, F16>::value) return static_cast<float>(__builtin_bit_cast(_Float16, v));
    else return __uint_as_float(static_cast<unsigned>(v) << 16);
}

// Sixteen bytes: N elements.
template <class T> struct Piece {
    typedef typename T::elem elem;
    static constexpr uint32_t N = 16 / sizeof(elem);

    template <bool STREAM = false> static __device__ __forceinline__ u4 load(const elem *from) { return fetch16<STREAM>(from); }
    template <bool STREAM = false> static __device__ __forceinline__ void store(elem *to, u4 raw) { put16<STREAM>(to, raw); }

    // the first `count` of them (all where count >= N); the others are zeros
    template <bool STREAM = false> static __device__ __forceinline__ u4 load(const elem *from, uint32_t count)
    {
        if (count >= N) return load<STREAM>(from);
        u4 raw = {0, 0, 0, 0};
        #pragma unroll
        for (uint32_t j = 0; j < N; ++j)
            if (j < count) {
                if constexpr (sizeof(elem) == 4) raw[j] = __float_as_uint(from[j]);
                else                             raw[j / 2] |= static_cast<unsigned>(from[j]) << (16 * (j % 2));
            }
        return raw;
    }
    template <bool STREAM = false> static __device__ __forceinline__ void store(elem *to, u4 raw, uint32_t count)
    {
        if (count >= N) { store<STREAM>(to, raw); return; }
        #pragma unroll
        for (uint32_t j = 0; j < N; ++j)
            if (j < count) {
                if constexpr (sizeof(elem) == 4) to[j] = __uint_as_float(raw[j]);
                else                             to[j] = static_cast<elem>(raw[j / 2] >> (16 * (j % 2)));
            }
    }
    static __device__ __forceinline__ float value(u4 raw, uint32_t j)
    {
        if constexpr (sizeof(elem) == 4) return __uint_as_float(raw[j]);
        else if constexpr (std::is_same<T, F16>::value) return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(raw[j / 2] >> (16 * (j % 2)))));
        else return __uint_as_float(j % 2 ? raw[j / 2] & 0xffff0000u : raw[j / 2] << 16);
    }
    // rounded to nearest, ties to even
    static __device__ __forceinline__ u4 pack(const float (&v)[N])
    {
        u4 raw;
        #pragma unroll
        for (int w = 0; w < 4; ++w) {
            if constexpr (sizeof(elem) == 4) raw[w] = __float_as_uint(v[w]);
            else                             raw[w] = T::pack(v[2 * w], v[2 * w + 1]);
        }
        return raw;
    }
};

}  // namespace
}  // namespace cocod
