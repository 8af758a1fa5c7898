// Rows of elements in pieces of 16 bytes, at any element's address.
#pragma once
#include "product_finish.hpp"

namespace cocod {
namespace {

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

    static __device__ __forceinline__ u4 load(const elem *from) { return *reinterpret_cast<const u4_any *>(from); }
    static __device__ __forceinline__ void store(elem *to, u4 raw) { *reinterpret_cast<u4_any *>(to) = raw; }

    // the first `count` of them (all where count >= N); the others are zeros
    static __device__ __forceinline__ u4 load(const elem *from, uint32_t count)
    {
        if (count >= N) return load(from);
        u4 raw = {0, 0, 0, 0};
        #pragma unroll
        for (uint32_t j = 0; j < N; ++j)
            if (j < count) {
                if constexpr (sizeof(elem) == 4) raw[j] = __float_as_uint(from[j]);
                else                             raw[j / 2] |= static_cast<unsigned>(from[j]) << (16 * (j % 2));
            }
        return raw;
    }
    static __device__ __forceinline__ void store(elem *to, u4 raw, uint32_t count)
    {
        if (count >= N) { store(to, raw); return; }
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
