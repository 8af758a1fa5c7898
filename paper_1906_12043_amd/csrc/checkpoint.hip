// Activations kept in 8 bits between forward and backward pass: 32 consecutive values of a row share a power of two.
//
// A value is stored as an e4m3 code (OCP, 1 + 4 + 3 bits) of value / 2^e, rounded to nearest even, with 2^e the smallest power of
// two for which the largest finite magnitude of the 32 is at most 448 * 2^e.  With a power of two every code times its scale is a value
// of all three element types, so expanding is exact, and so is a product that expands on its way into the matrix cores.  What is
// not zero is stored as not zero (the smallest code instead of none): the mask of a relu survives.  What is not finite is stored as
// NaN and does not count for the scale.
//
// Bound by memory: s + 1 + 1/32 bytes per value in either direction; a thread takes eight values, four threads a scale.
#include "operator_call.hpp"
#include "product_finish.hpp"

namespace cocod {
namespace {

constexpr int kCheckpointThreads = 256;

struct CheckpointParams {
    uint64_t rows;
    uint32_t cols;
    uint32_t per_row;                 // chunks of eight values, whole blocks of 32
    const void *x;
    void *out;
    uint64_t ldx;
    uint8_t *codes, *scales;
    uint64_t ld_codes, ld_scales;
    uint64_t step_rows;               // a thread's chunks lie as far apart as the launch has threads, which is so many rows
    uint32_t step_chunks;             //   and so many chunks
};

template <class T> struct Range;      // exponents of the smallest scale and of the largest magnitude
template <> struct Range<Bf16> { static constexpr int low = -117; static constexpr unsigned most = 0x7f700000u; };   // 1.875 * 2^127
template <> struct Range<F32> : Range<Bf16> {};
template <> struct Range<F16> { static constexpr int low = -15; static constexpr unsigned most = 0x47700000u; };     // 1.875 * 2^15

// this thread's next chunk; false behind the last
struct Walk {
    uint64_t row;
    uint32_t chunk;
    __device__ __forceinline__ explicit Walk(const CheckpointParams &p)
    {
        const uint64_t i = static_cast<uint64_t>(blockIdx.x) * kCheckpointThreads + threadIdx.x;
        if (i >> 32) { row = i / p.per_row; chunk = static_cast<uint32_t>(i % p.per_row); }
        else { row = static_cast<uint32_t>(i) / p.per_row; chunk = static_cast<uint32_t>(i) % p.per_row; }
    }
    __device__ __forceinline__ void next(const CheckpointParams &p)
    {
        row += p.step_rows;
        chunk += p.step_chunks;
        if (chunk >= p.per_row) { chunk -= p.per_row; ++row; }
    }
};

template <class T> __device__ __forceinline__ float widen(typename T::elem v)
{
    if constexpr (sizeof(v) == 4) return v;
    else if constexpr (std::is_same<T, F16>::value) return static_cast<float>(__builtin_bit_cast(_Float16, v));
    else return __uint_as_float(static_cast<unsigned>(v) << 16);
}

typedef unsigned short us2 __attribute__((ext_vector_type(2)));
typedef short s2 __attribute__((ext_vector_type(2)));

// Eight values: bit patterns of magnitudes (16-bit types: two to a word) reduced without unpacking them.
template <class T> struct Eight {
    static constexpr bool wide = sizeof(typename T::elem) == 4;
    static constexpr int WORDS = wide ? 8 : 4;
    unsigned w[WORDS];

    static __device__ __forceinline__ unsigned larger(unsigned a, unsigned b)
    {
        return wide ? (a > b ? a : b) : __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(us2, a), __builtin_bit_cast(us2, b)));
    }
    static __device__ __forceinline__ unsigned smaller(unsigned a, unsigned b)
    {
        return wide ? (a < b ? a : b) : __builtin_bit_cast(unsigned, __builtin_elementwise_min(__builtin_bit_cast(us2, a), __builtin_bit_cast(us2, b)));
    }
    __device__ __forceinline__ unsigned magnitude(int i) const { return w[i] & (wide ? 0x7fffffffu : 0x7fff7fffu); }
    // the largest magnitude
    __device__ __forceinline__ unsigned largest() const
    {
        unsigned m = magnitude(0);
        #pragma unroll
        for (int i = 1; i < WORDS; ++i) m = larger(m, magnitude(i));
        return wide ? m : (m >> 16 > (m & 0xffffu) ? m >> 16 : m & 0xffffu);
    }
    // the smallest magnitude that is not zero, less one (all ones: none)
    __device__ __forceinline__ unsigned smallest_less_one() const
    {
        unsigned m = ~0u;
        #pragma unroll
        for (int i = 0; i < WORDS; ++i)
            m = smaller(m, wide ? magnitude(i) - 1 : __builtin_bit_cast(unsigned, __builtin_bit_cast(us2, magnitude(i)) - us2{1, 1}));
        return wide ? m : (m >> 16 < (m & 0xffffu) ? m >> 16 : m & 0xffffu);
    }
    __device__ __forceinline__ float value(int i) const
    {
        if constexpr (wide) return __uint_as_float(w[i]);
        else return widen<T>(static_cast<uint16_t>(w[i / 2] >> (16 * (i % 2))));
    }
};

// bit pattern of a magnitude as fp32 bits
template <class T> __device__ __forceinline__ unsigned bits32(unsigned m)
{
    if constexpr (sizeof(typename T::elem) == 4) return m;
    else return __float_as_uint(widen<T>(static_cast<uint16_t>(m)));
}

// Two values as codes of value / scale in the low half of a word.
template <class T> __device__ __forceinline__ unsigned two_codes(const Eight<T> &v, int i, float scale)
{
    s2 out;
    if constexpr (Eight<T>::wide)                    out = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(s2{0, 0}, __uint_as_float(v.w[2 * i]), __uint_as_float(v.w[2 * i + 1]), scale, false);
    else if constexpr (std::is_same<T, F16>::value)  out = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(s2{0, 0}, __builtin_bit_cast(hf2, v.w[i]), scale, false);
    else                                             out = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(s2{0, 0}, __builtin_bit_cast(bf2, v.w[i]), scale, false);
    return static_cast<unsigned short>(out[0]);
}

// Codes value by value, for a thread that holds something not finite, beyond the largest stored magnitude or below half the smallest code.
template <class T> __device__ __noinline__ u2 rare_codes(const Eight<T> v, float scale)
{
    u2 code = {0, 0};
    #pragma unroll 1
    for (int i = 0; i < 8; ++i) {
        float x = v.value(0);
        #pragma unroll
        for (int j = 1; j < 8; ++j) if (j == i) x = v.value(j);
        const unsigned b = __float_as_uint(x), m = b & 0x7fffffffu, sign = b >> 24 & 0x80u;
        unsigned c;
        if (m >= 0x7f800000u) {
            c = 0x7fu | sign;
        } else {
            const float y = m > Range<T>::most ? __uint_as_float(Range<T>::most | (b & 0x80000000u)) : x;
            c = static_cast<unsigned short>(__builtin_amdgcn_cvt_scalef32_pk_fp8_f32(s2{0, 0}, y, 0.0f, scale, false)[0]) & 0xffu;
            if (m != 0 && (c & 0x7fu) == 0) c = 1u | sign;
        }
        code[i / 4] |= c << (8 * (i % 4));
    }
    return code;
}

template <class T> __global__ __launch_bounds__(kCheckpointThreads) void store_kernel(const CheckpointParams p)
{
    typedef typename T::elem elem;
    constexpr unsigned infinity = sizeof(elem) == 4 ? 0x7f800000u : std::is_same<T, F16>::value ? 0x7c00u : 0x7f80u;
    for (Walk at(p); at.row < p.rows; at.next(p)) {            // four threads of a block of 32 leave together
        const uint32_t q = at.chunk * 8;
        const elem *x = static_cast<const elem *>(p.x) + at.row * p.ldx + q;
        Eight<T> v;
        if (q + 8 <= p.cols) {
            #pragma unroll
            for (int j = 0; j < Eight<T>::WORDS / 4; ++j) {
                const u4 four = reinterpret_cast<const u4_any *>(x)[j];
                #pragma unroll
                for (int i = 0; i < 4; ++i) v.w[4 * j + i] = four[i];
            }
        } else {
            #pragma unroll
            for (int j = 0; j < Eight<T>::WORDS; ++j) {
                if constexpr (Eight<T>::wide) v.w[j] = q + j < p.cols ? __float_as_uint(x[j]) : 0u;
                else v.w[j] = (q + 2 * j < p.cols ? x[2 * j] : 0u) | (q + 2 * j + 1 < p.cols ? static_cast<unsigned>(x[2 * j + 1]) << 16 : 0u);
            }
        }
        unsigned top = v.largest();
        if (top >= infinity) {                                 // what is not finite does not count
            top = 0;
            #pragma unroll
            for (int j = 0; j < 8; ++j) {
                const unsigned m = sizeof(elem) == 4 ? v.magnitude(j) : v.magnitude(j / 2) >> (16 * (j % 2)) & 0xffffu;
                if (m < infinity && m > top) top = m;
            }
        }
        unsigned other = __shfl_xor(top, 1, 64);
        top = other > top ? other : top;
        other = __shfl_xor(top, 2, 64);
        top = bits32<T>(other > top ? other : top);
        // top = f 2^t with f in [1, 2): 448 = 1.75 * 2^8
        int e = static_cast<int>(top >> 23) - 135 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
        e = e < Range<T>::low ? Range<T>::low : e;
        const float scale = __uint_as_float(static_cast<unsigned>(e + 127) << 23);
        // 2^(e - 10) and less would round to no code at all
        const unsigned least = bits32<T>(v.smallest_less_one() + 1), half = e < -116 ? 0x00800000u : static_cast<unsigned>(e + 117) << 23;
        const bool none = v.smallest_less_one() == (sizeof(elem) == 4 ? ~0u : 0xffffu);
        u2 code;
        if (v.largest() >= infinity || top > Range<T>::most || (!none && least <= half)) {
            code = rare_codes(v, scale);
        } else {
            code = u2{two_codes(v, 0, scale) | two_codes(v, 1, scale) << 16, two_codes(v, 2, scale) | two_codes(v, 3, scale) << 16};
        }
        uint8_t *to = p.codes + at.row * p.ld_codes + q;
        if (q + 8 <= p.cols) {
            *reinterpret_cast<u2_any *>(to) = code;
        } else {
            #pragma unroll
            for (int j = 0; j < 8; ++j) if (q + j < p.cols) to[j] = static_cast<uint8_t>(code[j / 4] >> (8 * (j % 4)));
        }
        if (at.chunk % 4 == 0 && q < p.cols) p.scales[at.row * p.ld_scales + at.chunk / 4] = static_cast<uint8_t>(e + 127);
    }
}

template <class T> __global__ __launch_bounds__(kCheckpointThreads) void load_kernel(const CheckpointParams p)
{
    typedef typename T::elem elem;
    for (Walk at(p); at.row < p.rows; at.next(p)) {
        const uint32_t q = at.chunk * 8;
        if (q >= p.cols) continue;
        const uint8_t *from = p.codes + at.row * p.ld_codes + q;
        const float scale = __uint_as_float(static_cast<unsigned>(p.scales[at.row * p.ld_scales + at.chunk / 4]) << 23);
        u2 code = {0, 0};
        if (q + 8 <= p.cols) {
            code = *reinterpret_cast<const u2_any *>(from);
        } else {
            #pragma unroll
            for (int j = 0; j < 8; ++j) if (q + j < p.cols) code[j / 4] |= static_cast<unsigned>(from[j]) << (8 * (j % 4));
        }
        const u4 two = {T::codes(code.x, scale, false), T::codes(code.x, scale, true), T::codes(code.y, scale, false), T::codes(code.y, scale, true)};
        elem *x = static_cast<elem *>(p.out) + at.row * p.ldx + q;
        if constexpr (sizeof(elem) == 4) {
            #pragma unroll
            for (int j = 0; j < 8; ++j)
                if (q + j < p.cols) x[j] = __uint_as_float(j % 2 ? two[j / 2] & 0xffff0000u : two[j / 2] << 16);
        } else {
            if (q + 8 <= p.cols) {
                *reinterpret_cast<u4_any *>(x) = two;
            } else {
                #pragma unroll
                for (int j = 0; j < 8; ++j) if (q + j < p.cols) x[j] = static_cast<elem>(two[j / 2] >> (16 * (j % 2)));
            }
        }
    }
}

template <class T> hipError_t launch(hipStream_t stream, CheckpointParams p, bool load)
{
    const uint64_t chunks = p.rows * p.per_row, blocks = (chunks + kCheckpointThreads - 1) / kCheckpointThreads;
    constexpr uint64_t kMostBlocks = 1u << 20;
    const uint32_t grid = static_cast<uint32_t>(blocks < kMostBlocks ? blocks : kMostBlocks);
    const uint64_t threads = static_cast<uint64_t>(grid) * kCheckpointThreads;
    p.step_rows = threads / p.per_row;
    p.step_chunks = static_cast<uint32_t>(threads % p.per_row);
    if (load) hipLaunchKernelGGL(load_kernel<T>, dim3(grid), dim3(kCheckpointThreads), 0, stream, p);
    else      hipLaunchKernelGGL(store_kernel<T>, dim3(grid), dim3(kCheckpointThreads), 0, stream, p);
    return hipGetLastError();
}

int checkpoint(void *stream, int dtype, uint64_t rows, uint64_t cols, const void *x, uint64_t ldx, const uint8_t *codes, uint64_t ld_codes,
               const uint8_t *scales, uint64_t ld_scales, bool load, const char *what)
{
    if (dtype < 0) return set_error(COCOD_ERR_INVALID, "unknown element type %d", dtype);
    if (int rc = check_dtype(static_cast<uint32_t>(dtype))) return rc;
    const Dtype t = static_cast<Dtype>(dtype);
    const uint64_t s = dtype_bytes(t), blocks = (cols + 31) / 32;
    if (rows > kMaxRows) return set_error(COCOD_ERR_INVALID, "rows must be below 2^31");
    if (cols < 1 || cols > kMaxWidth) return set_error(COCOD_ERR_INVALID, "cols must be in 1..2^30");
    if (int rc = check_matrix("x", x, cols, ldx, s, rows)) return rc;
    if (int rc = check_matrix("codes", codes, cols, ld_codes, 1, rows)) return rc;
    if (int rc = check_matrix("scales", scales, blocks, ld_scales, 1, rows)) return rc;
    const Extent all[] = {{"x", x, matrix_bytes(rows, cols, ldx, s)}, {"codes", codes, matrix_bytes(rows, cols, ld_codes, 1)}, {"scales", scales, matrix_bytes(rows, blocks, ld_scales, 1)}};
    for (int i = 0; i < 2; ++i)
        if (int rc = check_apart(all[i], all + i + 1, 2 - i)) return rc;
    if (rows == 0) return COCOD_OK;
    const hipStream_t q = static_cast<hipStream_t>(stream);
    const OnStreamDevice device(q);
    if (device.status() != hipSuccess) return launch_status(device.status(), what);
    CheckpointParams p{};
    p.rows = rows;
    p.cols = static_cast<uint32_t>(cols);
    p.per_row = static_cast<uint32_t>(blocks * 4);
    p.x = x;
    p.out = const_cast<void *>(x);
    p.ldx = ldx;
    p.codes = const_cast<uint8_t *>(codes);
    p.scales = const_cast<uint8_t *>(scales);
    p.ld_codes = ld_codes;
    p.ld_scales = ld_scales;
    return launch_status(t == Dtype::F32 ? launch<F32>(q, p, load) : t == Dtype::BF16 ? launch<Bf16>(q, p, load) : launch<F16>(q, p, load), what);
}

}  // namespace
}  // namespace cocod

extern "C" {

int cocod_checkpoint_store(void *stream, int dtype, uint64_t rows, uint64_t cols, const void *x, uint64_t ldx, uint8_t *codes, uint64_t ld_codes,
                           uint8_t *scales, uint64_t ld_scales)
{
    return cocod::checkpoint(stream, dtype, rows, cols, x, ldx, codes, ld_codes, scales, ld_scales, false, "cocod_checkpoint_store");
}

int cocod_checkpoint_load(void *stream, int dtype, uint64_t rows, uint64_t cols, const uint8_t *codes, uint64_t ld_codes, const uint8_t *scales,
                          uint64_t ld_scales, void *x, uint64_t ldx)
{
    return cocod::checkpoint(stream, dtype, rows, cols, x, ldx, codes, ld_codes, scales, ld_scales, true, "cocod_checkpoint_load");
}

}  // extern "C"
