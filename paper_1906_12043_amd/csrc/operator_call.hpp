// What the calls without a context share: checks of arguments, the device of a stream.
#pragma once
#include "../../include/cocod.h"
#include "internal.hpp"
#include "product.hpp"

namespace cocod {

constexpr uint64_t kMaxPitch = 1ull << 30;           // elements between rows; with 2^31 rows byte extents stay below 2^63
constexpr uint64_t kMaxGroupStride = 1ull << 44;     // elements between groups
constexpr uint32_t kMaxGroups = 65535;
constexpr uint64_t kMaxRows = (1ull << 31) - 1;
constexpr uint32_t kMaxWidth = 1u << 30;

// Makes the stream's device current for the calls of one scope (the null stream belongs to the current one).
class OnStreamDevice {
public:
    explicit OnStreamDevice(hipStream_t stream)
    {
        int own = 0;
        if (!stream || hipStreamGetDevice(stream, &own) != hipSuccess || hipGetDevice(&before_) != hipSuccess) { before_ = -1; return; }
        if (own == before_) before_ = -1;
        else status_ = hipSetDevice(own);
    }
    ~OnStreamDevice() { if (before_ >= 0) (void)hipSetDevice(before_); }
    hipError_t status() const { return status_; }

private:
    int before_ = -1;
    hipError_t status_ = hipSuccess;
};

struct Extent { const char *name; const void *ptr; uint64_t bytes; };

inline uint64_t matrix_bytes(uint64_t rows, uint64_t cols, uint64_t ld, uint64_t size) { return rows == 0 ? 0 : ((rows - 1) * ld + cols) * size; }
inline uint64_t stack_bytes(uint64_t groups, uint64_t stride, uint64_t rows, uint64_t cols, uint64_t ld, uint64_t size)
{
    return (groups - 1) * stride * size + matrix_bytes(rows, cols, ld, size);
}

// A matrix argument: not NULL (unless it has no rows), aligned to its elements, rows that do not run into each other.
inline int check_matrix(const char *name, const void *ptr, uint64_t cols, uint64_t ld, uint64_t size, uint64_t rows = 1)
{
    if (!ptr && !rows) return COCOD_OK;
    if (!ptr) return set_error(COCOD_ERR_INVALID, "%s is NULL", name);
    if (reinterpret_cast<uintptr_t>(ptr) % size) return set_error(COCOD_ERR_INVALID, "%s is not aligned to its elements", name);
    if (ld < cols || ld > kMaxPitch) return set_error(COCOD_ERR_INVALID, "rows of %s: pitch %llu, must be in %llu .. 2^30", name, (unsigned long long)ld, (unsigned long long)cols);
    return COCOD_OK;
}
// One matrix per group; stride 0 (shared by all groups) only where `shared` allows it.
inline int check_stride(const char *name, uint64_t stride, uint32_t groups, uint64_t rows, uint64_t cols, uint64_t ld, bool shared)
{
    if (stride > kMaxGroupStride) return set_error(COCOD_ERR_INVALID, "%s: more than 2^44 elements between groups", name);
    if (groups > 1 && !(shared && stride == 0) && stride < (rows - 1) * ld + cols)
        return set_error(COCOD_ERR_INVALID, "%s: %llu elements between groups, the matrices overlap", name, (unsigned long long)stride);
    return COCOD_OK;
}

// An output must not touch any other argument.
inline int check_apart(const Extent &out, const Extent *others, int n)
{
    const uintptr_t o = reinterpret_cast<uintptr_t>(out.ptr);
    for (int i = 0; i < n; ++i) {
        const uintptr_t q = reinterpret_cast<uintptr_t>(others[i].ptr);
        if (!out.ptr || !others[i].ptr || !out.bytes || !others[i].bytes) continue;
        if (o < q + others[i].bytes && q < o + out.bytes) return set_error(COCOD_ERR_INVALID, "%s and %s overlap", out.name, others[i].name);
    }
    return COCOD_OK;
}

inline int check_dtype(uint32_t dtype)
{
    return dtype <= COCOD_F16 ? COCOD_OK : set_error(COCOD_ERR_INVALID, "unknown element type %u", dtype);
}

// What cocod_debug_*_plan says of a product that runs with these parameters.
inline cocod_product_plan plan_as_run(Dtype type, Layout layout, Tile tile, uint32_t splits, const ProductParams &p)
{
    const bool direct_b_too = type != Dtype::F32 && direct_b(layout, p);
    return {static_cast<uint32_t>(tile), splits, !p.a ? 2u : direct_b_too && direct_a(layout, p) ? 0u : 1u};
}

inline int launch_status(hipError_t e, const char *what)
{
    if (e == hipSuccess) return COCOD_OK;
    if (e == hipErrorInvalidConfiguration) return set_error(COCOD_ERR_UNSUPPORTED, "%s: more tiles than one launch holds", what);
    return set_error(COCOD_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace cocod
