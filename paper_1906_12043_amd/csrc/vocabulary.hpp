// What the operators at a vocabulary share: the groups' rows and their targets, gathered copies of rows, pieces of the vocabulary.
#pragma once
#include "operator_call.hpp"
#include "product_finish.hpp"

namespace cocod {
namespace {

const Dtype kTypes[] = {Dtype::F32, Dtype::BF16, Dtype::F16};
constexpr uint32_t kPieceUnit = 256;
constexpr uint64_t kPieceElements = 1ull << 28;      // of slopes in memory at a time, unless the caller says otherwise

// Pieces of the vocabulary whose slopes are in memory at a time: whole units, of equal size unless the caller asks for one.
struct Pieces { uint64_t size; uint32_t count; };
inline Pieces pieces_of(uint32_t asked, uint64_t rows, uint32_t vocab)
{
    uint64_t piece = asked ? asked : kPieceElements / (rows ? rows : 1);
    Pieces p{};
    const uint64_t whole = (static_cast<uint64_t>(vocab) + kPieceUnit - 1) / kPieceUnit * kPieceUnit;
    piece = (piece < kPieceUnit ? kPieceUnit : piece) / kPieceUnit * kPieceUnit;
    if (piece > whole) piece = whole;
    p.count = static_cast<uint32_t>((whole + piece - 1) / piece);
    p.size = asked ? piece : (whole / kPieceUnit + p.count - 1) / p.count * kPieceUnit;      // of equal size
    p.count = static_cast<uint32_t>((whole + p.size - 1) / p.size);
    return p;
}

struct Rows {
    const int64_t *offsets;
    uint32_t groups;
    uint64_t rows;
    const int32_t *target;
    uint32_t vocab;
};

__device__ __forceinline__ uint64_t clamped(const Rows &p, uint32_t i)
{
    const int64_t v = p.offsets[i];
    return v < 0 ? 0 : static_cast<uint64_t>(v) > p.rows ? p.rows : static_cast<uint64_t>(v);
}
__device__ __forceinline__ bool has_target(const Rows &p, uint64_t r)
{
    return static_cast<uint32_t>(p.target[r]) < p.vocab;          // negative ones are large
}

// A copy of a row (pitch a multiple of 8, zeros behind dim) by the lanes of a wave.
template <class E> __device__ __forceinline__ void copy_row(const E *src, uint32_t dim, E *dst, uint64_t pitch, uint32_t lane)
{
    constexpr uint32_t V = 16 / sizeof(E);
    if ((reinterpret_cast<uintptr_t>(src) & 15) == 0 && dim % V == 0) {
        for (uint32_t j = lane * V; j < dim; j += 64 * V) *reinterpret_cast<float4 *>(dst + j) = *reinterpret_cast<const float4 *>(src + j);
        for (uint32_t j = dim + lane; j < pitch; j += 64) dst[j] = 0;
    } else {
        for (uint32_t j = lane; j < pitch; j += 64) dst[j] = j < dim ? src[j] : E(0);
    }
}

}  // namespace
}  // namespace cocod
