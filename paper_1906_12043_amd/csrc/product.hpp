// Parameters and launcher of the grouped matrix products (product_tiles.hpp holds the kernels).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cocod {

constexpr uint32_t kNoRow = ~0u;

// Element types, in the order of cocod_dtype.
enum class Dtype : uint32_t { F32 = 0, BF16 = 1, F16 = 2 };
inline uint64_t dtype_bytes(Dtype t) { return t == Dtype::F32 ? 4 : 2; }

// C = A B by group.  The kinds differ in which axis is ragged and in how the operands lie in memory:
//   Rows_KN  C[r][n] = sum_k A[r][k] B_g[k][n]    forward; gradient of the hidden states of the loss
//   Rows_NK  C[r][n] = sum_k A[r][k] B_g[n][k]    gradient of the input; logits
//   Weights  C_g[m][n] = sum_r A[r][m] B[r][n]    gradient of the weights: the ragged axis is summed over
// with r running over the rows offsets[g] .. offsets[g + 1] - 1.
enum class Layout { Rows_KN, Rows_NK, Weights };

// What becomes of a tile of C.
enum class Finish {
    Store,       // relu, mask, scale, running sum; store in the element type or fp32
    Stats,       // logits: maximum and sum of exponentials of the tile's part of every row but its target, and the target's logit
    Keep,        //   the same, and the exponentials stored (bf16: in fp16 times 2^14; pitch and columns to the end of the last tile are the buffer's)
    Slope        // logits: softmax minus one-hot, stored in the element type
};

struct ProductParams {
    const void *a;                    // [rows][lda] elements of the type; nullptr: codes and scales below
    uint64_t lda;
    const uint8_t *a_codes, *a_scales;
    uint64_t ld_codes, ld_scales;
    const void *b;
    uint64_t ldb, b_group;            // b_group: elements between the groups' matrices (Rows_*)
    const int64_t *offsets;           // device [groups + 1]; values outside 0 .. rows are taken as the nearer end
    const int64_t *ends;              // non-null: group g ends at row ends[g], not where the next one begins
    uint32_t groups;
    uint64_t rows;                    // bound of the ragged axis
    uint32_t m;                       // Weights: rows of C_g
    uint32_t n;                       // columns of C
    uint32_t k;                       // Rows_*: terms of a sum
    uint32_t a_zero_padded;           // A holds zeros from column k to the next multiple of 8
    void *out;
    uint64_t ldc, out_group;          // out_group: Weights
    uint32_t out_f32;                 // C is stored in fp32 whatever the element type
    const uint32_t *out_row;          // non-null: row r of C is stored at row out_row[r] (kNoRow: not at all)
    uint32_t relu;
    const void *mask;                 // non-null: C is zero where mask[r][n] (or the code) is not above zero
    const uint8_t *mask_codes;
    uint64_t ld_mask;
    float scale;                      // C is multiplied by it
    const float *row_scale;           // Rows_*, non-null: or by this, row by row
    uint32_t mean;                    // Weights: C is divided by the group's number of rows (no rows: C is zero)
    float *sum;                       // non-null: fp32 [rows][ld_sum], C so far (before the scale);
    uint64_t ld_sum;
    uint32_t sum_read, sum_write;     //   C is added to it / stays there and is not stored to out
    float *part;                      // splits > 1: fp32 [splits][rows of all groups][ld_part]
    uint64_t ld_part;
    uint32_t splits;
    // logits
    const int32_t *target;            // [rows]
    float2 *stats;                    // [column tiles][rows]: maximum, sum of exponentials, of all but the target
    float *target_logit;              // [rows]
    const float *top, *inverse;       // [rows]: largest logit; 1 / sum of the exponentials below it
    const float *target_slope;        // [rows]: probability of the target, less one
    uint32_t v0;                      // vocabulary entry of column 0
    uint32_t ldc_zero;                // Slope: columns up to here are stored, those from n on as zeros
};

// Tile shapes a launch can take (plan_product picks one).
enum class Tile : uint32_t { Large = 0, Medium = 1, Small = 2, Deep = 3, Tall = 4, Square = 5 };

// C = A B, stored (Finish::Store) or as logits (Rows_NK with Finish::Stats, Keep or Slope), one launch, with splits one more that joins
// them.  hipErrorInvalidConfiguration: the grid would exceed a launch's limits.
hipError_t launch_store_bf16(hipStream_t stream, Layout layout, Tile tile, const ProductParams &p);
hipError_t launch_store_f16(hipStream_t stream, Layout layout, Tile tile, const ProductParams &p);
hipError_t launch_store_f32(hipStream_t stream, Layout layout, Tile tile, const ProductParams &p);
hipError_t launch_logits_bf16(hipStream_t stream, Finish finish, Tile tile, const ProductParams &p);
hipError_t launch_logits_f16(hipStream_t stream, Finish finish, Tile tile, const ProductParams &p);
hipError_t launch_logits_f32(hipStream_t stream, Finish finish, Tile tile, const ProductParams &p);

// Rows, columns and threads of a tile as it runs (product_tiles.hpp asserts them), and whether a launch holds all tiles of a product.
struct TileSize { uint32_t bm, bn, threads; };
constexpr TileSize tile_size(Dtype type, Tile tile)
{
    return tile == Tile::Small ? TileSize{32, 64, 256} : tile == Tile::Square ? TileSize{64, 64, 256} : type == Dtype::F32 ? TileSize{128, 128, 512}
           : tile == Tile::Large ? TileSize{256, 256, 512} : tile == Tile::Tall ? TileSize{192, 128, 512} : TileSize{128, 128, tile == Tile::Deep ? 512u : 256u};
}
inline uint64_t blocks_of(const TileSize &t, bool weights, uint64_t rows, uint32_t groups, uint32_t m, uint32_t n, uint32_t splits)
{
    // of the rows, a tile begun per group
    const uint64_t row_tiles = weights ? static_cast<uint64_t>(groups) * ((m + t.bm - 1) / t.bm) : rows / t.bm + groups;
    return row_tiles * ((n + t.bn - 1) / t.bn) * splits;
}
inline bool fits_a_launch(const TileSize &t, uint64_t blocks) { return blocks * t.threads < (1ull << 32); }

// Columns of the tiles in which Finish::Stats forms its statistics (ProductParams::stats holds one row of them per column tile).
inline uint32_t tile_cols(Dtype type, Tile tile)
{
    return tile_size(type, tile).bn;
}

// 16-bit operands that start on a 16-byte address, with rows of whole 16-byte pieces, go to LDS without passing through registers.
inline bool direct_operand(const void *base, uint64_t ld, uint64_t group, bool whole)
{
    return (reinterpret_cast<uintptr_t>(base) & 15) == 0 && ld % 8 == 0 && group % 8 == 0 && ld <= (1u << 22) && whole;
}
inline bool direct_a(Layout layout, const ProductParams &p)
{
    return p.a && direct_operand(p.a, p.lda, 0, layout == Layout::Weights || p.k % 8 == 0 || p.a_zero_padded);
}
inline bool direct_b(Layout layout, const ProductParams &p)
{
    return direct_operand(p.b, p.ldb, layout == Layout::Weights ? 0 : p.b_group, layout != Layout::Rows_NK || p.k % 8 == 0);
}
// The tile that a launch takes where `planned` was planned: the large, the deep and the tall one need operands that go to LDS directly (the large
// one also takes codes).
inline Tile settle_tile(Dtype type, Layout layout, Tile planned, const ProductParams &p)
{
    if ((planned == Tile::Deep || planned == Tile::Tall) && (type == Dtype::F32 || !direct_a(layout, p) || !direct_b(layout, p))) return Tile::Medium;
    return planned == Tile::Large && (type == Dtype::F32 || (p.a && !direct_a(layout, p)) || !direct_b(layout, p)) ? Tile::Medium : planned;
}

// Tile and splits of a product, from its sizes alone; direct: 16-bit operands are expected to go to LDS directly; stored: Finish::Store.
struct ProductPlan { Tile tile; uint32_t splits; };
ProductPlan plan_product(Layout layout, Dtype type, bool direct, uint64_t rows, uint32_t groups, uint32_t m, uint32_t n, uint32_t k, bool may_split,
                         bool stored = true);
// Bytes of ProductParams::part (0 with one split), whose rows hold part_pitch(n) floats.
inline uint64_t part_pitch(uint32_t n) { return (static_cast<uint64_t>(n) + 3) / 4 * 4; }
uint64_t part_bytes(const ProductPlan &plan, Layout layout, uint64_t rows, uint32_t groups, uint32_t m, uint32_t n);
hipError_t launch_join(hipStream_t stream, Dtype type, Layout layout, const ProductParams &p);

inline hipError_t launch_store(hipStream_t stream, Dtype type, Layout layout, Tile tile, const ProductParams &p)
{
    const hipError_t e = type == Dtype::BF16 ? launch_store_bf16(stream, layout, tile, p)
                         : type == Dtype::F16 ? launch_store_f16(stream, layout, tile, p) : launch_store_f32(stream, layout, tile, p);
    return e != hipSuccess || p.splits <= 1 ? e : launch_join(stream, type, layout, p);
}
inline hipError_t launch_logits(hipStream_t stream, Dtype type, Finish finish, Tile tile, const ProductParams &p)
{
    return type == Dtype::BF16 ? launch_logits_bf16(stream, finish, tile, p)
           : type == Dtype::F16 ? launch_logits_f16(stream, finish, tile, p) : launch_logits_f32(stream, finish, tile, p);
}

}  // namespace cocod
