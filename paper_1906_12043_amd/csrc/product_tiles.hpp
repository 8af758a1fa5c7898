// Grouped matrix products on the matrix cores: C = A B for every group of a ragged batch, one launch for all groups.
//
// A block computes a BM x BN tile of C.  Slices of BK terms of both operands pass through LDS, several on their way at a time, one meeting of the
// waves per slice.  The matrix instruction, 32x32x16 or 16x16x32, has the operands exchanged (C^T = B^T A^T), so that a lane holds one row of C and runs of four
// consecutive columns of it.
//
// What bounds it: long sums the chip's power (8 groups of 8192 rows, 4096 x 4096 bf16: forward 1796 us, 1.22 PFLOP/s; with
// 32x32x16 1.14 at 1.75 GHz, without loads to LDS 1.41, without reads from it 1.40, without both 1.94 PFLOP/s), short ones the start and end
// of blocks and the latency of slices out of memory, few rows the stream of the weights (16 matrices of 1024 x 1024, a row each: 9.4 us,
// 3.6 TB/s).
//
// In LDS an operand lies as it does in memory: with the summed axis contiguous ([BX][BK], read as 16-byte pieces of eight
// terms) or with the other axis contiguous ([BK][BX], read by the transposing 8-byte LDS loads, which give a lane four
// terms of one column).  16-byte chunks are permuted inside a row so that the lanes of one read hit all banks.
#pragma once
#include "product_finish.hpp"

namespace cocod {
namespace {

constexpr uint32_t kXcdCount = 8;
constexpr uint32_t kBandTiles = 8;                   // row tiles that take turns in front of one column tile

// Largest factor of softmax minus one-hot kept in the element type: fp16 would lose probabilities below 2^-24.
template <class T> constexpr float slope_scale() { return std::is_same<T, F16>::value ? 0x1p14f : 1.0f; }

template <int BM_, int BN_, int BK_, int WM_, int WN_, int WK_, int STAGES_ = 2, int MI_ = 32, bool ONCE_ = false> struct TileShape {
    static constexpr bool ONCE = ONCE_;              // what a block reads of B is not read again soon: past the caches
    static constexpr int STAGES = STAGES_;           // slices in LDS
    static constexpr int MI = MI_, MK = MI == 32 ? 16 : 32, X = MI * MI / 64;        // the matrix instruction: MI x MI x MK, X values a lane
    static constexpr int BM = BM_, BN = BN_, BK = BK_, WM = WM_, WN = WN_, WK = WK_;
    static constexpr int threads = 64 * WM * WN * WK;
    static constexpr int MB = BM / WM / MI, NB = BN / WN / MI;       // blocks of a wave
};

// How a tile of [ROWS][COLS] 16-bit elements lies in LDS.  KC: the summed axis is the contiguous one.
template <bool KC, int BX, int BK> struct LdsTile {
    static constexpr int ROWS = KC ? BX : BK, COLS = KC ? BK : BX, CH = COLS / 8;
    static constexpr int bytes = ROWS * COLS * 2;
    static __device__ __forceinline__ uint32_t swizzle(uint32_t row)
    {
        if (KC) return CH >= 16 ? row & 15 : CH == 8 ? (row >> 1) & 7 : (row >> 2) & 3;      // sixteen rows of one chunk: sixteen places
        return CH >= 16 ? (row & 3) << 2 : CH == 8 ? (row & 2) << 1 : 0;
    }
    // eight terms k0 + 8 (lane / MI) .. of the element x0 + lane % MI of the other axis
    template <int MI> static __device__ __forceinline__ u4 fragment(const uint8_t *lds, uint32_t x0, uint32_t k0, uint32_t lane)
    {
        if constexpr (KC) {
            const uint32_t row = x0 + lane % MI, c = k0 / 8 + lane / MI;
            return *reinterpret_cast<const u4 *>(lds + row * (COLS * 2) + ((c ^ swizzle(row)) * 16));
        } else {
            const uint32_t i = lane % 16, row = k0 + 8 * (lane / MI) + i / 4, c = (x0 + (lane % MI - i)) / 8 + (i % 4) / 2;
            const uint8_t *at = lds + row * (COLS * 2) + ((c ^ swizzle(row)) * 16) + (i % 2) * 8;
            union { s4 h[2]; u4 v; } out;
            out.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)at);
            out.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)(at + 4 * COLS * 2));
            return out.v;
        }
    }
};

__device__ __forceinline__ u4 zero4() { return u4{0, 0, 0, 0}; }

// How an operand gets from memory into LDS: 16-byte pieces that the loads themselves put there; through registers, with any alignment and any
// type; or as codes of 8 bits with a scale for every 32, expanded on the way.
enum { kDirect = 0, kRegs = 1, kCodes = 2 };
__device__ __attribute__((aligned(16))) const unsigned int kZeroChunk[4] = {0, 0, 0, 0};

template <class T, int HOW, bool KC, int BX, int BK, int THREADS, bool PAST = false> struct Loader {
    typedef LdsTile<KC, BX, BK> L;
    typedef typename T::elem elem;
    static constexpr int planes = HOW == kCodes ? 1 : T::planes;
    static constexpr int CHUNKS = L::ROWS * L::CH / THREADS;        // 16-byte chunks of LDS per thread
    static_assert(CHUNKS >= 1 && CHUNKS * THREADS == L::ROWS * L::CH, "whole chunks per thread");
    static constexpr int W = HOW == kCodes && CHUNKS % 2 == 0 ? 2 : 1;   // chunks per load: sixteen codes are two
    static constexpr int N = CHUNKS / W;                            // loads per thread
    static constexpr int bytes = planes * L::bytes;
    static constexpr int RAW = HOW == kDirect ? 1 : (sizeof(elem) == 4 && HOW == kRegs ? 2 : 1);

    const elem *src;                  // element (0, 0) of the operand's matrix of this group
    uint64_t ld;
    const uint8_t *codes, *scales;
    uint64_t ld_codes, ld_scales;
    uint32_t x0, x_end;               // the other axis: first element of the tile, end
    uint32_t k_end;                   // end of the summed axis
    u4 raw[HOW == kDirect ? 1 : N][RAW];
    float sc[HOW == kCodes ? N : 1];
    uint32_t off[N], scale_off[HOW == kCodes ? N : 1];      // of a thread's chunks in a slice (bytes / elements / codes; scales)

    uint32_t down[HOW != kDirect && !KC ? N : 1];           // elements by which a load of a cut chunk lies too far back
    bool fits;                        // slices within the sum can be loaded without checks
    bool cut;                         // some chunk is cut
    bool moved = false;               //   and the requested slice was loaded that way

    // load i of this thread: row of the tile, first chunk (pairs of chunks stay side by side in LDS)
    __device__ __forceinline__ static uint32_t row_of(int i) { return (i * THREADS + threadIdx.x) / (L::CH / W); }
    __device__ __forceinline__ static uint32_t place_of(int i) { return (i * THREADS + threadIdx.x) * W; }
    __device__ __forceinline__ static uint32_t chunk_of(int i) { return (place_of(i) % L::CH) ^ L::swizzle(row_of(i)); }
    static_assert(W == 1 || !KC, "the permutation of whole pairs");

    __device__ __forceinline__ void start()
    {
        // Rows past the end repeat the last one, chunks of columns past the end the last one: their products are not stored.  A chunk that
        // the end of a row cuts is loaded from as far back as it has to and moved down on its way to LDS (direct: it is read to its
        // end, which lies within the pitch).
        const uint64_t pitch = HOW == kCodes ? ld_codes : ld;
        constexpr uint32_t E = 8 * W;
        fits = HOW == kDirect || ((KC || x_end >= E) && pitch <= (1u << 22) && (HOW != kCodes || ld_scales <= (1u << 22)));
        cut = HOW != kDirect && !KC && x0 + BX > x_end;
        #pragma unroll
        for (int i = 0; i < N; ++i) {
            uint32_t row = row_of(i), q = chunk_of(i) * 8, back = 0;
            if (KC) {
                const uint32_t last = x_end - 1 - x0;
                row = row < last ? row : last;
            } else if (HOW == kDirect) {
                const uint32_t last = (x_end - 1 - x0) / 8 * 8;
                q = q < last ? q : last;
            } else {
                if constexpr (HOW == kCodes) {
                    static_assert(BX % 32 == 0, "codes of whole blocks, rows summed over");
                    const uint32_t last = x_end - 1 - x0;
                    scale_off[i] = row * static_cast<uint32_t>(ld_scales) + (q < last ? q : last) / 32;
                }
                if (x0 + q + E > x_end) back = x0 + q + E - x_end;
                down[i] = back < E ? back : 0;
            }
            off[i] = (row * static_cast<uint32_t>(pitch) + q - back) * (HOW == kDirect ? 2 : 1);
        }
    }

    // request the slice that begins at term k0, zeros behind the sum's end
    __device__ __forceinline__ void request(uint8_t *lds, uint32_t k0, uint32_t wave)
    {
        if constexpr (HOW == kDirect) {
            const char *base = reinterpret_cast<const char *>(src) + 2 * (KC ? static_cast<uint64_t>(x0) * ld + k0 : static_cast<uint64_t>(k0) * ld + x0);
            #pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t row = row_of(i), c = chunk_of(i);
                const char *from = k0 + (KC ? c * 8 : row) < k_end ? base + off[i] : reinterpret_cast<const char *>(kZeroChunk);
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                                 (__attribute__((address_space(3))) void *)(lds + (i * THREADS + wave * 64) * 16), 16, 0, PAST ? 2 : 0);
            }
        } else {
            moved = false;
            #pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t row = row_of(i), c = chunk_of(i);
                const uint32_t r = (KC ? x0 : k0) + row, r_end = KC ? x_end : k_end, q = (KC ? k0 : x0) + c * 8, q_end = KC ? k_end : x_end;
                #pragma unroll
                for (int j = 0; j < RAW; ++j) raw[i][j] = zero4();
                if constexpr (HOW == kCodes) sc[i] = 1.0f;
                if (r < r_end && q < q_end) {
                    if constexpr (HOW == kCodes) {
                        const uint8_t *at = codes + r * ld_codes + q;
                        sc[i] = __uint_as_float(static_cast<unsigned>(scales[r * ld_scales + q / 32]) << 23);
                        u4 v = zero4();
                        #pragma unroll
                        for (int e = 0; e < 8 * W; ++e)
                            if (q + e < q_end) v[e / 4] |= static_cast<unsigned>(at[e]) << (8 * (e % 4));
                        raw[i][0] = v;
                    } else {
                        const elem *at = src + r * ld + q;
                        if (q + 8 <= q_end) {
                            #pragma unroll
                            for (int j = 0; j < RAW; ++j) raw[i][j] = reinterpret_cast<const u4_any *>(at)[j];
                        } else {
                            #pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (q + e < q_end) {
                                    if constexpr (sizeof(elem) == 4) raw[i][e / 4][e % 4] = __float_as_uint(at[e]);
                                    else                             raw[i][0][e / 2] |= static_cast<unsigned>(at[e]) << (16 * (e % 2));
                                }
                        }
                    }
                }
            }
        }
    }

    // a slice that lies within the sum, of an operand that fits: nothing to check
    __device__ __forceinline__ void request_whole(uint8_t *lds, uint32_t k0, uint32_t wave)
    {
        if constexpr (HOW == kDirect) {
            const char *base = reinterpret_cast<const char *>(src) + 2 * (KC ? static_cast<uint64_t>(x0) * ld + k0 : static_cast<uint64_t>(k0) * ld + x0);
            #pragma unroll
            for (int i = 0; i < N; ++i)
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(base + off[i]),
                                                 (__attribute__((address_space(3))) void *)(lds + (i * THREADS + wave * 64) * 16), 16, 0, PAST ? 2 : 0);
        } else {
            const uint64_t r = KC ? x0 : k0, q = KC ? k0 : x0;
            #pragma unroll
            for (int i = 0; i < N; ++i) {
                if constexpr (HOW == kCodes) {
                    const uint8_t *at = codes + r * ld_codes + q + static_cast<int32_t>(off[i]);
                    if constexpr (W == 2) {
                        raw[i][0] = *reinterpret_cast<const u4_bytes *>(at);
                    } else {
                        const u2 v = *reinterpret_cast<const u2_any *>(at);
                        raw[i][0] = u4{v.x, v.y, 0, 0};
                    }
                    sc[i] = __uint_as_float(static_cast<unsigned>((scales + r * ld_scales + q / 32)[scale_off[i]]) << 23);
                } else {
                    #pragma unroll
                    for (int j = 0; j < RAW; ++j) raw[i][j] = reinterpret_cast<const u4_any *>(src + r * ld + q + static_cast<int32_t>(off[i]))[j];
                }
            }
            moved = cut;
        }
    }

    // the elements of load i by down[i] towards the first
    __device__ __forceinline__ void move_down(int i)
    {
        constexpr int SIZE = HOW == kCodes ? 1 : sizeof(elem), WORDS = 8 * W * SIZE / 4;
        unsigned w[WORDS + 1];
        #pragma unroll
        for (int j = 0; j < WORDS; ++j) w[j] = raw[i][j / 4][j % 4];
        w[WORDS] = 0;
        const uint32_t bytes = down[i] * SIZE;
        #pragma unroll
        for (int step = 1; step < WORDS; step <<= 1)
            #pragma unroll
            for (int j = 0; j < WORDS; ++j) w[j] = bytes & (4 * step) ? (j + step < WORDS ? w[j + step] : 0) : w[j];
        if constexpr (SIZE < 4) {
            #pragma unroll
            for (int j = 0; j < WORDS; ++j) w[j] = __builtin_amdgcn_alignbyte(w[j + 1], w[j], bytes & 3);
        }
        #pragma unroll
        for (int j = 0; j < WORDS; ++j) raw[i][j / 4][j % 4] = w[j];
    }

    __device__ __forceinline__ void ask(uint8_t *lds, uint32_t k0, uint32_t wave)
    {
        if (fits && k0 + BK <= k_end) request_whole(lds, k0, wave);
        else                          request(lds, k0, wave);
    }

    // put the requested slice into LDS
    __device__ __forceinline__ void deliver(uint8_t *lds)
    {
        if constexpr (HOW == kDirect) return;
        if constexpr (HOW != kDirect && !KC) {
            if (moved) {
                #pragma unroll
                for (int i = 0; i < N; ++i) move_down(i);
            }
        }
        #pragma unroll
        for (int i = 0; i < N; ++i) {
            uint8_t *at = lds + place_of(i) * 16;
            if constexpr (HOW == kCodes) {
                #pragma unroll
                for (int w = 0; w < W; ++w)
                    reinterpret_cast<u4 *>(at)[w] = u4{T::codes(raw[i][0][2 * w], sc[i], false), T::codes(raw[i][0][2 * w], sc[i], true),
                                                       T::codes(raw[i][0][2 * w + 1], sc[i], false), T::codes(raw[i][0][2 * w + 1], sc[i], true)};
            } else if constexpr (T::planes == 1) {
                *reinterpret_cast<u4 *>(at) = raw[i][0];
            } else {
                u4 p[3];
                #pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float a = __uint_as_float(raw[i][j / 2][2 * j % 4]) * kPlaneScale, b = __uint_as_float(raw[i][j / 2][2 * j % 4 + 1]) * kPlaneScale;
                    #pragma unroll
                    for (int pl = 0; pl < 3; ++pl) {
                        const unsigned pair = T::pack(a, b);
                        p[pl][j] = pair;
                        a -= __uint_as_float(pair << 16);
                        b -= __uint_as_float(pair & 0xffff0000u);
                    }
                }
                #pragma unroll
                for (int pl = 0; pl < 3; ++pl) *reinterpret_cast<u4 *>(at + pl * L::bytes) = p[pl];
            }
        }
    }

    // element (x of the other axis, term k) in fp32, zero outside (the exact path for sums that are not finite)
    __device__ __forceinline__ float element(uint32_t x, uint32_t k) const
    {
        if (x >= x_end || k >= k_end) return 0.0f;
        const uint64_t r = KC ? x : k, q = KC ? k : x;
        if constexpr (HOW == kCodes)
            return __uint_as_float(T::codes(codes[r * ld_codes + q], __uint_as_float(static_cast<unsigned>(scales[r * ld_scales + q / 32]) << 23), false) << 16);
        else
            return static_cast<float>(src[r * ld + q]);
    }
};

// Where a block's tile lies.
struct Place { uint32_t group; uint32_t n0; uint64_t row0; uint32_t rows; uint32_t m0; uint32_t terms; uint32_t split; };

// Blocks go round the eight dies in turn: each die gets a run of consecutive tiles (of one split after another), which share operands
// in its cache.  In a band of row tiles the row tiles take turns in front of one column tile.
__device__ __forceinline__ bool tile_of_block(uint32_t row_tiles, uint32_t col_tiles, uint32_t splits, uint32_t &row_tile, uint32_t &col_tile, uint32_t &split)
{
    const uint32_t tiles = row_tiles * col_tiles, total = tiles * splits;
    if (blockIdx.x >= total) return false;
    const uint32_t x = blockIdx.x % kXcdCount, q = total / kXcdCount, r = total % kXcdCount;
    uint32_t idx = x * q + (x < r ? x : r) + blockIdx.x / kXcdCount;
    split = idx / tiles;
    idx -= split * tiles;
    const uint32_t band = idx / (kBandTiles * col_tiles), in = idx - band * kBandTiles * col_tiles;
    const uint32_t left = row_tiles - band * kBandTiles, high = left < kBandTiles ? left : kBandTiles;
    row_tile = band * kBandTiles + in % high;
    col_tile = in / high;
    return true;
}

// The row tiles of all groups in order; every wave scans the groups' lengths for itself, 64 at a time.
template <int BM> __device__ __forceinline__ bool place_rows(const ProductParams &p, uint32_t col_tiles, Place &at, int BN)
{
    const uint32_t lane = threadIdx.x % 64;
    uint32_t total = 0, incl = 0, tiles = 0;
    uint64_t first = 0, len = 0;
    auto scan = [&](uint32_t g0) {
        const uint32_t g = g0 + lane;
        first = 0; len = 0;
        if (g < p.groups) { first = bound_at(p, g); len = length_at(p, g); }
        tiles = static_cast<uint32_t>((len + BM - 1) / BM);
        incl = tiles;
        #pragma unroll
        for (int d = 1; d < 64; d <<= 1) { const uint32_t v = __shfl_up(incl, d, 64); if (lane >= static_cast<uint32_t>(d)) incl += v; }
        return __shfl(incl, 63, 64);
    };
    for (uint32_t g0 = 0; g0 < p.groups; g0 += 64) total += scan(g0);
    uint32_t row_tile, col_tile;
    if (!tile_of_block(__builtin_amdgcn_readfirstlane(total), col_tiles, p.splits, row_tile, col_tile, at.split)) return false;
    uint32_t g0 = 0;
    if (p.groups > 64)
        for (;; g0 += 64) {
            if (g0 >= p.groups) return false;                  // offsets that do not ascend
            const uint32_t n = scan(g0);
            if (row_tile < n) break;
            row_tile -= n;
        }
    const unsigned long long beyond = __ballot(incl > row_tile);
    if (!beyond) return false;
    const uint32_t who = __ffsll(beyond) - 1;
    const uint32_t tile = row_tile - (__shfl(incl, who, 64) - __shfl(tiles, who, 64));
    at.group = __builtin_amdgcn_readfirstlane(g0 + who);
    const uint64_t f = __shfl(first, who, 64), l = __shfl(len, who, 64);
    const uint64_t r0 = f + static_cast<uint64_t>(tile) * BM, left = f + l - r0;
    at.row0 = (static_cast<uint64_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(r0 >> 32))) << 32) | __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(r0));
    at.rows = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(left < BM ? left : BM));
    at.n0 = col_tile * BN;
    at.m0 = 0;
    at.terms = p.k;
    return true;
}

template <int BM> __device__ __forceinline__ bool place_weights(const ProductParams &p, uint32_t col_tiles, Place &at, int BN)
{
    const uint32_t per = (p.m + BM - 1) / BM;
    uint32_t row_tile, col_tile;
    if (!tile_of_block(per * p.groups, col_tiles, p.splits, row_tile, col_tile, at.split)) return false;
    at.group = row_tile / per;
    at.m0 = row_tile % per * BM;
    at.rows = p.m - at.m0 < BM ? p.m - at.m0 : BM;
    at.n0 = col_tile * BN;
    at.row0 = bound_at(p, at.group);
    at.terms = static_cast<uint32_t>(length_at(p, at.group));
    return true;
}

// ---- the kernel ---------------------------------------------------------------------------------------------

// All but the last LEFT requests of every wave have arrived in LDS, and every wave has the fragments it has read.
template <int LEFT> __device__ __forceinline__ void slices_arrived()
{
    static_assert(LEFT < 64, "the wait's counter");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LEFT) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <class T, Layout LAYOUT, class S, int HOW_A, int HOW_B> struct Product {
    static constexpr bool WEIGHTS = LAYOUT == Layout::Weights;
    static constexpr bool A_KC = !WEIGHTS, B_KC = LAYOUT == Layout::Rows_NK;
    typedef Loader<T, HOW_A, A_KC, S::BM, S::BK, S::threads> LoadA;
    typedef Loader<T, HOW_B, B_KC, S::BN, S::BK, S::threads, S::ONCE> LoadB;
    static constexpr int PA = LoadA::planes, PB = LoadB::planes, SUMS = PB == 1 ? 1 : 2;
    static constexpr int stage = LoadA::bytes + LoadB::bytes;
    static constexpr int join_bytes = S::WK > 1 ? S::WK * S::BM * (S::BN + 4) * 4 : S::threads / 64 * S::MI * (S::NB * S::MI + 4) * 4;
    static constexpr int ST = S::STAGES, REQUESTS = LoadA::N + LoadB::N;
    static_assert(ST == 2 || (HOW_A == kDirect && HOW_B == kDirect), "operands in registers hold one slice");
    static constexpr int lds_bytes = ST * stage > join_bytes ? ST * stage : join_bytes;

    // The pipeline.  While the matrix cores work on one part of a step of MK terms (times WK), the fragments of the next part are read: of B
    // those of a step, of A those of PARTS of its row blocks, two where all of them twice would not leave registers for the sums.  In front of a
    // slice's last part all waves meet: their last fragments of the slice are in registers, so its buffer takes the slice STAGES
    // further on, which then has the time of STAGES - 1 slices to arrive; and the next slice, requested that long ago, is there, so that its first
    // fragments are read beside the last part's products.  An operand that passes through registers is requested at the same place and
    // put into LDS a part before the waves meet.
    typedef typename std::conditional<S::MI == 32, f16v, f4>::type Block;
    typedef Block Sums[SUMS][S::MB][S::NB];
    static constexpr int STEPS = S::BK / S::MK / S::WK;
    static constexpr int PARTS = SUMS * S::MB * S::NB * S::X + 8 * (PA * S::MB + PB * S::NB) > 192 ? 2 : 1, MP = S::MB / PARTS, LAST = STEPS * PARTS - 1;
    static_assert(STEPS % 2 == 0 && S::MB % PARTS == 0, "the first fragments of a slice are always the same registers'");
    // where both operands pass through registers, these are free for the next request as soon as they are in LDS
    static constexpr bool EARLY = HOW_A != kDirect && HOW_B != kDirect;
    struct Fragments { u4 a[2][PA][MP], b[2][PB][S::NB]; };

    // the fragments of part kk
    template <int kk> static __device__ __forceinline__ void read(Fragments &f, const uint8_t *lds, uint32_t wm, uint32_t wn, uint32_t wk, uint32_t lane)
    {
        const uint32_t k0 = (kk / PARTS * S::WK + wk) * S::MK;
        if constexpr (kk % PARTS == 0)
            #pragma unroll
            for (int pl = 0; pl < PB; ++pl)
                #pragma unroll
                for (int j = 0; j < S::NB; ++j)
                    f.b[kk / PARTS % 2][pl][j] = LoadB::L::template fragment<S::MI>(lds + LoadA::bytes + pl * LoadB::L::bytes, (wn * S::NB + j) * S::MI, k0, lane);
        #pragma unroll
        for (int pl = 0; pl < PA; ++pl)
            #pragma unroll
            for (int i = 0; i < MP; ++i)
                f.a[kk % 2][pl][i] = LoadA::L::template fragment<S::MI>(lds + pl * LoadA::L::bytes, (wm * S::MB + kk % PARTS * MP + i) * S::MI, k0, lane);
    }

    template <int kk> static __device__ __forceinline__ void multiply(const Fragments &f, Sums &acc)
    {
        const auto &a = f.a[kk % 2];
        const auto &b = f.b[kk / PARTS % 2];
        #pragma unroll
        for (int i = 0; i < MP; ++i)
            #pragma unroll
            for (int j = 0; j < S::NB; ++j) {
                constexpr int first = kk % PARTS * MP;
                acc[0][first + i][j] = T::mfma(b[0][j], a[0][i], acc[0][first + i][j]);
                if constexpr (PB == 3) {
                    Block s = acc[1][first + i][j];
                    if constexpr (PA == 3) {
                        s = T::mfma(b[0][j], a[2][i], s);
                        s = T::mfma(b[2][j], a[0][i], s);
                        s = T::mfma(b[1][j], a[1][i], s);
                        s = T::mfma(b[0][j], a[1][i], s);
                    } else {
                        s = T::mfma(b[2][j], a[0][i], s);
                    }
                    acc[1][first + i][j] = T::mfma(b[1][j], a[0][i], s);
                }
            }
    }

    // Part kk of the slice in `cur`.  (fill is cur: a name of its own tells the compiler that reads need not wait for what is requested into
    // it; the meeting of the waves keeps the reads of the old slice in front.)  WHOLE: the slice that is requested needs no checks.
    template <bool WHOLE, int kk = 0>
    static __device__ __forceinline__ void parts(const uint8_t *__restrict__ cur, uint8_t *__restrict__ next, uint8_t *__restrict__ fill, LoadA &la, LoadB &lb,
                                                 bool more, uint32_t k_fill, Fragments &f, Sums &acc, uint32_t wm, uint32_t wn, uint32_t wk, uint32_t lane,
                                                 uint32_t wave)
    {
        if constexpr (kk <= LAST) {
            if constexpr (kk + 1 == LAST) {
                la.deliver(next);
                lb.deliver(next + LoadA::bytes);
            }
            if constexpr (kk == LAST) { if (WHOLE) slices_arrived<EARLY ? 63 : (ST - 2) * REQUESTS>(); else slices_arrived<EARLY ? 63 : 0>(); }
            if constexpr (kk == LAST - EARLY) {
                if constexpr (WHOLE) {
                    la.request_whole(fill, k_fill, wave);
                    lb.request_whole(fill + LoadA::bytes, k_fill, wave);
                } else if (more) {
                    la.ask(fill, k_fill, wave);
                    lb.ask(fill + LoadA::bytes, k_fill, wave);
                }
            }
            if constexpr (kk == LAST) read<0>(f, next, wm, wn, wk, lane); else read<kk + 1>(f, cur, wm, wn, wk, lane);
            multiply<kk>(f, acc);
            // the reads between the first products, so that the last of them has arrived when the next part begins, the requests beside them
            constexpr int READS = PA * MP * (A_KC ? 1 : 2) + ((kk + 1) % PARTS ? 0 : PB * S::NB * (B_KC ? 1 : 2)), PRODUCTS = MP * S::NB * (PB == 1 ? 1 : PA == 3 ? 6 : 3);
            constexpr int PER = (READS + PRODUCTS - 1) / PRODUCTS, ASKED = LoadA::N * LoadA::RAW + LoadB::N * LoadB::RAW;
            constexpr int ASK = kk == LAST - EARLY && WHOLE ? (ASKED + PRODUCTS - 1) / PRODUCTS : 0;
            #pragma unroll
            for (int r = 0; r < PRODUCTS; ++r) {
                __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                if (r * PER < READS) __builtin_amdgcn_sched_group_barrier(0x100, PER, 0);
                if constexpr (ASK > 0) if (r * ASK < ASKED) __builtin_amdgcn_sched_group_barrier(0x20, ASK, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            parts<WHOLE, kk + 1>(cur, next, fill, la, lb, more, k_fill, f, acc, wm, wn, wk, lane, wave);
        }
    }
};

// Rows of a tile that lies within C, eight columns of a row per lane: what finish (below) does to four, with its decisions taken once.  Lanes that stand
// side by side store whole lines, past the caches (8192 x 1024 x 32000 bf16 223 -> 205 us): in 16 bits eight neighbouring columns each, in
// 32 bits four and four more a lane row further on.
template <class T, bool WEIGHTS, Finish FINISH> struct RowFinish {
    char *to;                         // first row of the tile (column 0 of C)
    uint64_t pitch;                   // bytes
    bool f32, part, aligned;
    float factor;

    __device__ __forceinline__ RowFinish(const ProductParams &p, const Place &at, float factor_)
    {
        part = FINISH == Finish::Store && p.splits > 1;
        f32 = part || p.out_f32 || sizeof(typename T::elem) == 4;
        factor = factor_;
        const uint64_t size = f32 ? 4 : 2;
        const uint64_t local = WEIGHTS ? at.m0 : at.row0;
        if (part) {
            const uint64_t all = WEIGHTS ? static_cast<uint64_t>(p.groups) * p.m : p.rows;
            pitch = p.ld_part * 4;
            to = reinterpret_cast<char *>(p.part + (at.split * all + (WEIGHTS ? static_cast<uint64_t>(at.group) * p.m : 0) + local) * p.ld_part);
        } else {
            pitch = p.ldc * size;
            to = static_cast<char *>(p.out) + (WEIGHTS ? at.group * p.out_group * size : 0) + (p.out_row && !WEIGHTS ? 0 : local * pitch);
        }
        aligned = ((reinterpret_cast<uintptr_t>(to) | pitch) & 15) == 0;
        if (!part && !WEIGHTS && FINISH == Finish::Store) {
            if (p.mask) aligned = aligned && ((reinterpret_cast<uintptr_t>(p.mask) | p.ld_mask * sizeof(typename T::elem)) & 15) == 0;
            if (p.mask_codes) aligned = aligned && ((reinterpret_cast<uintptr_t>(p.mask_codes) | p.ld_mask) & 7) == 0;
        }
    }

    // rows r0 + first, r0 + first + PASS, ... of ROWS; v: the turned tile, PITCH floats a row, its column 0 is column c0 of C
    template <int LANES, int PITCH, int ROWS> __device__ __forceinline__ void rows(const ProductParams &p, const Place &at, uint32_t r0, uint32_t c0, const float *v) const
    {
        constexpr uint32_t PASS = 64 / LANES;
        const uint32_t first = threadIdx.x % 64 / LANES, l = threadIdx.x % LANES, qa = f32 ? 4 * l : 8 * l, qb = f32 ? qa + 4 * LANES : qa + 4;
        const uint32_t ca = c0 + qa, cb = c0 + qb;
        // what belongs to a row is fetched once, by the lane of its number
        const uint32_t lane = threadIdx.x % 64, mine = r0 + lane % ROWS;
        const uint64_t my_row = at.row0 + mine;
        float row_factor = factor, row_top = 0.0f, row_one = 0.0f;
        uint32_t row_number = 0;
        constexpr bool SLOPE = FINISH == Finish::Slope || FINISH == Finish::Score;
        const bool by_row = !WEIGHTS && !part && (SLOPE || p.row_scale || p.out_row);
        if (by_row && mine < at.rows) {
            if (FINISH == Finish::Score) { row_top = p.top[my_row]; row_factor = p.inverse[my_row]; row_one = p.slope_one[my_row]; row_number = static_cast<uint32_t>(p.target[my_row]) - p.v0; }
            if (FINISH == Finish::Slope) { row_top = p.top[my_row]; row_factor = p.inverse[my_row] * slope_scale<T>(); row_number = static_cast<uint32_t>(p.target[my_row]) - p.v0; }
            if (FINISH == Finish::Store && p.row_scale) row_factor = p.row_scale[my_row];
            if (FINISH == Finish::Store && p.out_row) row_number = p.out_row[my_row];
        }
        #pragma unroll 4
        for (uint32_t k = 0; k < ROWS; k += PASS) {
            const uint32_t r = k + first;
            const float f = by_row ? __shfl(row_factor, r, 64) : factor;
            const uint32_t number = by_row ? __shfl(row_number, r, 64) : 0;
            const float top = SLOPE ? __shfl(row_top, r, 64) : 0.0f;
            const float one = FINISH == Finish::Score ? __shfl(row_one, r, 64) : 0.0f;
            f4 a = *reinterpret_cast<const f4 *>(v + r * PITCH + qa), b = *reinterpret_cast<const f4 *>(v + r * PITCH + qb);
            if (r0 + r >= at.rows) continue;
            const uint64_t row = at.row0 + r0 + r;
            char *at_row = to + static_cast<uint64_t>(r0 + r) * pitch;
            if constexpr (FINISH == Finish::Slope) {
                #pragma unroll
                for (uint32_t j = 0; j < 4; ++j) { a[j] = T::exp(a[j], top) * f; b[j] = T::exp(b[j], top) * f; }
                if (number - ca < 4 || number - cb < 4) {      // the target is one of these columns
                    const float t = p.target_slope[row] * slope_scale<T>();
                    #pragma unroll
                    for (uint32_t j = 0; j < 4; ++j) { if (number - ca == j) a[j] = t; if (number - cb == j) b[j] = t; }
                }
            } else if constexpr (FINISH == Finish::Score) {
                #pragma unroll
                for (uint32_t j = 0; j < 4; ++j) { a[j] = score_slope<T>(a[j] * p.logit_scale, top, f, one); b[j] = score_slope<T>(b[j] * p.logit_scale, top, f, one); }
                if (number - ca < 4 || number - cb < 4) {
                    const float t = p.target_slope[row];
                    #pragma unroll
                    for (uint32_t j = 0; j < 4; ++j) { if (number - ca == j) a[j] = t; if (number - cb == j) b[j] = t; }
                }
            } else if (!part) {
                if (!WEIGHTS) {
                    if (p.out_row) { if (number == kNoRow) continue; at_row = to + number * pitch; }
                    if (p.sum) {
                        float *s = p.sum + row * p.ld_sum;
                        if (p.sum_read) { a += *reinterpret_cast<const f4 *>(s + ca); b += *reinterpret_cast<const f4 *>(s + cb); }
                        if (p.sum_write) { *reinterpret_cast<f4 *>(s + ca) = a; *reinterpret_cast<f4 *>(s + cb) = b; continue; }
                    }
                }
                a *= f;
                b *= f;
                if (!WEIGHTS && p.relu) {
                    #pragma unroll
                    for (int j = 0; j < 4; ++j) { a[j] = a[j] < 0.0f ? 0.0f : a[j]; b[j] = b[j] < 0.0f ? 0.0f : b[j]; }
                }
                if (!WEIGHTS && (p.mask || p.mask_codes)) mask(p, row, ca, cb, a, b);
            }
            if (f32) {
                float *o = reinterpret_cast<float *>(at_row);
                __builtin_nontemporal_store(a, reinterpret_cast<f4 *>(o + ca));
                __builtin_nontemporal_store(b, reinterpret_cast<f4 *>(o + cb));
            } else {
                const u4 o = {T::pack(a.x, a.y), T::pack(a.z, a.w), T::pack(b.x, b.y), T::pack(b.z, b.w)};
                __builtin_nontemporal_store(o, reinterpret_cast<u4 *>(at_row) + ca / 8);
            }
        }
    }

    __device__ __forceinline__ void mask(const ProductParams &p, uint64_t row, uint32_t ca, uint32_t cb, f4 &a, f4 &b) const
    {
        if (p.mask_codes) {
            const uint8_t *m = p.mask_codes + row * p.ld_mask;
            const unsigned x = *reinterpret_cast<const unsigned *>(m + ca), y = *reinterpret_cast<const unsigned *>(m + cb);
            #pragma unroll
            for (int j = 0; j < 4; ++j) {
                if ((x >> (8 * j) & 0xffu) - 1u >= 0x7eu) a[j] = 0.0f;            // 1 .. 0x7e are above zero
                if ((y >> (8 * j) & 0xffu) - 1u >= 0x7eu) b[j] = 0.0f;
            }
        } else if constexpr (sizeof(typename T::elem) == 4) {
            const float *m = static_cast<const float *>(p.mask) + row * p.ld_mask;
            const f4 x = *reinterpret_cast<const f4 *>(m + ca), y = *reinterpret_cast<const f4 *>(m + cb);
            #pragma unroll
            for (int j = 0; j < 4; ++j) { if (!(x[j] > 0.0f)) a[j] = 0.0f; if (!(y[j] > 0.0f)) b[j] = 0.0f; }
        } else {
            constexpr unsigned most = std::is_same<T, F16>::value ? 0x7c00u : 0x7f80u;
            const uint16_t *m = static_cast<const uint16_t *>(p.mask) + row * p.ld_mask;
            const u2 x = *reinterpret_cast<const u2 *>(m + ca), y = *reinterpret_cast<const u2 *>(m + cb);
            #pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (((x[j / 2] >> (16 * (j % 2))) & 0xffffu) - 1u >= most) a[j] = 0.0f;
                if (((y[j / 2] >> (16 * (j % 2))) & 0xffffu) - 1u >= most) b[j] = 0.0f;
            }
        }
    }
};

// Sums over entries of a row below its largest logit `top`: exponentials of those below it, number of those equal to it, distances times exponentials.
// The sum of the exponentials is 1 + rest, rest = below + largest - 1: the 1 stays apart, so that log(1 + rest) keeps its digits where the row is sure.
template <class T> struct Moment {
    float below = 0.0f, largest = 0.0f, far = 0.0f;
    __device__ __forceinline__ void add(float z, float top)
    {
        // z is a product, rounded, and `top` one of them: taken from it unrounded, the largest would not lie at distance zero, and the rounding of `top` in the place of what a sure row keeps apart.
        #pragma clang fp contract(off)
        const float d = z - (top == -INFINITY ? 0.0f : top), e = T::exp(d, 0.0f);       // (what is not finite stays so in `below`)
        below += d == 0.0f ? 0.0f : e;
        largest += d == 0.0f ? 1.0f : 0.0f;
        far = fmaf(e, fmaxf(d, kFarBelow), far);
    }
    __device__ __forceinline__ void add_lane(int d)
    {
        below += __shfl_xor(below, d, 64);
        largest += __shfl_xor(largest, d, 64);
        far += __shfl_xor(far, d, 64);
    }
    __device__ __forceinline__ float4 result(float top) const { return make_float4(top, below + (largest - 1.0f), far, 0.0f); }
};

template <class T, Layout LAYOUT, class S, Finish FINISH, int HOW_A, int HOW_B>
__global__ __launch_bounds__(S::threads) void product_kernel(const ProductParams p)
{
    typedef Product<T, LAYOUT, S, HOW_A, HOW_B> P;
    constexpr bool WEIGHTS = P::WEIGHTS;
    static_assert(S::WN * S::BM * 8 <= P::lds_bytes, "the statistics' waves meet in the operands' buffers");
    __shared__ __attribute__((aligned(16))) uint8_t lds[P::lds_bytes];
    Place at;
    const uint32_t col_tiles = (p.n + S::BN - 1) / S::BN;
    if (!(WEIGHTS ? place_weights<S::BM>(p, col_tiles, at, S::BN) : place_rows<S::BM>(p, col_tiles, at, S::BN))) return;

    typedef typename T::elem elem;
    typename P::LoadA la;
    typename P::LoadB lb;
    la.ld = p.lda; la.ld_codes = p.ld_codes; la.ld_scales = p.ld_scales;
    la.src = static_cast<const elem *>(p.a) + at.row0 * p.lda;
    la.codes = p.a_codes + at.row0 * p.ld_codes;
    la.scales = p.a_scales + at.row0 * p.ld_scales;
    la.x0 = at.m0; la.x_end = at.m0 + at.rows; la.k_end = at.terms;
    lb.ld = p.ldb;
    lb.src = static_cast<const elem *>(p.b) + (WEIGHTS ? at.row0 * p.ldb : at.group * p.b_group);
    lb.x0 = at.n0; lb.x_end = p.n; lb.k_end = at.terms;
    la.start();
    lb.start();

    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t wk = wave % S::WK, wn = wave / S::WK % S::WN, wm = wave / S::WK / S::WN;
    typename P::Sums acc;
    #pragma unroll
    for (int s = 0; s < P::SUMS; ++s)
        #pragma unroll
        for (int i = 0; i < S::MB; ++i)
            #pragma unroll
            for (int j = 0; j < S::NB; ++j) acc[s][i][j] = typename P::Block{0};

    // this split's slices
    uint32_t slices = (at.terms + S::BK - 1) / S::BK, slice0 = 0;
    if (p.splits > 1) {
        const uint32_t per = (slices + p.splits - 1) / p.splits;
        slice0 = per * at.split < slices ? per * at.split : slices;
        slices = slices - slice0 < per ? slices - slice0 : per;
    }
    if (slices) {
        const uint32_t k0 = slice0 * S::BK;
        la.ask(lds, k0, wave);
        lb.ask(lds + P::LoadA::bytes, k0, wave);
        la.deliver(lds);
        lb.deliver(lds + P::LoadA::bytes);
        #pragma unroll
        for (uint32_t i = 1; i < P::ST; ++i)
            if (i < slices) {
                la.ask(lds + i * P::stage, k0 + i * S::BK, wave);
                lb.ask(lds + i * P::stage + P::LoadA::bytes, k0 + i * S::BK, wave);
            }
        if (HOW_A == kDirect && HOW_B == kDirect && slices >= P::ST) slices_arrived<(P::ST - 1) * P::REQUESTS>(); else slices_arrived<0>();
        uint32_t t = 0, cur = 0, next = P::stage;
        auto turn = [&] { cur = next; next = next + P::stage == P::ST * P::stage ? 0 : next + P::stage; };
        auto whole = [&] { return la.fits && lb.fits && t + P::ST < slices && k0 + (t + P::ST + 1) * S::BK <= at.terms; };
        // (the empty statements keep the compiler from joining the first reads with the loop's last ones at the head of the loop, where nothing hides them)
        typename P::Fragments f;
        P::template read<0>(f, lds, wm, wn, wk, lane);
        #pragma unroll
        for (int pl = 0; pl < P::PA; ++pl)
            #pragma unroll
            for (int i = 0; i < P::MP; ++i) asm volatile("" : "+v"(f.a[0][pl][i]));
        #pragma unroll
        for (int pl = 0; pl < P::PB; ++pl)
            #pragma unroll
            for (int j = 0; j < S::NB; ++j) asm volatile("" : "+v"(f.b[0][pl][j]));
        for (; whole(); ++t) {
            P::template parts<true>(lds + cur, lds + next, lds + cur, la, lb, true, k0 + (t + P::ST) * S::BK, f, acc, wm, wn, wk, lane, wave);
            turn();
        }
        #pragma unroll 1
        for (; t < slices; ++t) {
            P::template parts<false>(lds + cur, lds + next, lds + cur, la, lb, t + P::ST < slices, k0 + (t + P::ST) * S::BK, f, acc, wm, wn, wk, lane, wave);
            turn();
        }
    }
    slices_arrived<0>();                                       // LDS is free

    float unscale = 1.0f;
    if constexpr (P::PB == 3) {
        unscale = P::PA == 3 ? kPlaneUnscale : 1.0f / kPlaneScale;
        bool fine = true;
        #pragma unroll
        for (int i = 0; i < S::MB; ++i) {
            // (a row without a target takes no part, so it has no say in how the others' sums are formed, nor have its repeats behind the last row)
            bool counts = true;
            if constexpr (FINISH == Finish::Moments) {
                const uint32_t r = (wm * S::MB + i) * S::MI + lane % S::MI;
                counts = r < at.rows && (!p.target || static_cast<uint32_t>(p.target[at.row0 + r]) < p.n);
            }
            #pragma unroll
            for (int j = 0; j < S::NB; ++j) {
                acc[0][i][j] += acc[P::SUMS - 1][i][j];
                #pragma unroll
                for (int r = 0; r < 16; ++r) fine = fine && (!counts || __builtin_isfinite(acc[0][i][j][r]));
            }
        }
        if (__syncthreads_or(!fine)) {
            // the same sums with fp32 products: what is not finite then is so by fp32 arithmetic
            unscale = 1.0f;
            #pragma unroll
            for (int i = 0; i < S::MB; ++i)
                #pragma unroll
                for (int j = 0; j < S::NB; ++j) acc[0][i][j] = f16v{0};
            const uint32_t k_end = (slice0 + slices) * S::BK < at.terms ? (slice0 + slices) * S::BK : at.terms;
            #pragma unroll 1
            for (uint32_t k0 = slice0 * S::BK + 2 * wk; k0 < k_end; k0 += 2 * S::WK) {
                const uint32_t k = k0 + lane / 32;
                float a[S::MB], b[S::NB];
                #pragma unroll
                for (int i = 0; i < S::MB; ++i) a[i] = k < k_end ? la.element(at.m0 + (wm * S::MB + i) * 32 + lane % 32, k) : 0.0f;
                #pragma unroll
                for (int j = 0; j < S::NB; ++j) b[j] = k < k_end ? lb.element(at.n0 + (wn * S::NB + j) * 32 + lane % 32, k) : 0.0f;
                #pragma unroll
                for (int i = 0; i < S::MB; ++i)
                    #pragma unroll
                    for (int j = 0; j < S::NB; ++j) acc[0][i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(b[j], a[i], acc[0][i][j], 0, 0, 0);
            }
        }
    }

    // Four consecutive columns of a row, r in the tile and c in C.
    const float factor = FINISH == Finish::Store && p.splits <= 1 ? group_factor(p, at.group) : 1.0f;
    auto finish = [&](uint32_t r, uint32_t c, f4 v) {
        if constexpr (FINISH == Finish::Store) {
            if (r >= at.rows || c >= p.n) return;
            const uint64_t row = WEIGHTS ? static_cast<uint64_t>(at.group) * p.m + at.m0 + r : at.row0 + r;
            if (p.splits > 1) {
                const uint64_t all = WEIGHTS ? static_cast<uint64_t>(p.groups) * p.m : p.rows;
                *reinterpret_cast<f4 *>(p.part + (at.split * all + row) * p.ld_part + c) = v;
            } else {
                finish_quad<T, WEIGHTS>(p, at.group, row, at.m0 + r, c, v, factor);
            }
        } else if constexpr (FINISH == Finish::Slope) {
            if (r >= at.rows || c >= p.ldc_zero) return;
            const float top = p.top[at.row0 + r], inverse = p.inverse[at.row0 + r] * slope_scale<T>(), slope = p.target_slope[at.row0 + r] * slope_scale<T>();
            const int32_t target = p.target[at.row0 + r];
            #pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j] = static_cast<int32_t>(p.v0 + c + j) == target ? slope : T::exp(v[j], top) * inverse;
                if (c + j >= p.n) v[j] = 0.0f;
            }
            store_values<T>(p.out, (at.row0 + r) * p.ldc + c, v, 4, false);
        } else if constexpr (FINISH == Finish::Score) {
            if (r >= at.rows || c >= p.ldc_zero) return;
            const float top = p.top[at.row0 + r], none = p.inverse[at.row0 + r], one = p.slope_one[at.row0 + r], slope = p.target_slope[at.row0 + r];
            const int32_t target = p.target[at.row0 + r];
            #pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j] = static_cast<int32_t>(p.v0 + c + j) == target ? slope : score_slope<T>(v[j] * p.logit_scale, top, none, one);
                if (c + j >= p.n) v[j] = 0.0f;
            }
            store_values<T>(p.out, (at.row0 + r) * p.ldc + c, v, 4, false);
        }
    };
    const bool find_target = FINISH != Finish::Moments || p.target;

    if constexpr (S::WK > 1) {
        // the waves' sums over their terms meet in LDS, row by row, in the order of the waves
        static_assert(S::WM == 1 && S::MB == 1 && S::MI == 32, "waves share the terms of 32 rows");
        constexpr int PITCH = S::BN + 4, LANES = S::BN / 4;
        float *part = reinterpret_cast<float *>(lds);
        #pragma unroll
        for (int j = 0; j < S::NB; ++j)
            #pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f4 *>(part + (wk * S::BM + lane % 32) * PITCH + (wn * S::NB + j) * 32 + 8 * g + 4 * (lane / 32)) =
                    f4{acc[0][0][j][4 * g], acc[0][0][j][4 * g + 1], acc[0][0][j][4 * g + 2], acc[0][0][j][4 * g + 3]};
        __syncthreads();
        #pragma unroll
        for (uint32_t r = threadIdx.x / LANES; r < S::BM; r += S::threads / LANES) {
            const uint32_t q = threadIdx.x % LANES * 4, c = at.n0 + q;
            f4 v = *reinterpret_cast<const f4 *>(part + r * PITCH + q);
            #pragma unroll
            for (int w = 1; w < S::WK; ++w) v += *reinterpret_cast<const f4 *>(part + (w * S::BM + r) * PITCH + q);
            v *= unscale;
            if constexpr (FINISH == Finish::Stats || FINISH == Finish::Keep) {
                static_assert(LANES <= 64 && 64 % LANES == 0, "a row within a wave");
                const int32_t target = r < at.rows ? p.target[at.row0 + r] : -1;
                float top = -INFINITY;
                #pragma unroll
                for (uint32_t j = 0; j < 4; ++j) {
                    if (c + j >= p.n) v[j] = -INFINITY;
                    else if (static_cast<int32_t>(p.v0 + c + j) == target) { p.target_logit[at.row0 + r] = v[j]; v[j] = -INFINITY; }
                    top = fmaxf(top, v[j]);
                }
                #pragma unroll
                for (int d = 1; d < LANES; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
                const float base = top == -INFINITY ? 0.0f : top;
                v = f4{T::exp(v[0], base), T::exp(v[1], base), T::exp(v[2], base), T::exp(v[3], base)};
                if (FINISH == Finish::Keep && r < at.rows) keep_values<T>(p.out, (at.row0 + r) * p.ldc + c, v);
                float sum = (v[0] + v[1]) + (v[2] + v[3]);
                #pragma unroll
                for (int d = 1; d < LANES; d <<= 1) sum += __shfl_xor(sum, d, 64);
                if (q == 0 && r < at.rows) p.stats[static_cast<uint64_t>(at.n0 / S::BN) * p.rows + at.row0 + r] = make_float2(top, sum);
            } else if constexpr (FINISH == Finish::Moments) {
                static_assert(LANES <= 64 && 64 % LANES == 0 && LANES == quad_order(T::dtype, Tile::Small).width, "a row within a wave, a quad a lane");
                const int32_t target = find_target && r < at.rows ? p.target[at.row0 + r] : -1;
                float most = -INFINITY;
                #pragma unroll
                for (uint32_t j = 0; j < 4; ++j) {
                    v[j] *= p.logit_scale;
                    if (c + j >= p.n) v[j] = -INFINITY;
                    else if (static_cast<int32_t>(c + j) == target) p.target_logit[at.row0 + r] = v[j];
                    most = fmaxf(most, v[j]);
                }
                if (p.quads && r < at.rows) p.quads[(at.row0 + r) * p.ld_quads + c / 4] = most;
                float top = most;
                #pragma unroll
                for (int d = 1; d < LANES; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
                Moment<T> sum;
                #pragma unroll
                for (int j = 0; j < 4; ++j) sum.add(v[j], top);
                #pragma unroll
                for (int d = 1; d < LANES; d <<= 1) sum.add_lane(d);
                if (q == 0 && r < at.rows) p.moments[(at.row0 + r) * p.moment_tiles + at.n0 / S::BN] = sum.result(top);
            } else {
                finish(r, c, v);
            }
        }
    } else if constexpr (FINISH == Finish::Stats || FINISH == Finish::Keep) {
        // The maximum over the wave's columns (lanes MI apart hold a row), over the waves, and the sums of exponentials below the tile's
        // maximum; kept or not, the same bits.  The target's logit goes apart and counts as minus infinity here.
        constexpr bool KEEP = FINISH == Finish::Keep;
        float *tops = reinterpret_cast<float *>(lds), *sums = tops + S::WN * S::BM;        // the operand buffers are free
        const uint32_t c0 = at.n0 + wn * S::NB * S::MI + 4 * (lane / S::MI);
        const bool whole = at.n0 + S::BN <= p.n;
        #pragma unroll
        for (int i = 0; i < S::MB; ++i) {
            const uint32_t r = (wm * S::MB + i) * S::MI + lane % S::MI;
            const int32_t target = r < at.rows ? p.target[at.row0 + r] - static_cast<int32_t>(p.v0) : -1;
            if (__ballot(target >= static_cast<int32_t>(at.n0) && target < static_cast<int32_t>(at.n0 + S::BN))) {
                #pragma unroll
                for (int j = 0; j < S::NB; ++j)
                    #pragma unroll
                    for (int x = 0; x < S::X; ++x)
                        if (static_cast<int32_t>(c0 + j * S::MI + 8 * (x / 4) + x % 4) == target) {
                            p.target_logit[at.row0 + r] = acc[0][i][j][x] * unscale;
                            acc[0][i][j][x] = -INFINITY;
                        }
            }
            float top = -INFINITY;
            if (!whole) {
                #pragma unroll
                for (int j = 0; j < S::NB; ++j)
                    #pragma unroll
                    for (int x = 0; x < S::X; ++x) if (c0 + j * S::MI + 8 * (x / 4) + x % 4 >= p.n) acc[0][i][j][x] = -INFINITY;
            }
            #pragma unroll
            for (int j = 0; j < S::NB; ++j)
                #pragma unroll
                for (int x = 0; x < S::X; ++x) top = fmaxf(top, acc[0][i][j][x]);
            #pragma unroll
            for (int d = S::MI; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
            top *= unscale;
            if (lane < S::MI) tops[wn * S::BM + r] = top;
            __builtin_amdgcn_sched_barrier(0);                 // one row block's values at a time
        }
        __syncthreads();
        constexpr int PITCH = S::NB * S::MI + 4, LANES = S::NB * S::MI / 4;
        static_assert(2 * S::WN * S::BM * 4 + S::threads / 64 * S::MI * PITCH * 4 <= P::lds_bytes, "statistics and the waves' turned rows");
        float *mine = sums + S::WN * S::BM + wave * S::MI * PITCH;
        #pragma unroll
        for (int i = 0; i < S::MB; ++i) {
            const uint32_t r0 = (wm * S::MB + i) * S::MI, r = r0 + lane % S::MI;
            float top = -INFINITY, sum = 0.0f;
            #pragma unroll
            for (int w = 0; w < S::WN; ++w) top = fmaxf(top, tops[w * S::BM + r]);
            const float base = top == -INFINITY ? 0.0f : top;
            #pragma unroll
            for (int j = 0; j < S::NB; ++j) {
                #pragma unroll
                for (int g = 0; g < S::X / 4; ++g) {
                    f4 e;
                    #pragma unroll
                    for (int x = 0; x < 4; ++x) e[x] = T::exp(acc[0][i][j][4 * g + x] * unscale, base);
                    sum += (e[0] + e[1]) + (e[2] + e[3]);
                    if (KEEP) *reinterpret_cast<f4 *>(mine + (lane % S::MI) * PITCH + j * S::MI + 8 * g + 4 * (lane / S::MI)) = e;
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            #pragma unroll
            for (int d = S::MI; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
            if (lane < S::MI) sums[wn * S::BM + r] = sum;
            if constexpr (KEEP) {
                __builtin_amdgcn_wave_barrier();
                #pragma unroll 4
                for (uint32_t k = lane / LANES; k < S::MI; k += 64 / LANES) {
                    const uint32_t q = lane % LANES * 4;
                    const f4 e = *reinterpret_cast<const f4 *>(mine + k * PITCH + q);
                    if (r0 + k < at.rows) keep_values<T>(p.out, (at.row0 + r0 + k) * p.ldc + at.n0 + wn * S::NB * S::MI + q, e);
                }
                __builtin_amdgcn_wave_barrier();
            }
        }
        __syncthreads();
        for (uint32_t r = threadIdx.x; r < at.rows; r += S::threads) {
            float top = -INFINITY, sum = 0.0f;
            #pragma unroll
            for (int w = 0; w < S::WN; ++w) top = fmaxf(top, tops[w * S::BM + r]);
            #pragma unroll
            for (int w = 0; w < S::WN; ++w) sum += sums[w * S::BM + r];
            p.stats[static_cast<uint64_t>(at.n0 / S::BN) * p.rows + at.row0 + r] = make_float2(top, sum);
        }
    } else if constexpr (FINISH == Finish::Moments) {
        // As above: the tile's maximum, then the sums below it.  The target is among them; it is one of the largest that is left out.
        float *tops = reinterpret_cast<float *>(lds), *sums = tops + S::WN * S::BM, *ones = sums + S::WN * S::BM, *far = ones + S::WN * S::BM;
        static_assert(4 * S::WN * S::BM * 4 <= P::lds_bytes, "the waves' sums");
        const uint32_t c0 = at.n0 + wn * S::NB * S::MI + 4 * (lane / S::MI);
        const bool whole = at.n0 + S::BN <= p.n;
        const float scale = unscale * p.logit_scale;
        #pragma unroll
        for (int i = 0; i < S::MB; ++i) {
            const uint32_t r = (wm * S::MB + i) * S::MI + lane % S::MI;
            const int32_t target = find_target && r < at.rows ? p.target[at.row0 + r] : -1;
            if (__ballot(target >= static_cast<int32_t>(at.n0) && target < static_cast<int32_t>(at.n0 + S::BN))) {
                #pragma unroll
                for (int j = 0; j < S::NB; ++j)
                    #pragma unroll
                    for (int x = 0; x < S::X; ++x)
                        if (static_cast<int32_t>(c0 + j * S::MI + 8 * (x / 4) + x % 4) == target) p.target_logit[at.row0 + r] = acc[0][i][j][x] * scale;
            }
            if (!whole) {
                #pragma unroll
                for (int j = 0; j < S::NB; ++j)
                    #pragma unroll
                    for (int x = 0; x < S::X; ++x) if (c0 + j * S::MI + 8 * (x / 4) + x % 4 >= p.n) acc[0][i][j][x] = -INFINITY;
            }
            constexpr int EACH = S::NB * S::X / 4;
            constexpr QuadOrder order = quad_order(T::dtype, S::BN == 256 ? Tile::Large : S::threads == 512 ? Tile::Deep : S::BN == 64 ? Tile::Square : Tile::Medium);
            static_assert(order.width == S::NB * S::MI / 4 && order.each == EACH, "quad_order");
            float quad[EACH], top = -INFINITY;
            #pragma unroll
            for (int j = 0; j < S::NB; ++j)
                #pragma unroll
                for (int g = 0; g < S::X / 4; ++g) {
                    const auto &v = acc[0][i][j];
                    const float most = fmaxf(fmaxf(v[4 * g], v[4 * g + 1]), fmaxf(v[4 * g + 2], v[4 * g + 3]));
                    quad[j * (S::X / 4) + g] = most * scale;
                    top = fmaxf(top, most);
                }
            if (p.quads && r < at.rows) {
                float *to = p.quads + (at.row0 + r) * p.ld_quads + (at.n0 + wn * S::NB * S::MI) / 4 + lane / S::MI * EACH;
                if constexpr (EACH == 2) *reinterpret_cast<float2 *>(to) = make_float2(quad[0], quad[1]);
                else
                    #pragma unroll
                    for (int e = 0; e < EACH; e += 4) *reinterpret_cast<f4 *>(to + e) = f4{quad[e], quad[e + 1], quad[e + 2], quad[e + 3]};
            }
            #pragma unroll
            for (int d = S::MI; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
            if (lane < S::MI) tops[wn * S::BM + r] = top * scale;
            __builtin_amdgcn_sched_barrier(0);                 // one row block's values at a time
        }
        __syncthreads();
        #pragma unroll
        for (int i = 0; i < S::MB; ++i) {
            const uint32_t r = (wm * S::MB + i) * S::MI + lane % S::MI;
            float top = -INFINITY;
            #pragma unroll
            for (int w = 0; w < S::WN; ++w) top = fmaxf(top, tops[w * S::BM + r]);
            Moment<T> sum;
            #pragma unroll
            for (int j = 0; j < S::NB; ++j) {
                #pragma unroll
                for (int x = 0; x < S::X; ++x) sum.add(acc[0][i][j][x] * scale, top);
                __builtin_amdgcn_sched_barrier(0);
            }
            #pragma unroll
            for (int d = S::MI; d < 64; d <<= 1) sum.add_lane(d);
            if (lane < S::MI) { sums[wn * S::BM + r] = sum.below; ones[wn * S::BM + r] = sum.largest; far[wn * S::BM + r] = sum.far; }
        }
        __syncthreads();
        for (uint32_t r = threadIdx.x; r < at.rows; r += S::threads) {
            float top = -INFINITY;
            Moment<T> sum;
            #pragma unroll
            for (int w = 0; w < S::WN; ++w) {
                top = fmaxf(top, tops[w * S::BM + r]);
                sum.below += sums[w * S::BM + r];
                sum.largest += ones[w * S::BM + r];
                sum.far += far[w * S::BM + r];
            }
            p.moments[(at.row0 + r) * p.moment_tiles + at.n0 / S::BN] = sum.result(top);
        }
    } else {
        // A block of rows at a time turns in the wave's own part of LDS, so that consecutive lanes take consecutive columns.  Tiles that lie
        // within C with every row on 16 bytes are finished eight columns at a time, without a decision per element.
        constexpr int PITCH = S::NB * S::MI + 4, LANES = S::NB * S::MI / 8, PASS = 64 / LANES;     // rows of one pass
        float *mine = reinterpret_cast<float *>(lds) + wave * S::MI * PITCH;
        const uint32_t q = lane % LANES * 8, c = at.n0 + wn * S::NB * S::MI + q;
        const RowFinish<T, WEIGHTS, FINISH> whole(p, at, factor);
        const bool fast = at.n0 + S::BN <= p.n && whole.aligned;
        #pragma unroll
        for (int i = 0; i < S::MB; ++i) {
            #pragma unroll
            for (int j = 0; j < S::NB; ++j)
                #pragma unroll
                for (int g = 0; g < S::X / 4; ++g)
                    *reinterpret_cast<f4 *>(mine + (lane % S::MI) * PITCH + j * S::MI + 8 * g + 4 * (lane / S::MI)) =
                        f4{acc[0][i][j][4 * g], acc[0][i][j][4 * g + 1], acc[0][i][j][4 * g + 2], acc[0][i][j][4 * g + 3]} * unscale;
            __builtin_amdgcn_wave_barrier();
            const uint32_t r0 = (wm * S::MB + i) * S::MI;
            if (fast) {
                whole.template rows<LANES, PITCH, S::MI>(p, at, r0, at.n0 + wn * S::NB * S::MI, mine);
            } else {
                #pragma unroll 1
                for (uint32_t r = lane / LANES; r < S::MI; r += PASS)
                    #pragma unroll
                    for (int h = 0; h < 2; ++h) finish(r0 + r, c + 4 * h, *reinterpret_cast<const f4 *>(mine + r * PITCH + q + 4 * h));
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
}

template <class T, Layout LAYOUT, class S, Finish FINISH, int HOW_A, int HOW_B>
hipError_t launch_one(hipStream_t stream, const ProductParams &p)
{
    constexpr TileSize size = {S::BM, S::BN, S::threads};
    const uint64_t blocks = blocks_of(size, LAYOUT == Layout::Weights, p.rows, p.groups, p.m, p.n, p.splits);
    if (!fits_a_launch(size, blocks)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((product_kernel<T, LAYOUT, S, FINISH, HOW_A, HOW_B>), dim3(static_cast<uint32_t>(blocks)), dim3(S::threads), 0, stream, p);
    return hipGetLastError();
}

// 16x16x32 draws less power for the same products than 32x32x16: 8 groups of 8192 rows, 4096 x 4096 1765 us instead of 1890, 16 of 1024, 2048 x 2048
// 119 instead of 128.  Codes leave no registers for its fragments beside those on their way (weight gradient of 16 groups of 1024 rows, 2048 x 2048:
// 236 us, with 32x32x16 214), and two medium tiles on a compute unit lose by it (16 of 512, 1024 x 1024: 27 instead of 24).
typedef TileShape<256, 256, 64, 2, 4, 1, 2, 16> Large16;
typedef TileShape<256, 256, 64, 2, 4, 1> Large16Codes;
typedef TileShape<128, 128, 64, 2, 2, 1> Medium16;
// where every compute unit has one block at most: the medium tile with four slices in LDS instead of two (and room for a second block).  2048 x 2048 x
// 2048: 24 us instead of 29, 4 groups of 1024 rows, 2048 to 512 columns: 22 instead of 26, out of memory 23 instead of 33 (1024 x 4096 x 4096 41 us, with
// 32x32x16 43, input gradient 38 and 43); with 512 blocks (16 groups of 512
// rows, 1024 x 1024) 30 instead of 24
typedef TileShape<128, 128, 64, 2, 4, 1, 4, 16> Deep16;
// Rows of a batch, stored: between the medium and the large one, where these need a turn of 256 blocks more or leave units idle.  7 groups, 5003 rows, 2056 to
// 1000 columns, fp16: 35 us instead of 45 (medium) and 60 (large); 4096 x 4160 x 4160 148 instead of 166 and 183; 16 of 256 rows, 1024 x 1024: 18 instead of
// 21 and 30; 16 of 1024, 2048 x 2048: 155 against 140 and 113.  Four waves instead of eight: 63 us, 256 x 128 or 128 x 256 the same or worse.
typedef TileShape<192, 128, 64, 2, 4, 1, 3, 16> Tall16;
typedef TileShape<32, 64, 128, 1, 1, 4> Small16;
// short sums and few blocks: a slice more in flight (one row, 4096 x 4096: 10.1 us instead of 11.0; the other tiles lose by four slices of 32: 8 groups
// of 8192 rows, 4096 x 4096, input gradient 1962 us instead of 1840: of a row of 64 bytes the other half of the line is fetched again)
typedef TileShape<32, 64, 128, 1, 1, 4, 3> Small16Direct;
// a large table that a few rows read once, past the caches: 4 rows, 131072 entries of 2048 105 us -> 90 (6.0 TB/s); two or four slices in flight 120
typedef TileShape<32, 64, 128, 1, 1, 4, 3, 32, true> Small16Once;
typedef TileShape<128, 128, 32, 2, 4, 1> Medium32;
typedef TileShape<32, 64, 64, 1, 2, 2> Small32;
// between these, three blocks on a compute unit: weight gradient of 4 groups of 250 rows, 512 x 768 13.7 us instead of 15.3 (medium) and 17.4 (small), of 2 of
// 254, 512 x 5003 38 instead of 45 and 49; 2048 x 2048 x 2048 132 against 101 and 180
typedef TileShape<64, 64, 32, 2, 2, 1> Square32;

template <class S> constexpr bool is_size(Dtype type, Tile tile)
{
    const TileSize t = tile_size(type, tile);
    return t.bm == S::BM && t.bn == S::BN && t.threads == S::threads;
}
static_assert(is_size<Large16>(Dtype::BF16, Tile::Large) && is_size<Large16Codes>(Dtype::BF16, Tile::Large) && is_size<Medium16>(Dtype::BF16, Tile::Medium) &&
              is_size<Deep16>(Dtype::BF16, Tile::Deep) && is_size<Tall16>(Dtype::BF16, Tile::Tall) && is_size<Small16>(Dtype::BF16, Tile::Small) &&
              is_size<Small16Direct>(Dtype::BF16, Tile::Small) && is_size<Medium32>(Dtype::F32, Tile::Medium) && is_size<Small32>(Dtype::F32, Tile::Small) &&
              is_size<Square32>(Dtype::F32, Tile::Square), "tile_size");

template <class T, Layout LAYOUT, Finish FINISH>
hipError_t launch_layout(hipStream_t stream, Tile tile, const ProductParams &p)
{
    constexpr bool WEIGHTS = LAYOUT == Layout::Weights;
    if constexpr (T::planes == 3) {
        if constexpr (WEIGHTS)
            if (!p.a) return tile == Tile::Small    ? launch_one<T, LAYOUT, Small32, FINISH, kCodes, kRegs>(stream, p)
                             : tile == Tile::Square ? launch_one<T, LAYOUT, Square32, FINISH, kCodes, kRegs>(stream, p)
                                                    : launch_one<T, LAYOUT, Medium32, FINISH, kCodes, kRegs>(stream, p);
        return tile == Tile::Small    ? launch_one<T, LAYOUT, Small32, FINISH, kRegs, kRegs>(stream, p)
               : tile == Tile::Square ? launch_one<T, LAYOUT, Square32, FINISH, kRegs, kRegs>(stream, p)
                                      : launch_one<T, LAYOUT, Medium32, FINISH, kRegs, kRegs>(stream, p);
    } else {
        const bool b_direct = direct_b(LAYOUT, p);
        if constexpr (WEIGHTS)
            if (!p.a) {
                if (b_direct && tile == Tile::Large) return launch_one<T, LAYOUT, Large16Codes, FINISH, kCodes, kDirect>(stream, p);
                if (b_direct) return tile == Tile::Small ? launch_one<T, LAYOUT, Small16, FINISH, kCodes, kDirect>(stream, p)
                                                         : launch_one<T, LAYOUT, Medium16, FINISH, kCodes, kDirect>(stream, p);
                return tile == Tile::Small ? launch_one<T, LAYOUT, Small16, FINISH, kCodes, kRegs>(stream, p)
                                           : launch_one<T, LAYOUT, Medium16, FINISH, kCodes, kRegs>(stream, p);
            }
        if (b_direct && direct_a(LAYOUT, p)) {
            if (tile == Tile::Large) return launch_one<T, LAYOUT, Large16, FINISH, kDirect, kDirect>(stream, p);
            if (tile == Tile::Deep) return launch_one<T, LAYOUT, Deep16, FINISH, kDirect, kDirect>(stream, p);
            if constexpr (FINISH == Finish::Store && !WEIGHTS)
                if (tile == Tile::Tall) return launch_one<T, LAYOUT, Tall16, FINISH, kDirect, kDirect>(stream, p);
            if constexpr (FINISH == Finish::Moments)
                if (tile == Tile::Small && p.b_once) return launch_one<T, LAYOUT, Small16Once, FINISH, kDirect, kDirect>(stream, p);
            return tile == Tile::Small ? launch_one<T, LAYOUT, Small16Direct, FINISH, kDirect, kDirect>(stream, p)
                                       : launch_one<T, LAYOUT, Medium16, FINISH, kDirect, kDirect>(stream, p);
        }
        return tile == Tile::Small ? launch_one<T, LAYOUT, Small16, FINISH, kRegs, kRegs>(stream, p)
                                   : launch_one<T, LAYOUT, Medium16, FINISH, kRegs, kRegs>(stream, p);
    }
}

template <class T> hipError_t launch_store(hipStream_t stream, Layout layout, Tile tile, const ProductParams &p)
{
    if (layout == Layout::Rows_KN) return launch_layout<T, Layout::Rows_KN, Finish::Store>(stream, tile, p);
    if (layout == Layout::Rows_NK) return launch_layout<T, Layout::Rows_NK, Finish::Store>(stream, tile, p);
    return launch_layout<T, Layout::Weights, Finish::Store>(stream, tile, p);
}

template <class T> hipError_t launch_logits(hipStream_t stream, Finish finish, Tile tile, const ProductParams &p)
{
    if (finish == Finish::Stats) return launch_layout<T, Layout::Rows_NK, Finish::Stats>(stream, tile, p);
    if (finish == Finish::Moments) return launch_layout<T, Layout::Rows_NK, Finish::Moments>(stream, tile, p);
    if (finish == Finish::Score) return launch_layout<T, Layout::Rows_NK, Finish::Score>(stream, tile, p);
    if constexpr (!std::is_same<T, F16>::value)                // (its slopes would be rounded twice to the same eleven bits)
        if (finish == Finish::Keep) return launch_layout<T, Layout::Rows_NK, Finish::Keep>(stream, tile, p);
    return finish == Finish::Slope ? launch_layout<T, Layout::Rows_NK, Finish::Slope>(stream, tile, p) : hipErrorInvalidValue;
}

}  // namespace
}  // namespace cocod
