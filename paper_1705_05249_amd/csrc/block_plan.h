// Which kernel a product of 8-bit matrices takes and in how many slices of its sum.  Host code alone: it can be asked without a GPU.
#pragma once

#include "experts.h"
#include "internal.h"

namespace mg {

// How a kernel sums: on the FP8 pipes with scales that are powers of two or any (SUMS_SQUARE: any, and square blocks of B, so that all of a
// fragment's rows of B have one), on the FP16 pipes with any scales, or on the bfloat16 pipes, whose operands take scales that are powers of two
// into their exponents while they are widened
enum BlockSums { SUMS_POW2 = 0, SUMS_ANY = 1, SUMS_FP32 = 2, SUMS_SQUARE = 3, SUMS_FP32_POW2 = 4 };
constexpr bool sums_fp32(int sums) { return sums == SUMS_FP32 || sums == SUMS_FP32_POW2; }

// Kernels for operands whose rows start on 16 bytes (block_dma_kernel.h), by their tile
enum BlockDmaTile { DMA_256 = 0, DMA_128 = 1, DMA_64 = 2 };
constexpr int block_dma_rows(int tile) { return tile == DMA_256 ? 256 : tile == DMA_128 ? 128 : 64; }
constexpr int block_dma_cols(int tile, int sums) { return tile == DMA_256 && sums_fp32(sums) ? 128 : block_dma_rows(tile); }
constexpr int TILE_ANY = -1, TILE_ANY_64 = -2; // the kernel for operands at any address
constexpr int TILE_FEW = -3;                   // the kernel for few rows in one operand

struct Plan {
    int tile;                                 // BlockDmaTile or one of those
    int tiles_m, tiles_n, slices;
    int fragments;                            // TILE_FEW
    bool few_b;
};

inline int64_t output_rows(int mode, int groups, int64_t m) { return mode == BLOCK_SUM ? groups * m : m; }

// What a kernel takes, in us, measured with random operands.  A compute unit that has one of its tiles: `alone` for a block of 128 of the sum while half of the
// chip is idle, `full` while all of it is busy; with n of them n * `each` (two work-groups of 128 x 128 share a compute unit, two to four of 64 x 64).
// Around the sum: `start`, and `more` for every round of tiles (C leaves).  Over 2048 x 2048 .. 8192 x 4096 with sums of 512 to 8192 within a tenth of what calls in a row take
// (8192 x 4096 x 4096 with activations: estimated 116 us, measured 121; with FP32 sums 4096 x 4096 x 8192 223 and 238 to 248; 16 experts' rows, 16384 x 4096 x 2048, 161 and 175),
// with two exceptions: `each` of 128 x 128 is 0.515 with uniform bits, where the clock stays up (with activations the smaller tiles slow down more than the large ones), and
// many tiles with short sums that write FP32, the experts' weights' gradient, take longer than their estimate (16384 rows of 16 experts, 4096 x 2048: 304 us, measured
// 338 with equal counts and 421 with a router's).
struct Cost {
    double alone, full, each, start, more;
};
inline Cost cost_of(int tile, int sums)
{
    const bool fp32 = sums_fp32(sums);
    Cost c{};
    switch (tile) {
        case DMA_256: c = fp32 ? Cost{1.47, 1.7, 1.6, 4, 7} : Cost{1.38, 1.6, 1.55, 4, 6.5}; break;
        case DMA_128: c = fp32 ? Cost{1.05, 1.19, 0.93, 3, 1.5} : Cost{0.6, 0.75, 0.6, 3, 1}; break;
        case DMA_64: c = fp32 ? Cost{0.5, 0.52, 0.37, 3, 0.7} : Cost{0.3, 0.31, 0.24, 3, 0.5}; break;
        case TILE_ANY: c = fp32 ? Cost{1.8, 2.1, 1.5, 4, 1.5} : Cost{1.2, 1.4, 1.0, 4, 1.5}; break;
        default: c = fp32 ? Cost{0.9, 1.0, 0.6, 3.5, 0.7} : Cost{0.6, 0.66, 0.4, 3.5, 0.7}; break;
    }
    // scales of any value are multiplied in beside the matrix instructions (4096^3: 66 -> 76 us; 128 x 4096 x 4096 on 64 x 64 tiles 13 -> 17)
    const double scaling = sums == SUMS_POW2 || sums == SUMS_FP32_POW2 ? 1. : tile == DMA_256 ? 1.17 : 1.4;
    c.alone *= scaling;
    c.full *= scaling;
    c.each *= scaling;
    return c;
}

// Which kernel and how many slices of the sum: the least of the estimates.  Slices cost a launch that reads what they wrote, and no slice gets fewer than four blocks.
inline Plan plan(int mode, int groups, int64_t m, int64_t n, int64_t k, int sums, bool aligned, size_t workspace)
{
    Plan best{};
    best.slices = 1;
    // The kernel for few rows reads them once for every 16 of the others.  8192 x 8192: 4 rows 15.9 us, 16 rows 22, 32 rows 33, 64 x 64 tiles 19; 4096 x 4096: 32 rows 10,
    // 64 x 64 tiles 11.5.
    // Experts' rows: only their mean is known, and an expert with more of them has its weights read again for every 16.  So it is taken where the 64 x 64 tiles of all experts
    // that can have rows do not outnumber the 256 compute units (twice for FP32 sums, in which tiles take longer), up to a mean of 8 rows, 16 where they reach half of the
    // units.  2048 x 4096, FP8 pipes, even counts and then a router's, this kernel / tiles: 4 experts, 1 row 8.8 / 11.7 and 8.5 / 11.5 us, 8 rows 10.2 / 11.5 and 10.3 / 11.6;
    // 16 experts, 1 row 29 / 22 and 17 / 13, 8 rows 36 / 22 and 37 / 21; 32 experts, 3 rows 56 / 40 and 34 / 30; 64 experts, 16 rows 155 / 107 and 191 / 105, and with
    // all rows in eight of them 148 / 21.  FP32 sums: 8 experts, 1 row 15.5 / 18.8 and 11.8 / 17.6; 32 experts, 1 row 53 / 47 and 28 / 25.
    const int64_t asked = m < groups ? m : groups;                                      // experts that can have rows
    const int64_t few = mode == BLOCK_ROWS ? ceil_div(m, groups) : m < n ? m : n;       // rows of A (for an expert), or of the smaller operand
    const int64_t small_tiles = asked * ceil_div(n, 64);
    if (mode == BLOCK_ROWS ? small_tiles <= (sums_fp32(sums) ? 512 : 256) && few <= (small_tiles <= 128 ? 16 : 8)
                           : mode == BLOCK_DENSE && (few <= 8 || (few <= 32 && (m < n ? n : m) * k <= int64_t(1) << 25))) {
        best.tile = TILE_FEW;
        best.few_b = mode == BLOCK_DENSE && n < m;
        best.fragments = few <= 16 ? 1 : 2;
        return best;
    }
    const int64_t batch = mode == BLOCK_SUM ? groups : 1;
    const double blocks = static_cast<double>(ceil_div(k, SCALE_BLOCK)) / batch + (mode == BLOCK_SUM ? 0.5 : 0.);
    const double one = static_cast<double>(output_rows(mode, groups, m)) * n * 4;
    double least = 0;
    for (const int tile : {int(DMA_256), int(DMA_128), int(DMA_64), TILE_ANY, TILE_ANY_64}) {
        if (aligned != (tile >= 0)) continue;
        const int64_t any = tile == TILE_ANY ? 128 : 64, bm = tile < 0 ? any : block_dma_rows(tile), bn = tile < 0 ? any : block_dma_cols(tile, sums);
        Plan p{};
        p.tile = tile;
        p.tiles_m = static_cast<int>(ceil_div(m, bm) + (mode == BLOCK_ROWS ? groups : 0));
        p.tiles_n = static_cast<int>(ceil_div(n, bn));
        // (every expert's last tile is half full, if it has rows at all; where their mean is small each has one tile)
        const int64_t ends = groups < m / bm ? groups / 2 : 0;
        const int64_t tiles = (mode == BLOCK_ROWS ? (few <= 16 ? asked : ceil_div(m, bm) + ends) : static_cast<int64_t>(p.tiles_m)) * p.tiles_n * batch;
        const Cost c = cost_of(tile, sums);
        for (int s = 1; s <= 16; s *= 2) {
            if (s > 1 && (blocks / s < 4 || one * s > static_cast<double>(workspace) || tiles * s > 512)) break;
            const double per_unit = static_cast<double>(ceil_div(tiles * s, 256));
            const double a_block = per_unit > 1 ? (c.each * per_unit > c.full ? c.each * per_unit : c.full) : tiles * s <= 128 ? c.alone : c.full;
            const double us = c.start + c.more * per_unit + blocks / s * a_block + (s > 1 ? 4 + one * (s + 1) / 4e6 : 0);
            if (least == 0 || us < least) {
                least = us;
                best = p;
                best.slices = s;
            }
        }
    }
    return best;
}

// Rows on 16 bytes, and 32-bit offsets: inside a tile of 256 rows, or from the first row of A where rows are indexed (of those there is one for every `fan` slots)
inline bool dma_operands(const BlockProblem &p)
{
    auto on16 = [](const void *x, int64_t a, int64_t b) { return reinterpret_cast<uintptr_t>(x) % 16 == 0 && a % 16 == 0 && b % 16 == 0; };
    if (!on16(p.A, p.lda, 0) || !on16(p.B, p.ldb, p.mode == BLOCK_ROWS ? p.stride_b : 0)) return false;
    const __int128 rows_a = p.mode == BLOCK_ROWS && p.groups.source != nullptr ? ceil_div(p.m, p.groups.fan) : 256, most = (__int128(1) << 31) - (1 << 20);
    const __int128 along = p.mode == BLOCK_SUM ? p.lda : p.k;
    return rows_a * p.lda + along < most && __int128(256) * p.ldb + along < most && (rows_a * p.ldsa + along / 128) * 4 < most &&
           (__int128(256) * p.ldsb + along / 128) * 4 < most;
}

// What a call takes
inline int block_sums(const BlockProblem &p) { return p.fp32_sums ? (p.pow2 ? SUMS_FP32_POW2 : SUMS_FP32) : p.pow2 ? SUMS_POW2 : p.b_square ? SUMS_SQUARE : SUMS_ANY; }
inline Plan plan(const BlockProblem &p) { return plan(p.mode, p.groups.count, p.m, p.n, p.k, block_sums(p), dma_operands(p), p.workspace == nullptr ? 0 : p.workspace_bytes); }

}  // namespace mg
