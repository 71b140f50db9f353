// Which kernel a product of 16-bit matrices takes and in how many slices of its sum.  Host code alone: it can be asked without a GPU.
#pragma once

#include "internal.h"
#include "layers.h"

namespace mg {

struct LinearPlan {
    int tile;                        // LinearTile
    int slices, k_per_slice;
    double us;                       // the estimate; 0: none was needed
};

// What a tile takes, in us, measured with random bfloat16 operands: `alone` for 64 values of the sum while a compute unit has one of its tiles, `pair` while it has two
// at a time (LDS has room for two of 128 or 64); around the sum `start`, and `more` for every tile of a compute unit (C leaves).  Operands across the sum cost more
// reads of LDS (`form`).  Estimated and measured: 2048^3 on 128_DEEP 23 and 21.7, 4096 x 4096 x 2048 on 256 55 and 57, on 128 74 and 72, 8192 x 8192 x 512 on 256
// 75 and 89, 1000 x 9999 x 1001 on 128 37 and 36, on 256 33 and 31, 8192 x 1024 x 1024 on 128 22 and 21.5, 512 x 2048 x 2048 on 64 10.6 and 10.7,
// with two sets of wavefronts 9.5 and 9.3; 1024^3 7.1 and 7.3, with two sets 7.0 and 6.9; 64 x 2048 x 8192 31.2 and 30.9, with two sets 24.3 and 23.7.
struct LinearCost {
    double alone, pair, start, more;
};
inline LinearCost linear_cost(int tile, int form)
{
    LinearCost c{};
    double one = 1, both = 1;              // FORM_KN, FORM_NN
    switch (tile) {
        case LINEAR_256: c = {1.4, 2.8, 4, 6.5}; one = 1.04; both = 1.08; break;
        case LINEAR_128: c = {0.82, 1.0, 3, 1.6}; one = 1.04; both = 1.08; break;
        case LINEAR_128_DEEP: c = {0.57, 1.14, 2.5, 2}; one = 1.04; both = 1.08; break;
        case LINEAR_64: c = {0.215, 0.4, 3.2, 0.5}; one = 1.42; both = 1.35; break;
        case LINEAR_64_TWICE: c = {0.155, 0.31, 2.5, 2}; one = 1.42; both = 1.35; break;
        default: c = {0.5, 0.7, 3, 1.5}; one = 1.25; both = 1.5; break;
    }
    const double factor = form == FORM_NN ? both : form == FORM_KN ? one : 1;
    c.alone *= factor;
    c.pair *= factor;
    return c;
}

// The least of the estimates.  Slices cost a launch that reads what they wrote; no slice gets fewer than four pieces of 64.
inline LinearPlan linear_plan(int form, int end, int64_t rows, int64_t cols, int64_t k, bool aligned, size_t room)
{
    LinearPlan best{LINEAR_ANY, 1, static_cast<int>(padded(k > 0 ? k : 1)), 0};
    const double pieces = static_cast<double>(ceil_div(k > 0 ? k : 1, LAYER_PIECE)), one = static_cast<double>(rows) * padded(cols) * 4;
    if (form == FORM_KK && end != END_SCORES_GRAD && rows <= LINEAR_FEW_ROWS) {
        // Few rows: whatever the other sizes.  One row, 4096 x 8192: 14.6 us, 64 x 64 tiles in four slices 12.2 and 4.5 for their sum; 24 rows: 2048 x 4096 6.7 and 10.2,
        // gate and up weights of 4096 x 2048 8.0 and 12.8; 8 rows, 512 x 8192: 7.1 and 12.8.  One row, gate and up weights of 8192 x 4096, out of the last-level cache 25 and
        // 21.5, but out of memory, where a model of some layers has them, a block's call takes 41 us and 49 with the tiles in it.
        best.tile = aligned ? LINEAR_FEW : LINEAR_ANY_FEW;
        return best;
    }
    for (const int tile : {int(LINEAR_256), int(LINEAR_128), int(LINEAR_128_DEEP), int(LINEAR_64), int(LINEAR_64_TWICE), int(LINEAR_ANY)}) {
        if (aligned != (tile != LINEAR_ANY)) continue;
        const int64_t size = linear_tile_size(tile), tiles = ceil_div(rows, size) * ceil_div(cols, size);
        const LinearCost c = linear_cost(tile, form);
        for (int s = 1; s <= 64; s *= 2) {
            if (s > 1 && (end != END_STORE || pieces / s < 4 || one * s > static_cast<double>(room) || tiles * s > 1024)) break;
            if (tile == LINEAR_64_TWICE && tiles * s > 256) break;      // (two of them do not share a compute unit: 700 x 1536 x 1536, 264 tiles, 11.8 and 14.6 us)
            const double per_unit = static_cast<double>(ceil_div(tiles * s, 256));
            const double pairs = static_cast<double>(ceil_div(tiles * s, 256) / 2), piece = pairs * c.pair + (per_unit - 2 * pairs) * c.alone;
            const double us = c.start + c.more * per_unit + pieces / s * piece + (s > 1 ? 6 + one * (s + 1) / 4e6 : 0);
            if (best.us == 0 || us < best.us) {
                best.us = us;
                best.tile = tile;
                best.k_per_slice = static_cast<int>(padded(ceil_div(k > 0 ? k : 1, s)));
                best.slices = static_cast<int>(ceil_div(k > 0 ? k : 1, best.k_per_slice));
            }
        }
    }
    return best;
}

// Products of END_STORE that do not wait for each other: the first of FORM_KN, the others of FORM_NN, aligned; rows 0: not there
struct LinearSize {
    int64_t rows, cols, k;
};

// The tile and the first one's slices on which they go in one launch; LINEAR_ANY: one by one.  It takes the work of all over 256 compute units that have two tiles at a time (`half` a K-tile),
// a part of the longest sum in the end, or that sum alone, or the rounds of all that are as long; tiles start and end in rounds.  Estimated and measured, and one by one, in us:
//   333 x 1001 x 4096 with 4096 x 1001 and 1001 x 1999 x 333     128 in four slices 25 and 25.6, 34.3    64 x 512 x 2048 with 2048 x 512 and 512 x 1024 x 64          64 in eight 10 and 10.2, 16.5
//   1024 x 1024 x 4096 with 4096 x 1024 and 1024 x 2048 x 1024   128 in two 45 and 40.5, 50.5            256 x 512 x 16384 with 16384 x 512 x 256                     128 in 16 27 and 30.3, 36.1
//   1000 x 1001 x 9999 with 9999 x 1001 x 1000                   128 in four 64 and 70.5, 71.0           4096 x 1024 x 4096 with 4096 x 1024 and 1024 x 2048 x 4096   one by one 118.8, 128 125.8
inline LinearPlan linear_plan_together(const LinearSize (&sizes)[3], size_t room)
{
    LinearPlan best{LINEAR_ANY, 1, 0, 0};
    int there = 0;
    double least = 0;
    for (int n = 0; n < 3; ++n)
        if (sizes[n].rows > 0) {
            ++there;
            least += 1.2 + linear_plan(n == 0 ? FORM_KN : FORM_NN, END_STORE, sizes[n].rows, sizes[n].cols, sizes[n].k, true, room).us;       // (a gap between launches)
        }
    if (there < 2) return best;
    const double one = static_cast<double>(sizes[0].rows) * padded(sizes[0].cols) * 4;
    for (const int tile : {int(LINEAR_128), int(LINEAR_64)}) {
        const int64_t size = linear_tile_size(tile);
        const bool large = tile == LINEAR_128;
        const double alone = large ? 0.82 : 0.19, half = large ? 0.5 : 0.2, tail = large ? 0.2 : 0.1, start = large ? 5.3 : 5.5, more = large ? 2 : 1.45;
        for (int s = 1; s <= 16; s *= 2) {
            const int64_t k = sizes[0].k > 0 ? sizes[0].k : 1, each = padded(ceil_div(k, s));
            if (s > 1 && (sizes[0].rows == 0 || k / s < 4 * LAYER_PIECE || one * s > static_cast<double>(room))) break;
            int64_t tiles[3], pieces[3], groups = 0, longest = 0, as_long = 0;
            double work = 0;
            for (int n = 0; n < 3; ++n) {
                tiles[n] = ceil_div(sizes[n].rows, size) * ceil_div(sizes[n].cols, size) * (n == 0 ? s : 1);
                pieces[n] = tiles[n] == 0 ? 0 : ceil_div(n == 0 ? each : sizes[n].k, LAYER_PIECE);
                groups += tiles[n];
                work += static_cast<double>(tiles[n]) * static_cast<double>(pieces[n]);
                longest = pieces[n] > longest ? pieces[n] : longest;
            }
            if (groups > 65536) break;
            for (int n = 0; n < 3; ++n) as_long += 2 * pieces[n] >= longest ? tiles[n] : 0;
            const double length = static_cast<double>(longest), last = as_long <= 256 ? length * alone : static_cast<double>(ceil_div(as_long, 512)) * length * 2 * half;
            const double body = work / 256 * half + length * alone * tail;
            const double us = start + more * static_cast<double>(groups) / 256 + (body > last ? body : last) + (s > 1 ? 2 + one * (2 * s + 1) / 8e6 : 0);
            if (us < 0.97 * least) {                     // (what is not clearly ahead is not taken)
                least = us;
                best = {tile, static_cast<int>(ceil_div(k, each)), static_cast<int>(each), us};
            }
        }
    }
    return best;
}

// Rows on 16 bytes, whole pieces along a sum where the operand is the caller's, 32-bit offsets inside a tile
inline bool linear_aligned(int form, int end, const LinearArgs &a)
{
    auto on16 = [](const void *x, int64_t ld) { return reinterpret_cast<uintptr_t>(x) % 16 == 0 && ld % 8 == 0 && ld <= int64_t(1) << 21; };
    if (!on16(a.P, a.ldp) || !on16(a.Q0, a.ldq0)) return false;
    if ((end == END_GATED || a.segment > 0) && !on16(a.Q1, a.ldq1)) return false;
    // a piece of an operand along the sum in which the sum ends has to hold zeros behind it, whatever the other operand is: nothing times infinity is no number
    if (form == FORM_NN || (a.k % 8 == 0 && a.segment == 0)) return true;
    return a.p_padded && (form == FORM_KN || a.q_padded);
}

}  // namespace mg
