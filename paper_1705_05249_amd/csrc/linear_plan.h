// Which kernel a product of 16-bit matrices takes and in how many slices of its sum.  Host code alone: it can be asked without a GPU.
#pragma once

#include "internal.h"
#include "layers.h"

namespace mg {

struct LinearPlan {
    int tile;                        // LinearTile
    int slices, k_per_slice;
};

// What a tile takes, in us: `alone` for 64 values of the sum while a compute unit has one of its tiles, with n of them n * `each`; around the sum `start`, and
// `more` for every round of tiles (C leaves).
struct LinearCost {
    double alone, each, start, more;
};
inline LinearCost linear_cost(int tile, int form)
{
    (void)form;
    switch (tile) {
        case LINEAR_256: return {1.5, 1.65, 4, 6};
        case LINEAR_128: return {0.6, 0.5, 3, 2};
        case LINEAR_64: return {0.3, 0.17, 3, 1};
        default: return {0.5, 0.35, 3, 1.5};
    }
}

// The least of the estimates.  Slices cost a launch that reads what they wrote; no slice gets fewer than four pieces of 64.
inline LinearPlan linear_plan(int form, int end, int64_t rows, int64_t cols, int64_t k, bool aligned, size_t room)
{
    LinearPlan best{LINEAR_ANY, 1, static_cast<int>(padded(k > 0 ? k : 1))};
    const double pieces = static_cast<double>(ceil_div(k > 0 ? k : 1, LAYER_PIECE)), one = static_cast<double>(rows) * padded(cols) * 4;
    double least = 0;
    for (const int tile : {int(LINEAR_256), int(LINEAR_128), int(LINEAR_64), int(LINEAR_ANY)}) {
        if (aligned != (tile != LINEAR_ANY)) continue;
        const int64_t size = linear_tile_size(tile), tiles = ceil_div(rows, size) * ceil_div(cols, size);
        const LinearCost c = linear_cost(tile, form);
        for (int s = 1; s <= 64; s *= 2) {
            if (s > 1 && (end != END_STORE || pieces / s < 4 || one * s > static_cast<double>(room) || tiles * s > 1024)) break;
            const double per_unit = static_cast<double>(ceil_div(tiles * s, 256));
            const double piece = c.each * per_unit > c.alone ? c.each * per_unit : c.alone;
            const double us = c.start + c.more * per_unit + pieces / s * piece + (s > 1 ? 4 + one * (s + 1) / 4e6 : 0);
            if (least == 0 || us < least) {
                least = us;
                best.tile = tile;
                best.k_per_slice = static_cast<int>(padded(ceil_div(k > 0 ? k : 1, s)));
                best.slices = static_cast<int>(ceil_div(k > 0 ? k : 1, best.k_per_slice));
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
