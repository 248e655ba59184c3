// Which prefill-shaped tiles run on which XCD. Block b of a launch runs on XCD
// b mod kXcds (up to a fixed rotation), and each XCD has its own L2: of every
// chunk of a longest-first list each XCD gets consecutive tiles, row blocks of
// one query head, which read the same K and V. Host and device code: the
// planner orders long launches (plan.cpp), the quantised mixed launch its own
// blocks (attn_quant.hip).
#pragma once

#include <stdint.h>

#include "mixed_order.h"
#include "plan_format.h"

namespace sangam {

constexpr int kXcds = 8;
constexpr int kXcdOrderMinRounds = 8;  // rounds of tiles per work-group slot from which the planner orders

// Place in the order of entry `at` of a list of n, and the entry at a place. A
// last, partial chunk keeps its remainder in order.
SANGAM_HD inline int xcd_place(int at, int n, int chunk) {
    const int base = at / chunk * chunk, q = at - base;
    const int each = (chunk < n - base ? chunk : n - base) / kXcds;
    return q < each * kXcds ? base + kXcds * (q % each) + q / each : at;
}
SANGAM_HD inline int xcd_entry(int place, int n, int chunk) {
    const int base = place / chunk * chunk, q = place - base;
    const int each = (chunk < n - base ? chunk : n - base) / kXcds;
    return q < each * kXcds ? base + q % kXcds * each + q / kXcds : place;
}

// Chunk of the order that the planner gave n tiles (the launch's slots), or 0: in list order.
inline int xcd_plan_chunk(int64_t n, int prefill_rows, int cus) {
    const int64_t slots = int64_t(cus / kXcds > 1 ? cus / kXcds : 1) * (prefill_rows == kWidePrefillRows ? 1 : 2) * kXcds;
    return n >= kXcdOrderMinRounds * slots ? int(slots) : 0;  // (n counts as int)
}

// A mixed launch's prefill block `index` of n, in rounds of `round`: the tile
// that it takes and which half of it (wide: two blocks a tile). Where the plan
// is ordered already, whose chunks are of whole tiles, that order is undone
// first. One after the other they would undo each other: 5 prefills of 3400
// rows of 32 heads, an XCD's blocks of a round are of 9.0 heads, in the plan's
// order alone of 5.6, with it undone of 2.8 (16 of 900 rows: 14.0, 8.8, 8.8).
struct XcdTile {
    int tile;
    int half;
};
SANGAM_HD inline XcdTile xcd_mixed_tile(int index, int n, int wide, int round, int plan_chunk) {
    const int block = xcd_entry(index, n, round);
    const int tile = block >> wide;
    return {plan_chunk > 0 ? xcd_place(tile, n >> wide, plan_chunk) : tile, block & wide};
}

}  // namespace sangam
