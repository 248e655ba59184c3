// Lists, for tests/test_xcd_order.py, the prefill tiles of mixed launches over
// a quantised cache: reads "tiles prefill_rows cus" lines and prints the chunk
// of the plan's order, then per block in launch order 2 x tile + half.
#include <cstdio>

#include "../../paper_2607_04206_amd/csrc/xcd_order.h"

using namespace sangam;

int main() {
    int tiles, rows, cus;
    while (std::scanf("%d %d %d", &tiles, &rows, &cus) == 3) {
        const int wide = rows == kWidePrefillRows, chunk = xcd_plan_chunk(tiles, rows, cus);
        std::printf("%d", chunk);
        for (int k = 0; k < tiles << wide; ++k) {
            const XcdTile x = xcd_mixed_tile(k, tiles << wide, wide, cus, chunk);
            std::printf(" %d", 2 * x.tile + x.half);
        }
        std::printf("\n");
    }
    return 0;
}
