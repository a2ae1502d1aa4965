// What the choice of a form for a product of 8-bit integers has to keep to, over sizes.  Exits with the number of failures.
#include <cstdio>

#include "../../paper_2410_17375_amd/csrc/amusd_plan.h"

using namespace amusd;

int main() {
    int bad = 0;
    long forms[9] = {}, ways[5] = {};
    auto check = [&](bool ok, const char* what, int tiles, int kblocks, int rows) {
        if (!ok && ++bad < 20) std::printf("%s: %d tiles, %d blocks, %d rows\n", what, tiles, kblocks, rows);
    };
    for (int cus : {64, 256, 304})
        for (int tiles = 1; tiles < 10000; tiles += 1 + tiles / 7)
            for (int kblocks = 1; kblocks <= 2048; kblocks += 1 + kblocks / 5)
                for (int rows = 1; rows < 200000; rows += 1 + rows / 6)
                    for (bool gated : {false, true}) {
                        if (gated && tiles % 2) continue;
                        const Q8Plan p = q8_gemm_plan(tiles, kblocks, gated, rows, cus, true), alone = q8_gemm_plan(tiles, kblocks, gated, rows, cus, false);
                        const Q8Plan top = q8_gemm_plan(tiles, kblocks, gated, (rows + 15) / 16 * 16, cus, true);
                        const long ft = q8_form_tiles(p.form), rt = q8_form_rows(p.form);
                        const long groups = (tiles + ft - 1) / ft * ((rows + rt * 16 - 1) / (rt * 16));
                        forms[p.form]++;
                        ways[p.ways]++;
                        check(alone.ways == 1, "shared without a workspace", tiles, kblocks, rows);
                        check(p.form == top.form && p.ways == top.ways, "depends on more than the tiles of 16 rows", tiles, kblocks, rows);
                        check(!gated || p.form != kQ8Few1x1, "a gate without its up half", tiles, kblocks, rows);
                        check(p.ways == 1 || p.ways == 2 || p.ways == 4, "ways", tiles, kblocks, rows);
                        if (p.ways == 1) continue;
                        check(rows > 16 && p.form != kQ8Tile256, "shared by a form that cannot", tiles, kblocks, rows);
                        check(kblocks >= p.ways * kQ8MinBlocks, "parts too short", tiles, kblocks, rows);
                        check(groups * (p.form >= kQ8Tile64 ? 4 : 1) <= kQ8Tickets, "more tickets than there are", tiles, kblocks, rows);
                        // the parts of whole pairs of blocks: none is empty
                        const int pairs = (kblocks + 1) / 2, share = (pairs + p.ways - 1) / p.ways * 2, few = (kblocks + p.ways - 1) / p.ways;
                        check((p.ways - 1) * share < kblocks && (p.ways - 1) * few < kblocks, "an empty part", tiles, kblocks, rows);
                        // past the bound of the workspace's search nobody shares
                        check(rows <= (kQ8Tickets / 4 + 1) * 128, "shared past the bound", tiles, kblocks, rows);
                    }
    for (int f = 0; f < 9; ++f) check(forms[f] > 0, "a form that nothing reaches", f, 0, 0);
    check(ways[1] && ways[2] && ways[4], "a number of ways that nothing reaches", 0, 0, 0);
    return bad != 0;
}
