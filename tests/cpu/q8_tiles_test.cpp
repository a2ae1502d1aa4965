// The room for chunk sums of attention over an 8-bit cache: enough for 16 rows, however they are spread over a cache's sequences, and no
// more than 128 MB or a 32nd of the cache beyond that.  Exits with the number of failures.
#include <cstdio>

#include "../../paper_2410_17375_amd/csrc/amusd_plan.h"

using namespace amusd;

// most tiles that `rows` rows can have in `segs` sequences of at least one row each
static int most_tiles(int rows, int segs, int group) {
    int best = 0;
    for (int n = 1; n <= rows - (segs - 1); ++n) {
        const int here = (n * group + 15) / 16, rest = segs == 1 ? 0 : most_tiles(rows - n, segs - 1, group);
        if (segs == 1 && n < rows) continue;
        if (here + rest > best) best = here + rest;
    }
    return best;
}

int main() {
    int bad = 0;
    auto check = [&](bool ok, const char* what, int n_seqs, int group, int heads, long tile) {
        if (!ok && ++bad < 20) std::printf("%s: %d sequences, groups of %d, %d heads, %ld bytes a tile\n", what, n_seqs, group, heads, tile);
    };
    for (int group : {1, 2, 4, 8}) {
        int need[17] = {};
        for (int segs = 1; segs <= 6; ++segs) need[segs] = most_tiles(16, segs, group);
        for (int n_seqs : {1, 2, 3, 4, 5, 6, 16, 100, 4096})
            for (int heads : {1, 2, 8, 32, 2048})
                for (long tile = 4096; tile < 1l << 30; tile *= 3) {
                    const long cache = tile * 37 * n_seqs, room = cache / 32 > 128 << 20 ? cache / 32 : 128 << 20;
                    const long tiles = q8_part_tiles(n_seqs, group, heads, 256, tile, cache);
                    for (int segs = 1; segs <= (n_seqs < 6 ? n_seqs : 6); ++segs)
                        check(tiles >= (long)need[segs] * heads, "no room for 16 rows", n_seqs, group, heads, tile);
                    check(n_seqs < 16 || tiles >= 16l * heads, "no room for a row of 16 sequences", n_seqs, group, heads, tile);
                    const long least = (group + (n_seqs < 16 ? n_seqs : 16)) * (long)heads;
                    check(tiles <= least || tiles * tile <= room, "more room than that", n_seqs, group, heads, tile);
                    check(tiles >= heads, "less than a tile", n_seqs, group, heads, tile);
                    check(n_seqs > 1 || tiles <= (long)group * heads || tiles * tile <= room, "more than a sequence's 16 rows", n_seqs, group, heads, tile);
                }
    }
    return bad != 0;
}
