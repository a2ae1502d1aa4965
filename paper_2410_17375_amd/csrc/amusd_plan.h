// Choices between forms of a stage that follow from sizes alone.  Host code, no GPU needed.
#pragma once
#include <cstdint>
#include <initializer_list>

namespace amusd {

// Attention of a prompt's rows: a workgroup per row tile and kv head that walks all keys (whole), or the keys split into
// stretches and the chunks' partials merged.
//
// The whole form takes, per 1000 keys, `alone` us while each of its workgroups has a compute unit for itself (the last tile's
// walk is its time), and `two` where some share one (a middling tile's; the longest begin first).  The split form fills the
// chip whatever the number of tiles: `split` us per 1000 keys and workgroup of the whole form per compute unit, the partials
// (stored and read back at 7.5 TB/s) on top, and a stretch and 2 us for its ends.  A key block at the end of an odd run takes
// 0.75 of a step of two.  From 1.9 workgroups a compute unit on the whole form is the faster one for any number of keys.
// Measured (MI355X, 1521 prompts of 17 to 2000 rows behind 0 to 14000 keys, 1 to 32 kv heads, the eight forms, contexts of 1000
// to 16384): the choice is 0.4 % from the better form on average, 20 % and more in six.  whole / split us: heads of 64 in fours,
// 8 kv heads, 768 rows behind 8000 keys 185 / 152, float32 622 / 465; in eights, 4 kv heads, 192 / 233; heads of 128 in fours, 250
// rows behind 1500 43 / 32, 600 rows behind none 22 / 55.
inline bool pf_attention_walks_whole_rows(bool bf16, int head_dim, int group, int kv_heads, int rows, int keys, int cus, int chunk, int run_blocks,
                                          int stretch) {
    struct Rates { double alone, two, split; };
    static const Rates rates[2][2][2] = {{{{48, 72, 30}, {76, 136, 70}}, {{81, 136, 69}, {137, 274, 158}}},      // float32: heads of 64, 128,
                                         {{{15, 20, 7}, {17, 38, 18}}, {{19, 28, 14}, {26, 56, 33}}}};           // in fours, eights
    if (group != 4 && group != 8) return false;
    const Rates& r = rates[bf16][head_dim == 128][group == 8];
    const int wgs = (rows + 15) / 16 * kv_heads;
    const double per_cu = (double)wgs / cus;
    if (per_cu >= 1.9) return true;
    const bool pairs = run_blocks == 1 && group == 4 && head_dim == 64;       // a chunk's two runs in one step
    const double odd = run_blocks % 2 && !pairs ? (run_blocks - 1 + 2 * 0.75) / run_blocks : 1.;
    const double partials = 1000. / chunk * 16 * group * wgs * (head_dim + 4) * 8 / 7.5e6;
    const double whole = per_cu <= 1 ? keys * r.alone * odd : (keys - 0.4 * rows) * r.two * odd;    // ns
    const double split = keys * (per_cu * r.split * odd + partials);
    return whole <= split + r.alone * stretch + 2000;
}

// Attention of a verify pass, groups of 4 or 8 heads: tiles of (row, head) pairs (true) or a tile per head, whose units are one
// (kv head, chunk) each.  units: of the latter; tiles: of pairs, per chunk on average; run_blocks: key blocks of a wave's run.
//
// A tile per head is a workgroup a compute unit, round after round, over blocks that are staged once for all heads.  Pairs need
// fewer products while rows are few, and their workgroups share a compute unit; with many rows each tile fetches the keys for
// itself.  So pairs
//   where there is more than one round (168 sizes of the eight forms: all faster, by 0.2 to 154 us a layer.  Many rows to a unit do
//     not occur there, as it takes three sequences and a pass has 16 rows: at most 0.47 tiles a head);
//   up to half as many tiles as heads (float32 heads of 128, twice the registers a block: fewer);
//   and for 16-bit heads of 64 in runs of up to 7 blocks whatever the rows: both of a unit's forms are then mostly its beginning and
//     end (40 sizes, 0.8 us a layer less in the mean, 0.8 more at most; with 8 and more blocks and every compute unit taken
//     1.2 more: 16 rows behind 16360 keys 18.8 / 20.0).
// The line holds for full contexts, whose units are about the compute units.  With fewer than 200 of 256 pairs were faster for any number
// of rows (191 sizes that this takes a tile per head for, 0.2 us a layer slower at worst, 1 to 10 faster in the mean of a form): not made use of.
// Measured (MI355X): the attention's and the O-projection's kernels over 990 sizes, 1 to 8 sequences of 1 to 16 rows behind 100 to 16360
// keys; where the rule says pairs they are 1 us a layer slower at worst.  Whole passes of 2 layers, us, tile per head / pairs: 8B, 8 rows
// behind 2000 keys 211 / 208, behind 12000 224 / 219, 16 rows 238 / 241; 8 sequences of one row to 4000 260 / 235; heads in eights, 12 rows
// behind 7000 234 / 238; float32, 8 rows behind 2000 359 / 365, 2 rows behind 7000 391 / 375; 1B (4 layers), 16 rows behind 4000 236 / 229.
inline bool attention_packs_rows(bool bf16, int head_dim, int group, int units, double tiles, int run_blocks, int cus) {
    if (units > cus) return true;
    if (tiles <= group * (head_dim == 128 && !bf16 ? 0.375 : 0.5)) return true;
    return bf16 && head_dim == 64 && run_blocks < 8;
}

// Attention over an 8-bit cache: (tile of 16 pairs, kv head)s while which a tile's chunks are split over waves, and those whose sums there
// is room for at a time: in 128 MB or a 32nd of the cache, but those of 16 rows always (of up to n_seqs sequences, whose last tiles
// need not be full).  us, 64 rows of the 8B heads behind 131072 keys, 128 tiles together 462, 43 at a time 534, 32 at a time 586;
// 100 rows a wave a tile 2159, 50 tiles at a time 807.
inline int q8_split_tiles(int cus) { return cus * 5 / 4; }
inline int q8_part_tiles(int n_seqs, int group, int kv_heads, int cus, int64_t tile_bytes, int64_t cache_bytes) {
    const int segs = n_seqs < 16 ? n_seqs : 16;
    const int64_t least = (int64_t)(16 * group + 15 * segs) / 16 * kv_heads, split = q8_split_tiles(cus);
    const int64_t bytes = cache_bytes / 32 < 128 << 20 ? 128 << 20 : cache_bytes / 32, room = bytes / tile_bytes;
    const int64_t most = split < room ? split : room;
    return (int)(least > most ? least : most);
}

// Products of 8-bit integers: forms for few rows, whose workgroups' eight waves split the contraction of MT x 16 rows and NT x 16 features
// (kQ8FewMTxNT), and for many, whose workgroups hold a tile of the result (kQ8Tile<features>x<rows>).
enum Q8Form { kQ8Few1x1, kQ8Few1x2, kQ8Few2x2, kQ8Few2x4, kQ8Few4x4, kQ8Tile64, kQ8Tile128x64, kQ8Tile128, kQ8Tile256 };
// .. tiles of 16 rows and of 16 features of a workgroup
inline int q8_form_rows(Q8Form f) { const int n[] = {1, 1, 2, 2, 4, 4, 4, 8, 16}; return n[f]; }
inline int q8_form_tiles(Q8Form f) { const int n[] = {1, 2, 2, 4, 4, 4, 8, 8, 16}; return n[f]; }
struct Q8Plan {
    Q8Form form;
    int ways;        // workgroups that share a tile's contraction: 1, or 2 or 4 whose sums meet in a workspace
};
constexpr int kQ8Tickets = 4096;        // of a workspace: a wave (few rows: a workgroup) and tile has one
constexpr int kQ8MinBlocks = 16;        // blocks of 64 columns of a workgroup that shares

// Which: up to 16 rows by the number of feature tiles alone (one a workgroup while there is a compute unit for each; us with 1x1 / 1x2, 8
// rows: 4096 x 4096 5.3 / 6.0, 6144 features 7.6 / 6.8, 28672 24.9 / 19.8; shared by two, 2048 x 8192 6.9 / 7.4 alone, every other
// 0.6 to 2 slower); with more rows by an estimate of each form's time, us:
//   few: 2.6 + 0.9 a workgroup of a compute unit + its rounds x blocks of 64 columns (a wave's whole ones) x (0.022 a feature tile + 0.021 a
//     row tile): what a compute unit loads at about 50 GB/s;
//   tiles: a block takes its workgroup at least `alone` (what a compute unit loads, again); where compute units are full, `full` a workgroup
//     of them.  256 x 256 has a compute unit to itself: rounds x (blocks x 0.55 to 0.70 + 9); clocks fall as more of the chip multiplies;
//   shared: 2.3 + 0.35 a megabyte of sums that are written and read.
// Measured (MI355X, five projections of the 8B and the 1B model, 20 to 1024 rows, all forms): 3 % over the best in the mean.  Sharing
// gives, us alone / shared: down 8B, 32 rows 22.8 / 17.2, 256 rows 45.8 / 33.7, 512 rows 71.3 / 49.9; QKV 8B, 128 rows 16.4 / 13.3;
// down 1B, 32 rows 12.0 / 9.2, 512 rows 26.6 / 19.7.
inline Q8Plan q8_gemm_plan(int tiles, int kblocks, bool gated, int rows, int cus, bool shared) {
    if (rows <= 16) return {!gated && tiles <= cus ? kQ8Few1x1 : kQ8Few1x2, 1};
    Q8Plan best = {kQ8Few2x2, 1};
    double least = 1e30;
    auto ceil_div = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
    auto groups_of = [&](Q8Form f) { return ceil_div(tiles, q8_form_tiles(f)) * ceil_div(rows, q8_form_rows(f) * 16); };
    auto offer = [&](Q8Form f, int waves, auto us) {     // us(workgroups, blocks of each)
        const int64_t groups = groups_of(f);
        for (int ways = 1; ways <= (shared ? 4 : 1); ways *= 2) {
            if (ways > 1 && (kblocks < ways * kQ8MinBlocks || groups * waves > kQ8Tickets)) break;
            const int64_t wgs = groups * ways;
            const double sums = 1e-6 * wgs * (q8_form_tiles(f) * q8_form_rows(f) * 1024);
            const double all = us((double)wgs, (double)ceil_div(kblocks, ways)) + (ways > 1 ? 2.3 + 0.35 * sums : 0);
            if (all < least) { least = all; best = {f, ways}; }
        }
    };
    for (Q8Form f : {kQ8Few2x2, kQ8Few2x4, kQ8Few4x4})
        offer(f, 1, [&](double wgs, double blocks) {
            const int64_t rounds = ceil_div((int64_t)wgs, cus), whole = ceil_div((int64_t)blocks, 8) * 8;
            return 2.6 + 0.9 * wgs / cus + rounds * whole * (0.022 * q8_form_tiles(f) + 0.021 * q8_form_rows(f));
        });
    auto tile = [&](Q8Form f, double alone, double full) {
        offer(f, 4, [&](double wgs, double blocks) { return 2.4 + blocks * (alone > wgs * full / cus ? alone : wgs * full / cus); });
    };
    tile(kQ8Tile64, 0.20, 0.12);
    tile(kQ8Tile128x64, 0.24, 0.18);
    tile(kQ8Tile128, 0.35, 0.285);
    const int64_t wgs = groups_of(kQ8Tile256), rounds = ceil_div(wgs, cus);
    const double us = 3 + rounds * (kblocks * (0.55 + 0.15 * (wgs < cus ? (double)wgs / cus : 1.)) + 9);
    return us < least ? Q8Plan{kQ8Tile256, 1} : best;
}

}  // namespace amusd
