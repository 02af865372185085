// How the tiles of a key/value head's rows are dealt to blocks (moe_attn.hip): integer arithmetic alone, shared by the kernel and a host test.
#pragma once

#ifndef MOE_HD
#if defined(__HIPCC__)
#define MOE_HD __host__ __device__ __forceinline__
#else
#define MOE_HD inline
#endif
#endif

namespace moe {

// Least tiles of a block: one for each of its wavefronts.  (us with 4 / 8: three short float32 requests 6.4 / 7.3, 36 requests of 60 to 700
// tokens 16 either way.)
constexpr int kLeastTiles = 4;
// How many tiles the end of a block may move to meet the end of a row, so that the row is not shared with another block.  (us
// with 0 / 2 / 4 / 8: 36 requests of 60 to 700 tokens 19.8 / 17.6 / 16.0 / 16.2, 830 prompt rows 40 / 40 / 37 / 37, long requests the same.)
constexpr int kNearTiles = 4;

// Block w has the tiles from run_end(w * share) to run_end((w + 1) * share).
struct Runs {
    int share, near;
};
MOE_HD Runs deal_tiles(int total, int runs) {
    Runs d;
    d.share = (total + runs - 1) / runs;
    if (d.share < kLeastTiles) d.share = kLeastTiles;
    d.near = d.share / 2 < kNearTiles ? d.share / 2 : kNearTiles;
    return d;
}
// Where the end x of a block, 0 < x < total, in a row with `tiles` tiles from `start` on, is moved.
MOE_HD int run_end(const Runs& d, int x, int start, int tiles) {
    return x - start <= d.near ? start : start + tiles - x <= d.near ? start + tiles : x;
}
// The blocks run0 .. run0 + n - 1 that a row is split over: one more than there are ends inside it that stay where they are.
MOE_HD int runs_of_row(const Runs& d, int start, int tiles, int& run0) {
    run0 = (start + d.near) / d.share;
    return (start + tiles - d.near - 1) / d.share - run0 + 1;
}
// The same, for the counters and partial results of `runs` blocks that the row is joined through.  Rows of the split are as they are above; a
// row whose length was changed while the call runs is cut to them, so that it reaches none but these.
MOE_HD int runs_within(const Runs& d, int start, int tiles, int runs, int& run0) {
    const int all = d.share * runs;              // no less than there are tiles
    if (start > all - 1) start = all - 1;
    if (tiles > all - start) tiles = all - start;
    int n = runs_of_row(d, start, tiles, run0);
    if (run0 > runs - 1) run0 = runs - 1;
    if (n > runs - run0) n = runs - run0;
    return n < 1 ? 1 : n;
}
// The tiles that `pack` rows of one request read together, or 0 where they are better read one by one, `sum` tiles: n tiles, `whole` of
// them seen whole by all rows; any other takes `pack` second products, each about a quarter of what a tile costs that is read once more from the L2.
// us together / one by one, 16 / 16 heads of 128, 20 groups of 16 rows with 1, 2, 3, 5, 8, 15 of 4000 tokens and the others of 10: 255 / 137, 253 / 165,
// 254 / 279, 254 / 486, 255 / 714, 281 / 1163 (the rule: one by one up to 3); 32 / 8 heads, 100 groups of 4 rows with 1, 2, 3 of 4000: 315 / 308, 304 / 574, 309 / 841
// (one by one with 1); rows 16 tokens apart with a window of 32, 16 / 16 heads: 67 / 28, one after another with a window of 10: 39 / 50.
MOE_HD int shared_tiles(int n, int whole, int pack, int sum) { return n + (n - whole) * pack / 4 <= sum ? n : 0; }

}  // namespace moe
