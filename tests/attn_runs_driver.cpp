// Host check of which counters and partial results of the workspace a split row is joined through (csrc/moe_attn_split.h): the blocks
// that share it where the lengths are those that the split was made from, and blocks of this launch whatever they are.
// tests/test_attention_host_runs.py builds and runs it.  Prints "all ok" or ends with a line that says what is wrong.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "moe_attn_split.h"

static void fail(const char* what, long a, long b, long c, long d) {
    std::printf("wrong: %s (%ld, %ld, %ld, %ld)\n", what, a, b, c, d);
    std::exit(1);
}

int main() {
    std::mt19937 g(1);
    long outside = 0;
    for (int round = 0; round < 200000; ++round) {
        const int rows = 1 + (int)(g() % 40), most = 1 + (int)(g() % (round % 5 ? 40u : 700u)), runs = 1 + (int)(g() % (round % 3 ? 70u : 512u));
        std::vector<int> tiles(rows);
        int total = 0;
        for (int& t : tiles) total += t = 1 + (int)(g() % (unsigned)most);
        const moe::Runs d = moe::deal_tiles(total, runs);
        for (int start = 0, i = 0; i < rows; start += tiles[i++]) {      // the rows that the split was made from
            int run0, first;
            const int n = moe::runs_of_row(d, start, tiles[i], first), m = moe::runs_within(d, start, tiles[i], runs, run0);
            if (n >= 2 && (m != n || run0 != first)) fail("a row that is split", n, m, first, run0);
            if (n >= 2 && run0 + n > runs) fail("more blocks than there are", run0, n, runs, total);
        }
        for (int i = 0; i < 20; ++i) {                                   // rows as other lengths give them
            const int start = (int)(g() >> (1 + g() % 31)), t = 1 + (int)(g() >> (1 + g() % 31)) % (1 << 27);
            int run0, first;
            const int n = (int64_t)start + t <= INT32_MAX ? moe::runs_of_row(d, start, t, first) : 1 << 30;
            outside += n >= 2 && (first < 0 || first + (long)n > runs);
            const int m = moe::runs_within(d, start, t, runs, run0);
            if (m < 1 || run0 < 0 || run0 + m > runs) fail("outside the workspace", run0, m, runs, start);
        }
    }
    for (int start : {0, 1, 1 << 30, INT32_MAX})
        for (int t : {0, 1, 1 << 27, INT32_MAX})
            for (int runs : {1, 2, 512})
                for (int total : {1, 1000, (1 << 30) - 1}) {
                    int run0;
                    const int m = moe::runs_within(moe::deal_tiles(total, runs), start, t, runs, run0);
                    if (m < 1 || run0 < 0 || run0 + m > runs) fail("outside the workspace", run0, m, runs, start);
                }
    // rows of one request that are read together: where that is less work, not where it is only no more tiles
    const struct { int n, whole, pack, sum, want; } groups[] = {
        {125, 125, 4, 500, 125}, {125, 1, 4, 376, 125}, {125, 0, 4, 128, 0}, {16, 0, 16, 16, 0}, {16, 0, 16, 79, 0}, {16, 0, 16, 80, 16}, {1, 0, 16, 16, 1}, {1, 0, 2, 2, 1},
        {2, 1, 3, 5, 2}, {9, 9, 2, 8, 0}, {1 << 26, 0, 16, (1 << 30) - 1, 1 << 26}, {1 << 26, 0, 16, 1 << 26, 0}};
    for (const auto& c : groups)
        if (moe::shared_tiles(c.n, c.whole, c.pack, c.sum) != c.want) fail("rows together", c.n, c.whole, c.pack, c.sum);
    if (!outside) fail("no row here leaves the workspace by itself", 0, 0, 0, 0);
    std::printf("all ok\n");
}
