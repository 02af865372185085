// Host check of how the attention's tiles are dealt to blocks (csrc/moe_attn_split.h) and of the division by multiplication
// (csrc/moe_host.h): tests/test_attention_host.py builds and runs it.  Prints "all ok" or ends with a line that says what is wrong.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "moe_attn_split.h"
#include "moe_host.h"

static void fail(const char* what, long a, long b, long c) {
    std::printf("wrong: %s (%ld, %ld, %ld)\n", what, a, b, c);
    std::exit(1);
}

// Deals rows of the given tiles to blocks as the kernel does; every tile has to belong to one block, and every row that several
// blocks share to exactly those that runs_of_row names, its first part in the one slot and the others in the other.
static void check(const std::vector<int>& tiles, int runs) {
    std::vector<int> start(tiles.size());
    int total = 0;
    for (size_t i = 0; i < tiles.size(); ++i) {
        start[i] = total;
        total += tiles[i];
    }
    const moe::Runs d = moe::deal_tiles(total, runs);
    if ((long)d.share * runs < total) fail("tiles are left over", d.share, runs, total);
    auto bound = [&](int w) {
        const long x = (long)w * d.share;
        if (w == 0 || x >= total) return (int)(x < total ? x : total);
        size_t row = 0;
        while (start[row] + tiles[row] <= x) ++row;
        return moe::run_end(d, (int)x, start[row], tiles[row]);
    };
    std::vector<int> parts(tiles.size(), 0);
    int at = 0;
    size_t row = 0;
    for (int w = 0; w < runs; ++w) {
        const int b0 = bound(w), b1 = bound(w + 1);
        if (b0 != at || b1 < b0) fail("ends of blocks", w, b0, b1);
        if (b1 - b0 > d.share + 2 * d.near) fail("a block has too much", w, b0, b1);
        int slots[2] = {0, 0};
        while (row < tiles.size() && b0 < b1) {
            const int r0 = start[row], r1 = r0 + tiles[row];
            if (r0 >= b1) break;
            const bool begins = r0 >= b0, ends = r1 <= b1;
            if (!(begins && ends)) {
                int run0;
                const int n = moe::runs_of_row(d, r0, tiles[row], run0);
                if (n < 2 || w < run0 || w >= run0 + n) fail("a part of a row that is not split there", (long)row, w, run0);
                if (begins != (w == run0)) fail("the first part of a row", (long)row, w, run0);
                if (ends != (w == run0 + n - 1)) fail("the last part of a row", (long)row, w, run0 + n - 1);
                if (++slots[begins] > 1) fail("two parts in one slot", (long)row, w, begins);
                ++parts[row];
            } else {
                int run0;
                if (moe::runs_of_row(d, r0, tiles[row], run0) > 1) fail("a whole row that should be split", (long)row, w, run0);
            }
            if (!ends) break;
            ++row;
        }
        at = b1;
    }
    if (at != total || row != tiles.size()) fail("tiles that no block has", at, total, (long)row);
    for (size_t i = 0; i < tiles.size(); ++i) {
        int run0;
        const int n = moe::runs_of_row(d, start[i], tiles[i], run0);
        if (parts[i] && parts[i] != n) fail("parts of a row", (long)i, parts[i], n);
    }
}

int main() {
    std::mt19937 g(1);
    for (int round = 0; round < 20000; ++round) {
        const int rows = 1 + (int)(g() % (round % 3 ? 9 : 200)), most = 1 + (int)(g() % (round % 5 ? 40 : 700)), runs = 1 + (int)(g() % 70);
        std::vector<int> tiles(rows);
        for (int& t : tiles) t = 1 + (int)(g() % (unsigned)(g() % 4 ? most : 3));
        check(tiles, runs);
    }
    check({1}, 512);
    check({1 << 20}, 512);
    check({5000000, 1, 1, 1}, 64);
    for (int round = 0; round < 3000000; ++round) {
        const int bits = 1 + (int)(g() % 31);
        int d = (int)(g() & ((1u << bits) - 1));
        if (d < 1) d = 1;
        int shift;
        const uint64_t magic = moe::division_magic(d, shift);
        const uint32_t near = (uint32_t)(g() % 64) * (uint32_t)d;
        for (uint32_t t : {(uint32_t)g() & 0x7fffffffu, 0x7fffffffu, near & 0x7fffffffu, (near - 1) & 0x7fffffffu, 0u, 1u})
            if (t && (uint64_t)t * magic / t != magic) fail("product out of range", t, d, shift);
            else if ((int)(((uint64_t)t * magic) >> shift) != (int)(t / (uint32_t)d)) fail("quotient", t, d, shift);
    }
    std::printf("all ok\n");
}
