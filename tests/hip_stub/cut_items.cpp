// The work items of a product by row whose last round of tiles is cut (csrc/ops_groups.hpp) on the host:
// every place and column is made once.  tests/test_cut_items_cpu.py builds and runs it.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <random>
#include <string>
#include <vector>

// (what the header's walk over groups exchanges between lanes is not called here)
int __shfl_up(int v, int) { return v; }
int __shfl_xor(int v, int) { return v; }
uint64_t __ballot(bool b) { return b; }
int __builtin_amdgcn_readlane(int v, int) { return v; }
int __builtin_amdgcn_readfirstlane(int v) { return v; }
using std::max;
using std::min;
#define __device__
#include "ops_groups.hpp"

int main() {
    int bad = 0;
    auto check = [&](bool ok, const std::string &what) {
        if (!ok && ++bad <= 20) std::printf("FAIL %s\n", what.c_str());
    };
    std::mt19937 rng(1);
    constexpr int bn = 256;
    for (int round = 0; round < 4000; ++round) {
        const int units = round % 5 == 0 ? 304 : 256, tiles = static_cast<int>(rng() % (round % 3 ? 40 : 400)), tail = static_cast<int>(rng() % 9);
        const int m = 200 + static_cast<int>(rng() % 5000), mw = std::max(m + static_cast<int>(rng() % 8), bn);
        const int ct = (m + bn - 1) / bn, items = (tiles + tail) * ct;
        const int blocks = (items + 7) / 8 * 8 + 3 * units / 4 + 24;
        const std::string what = std::to_string(tiles) + " + " + std::to_string(tail) + " tiles, " + std::to_string(m) + " of " +
                                 std::to_string(mw) + " columns: ";
        // quarters of every tile, in columns of tiles
        std::vector<int> made((tiles + tail) * ct * 4);
        int whole = 0, quarters = 0;
        for (int id = 0; id < blocks + 64; ++id) {
            int t = -1, c0 = -1, quarter = -2;
            if (!hwr::cut_item(id, tiles, tail, m, mw, bn, units, t, c0, quarter)) continue;
            check(id < blocks, what + "an item past the grid");
            check(t >= 0 && t < tiles + tail && c0 >= 0 && c0 + bn <= mw && quarter >= -1 && quarter < 4, what + "in range");
            check(t < tiles || quarter < 0, what + "rows in no group whole");
            if (t < 0 || t >= tiles + tail || c0 < 0) continue;
            const int j = (c0 + bn - 1) / bn;            // (the last column of tiles may start early)
            (quarter < 0 ? whole : quarters) += t < tiles;
            for (int q = quarter < 0 ? 0 : quarter; q <= (quarter < 0 ? 3 : quarter); ++q) ++made[(t * ct + std::min(j, ct - 1)) * 4 + q];
        }
        bool once = true;
        for (int v : made) once = once && v == 1;
        check(once, what + "every quarter once");
        check(whole % units == 0 || (quarters == 0 && whole % units * 4 > units), what + std::to_string(whole) + " whole and " + std::to_string(quarters));
    }
    std::printf(bad ? "%d failed\n" : "ok\n", bad);
    return bad ? 1 : 0;
}
