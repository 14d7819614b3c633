// The walk over ragged groups (csrc/ops_groups.hpp) on the host: 64 lanes as
// coroutines that meet at every exchange.  tests/test_ops_host_cpu.py builds and runs it.
//
//   group_walk <scenario>      prints "ok", or the failed checks (exit 1)
#include <ucontext.h>

#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <functional>
#include <random>
#include <string>
#include <vector>

namespace {

constexpr int kLanes = 64;
struct Lanes {
    ucontext_t main, lane[kLanes];
    std::vector<char> stack[kLanes];
    int64_t slot[2][kLanes];
    int turn[kLanes], now = 0, left = 0;
    std::function<void(int)> body;
} L;

void run_lane() {
    L.body(L.now);
    const int me = L.now;
    --L.left;
    if (me + 1 < kLanes) {
        L.now = me + 1;
        setcontext(&L.lane[me + 1]);
    }
    setcontext(&L.main);
}
// Every lane's value; the lanes take turns, so that all have given theirs when one goes on.
const int64_t *exchange(int64_t v) {
    const int me = L.now, s = L.turn[me];
    L.turn[me] ^= 1;
    L.slot[s][me] = v;
    L.now = (me + 1) % kLanes;
    swapcontext(&L.lane[me], &L.lane[L.now]);
    return L.slot[s];
}
void wave(std::function<void(int)> body) {
    L.body = std::move(body);
    L.left = kLanes;
    for (int i = 0; i < kLanes; ++i) {
        L.stack[i].resize(1 << 16);
        L.turn[i] = 0;
        getcontext(&L.lane[i]);
        L.lane[i].uc_stack.ss_sp = L.stack[i].data();
        L.lane[i].uc_stack.ss_size = L.stack[i].size();
        L.lane[i].uc_link = nullptr;
        makecontext(&L.lane[i], run_lane, 0);
    }
    L.now = 0;
    swapcontext(&L.main, &L.lane[0]);
}

int __shfl_up(int v, int d) {
    const int me = L.now;
    const int64_t *all = exchange(v);
    return static_cast<int>(all[me >= d ? me - d : me]);
}
int __shfl_xor(int v, int d) {
    const int me = L.now;
    return static_cast<int>(exchange(v)[me ^ d]);
}
uint64_t __ballot(bool b) {
    const int64_t *all = exchange(b);
    uint64_t m = 0;
    for (int i = 0; i < kLanes; ++i) m |= static_cast<uint64_t>(all[i] != 0) << i;
    return m;
}
int __builtin_amdgcn_readlane(int v, int lane) { return static_cast<int>(exchange(v)[lane]); }
int __builtin_amdgcn_readfirstlane(int v) { return static_cast<int>(exchange(v)[0]); }
using std::max;
using std::min;

}  // namespace

#define __device__
#include "ops_groups.hpp"

namespace {

int g_bad = 0;
void check(bool ok, const std::string &what) {
    if (!ok && ++g_bad <= 20) std::printf("FAIL %s\n", what.c_str());
}

int count(const hwr::GroupsArg &g, int bm, bool tail) {
    int n = 0;
    wave([&](int lane) {
        const int v = hwr::count_tiles(g, bm, tail, lane);
        if (lane == 0) n = v;
    });
    return n;
}
hwr::RowTile find(const hwr::GroupsArg &g, int t, int bm, bool tail) {
    hwr::RowTile r{};
    wave([&](int lane) {
        const hwr::RowTile v = hwr::find_tile(g, t, bm, tail, lane);
        if (lane == 0) r = v;
    });
    return r;
}

// Tiles of groups that are as they should be: every place once, in order.
void tiles_cover_the_places() {
    std::mt19937 rng(1);
    for (int G : {1, 5, 63, 64, 65, 200}) {
        for (int bm : {16, 64, 256}) {
            std::vector<int32_t> off(G + 1);
            for (int i = 0; i < G; ++i) off[i + 1] = off[i] + (rng() % 3 ? static_cast<int>(rng() % 300) : 0);
            const int n = off[G] + 37;
            const hwr::GroupsArg g{n, G, off.data(), nullptr};
            for (bool tail : {false, true}) {
                const int tiles = count(g, bm, tail);
                int at = 0;
                for (int t = 0; t < tiles; ++t) {
                    const hwr::RowTile r = find(g, t, bm, tail);
                    const int p0 = r.g < G ? off[r.g] : off[G], p1 = r.g < G ? off[r.g + 1] : n;
                    check(r.p0 == at && r.p1 > r.p0 && r.p1 <= r.p0 + bm && r.p0 >= p0 && r.p1 <= p1 && (r.p0 - p0) % bm == 0,
                          "tile " + std::to_string(t) + " of " + std::to_string(G) + " groups");
                    at = r.p1;
                }
                check(at == (tail ? n : off[G]), "every place");
            }
        }
    }
}

// Offsets that hold anything: counts stay within the grid's, tiles within the places,
// and columns within the row.
void anything_in_offsets() {
    std::mt19937 rng(2);
    for (int n : {1, 1000, 1 << 20, 1 << 28, 700000000, INT32_MAX - 511})
        for (int G : {1, 63, 64, 65, 130, 1000, 1024})
            for (int kind = 0; kind < 4; ++kind) {
                std::vector<int32_t> off(G + 1);
                for (int i = 0; i <= G; ++i)
                    off[i] = kind == 0   ? (i & 1 ? n : 0)
                             : kind == 1 ? (i & 1 ? INT32_MAX : INT32_MIN)
                             : kind == 2 ? static_cast<int32_t>(rng())
                                         : static_cast<int32_t>(rng() % n) - (i & 1 ? 0 : n / 2);
                const hwr::GroupsArg g{n, G, off.data(), nullptr};
                for (int bm : {16, 32, 64, 128, 256})
                    for (bool tail : {false, true}) {
                        const std::string what = std::to_string(n) + " rows, " + std::to_string(G) + " groups, kind " +
                                                 std::to_string(kind) + ", tiles of " + std::to_string(bm);
                        const int tiles = count(g, bm, tail);
                        check(tiles >= 0 && tiles <= n / bm + std::min(n, G + 1), what + ": " + std::to_string(tiles) + " tiles");
                        if (tiles <= 0) continue;
                        for (int i = 0; i < 6; ++i) {
                            const int t = i == 0 ? 0 : i == 1 ? tiles - 1 : static_cast<int>(rng() % tiles);
                            const hwr::RowTile r = find(g, t, bm, tail);
                            check(r.g >= 0 && r.g <= G && r.p0 >= 0 && r.p0 <= r.p1 && r.p1 <= n && r.p1 - r.p0 <= bm,
                                  what + ", tile " + std::to_string(t) + ": " + std::to_string(r.p0) + " to " + std::to_string(r.p1));
                            check(tail || r.g < G, what + ": a group");
                        }
                        if (bm < 32) continue;
                        const int m = 2 * bm + 5;
                        const int64_t ids = std::min<int64_t>((n / bm + std::min(n, G + 1)) * int64_t{3} + 8, INT32_MAX);
                        for (int i = 0; i < 20; ++i) {
                            const int id = static_cast<int>(rng() % ids);
                            int t = 0, c0 = 0, part = 0;
                            if (!hwr::row_item(id, tiles, m, m, bm, 1, t, c0, part)) continue;
                            check(t >= 0 && t < tiles && c0 >= 0 && c0 + bm <= m && part == 0,
                                  what + ", item " + std::to_string(id) + ": column " + std::to_string(c0));
                        }
                    }
            }
}

// An order that holds anything gives a row of the batch or none.
void anything_in_order() {
    std::mt19937 rng(3);
    for (int n : {1, 7, 1000, INT32_MAX - 511}) {
        std::vector<int32_t> order = {0, -1, n - 1, n, INT32_MIN, INT32_MAX};
        for (int i = 0; i < 100; ++i) order.push_back(static_cast<int32_t>(rng()));
        const hwr::GroupsArg g{n, 1, nullptr, order.data()}, plain{n, 1, nullptr, nullptr};
        for (size_t p = 0; p < order.size(); ++p)
            check(hwr::row_at(g, static_cast<int>(p)) == (order[p] >= 0 && order[p] < n ? order[p] : -1), "order " + std::to_string(order[p]));
        check(hwr::row_at(plain, n - 1) == n - 1, "without an order");
    }
}

struct Scenario {
    const char *name;
    void (*run)();
};
const Scenario kScenarios[] = {{"tiles_cover_the_places", tiles_cover_the_places}, {"anything_in_offsets", anything_in_offsets},
                               {"anything_in_order", anything_in_order}};

}  // namespace

int main(int argc, char **argv) {
    if (argc != 2) return 2;
    for (const Scenario &s : kScenarios)
        if (std::strcmp(argv[1], s.name) == 0) {
            s.run();
            std::printf(g_bad ? "%d failed\n" : "ok\n", g_bad);
            return g_bad ? 1 : 0;
        }
    return 2;
}
