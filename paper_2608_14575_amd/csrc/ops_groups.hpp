// The walk over the ragged groups of a routed batch: tiles of places, and the
// work items of a product by row.  Integer arithmetic and lane exchanges alone, so
// that it also compiles for the host, where a test runs it lane by lane.
//
// The contents of offsets and order are not checked, so they may hold anything:
// whatever they do, places lie in [0, n), rows are checked before they are used, and
// nothing here passes 32 bits (n <= 2^31 - 512).
#pragma once

#include <cstdint>

namespace hwr {

struct GroupsArg {
    int n, G;
    const int32_t *offsets, *order;   // order may be null
};

// offsets as places: clamped to [0, n], so that whatever the array holds stays in bounds
__device__ inline int place_of(const GroupsArg &g, int i) {
    const int v = g.offsets[i];
    return v < 0 ? 0 : v > g.n ? g.n : v;
}

// Row at place p, or -1.
__device__ inline int row_at(const GroupsArg &g, int p) {
    const int r = g.order ? g.order[p] : p;
    return static_cast<unsigned>(r) < static_cast<unsigned>(g.n) ? r : -1;
}

// Rows of a tile: places [p0, p1) of group g (g == G: the rows in no group).
struct RowTile {
    int g, p0, p1;
};

// Every group is cut into tiles of bm places.  The tiles of lane i's groups in
// a block of 64 groups; group G are the rows in no group.
__device__ inline int lane_tiles(const GroupsArg &g, int i, int bm, bool tail, int &p0, int &p1) {
    p0 = p1 = 0;
    if (i < g.G) {
        p0 = place_of(g, i);
        p1 = place_of(g, i + 1);
    } else if (i == g.G && tail) {
        p0 = place_of(g, i);
        p1 = g.n;
    }
    return p1 > p0 ? (p1 - p0 + bm - 1) / bm : 0;
}

__device__ inline int wave_scan(int v, int lane) {   // inclusive
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// Tiles of all groups; one wave.  At most as many as n rows can make, which is what the
// grid has: offsets that do not ascend can list rows many times over.
__device__ inline int count_tiles(const GroupsArg &g, int bm, bool tail, int lane) {
    const int most = g.n / bm + min(g.n, g.G + 1);
    int sum = 0, p0, p1;
    for (int b = 0; b <= g.G; b += 64) sum = min(sum + lane_tiles(g, b + lane, bm, tail, p0, p1), most);
#pragma unroll
    for (int d = 32; d; d >>= 1) sum = min(sum + __shfl_xor(sum, d), most);
    return __builtin_amdgcn_readfirstlane(sum);
}

// Tile t of all groups (t < count_tiles); one wave.
__device__ inline RowTile find_tile(const GroupsArg &g, int t, int bm, bool tail, int lane) {
    for (int b = 0; b <= g.G; b += 64) {
        int p0, p1;
        const int mine = lane_tiles(g, b + lane, bm, tail, p0, p1);
        const int upto = wave_scan(mine, lane);
        const uint64_t hit = __ballot(upto > t);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            const int first = __builtin_amdgcn_readlane(upto - mine, l);
            const int a = __builtin_amdgcn_readlane(p0, l) + (t - first) * bm, e = __builtin_amdgcn_readlane(p1, l);
            return {b + l, a, a + bm < e ? a + bm : e};
        }
        t -= __builtin_amdgcn_readlane(upto, 63);
    }
    return {g.G, 0, 0};
}

// First group that ends past place p (G if none); one wave.
__device__ inline int group_of(const GroupsArg &g, int p, int lane) {
    for (int b = 0; b < g.G; b += 64) {
        const uint64_t hit = __ballot(b + lane < g.G && place_of(g, b + lane + 1) > p);
        if (hit) return b + __builtin_ctzll(hit);
    }
    return g.G;
}

// Workgroup id -> work item, so that the items of one of the 8 L2s (ids are
// dealt out in turn) are neighbours.  Returns -1 past the last item.
__device__ inline int xcd_item(int id, int items) {
    const int share = (items + 7) >> 3;
    const int at = id >> 3, i = (id & 7) * share + at;
    return at < share && i < items ? i : -1;
}

// Work item of a product by row: tile t of places, first column c0, part.  Tiles go in
// panels of 8 row tiles, column by column, so that the workgroups that run together on
// one L2 share rows and weights.  False past the last.
__device__ inline bool row_item(int id, int tiles, int m, int mw, int bn, int parts, int &t, int &c0, int &part) {
    const int ct = (m + bn - 1) / bn;
    int item = xcd_item(id, tiles * ct * parts);
    if (item < 0) return false;
    part = item / (tiles * ct);
    item -= part * (tiles * ct);
    const int panel = item / (8 * ct) * 8, in = item - panel * ct, rp = min(8, tiles - panel);
    t = panel + in % rp;
    // the last tile of columns ends with the row: it shares columns with the one before
    // (both give them the same bits), and no chunk is cut
    c0 = mw < bn ? 0 : min(in / rp * bn, mw - bn);
    return true;
}

}  // namespace hwr
