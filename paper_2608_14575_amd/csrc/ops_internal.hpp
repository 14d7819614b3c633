// Arguments and launchers of the operators on a routed batch (hwr_ops.h).
#pragma once

#include "hwr_internal.hpp"
#include "ops_groups.hpp"

namespace hwr {

// A grid of many workgroups: the runtime takes fewer than 2^32 threads in a dimension, so
// past this many they go in several rows (block_id numbers them; up to a row too many).
constexpr int64_t grid_row(int threads) { return ((int64_t{1} << 32) - 1) / threads / 16 * 16; }
inline dim3 wide_grid(int64_t blocks, int threads) {
    const int64_t most = grid_row(threads);
    if (blocks <= most) return dim3(static_cast<uint32_t>(blocks));
    return dim3(static_cast<uint32_t>(most), static_cast<uint32_t>((blocks + most - 1) / most));
}

// Copies of matrices with rows padded by zeros to whole, aligned chunks of 16 bytes.
constexpr int kMaxPads = 3;
struct PadArgs {
    struct Matrix {
        const void *src;
        void *dst;
        int64_t rows, ld;         // elements
        int width;
    } m[kMaxPads];
    int count;
};
int64_t padded_width(bool bf16, int width);   // elements
hipError_t launch_pad(bool bf16, const PadArgs &a, hipStream_t s);

// Low-rank intermediates (s x A, u) are kept by place, in blocks of kRankBlock
// columns of 128 bytes: fp32 values, or bf16 pairs hi[kRankBlock], lo[kRankBlock]
// with hi + lo the value to 16 significant bits.
constexpr int kRankBlock = 32;
constexpr int kLowBytes = 128;

// Products by row: out[r][c] = sum_e x[r][e] w_g(e, c), and for the adapter
// plus sum_e low[place][e] lw_g(e, c).
struct RowsArgs {
    GroupsArg g;
    int k, m;                     // contraction width (e), output width (c)
    const void *x;
    int64_t ldx;                  // elements
    const void *w;                // KS: [k][m], else [m][k] (transposed use)
    int64_t w_stride;             // elements between groups
    int ldw, mw;                  // elements between rows of w; columns there are (KS: m, or more that are not used)
    bool padded;                  // rows of x (and of w, not KS) go on with zeros up to a whole chunk
    void *y;
    int64_t ldy;
    const void *zeros;            // 256 zero bytes
    int parts;                    // workgroups that share a tile's contraction (rows_plan)
    int m_pad;                    // m up to a multiple of 4
    float *partial;               // [parts][n][m_pad], with parts > 1
    // adapter
    const void *low;              // [n][blocks] low-rank intermediates
    const void *lw;               // [G][rank][m] (KS) or [G][m][rank]
    int rank;
};

// low[place] = scale[g] x[row] w_g
struct ShrinkArgs {
    GroupsArg g;
    int k, rank;
    const void *x;
    int64_t ldx;                  // elements
    const void *w;                // [G][k][rank] (KS) or [G][rank][k]
    const float *scale;           // [G] or null
    void *low;
};

// Weight gradients: out[g][p][q] = sum over places of g of P[place][p] Q[place][q].
struct ColsArgs {
    GroupsArg g;
    int np, nq;                   // widths of P and Q as they stand in out (rows may go on to a whole chunk)
    bool padded;                  // they do
    const void *p, *q;            // rows through order, or low-rank intermediates by place
    int64_t ldp, ldq;             // elements
    void *out;                    // [G][np][nq]
    int blocks;                   // rank blocks (low-rank side)
    int parts;                    // workgroups that share a tile's places
    float *partial;               // [parts][G][np][nq], with parts > 1
    const void *zeros;
};

// Few rows: y = x w_g, or with an adapter x w + scale[g] (x a_g) b_g, by streaming the weights.
constexpr int kFewTile = 16;
struct FewArgs {
    GroupsArg g;
    int k, m, m_pad, rank;        // m_pad: m up to a multiple of 4
    const void *x;
    int64_t ldx;                  // elements
    const void *w;                // [k][m], groups w_stride elements apart
    int64_t w_stride;
    void *y;
    int64_t ldy;
    const void *a, *b;            // adapters
    const float *scale;
    int parts, low_parts;         // parts of the contraction
    float *partial;               // [parts][n][m_pad], with parts > 1 or an adapter
    float *low;                   // [low_parts][n][rank]
};

struct GroupRowsArgs {
    int n, n_table, G;
    const int32_t *choice, *table;
    int32_t *offsets, *order;
    int blocks;                   // 1: one launch, without work space
    int32_t *hist, *totals;       // [G + 1][blocks], [G + 1] work space
};

enum class RowsKind { kGrouped, kAdapter };

hipError_t launch_group_rows(const GroupRowsArgs &a, hipStream_t s);
int group_rows_blocks(int n);
// Tile of places and columns, and parts, for a product by row.
struct RowsPlan {
    bool direct;                  // whole chunks: straight into LDS
    int bm, bn, parts;
};
// ks: weights [k][m]; else [m][k]
RowsPlan rows_plan(bool bf16, RowsKind kind, bool ks, const RowsArgs &a, int cus);
hipError_t launch_rows(bool bf16, RowsKind kind, bool ks, const RowsArgs &a, int cus, hipStream_t s);
hipError_t launch_shrink(bool bf16, bool ks, const ShrinkArgs &a, int cus, hipStream_t s);
// Two of the same rows and rank in one launch: with [rank][k] and with [k][rank] weights.
hipError_t launch_shrink_pair(bool bf16, const ShrinkArgs &direct, const ShrinkArgs &ks, int cus, hipStream_t s);
bool few_rows(int n, int G, int k, int m, bool adapter, bool bf16);  // whether launch_few is meant for the batch
int few_tiles(int n, int G, bool adapter);
int few_parts(int n, int G, int k, int m, bool bf16, bool adapter, int cus);
hipError_t launch_few(bool bf16, bool adapter, const FewArgs &a, hipStream_t s);
// y[row] = sum of the partial sums of its place
hipError_t launch_join(bool bf16, const FewArgs &a, hipStream_t s);
enum class ColsKind { kDense, kLowP, kLowQ };
// Tile, and parts of the places, for a weight gradient.
struct ColsPlan {
    bool direct;                  // whole chunks: straight into LDS
    int tile, parts;
};
ColsPlan cols_plan(bool bf16, ColsKind kind, const ColsArgs &a, int cus);
hipError_t launch_cols(bool bf16, ColsKind kind, const ColsArgs &a, int cus, hipStream_t s);
// kLowQ and kLowP of the same groups and rank in one launch; both plans direct
hipError_t launch_cols_low_pair(bool bf16, const ColsArgs &q, const ColsArgs &p, hipStream_t s);

}  // namespace hwr
