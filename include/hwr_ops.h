/*
 * hwr_ops.h -- operators on a routed batch.
 *
 * hwr_route_batch answers a batch with one pair per query.  What a program
 * that serves or trains the pool's models on this card does next is to run
 * every row of the batch with the weights of the model it went to:
 *
 *   hwr_group_rows           the rows of every group (model), in row order,
 *                            from the choices and a pair -> group table;
 *   hwr_grouped_matmul       y[r] = x[r] W[g(r)]
 *   hwr_grouped_matmul_grad  dx[r] = dy[r] W[g(r)]^T,
 *                            dW[g] = sum over rows r of g of x[r]^T dy[r]
 *   hwr_adapter_matmul       y[r] = x[r] W + s[g(r)] (x[r] A[g(r)]) B[g(r)],
 *                            one projection shared by all rows and the
 *                            low-rank adapter of the row's group
 *   hwr_adapter_matmul_grad  with u[r] = s[g] dy[r] B[g]^T:
 *                            dx[r] = dy[r] W^T + u[r] A[g]^T,
 *                            dA[g] = sum over rows r of g of x[r]^T u[r],
 *                            dB[g] = sum of s[g] (x[r] A[g])^T dy[r]
 *                            (the shared W is frozen)
 *
 * Groups.  `order` lists the rows of group 0, then of group 1, ..., and last
 * the rows in no group; group g has the places offsets[g] .. offsets[g+1]-1,
 * and the places from offsets[n_groups] on hold the rows in no group.  Groups
 * may be empty.  A row in no group gets zeros from the grouped products and the
 * shared projection alone from the adapter's.  The gradients of an empty
 * group's weights are zeros.  order may be NULL: place i is row i.
 *
 * Layouts.  Weights are dense and row-major, [in][out]: W [G][k][m] (grouped) or
 * [k][m] (adapter), A [G][k][rank], B [G][rank][m]; gradients have the layout of
 * what they belong to.  Rows of x, y, dy and dx may be strided: ldx etc. are the
 * distances of rows in elements, 0 for dense.  Every pointer is device memory
 * and no output overlaps an input.  Any number of rows up to 2^31 - 512 (hwr_group_rows:
 * 2^31 - 1), any width up to 65536 and any element alignment is accepted; products run
 * fastest where widths, row strides and pointers are multiples of 16 bytes.
 *
 * Precision.  HWR_BF16 (raw bit patterns) or HWR_F32, one type for every matrix
 * of a call; scale is fp32.  Products accumulate in fp32 and each output is
 * rounded once (nearest, ties to even).  The low-rank intermediates s (x A) and u are not
 * rounded to bf16: HWR_F32 calls hold them in fp32; HWR_BF16 calls as the sum of two bf16
 * values (16 significant bits, so that the second product runs on bf16 operands),
 * except hwr_adapter_matmul of few rows (at most 192, fewer with large weights), which
 * holds them in fp32.  So the number of rows in a batch can change a row's last bits.
 * Sums have a fixed order: the same call on the same device gives the same bits.  An
 * infinity or a NaN stays in the rows (and groups) that it belongs to.
 *
 * Gradients are calls of their own; nothing is recorded for automatic differentiation.
 *
 * Every call is queued on the context's stream and returns without waiting; the
 * calling thread's current device is left as it was.  Inputs written and outputs read
 * on another stream have to be ordered against it by the caller.
 *
 * Work space belongs to the context: a call that needs more than it has allocates,
 * before it queues anything (and keeps what it had until hwr_ops_free, so that captured
 * graphs stay valid); under stream capture it is HWR_ERR_STATE instead, with nothing
 * recorded: make the call once outside, or reserve what the message names
 * (hwr_ops_reserve), before capturing.  All calls of a context, and all replays of graphs
 * captured from it, use the same work space: a replay has to be ordered against the
 * context's other calls and against its other graphs' replays (an event does), or each
 * graph captured from a context of its own.
 *
 * A context is not thread-safe.  Sizes and pointers are checked; the contents of offsets,
 * order, choice and table are not: values out of range give unspecified results, and all
 * memory accesses stay in bounds.
 */
#ifndef HWR_OPS_H
#define HWR_OPS_H

#include <stdint.h>

#include "hwr.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct hwr_ops hwr_ops;   /* opaque, owned by the library */

/* A context on one device and stream (hipStream_t or NULL). */
hwr_status hwr_ops_init(int32_t device, void *stream, hwr_ops **out);
/* Destroy it (NULL is allowed); waits for its stream first. */
void hwr_ops_free(hwr_ops *ops);
/* Message of the last error on ops, or of the last failed hwr_ops_init on this
 * thread when ops is NULL.  Never NULL; owned by the library. */
const char *hwr_ops_last_error(const hwr_ops *ops);
/* Work space for later calls: at least `bytes`. */
hwr_status hwr_ops_reserve(hwr_ops *ops, uint64_t bytes);

typedef struct {
    int32_t n;                    /* rows, 0..2147483136 (2^31 - 512)            */
    int32_t n_groups;             /* G, 1..1024 (as many as pairs)              */
    const int32_t *offsets;       /* [G + 1]                                    */
    const int32_t *order;         /* [n] row at each place, or NULL             */
} hwr_groups;

/* Rows by group, stable.  The group of row r is table[choice[r]], or choice[r]
 * where table is NULL; a choice outside [0, n_table) (outside [0, n_groups)
 * without a table) or a table entry outside [0, n_groups) leaves the row in no
 * group.  n == 0 writes offsets of zeros. */
hwr_status hwr_group_rows(hwr_ops *ops, int32_t n, const int32_t *choice, const int32_t *table, int32_t n_table,
                          int32_t n_groups, int32_t *offsets, int32_t *order);

typedef struct {
    int32_t dtype;                /* hwr_dtype of every matrix                  */
    int32_t k, m;                 /* widths of x and of y, 1..65536             */
    const void *x; int64_t ldx;   /* [n][k]                                     */
    const void *w;                /* [G][k][m]                                  */
    void *y; int64_t ldy;         /* [n][m]                                     */
} hwr_matmul_args;
hwr_status hwr_grouped_matmul(hwr_ops *ops, const hwr_groups *g, const hwr_matmul_args *a);

typedef struct {
    int32_t dtype;
    int32_t k, m;
    const void *dy; int64_t lddy; /* [n][m]                                     */
    const void *x; int64_t ldx;   /* [n][k]; needed for dw                      */
    const void *w;                /* [G][k][m]; needed for dx                   */
    void *dx; int64_t lddx;       /* [n][k] or NULL                             */
    void *dw;                     /* [G][k][m] or NULL                          */
} hwr_matmul_grad_args;
hwr_status hwr_grouped_matmul_grad(hwr_ops *ops, const hwr_groups *g, const hwr_matmul_grad_args *a);

typedef struct {
    int32_t dtype;
    int32_t k, m;
    int32_t rank;                 /* 1..128                                     */
    const void *x; int64_t ldx;   /* [n][k]                                     */
    const void *w;                /* [k][m]                                     */
    const void *a;                /* [G][k][rank]                               */
    const void *b;                /* [G][rank][m]                               */
    const float *scale;           /* [G], or NULL: 1                            */
    void *y; int64_t ldy;         /* [n][m]                                     */
} hwr_adapter_args;
hwr_status hwr_adapter_matmul(hwr_ops *ops, const hwr_groups *g, const hwr_adapter_args *a);

typedef struct {
    int32_t dtype;
    int32_t k, m;
    int32_t rank;
    const void *dy; int64_t lddy; /* [n][m]                                     */
    const void *x; int64_t ldx;   /* [n][k]; needed for da and db               */
    const void *w;                /* [k][m]; needed for dx                      */
    const void *a;                /* [G][k][rank]; needed for dx and db         */
    const void *b;                /* [G][rank][m]; needed for dx and da         */
    const float *scale;           /* [G], or NULL: 1                            */
    void *dx; int64_t lddx;       /* [n][k] or NULL                             */
    void *da;                     /* [G][k][rank] or NULL                       */
    void *db;                     /* [G][rank][m] or NULL                       */
} hwr_adapter_grad_args;
hwr_status hwr_adapter_matmul_grad(hwr_ops *ops, const hwr_groups *g, const hwr_adapter_grad_args *a);

#ifdef __cplusplus
}
#endif
#endif /* HWR_OPS_H */
