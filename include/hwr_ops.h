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
 *   hwr_grouped_linear       y[r] = act(x[r] W[g(r)] + bias[g(r)]) + residual[r]
 *   hwr_grouped_linear_grad  with dz[r] = dy[r] act'(z[r]): dx and dW as above from dz,
 *                            dbias[g] = sum over rows r of g of dz[r]
 *   hwr_adapter_matmul       y[r] = x[r] W + s[g(r)] (x[r] A[g(r)]) B[g(r)],
 *                            one projection shared by all rows and the
 *                            low-rank adapter of the row's group
 *   hwr_adapter_matmul_grad  with u[r] = s[g] dy[r] B[g]^T:
 *                            dx[r] = dy[r] W^T + u[r] A[g]^T,
 *                            dA[g] = sum over rows r of g of x[r]^T u[r],
 *                            dB[g] = sum of s[g] (x[r] A[g])^T dy[r]
 *                            (the shared W is frozen)
 *   hwr_log_probs            of rows of logits: the log probability of a given token,
 *                            the entropy, the most likely tokens
 *   hwr_log_probs_grad       the gradient of the logits
 *   hwr_adamw_step           one step of AdamW over many tensors
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
 * and no output overlaps an input (but dx of hwr_log_probs_grad).  Any number of rows up to 2^31 - 512 (hwr_group_rows:
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
 * (hwr_ops_reserve), before capturing.  (Both gradients of a grouped product or layer run in one launch, or, in
 * less space and more time, where there is not enough for that, in two, with the same bits.)  All calls of a context, and all replays of graphs
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

/* A layer: z[r] = x[r] W[g] + bias[g], y[r] = act(z[r]) + residual[r].  A row in no group has
 * y the residual (zeros without one) and z zeros.  z, which the gradient reads, is written where
 * it is not NULL; y is made of the sums before z is rounded.  y and z may not be x, the residual or each other. */
typedef struct {
    int32_t dtype;
    int32_t k, m;
    int32_t act;                  /* hwr_act (hwr.h)                            */
    const void *x; int64_t ldx;   /* [n][k]                                     */
    const void *w;                /* [G][k][m]                                  */
    const void *bias;             /* [G][m] or NULL                             */
    const void *residual; int64_t ldr;   /* [n][m] or NULL                      */
    void *y; int64_t ldy;         /* [n][m]                                     */
    void *z; int64_t ldz;         /* [n][m] or NULL                             */
} hwr_linear_args;
hwr_status hwr_grouped_linear(hwr_ops *ops, const hwr_groups *g, const hwr_linear_args *a);

/* With dz[r] = dy[r] act'(z[r]) (rounded once to the type of the matrices for dx and dw, not for
 * dbias).  The gradient of the residual is dy itself.  dx may not be dy, z or x. */
typedef struct {
    int32_t dtype;
    int32_t k, m;
    int32_t act;
    const void *dy; int64_t lddy; /* [n][m]                                     */
    const void *z; int64_t ldz;   /* [n][m]; needed but for HWR_ACT_NONE        */
    const void *x; int64_t ldx;   /* [n][k]; needed for dw                      */
    const void *w;                /* [G][k][m]; needed for dx                   */
    void *dx; int64_t lddx;       /* [n][k] or NULL                             */
    void *dw;                     /* [G][k][m] or NULL                          */
    void *dbias;                  /* [G][m] or NULL                             */
} hwr_linear_grad_args;
hwr_status hwr_grouped_linear_grad(hwr_ops *ops, const hwr_groups *g, const hwr_linear_grad_args *a);

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

/* Of every row r of logits x, with z = scale x:
 *   lse[r]     = ln sum over tokens c of exp(z[c])
 *   logp[r]    = z[token[r]] - lse[r]; 0 where token[r] is outside [0, m): no token
 *   entropy[r] = - sum over c of p[c] ln p[c], p[c] = exp(z[c] - lse[r])
 *   top_token[r], top_logp[r]: the `top` most likely tokens, the most likely first, of
 *                equal logits the lower token, and their log probabilities.
 * Outputs may be NULL.  A token at -inf is not allowed: p is 0, and it comes last among the most
 * likely.  Logits below -3.3e38 (the lowest finite values of either type) count as -inf;
 * a row of nothing else has lse -inf, logp -inf (0 without a token), entropy 0 and top_logp -inf.  A NaN or +inf in a
 * row makes its lse, logp, entropy and top_logp NaN (which tokens are listed is then unspecified).
 * Sums are fp32; how many rows a call has, and whether it asks for the most likely tokens, can change a
 * row's last bits. */
typedef struct {
    int32_t dtype;                /* hwr_dtype of x                             */
    int32_t n, m;                 /* rows, 0 or more; tokens, 1..16777216       */
    int32_t top;                  /* 0..32, at most m                           */
    float scale;                  /* 2^-64..2^64 (1 / temperature)              */
    const void *x; int64_t ldx;   /* [n][m]                                     */
    const int32_t *token;         /* [n]; needed for logp                       */
    float *logp, *lse, *entropy;  /* [n]                                        */
    float *top_logp;              /* [n][top]                                   */
    int32_t *top_token;           /* [n][top]                                   */
} hwr_log_probs_args;
hwr_status hwr_log_probs(hwr_ops *ops, const hwr_log_probs_args *a);

/* The gradient of the logits from those of logp and entropy, with ln p[c] = scale x[c] - lse[r]:
 *   dx[r][c] = scale (dlogp[r] (1[c = token[r]] - p[c]) - dentropy[r] p[c] (ln p[c] + entropy[r]))
 * A row without a token has no first term; without both terms, or with lse -inf, it gets zeros.
 * dx may be x itself, with the same row stride.  lse holds ln p to 2^-24 of its magnitude. */
typedef struct {
    int32_t dtype;
    int32_t n, m;
    float scale;
    const void *x; int64_t ldx;   /* [n][m]                                     */
    const int32_t *token;         /* [n]; needed with dlogp                     */
    const float *lse;             /* [n]                                        */
    const float *dlogp;           /* [n] or NULL: zeros                         */
    const float *entropy;         /* [n]; with dentropy, and only then          */
    const float *dentropy;        /* [n] or NULL: zeros                         */
    void *dx; int64_t lddx;       /* [n][m]                                     */
} hwr_log_probs_grad_args;
hwr_status hwr_log_probs_grad(hwr_ops *ops, const hwr_log_probs_grad_args *a);

/* AdamW.  A step number t over all values of some tensors at once, in fp32:
 *   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
 *   p = p (1 - lr weight_decay) - lr / (1 - beta1^t) m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
 * Weights p and gradients g are of one type.  Weights in HWR_BF16 have an fp32 master, which
 * is what is stepped (p is its rounding), or none: p is then rounded up or down at random.
 * States have 32 bits, m and v in fp32; or 8: e4m3 (1 sign, 4 exponent, 3 mantissa bits, no
 * infinities) with an fp32 scale for every 256 values of a tensor from its first on, rounded up or
 * down at random, and sqrt(v) in place of v (one below 2^-9 scales is rounded up to that, never down to
 * 0).  Each is the stored value times its scale.  Zeros (with any finite scales) are a beginning for all.
 * A block of which every value is below 2^-100 becomes zeros.  The roots are rounded without a bias, so
 * their squares have one, and noise: with normal gradients and beta2 0.999 (0.98) v settles 5% (4%) too
 * large on the mean, with a standard deviation of 0.35 (0.30) of itself; 98% of the values' updates are
 * within 0.70 to 1.42 (0.73 to 1.36) of what they should be, their mean 1.4% (1.2%) above.
 * The random numbers are a function of seed, t and the value's number (tensors are numbered
 * one after the other, each from a multiple of 256 on): the same call gives the same bits.
 * A NaN or infinity in g (with 8 bits, in its square) stays in its value, with states of 8 bits in its block of 256.  (With eps 0 a value whose
 * moments are 0 becomes NaN: 0 / 0.)
 *
 * hwr_adamw_init keeps what it needs of the tensors' addresses and sizes (not their contents) in
 * device memory; their memory has to stay until hwr_adamw_free.  Nothing that is written may overlap
 * anything else.  Steps of one hwr_adamw have to be ordered among each other.  Init copies from the host and waits: HWR_ERR_STATE
 * while the stream of ops is captured, with nothing recorded (while another of the thread's is, it is not to be called).  hwr_adamw_free
 * waits for the device, and is not to be called while a stream is captured; the context may be freed before. */
typedef struct hwr_adamw hwr_adamw;   /* opaque, owned by the library */

typedef struct {
    int64_t count;                /* values, 0..2^40                            */
    void *p;                      /* [count]                                    */
    const void *g;                /* [count]                                    */
    float *master;                /* [count]; all tensors of a step or none     */
    void *m, *v;                  /* [count]                                    */
    float *m_scale, *v_scale;     /* [(count + 255) / 256]; 8 bits              */
} hwr_adamw_tensor;

typedef struct {
    int32_t dtype;                /* hwr_dtype of p and g                       */
    int32_t bits;                 /* of m and v: 8 or 32                        */
    int32_t n_tensors;            /* 0..1048576                                 */
    const hwr_adamw_tensor *tensors;   /* host memory, not kept                 */
} hwr_adamw_config;
hwr_status hwr_adamw_init(hwr_ops *ops, const hwr_adamw_config *config, hwr_adamw **out);
void hwr_adamw_free(hwr_adamw *adamw);

typedef struct {
    double lr, beta1, beta2;      /* lr 0 or more; betas in [0, 1)              */
    double eps, weight_decay;     /* eps in [0, 1) (2^-126 for less, but for 0); weight_decay 0 or more */
    uint64_t seed;
    int64_t step;                 /* t, 1 or more                               */
    int64_t *steps;               /* or, in device memory, the steps before this one: counted up
                                     by the call, which may then be captured (without, a captured
                                     call is HWR_ERR_STATE); step is not read   */
    const float *lr_device;       /* with steps: in place of lr, or NULL        */
} hwr_adamw_args;
/* On the stream of ops, a context of the device that the adamw was made on. */
hwr_status hwr_adamw_step(hwr_ops *ops, hwr_adamw *adamw, const hwr_adamw_args *a);

#ifdef __cplusplus
}
#endif
#endif /* HWR_OPS_H */
