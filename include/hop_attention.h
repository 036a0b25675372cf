/*
 * hop_attention.h - attention over the sequences of all replicas at once, and the norm and rotation of its queries and keys.
 *
 * With the products and norms of hop_layers.h these are the layers of a language model for callers that compute their own gradients
 * (HOP_GRAD_EXTERNAL): one hop_product makes queries, keys and values of all workers' tokens as columns of one matrix, hop_rotate norms and
 * turns the first two where they lie, hop_attention reads all three, another hop_product takes its result.
 *
 *   hop_rotate          y_h = R(position) (norm(x_h) w_g)         every head h of every row
 *   hop_rotate_grad     gradients of x and w
 *   hop_attention       o_i = sum_j p_ij v_j,  p_i = softmax_j(scale q_i k_j),  lse_i = log sum_j exp(scale q_i k_j)
 *   hop_attention_grad  gradients of q, k and v
 *
 * The conventions are those of hop_layers.h (types, distances between rows, indexes of parameters, scratch, streams, errors).  Beyond them
 *  - A head is `cols` consecutive columns of a row.  Query head h belongs to key head h / (q_heads / k_heads); q_heads is a multiple of k_heads.
 *  - Sequences lie packed in the rows: sequence s has the query rows q_begin[s] to q_begin[s + 1] and the key rows k_begin[s] to k_begin[s + 1],
 *    two tables of S + 1 ascending row numbers on the device (the same one where queries and keys are the same rows).  A sequence may have none of
 *    either; so room behind a sequence's keys, where a cache grows, is a sequence without queries.  Rows in front of the first and behind the last sequence are neither read nor written.
 *  - `causal`: the queries are the last rows of their sequence, query i of nq sees the keys up to i + nk - nq of nk.  So one query sees all keys of
 *    its sequence, and with more queries than keys the first ones see none: their o is 0, their lse -infinity, they have no gradient.
 *  - What a query does not see has no influence, whatever it holds: infinities and NaN in keys and values behind a query, or in queries (and
 *    their gradients) in front of a key, or in rows of other sequences, change nothing.
 *  - Sums, statistics and scores are held in fp32.  With bfloat16 rows the softmax's terms and the gradients of the scores are rounded to
 *    bfloat16 as operands of the products that follow.  A row's results depend on its sequence and on how many rows all of them have, not on other
 *    rows' values, and are the same bits every time.
 *  - Results may not overlap what a call reads, except where it is said.
 *  - Sizes: heads of up to HOP_MAX_HEAD_COLS columns, rows times query heads below 2^30, distances between rows up to 2^22 elements, up to
 *    HOP_MAX_GROUPS sequences.  Fastest are heads of 64 and 128 columns in rows whose addresses and distances are multiples of 16 bytes; others
 *    are copied into the scratch first, except where a few queries read the keys of bfloat16 rows, or of fp32 heads of up to 64 columns.
 */
#ifndef HOP_ATTENTION_H
#define HOP_ATTENTION_H

#include "hop_layers.h"

#ifdef __cplusplus
extern "C" {
#endif

#define HOP_MAX_HEAD_COLS 128
#define HOP_MAX_HEADS 1024

/* x: rows x (q_heads + k_heads) cols, the queries' heads first; either number may be 0.  For a head x_h:
 *   n = norm(x_h) over its columns,  t = n w,  w of the row's group: q_weight for the queries' heads, k_weight for the keys' (NULL: 1)
 *   the first `rotary` columns (even; 0: none) are turned in pairs (c, c'), c' = c + rotary / 2 or with `adjacent` c = 2 i, c' = 2 i + 1:
 *   y_c = t_c cos a - t_c' sin a,  y_c' = t_c' cos a + t_c sin a,  a = position base^(-2 i / rotary) for pair i
 * The angle is held in 64 bits up to its sine and cosine, so far positions lose nothing.
 * positions: device, a number of each row; NULL: the row's number in its sequence of seq_begin (device, S + 1, NULL with S = 1). */
typedef struct {
    hop_groups groups;             /* whose weights: workers */
    const int32_t* positions;
    const int32_t* seq_begin;
    int32_t S;
    int32_t q_heads, k_heads, cols, rotary, adjacent;
    const float* q_weight;         /* cols per group, or NULL */
    int64_t q_weight_stride;
    const float* k_weight;
    int64_t k_weight_stride;
    const int32_t* index;          /* host, G, or NULL: of q_weight and k_weight */
    double base;
    float eps;
    int32_t norm;                  /* HOP_NORM_* */
} hop_rotate_args;

/* y may be x, with the same distance between rows (its gradient needs x, then). */
int hop_rotate(const hop_rotate_args* a, const void* x, int64_t ldx, void* y, int64_t ldy, void* stream);

/* dy: gradient of y, x as hop_rotate got it.  dx may be dy, with the same distance; any output may be NULL.  dq_weight and dk_weight are written,
 * zeros for a group without rows. */
typedef struct {
    const void* dy;
    int64_t lddy;
    const void* x;
    int64_t ldx;
    void* dx;
    int64_t lddx;
    float* dq_weight;
    int64_t dq_weight_stride;
    float* dk_weight;
    int64_t dk_weight_stride;
    const int32_t* index;          /* host, G, or NULL: of dq_weight and dk_weight */
} hop_rotate_grads;

size_t hop_rotate_grad_scratch_bytes(const hop_rotate_args* a, const hop_rotate_grads* g);
int hop_rotate_grad(const hop_rotate_args* a, const hop_rotate_grads* g, void* scratch, size_t scratch_bytes, void* stream);

/* q: q_rows x q_heads cols, k and v: k_rows x k_heads cols. */
typedef struct {
    int64_t q_rows, k_rows;
    const int32_t* q_begin;        /* device, S + 1; NULL with S = 1: all rows */
    const int32_t* k_begin;
    int32_t S, dtype;
    const void* q;
    int64_t ldq;
    const void* k;
    int64_t ldk;
    const void* v;
    int64_t ldv;
    int32_t q_heads, k_heads, cols, causal;
    float scale;                   /* above zero */
    int32_t reserved;
} hop_attention_args;

/* o: q_rows x q_heads cols; lse: q_heads x q_rows floats, or NULL. */
size_t hop_attention_scratch_bytes(const hop_attention_args* a);
int hop_attention(const hop_attention_args* a, void* o, int64_t ldo, float* lse, void* scratch, size_t scratch_bytes, void* stream);

/* o and lse as hop_attention wrote them, grad: the gradient of o.  dq, dk, dv as q, k, v; all are written (zeros for rows that nothing sees or that see nothing). */
typedef struct {
    const void* grad;
    int64_t ldgrad;
    const void* o;
    int64_t ldo;
    const float* lse;
    void* dq;
    int64_t lddq;
    void* dk;
    int64_t lddk;
    void* dv;
    int64_t lddv;
} hop_attention_grads;

size_t hop_attention_grad_scratch_bytes(const hop_attention_args* a, const hop_attention_grads* g);
int hop_attention_grad(const hop_attention_args* a, const hop_attention_grads* g, void* scratch, size_t scratch_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HOP_ATTENTION_H */
