/*
 * hop_layers.h - layers of a model on all replicas at once, for callers that compute their own gradients (HOP_GRAD_EXTERNAL).
 *
 * A program that trains more than the linear SVM of hop.h fills N x d floats of gradients before every wave.  These calls do
 * the work of a residual block for all workers of the wave together: the rows (samples, tokens) of all workers lie stacked in
 * one matrix, and every worker - every *group* of rows - has parameters of its own, read where they are, in the ring slots of
 * its replica.  A layer of experts is the same thing with the experts' weights stacked and the rows sorted by expert.
 *
 *   hop_product       y[r, n] = sum_k x[r, k] w_g[n, k]        rows r of group g (transposed: w_g[k, n])
 *   hop_product_grad  dw_g[n, k] = sum_{r in g} dy[r, n] x[r, k]
 *   hop_residual      y = x + scale dropout(gate norm(b) post_g),  h = next_norm(y) pre_g
 *   hop_residual_grad gradients of x, b, post, pre and gate
 *   hop_dropout       y = x / (1 - p) where the counter-based generator keeps it, else 0
 *
 * Conventions beyond those of hop.h
 *  - Tensors are matrices of rows with a distance between rows (ld, in elements, at least the number of columns), fp32 or
 *    bfloat16 (`dtype`); norms' and gates' parameters and all gradients of parameters are fp32.  Pointers need the alignment of an element; the
 *    fastest forms want addresses and distances that are multiples of 16 bytes.
 *  - Sums, statistics and everything between reading and writing are held in fp32; what is written as bfloat16 is rounded once.
 *  - Outputs may not overlap inputs or each other, except that hop_dropout may work in place and that y of hop_residual may be
 *    x or b, with the same distance between rows.
 *  - Parameters of group g: element 0 at base + (index ? index[g] : g) * stride elements.  For replicas in a context's arena the
 *    base is the arena plus the layer's place in the vector, the stride that of hop_layout, and index[g] = worker * depth + slot.
 *    `index` is host memory, read during the call.
 *    Gradients of parameters go to different places for different groups: no number twice in their index, and the groups' matrices (vectors)
 *    lie behind each other or row by row side by side; a distance that has them overlap is refused.
 *  - row_begin is device memory, G + 1 ascending row numbers from 0 to `rows`; a group may have none.  Kernels hold every row
 *    number they read against `rows` and touch nothing outside the tensors; what a table that breaks the rule gives is not specified.
 *  - Calls enqueue kernels on `stream` and return (no allocation, no copy, no wait); they can be captured into a HIP graph.
 *    `scratch` is device memory, 16-byte aligned, of at least the bytes that the matching *_scratch_bytes call names (which may
 *    be 0); it is free again when the call's kernels have run.  Results are the same bits on every call with the same arguments.
 *  - Sizes: rows below 2^30 - 65536, products' columns up to 2^21 and results up to 2^40 elements, dropout's columns up to 2^29; anything
 *    else, like every null pointer, misaligned address, distance below the columns, unknown enum value and index below zero, is
 *    HOP_ERR_INVALID_ARG and nothing is launched; too little scratch is HOP_ERR_ARENA_TOO_SMALL.
 *  - No rows (rows = 0): nothing is written except the gradients of parameters, which are zero.
 */
#ifndef HOP_LAYERS_H
#define HOP_LAYERS_H

#include "hop.h"

#ifdef __cplusplus
extern "C" {
#endif

#define HOP_MAX_GROUPS 4096        /* most groups of a call */
#define HOP_MAX_INDEXED 256        /* most groups of a call with an index list */
#define HOP_MAX_NORM_COLS 32768    /* widest row of hop_residual; up to 8192 are what it is fast for */

enum { HOP_F32 = 0, HOP_BF16 = 1 };
/* none; x / sqrt(mean x^2 + eps); (x - mean x) / sqrt(var x + eps) */
enum { HOP_NORM_NONE = 0, HOP_NORM_RMS = 1, HOP_NORM_CENTRED = 2 };
/* no gate; a vector of each group, as it is; a tensor of the rows' type, through the logistic function */
enum { HOP_GATE_NONE = 0, HOP_GATE_VECTOR = 1, HOP_GATE_ELEMENT = 2 };

typedef struct {
    int64_t rows;
    const int32_t* row_begin;      /* device, G + 1; NULL with G = 1: all rows */
    int32_t G;
    int32_t dtype;                 /* HOP_F32 / HOP_BF16: of the rows (and of hop_product's weights) */
} hop_groups;

/* x: rows x in, y: rows x out.  w_g: out x in, or in x out with `transposed` (the gradient to the rows of a layer is the
 * transposed product of the gradient to its result with the same weights). */
typedef struct {
    hop_groups groups;
    const void* x;
    int64_t ldx;
    const void* w;
    int64_t ldw, w_stride;
    const int32_t* w_index;        /* host, G, or NULL */
    void* y;
    int64_t ldy;
    int64_t in, out;
    int32_t transposed;
    int32_t reserved;
} hop_product_args;

/* dy: rows x out, x: rows x in, dw_g: out x in floats, written (zeros for a group without rows). */
typedef struct {
    hop_groups groups;
    const void* dy;
    int64_t lddy;
    const void* x;
    int64_t ldx;
    float* dw;
    int64_t lddw, dw_stride;
    const int32_t* dw_index;       /* host, G, or NULL */
    int64_t in, out;
} hop_product_grad_args;

size_t hop_product_scratch_bytes(const hop_product_args* a);
int hop_product(const hop_product_args* a, void* scratch, size_t scratch_bytes, void* stream);
size_t hop_product_grad_scratch_bytes(const hop_product_grad_args* a);
int hop_product_grad(const hop_product_grad_args* a, void* scratch, size_t scratch_bytes, void* stream);

/* A dropout mask that is never stored: Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011) with the key that all draws of the
 * library have, SplitMix64 folded over (seed, stream 8, worker, iter, site), and the counter (column / 8, row low, row high, 0).
 * Column c of a row takes 16 bits, word (c mod 8) / 2, low half first, and is kept if they are at least t = p * 65536 rounded
 * (half up); what is kept is multiplied by 65536 / (65536 - t), so the expectation is exact for the p that 16 bits can hold.
 * p = 0 keeps all, p = 1 nothing; what is dropped is 0 whatever it was.  `first_row` is the row number of the first row: a batch
 * cut in pieces has the mask of the whole.  A call has one mask, whatever its groups: workers with draws of their own are calls of their own. */
typedef struct {
    uint64_t seed;
    int64_t first_row;
    int32_t worker, iter, site;
    float p;
} hop_drop;

int hop_dropout(int32_t dtype, const void* x, int64_t ldx, void* y, int64_t ldy, int64_t rows, int64_t cols, const hop_drop* drop,
                void* stream);

/* n = norm(b); t = n post; u = gate t; y = x + scale dropout(u); h = next_norm(y) pre.
 * b NULL: y is x, only h is written (a norm by itself).  next_norm NONE: no h.  post, pre NULL: 1.  drop NULL: none. */
typedef struct {
    hop_groups groups;
    int64_t cols;
    const void* b;                 /* rows x cols, or NULL */
    int64_t ldb;
    const void* z;                 /* rows x cols, HOP_GATE_ELEMENT only */
    int64_t ldz;
    const float* post;             /* cols per group, or NULL */
    int64_t post_stride;
    const float* pre;              /* cols per group, or NULL */
    int64_t pre_stride;
    const float* gate;             /* cols per group, HOP_GATE_VECTOR only */
    int64_t gate_stride;
    const int32_t* index;          /* host, G, or NULL: of post, pre and gate */
    const hop_drop* drop;          /* host, or NULL */
    int32_t norm, next_norm, gate_kind;
    float scale, eps;
    int32_t reserved;
} hop_residual_args;

/* x: rows x cols; y: rows x cols (NULL with b NULL); h: rows x cols (NULL without next_norm). */
int hop_residual(const hop_residual_args* a, const void* x, int64_t ldx, void* y, int64_t ldy, void* h, int64_t ldh, void* stream);

/* Gradients: dy (or NULL: zero) and dh (or NULL: none) of the results, y as hop_residual wrote it (the argument x with b NULL).
 *   e = dy + next_norm'(dh pre; y), dx = e; f = scale dropout(e); dgate = sum of f t over the group's rows, or dz = f t s (1 - s)
 *   with s the logistic function of z; q = f gate; dpost = sum q n; db = norm'(q post; b); dpre = sum dh next_norm(y).
 * Any output may be NULL and is then not computed.  dpost, dpre and dgate are written, zeros for a group without rows. */
typedef struct {
    const void* dy;
    int64_t lddy;
    const void* dh;
    int64_t lddh;
    const void* y;
    int64_t ldy;
    void* dx;
    int64_t lddx;
    void* db;
    int64_t lddb;
    void* dz;
    int64_t lddz;
    float* dpost;
    int64_t dpost_stride;
    float* dpre;
    int64_t dpre_stride;
    float* dgate;
    int64_t dgate_stride;
    const int32_t* index;          /* host, G, or NULL: of dpost, dpre and dgate */
} hop_residual_grads;

size_t hop_residual_grad_scratch_bytes(const hop_residual_args* a, const hop_residual_grads* g);
int hop_residual_grad(const hop_residual_args* a, const hop_residual_grads* g, void* scratch, size_t scratch_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HOP_LAYERS_H */
