// Internal declarations shared by the host side (hop_attention.cpp) and the kernels (hop_attention.hip, hop_attention_grad.hip,
// hop_rotate.hip) of include/hop_attention.h.  Nothing here is part of the public ABI.
#pragma once

#include <cstdint>

#include "hop_attention.h"
#include "hop_layers_internal.h"

// A tile's rows lie within the 31 bits of a buffer's places: the gradients' tiles are the largest, 128 rows of keys, or as many pairs, which are that many rows where a
// group has one head and 65 at most where it has more.
constexpr int64_t kHopaMostDistance = (int64_t)1 << 22;
constexpr int kHopaMostTileRows = 128;
static_assert((kHopaMostTileRows - 1) * kHopaMostDistance * 4 + HOP_MAX_HEAD_COLS * 4 < (int64_t)1 << 31, "rows of a tile");
static_assert(kHopaMostTileRows / 2 * kHopaMostDistance * 4 + (int64_t)HOP_MAX_HEADS * HOP_MAX_HEAD_COLS * 4 < (int64_t)1 << 31, "pairs of a tile");

// A head of queries and a row are a *pair*; the pairs of a key head's group are numbered row by row, head by head within a row, and the
// kernels work on runs of pairs: every key and value that is read serves all heads of the group.
struct HopAttentionTask {
    const int32_t *q_begin, *k_begin;      // null: one sequence of all rows
    int32_t S, q_rows, k_rows;
    int32_t k_heads, group, cols;          // group: query heads of a key head
    int32_t head;                          // columns from a head to the next one where q, k, v, o and grad are read
    uint32_t group_inverse;                // see hopa_divide
    int32_t group_shift;
    int32_t causal, parts;
    float scale, scale_log2;               // scale_log2 = scale log2(e)
    const void *q, *k, *v;
    int64_t ldq, ldk, ldv;
    void* o;                               // forward (gradient: read)
    int64_t ldo;
    float* lse;
    float* partial;                        // sums of parts of the contraction, see the kernels
    const void* grad;                      // gradient
    int64_t ldgrad;
    void *dq, *dk, *dv;
    int64_t lddq, lddk, lddv;
    float* terms;                          // of every pair, [2][k_heads][q_rows group]: lse log2(e) and sum do o
    void *q_plan, *k_plan;                 // how pairs and keys are shared out
};

// Pairs' rows: x / group, exact for all x below 2^31.  shift = ceil(log2 group) - 1 and inverse = ceil(2^(32 + shift) / group), below 2^32; rounding it up by e / group, e < group <=
// 2^(shift + 1), makes the quotient too large by x e / (2^(32 + shift) group) < 1 / group, which never reaches the next whole number.  A group of 1 has no inverse: 0.
constexpr int32_t hopa_group_shift(int32_t group) {
    int32_t shift = 0;
    while (2 << shift < group) ++shift;
    return shift;
}
constexpr uint32_t hopa_group_inverse(int32_t group) {
    return group == 1 ? 0 : (uint32_t)((((uint64_t)1 << (32 + hopa_group_shift(group))) + group - 1) / group);
}
constexpr int hopa_divide(int x, uint32_t inverse, int32_t shift) {
    return (int)((uint32_t)((uint64_t)(uint32_t)x * inverse >> 32) >> shift) + (int)((uint32_t)x & (inverse ? 0u : ~0u));
}

// Matrices that are copied first, each to rows of `heads` heads `head` columns apart.
struct HopAttentionCopies {
    struct {
        const void* from;
        void* to;
        int64_t ld;
        const int32_t* begin;
        int32_t rows, heads;
    } of[5];
    int32_t n, cols, head, S;
};
// What a call needs besides its task: copies to make, bytes of scratch, most tiles of the gradient's pairs and keys.
struct HopAttentionPlan {
    HopAttentionCopies copies;
    size_t bytes;
    int64_t q_tiles, k_tiles;
};

struct HopRotateTask {
    HopRows rows;
    HopRows sequences;
    const int32_t* positions;
    int32_t q_heads, heads, cols, rotary, adjacent, norm, indexed, dindexed;
    float eps, inv_cols;
    const float *q_weight, *k_weight;
    int64_t q_stride, k_stride;
    const void *x, *dy;
    void *y, *dx;
    int64_t ldx, ldy, lddy, lddx;
    float *dq_weight, *dk_weight;
    int64_t dq_stride, dk_stride;
    float* partial;                        // sums of the weights' gradients over the rows of a chunk: [chunk][2][cols]
    int32_t shift;                         // rows of a chunk: 1 << shift
    double turns[HOP_MAX_HEAD_COLS / 2];   // a pair's turns per position: base^(-2 i / rotary) / (2 pi)
};

// They set the task's parts of the scratch (null: only the bytes are asked for) and what is read instead of its matrices.
HopAttentionPlan hopa_forward_plan(HopAttentionTask* t, int dtype, char* scratch);
HopAttentionPlan hopa_grad_plan(HopAttentionTask* t, int dtype, char* scratch);
int hopa_forward(const HopAttentionTask& t, int dtype, const HopAttentionPlan& plan, void* stream);
int hopa_grad(const HopAttentionTask& t, int dtype, const HopAttentionPlan& plan, void* stream);

int hopa_rotate(const HopRotateTask& t, int dtype, const HopIndex& index, void* stream);
int hopa_rotate_grad(const HopRotateTask& t, int dtype, const HopIndex& index, const HopIndex& dindex, void* stream);
// The gradient to weights: rows of a chunk, 1 << shift, and how many chunks there are at most.
constexpr int64_t kHopaMostChunks = 1 << 20;
inline int hopa_rotate_shift(int64_t rows) {
    int shift = 0;
    while ((shift < 6 && (rows >> shift) > 1024) || (rows >> shift) > kHopaMostChunks) ++shift;
    return shift;
}
inline int64_t hopa_rotate_chunks(int64_t rows, int G) {
    const int shift = hopa_rotate_shift(rows);
    return ((rows + (1 << shift) - 1) >> shift) + G;
}
