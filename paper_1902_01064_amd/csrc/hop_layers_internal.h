// Internal declarations shared by the host side (hop_layers.cpp) and the kernels (hop_product.hip, hop_residual.hip) of
// include/hop_layers.h.  Nothing here is part of the public ABI.
#pragma once

#include <cstdint>

#include "hop_layers.h"

// Which vector of a lattice belongs to each group, as a kernel argument (1 KB): a stand-alone call has nowhere to upload it.
struct HopIndex {
    int32_t at[HOP_MAX_INDEXED];
};
inline void hop_index_fill(HopIndex* d, const int32_t* index, int G) {
    for (int g = 0; index && g < G; ++g) d->at[g] = index[g];
}

struct HopRows {                   // the groups' rows, as a kernel's argument
    const int32_t* begin;          // null: one group of all rows
    int32_t G, rows;
};

struct HopProductTask {            // y = x w^T or x w, row by row with the group's w
    HopRows rows;
    const void *x, *w;
    void* y;
    int64_t ldx, ldw, w_stride, ldy;
    float* partial;                // [parts][rows][out] where the contraction is cut in parts
    int32_t in, out, indexed;
};

struct HopProductGradTask {        // dw = dy^T x over the group's rows
    HopRows rows;
    const void *dy, *x;
    float* dw;
    int64_t lddy, ldx, lddw, dw_stride;
    float* partial;                // [parts][G][out][in] where the rows are cut in parts
    int32_t in, out, indexed;
};

// How a product is computed: by tiles fed through registers, of any alignment; by tiles fed to LDS by the memory unit; by tiles of few
// rows whose weights go straight to registers.  Decided from sizes, types and alignment alone.
enum { HOPL_ANY = 0, HOPL_FED = 1, HOPL_FEW = 2 };
struct HopProductPlan {
    int kind, parts, tile;
};

struct HopMask {                   // of a dropout: key, first row, threshold and factor
    uint32_t k0, k1;
    int64_t first_row;
    uint32_t threshold;            // kept: the draw's 16 bits, as the upper half of a word, are at least this; 0: all
    int32_t none;                  // p = 1: nothing is kept, whatever the draw
    float factor;
};

struct HopResidualTask {
    HopRows rows;
    int32_t cols, norm, next_norm, gate_kind, indexed, dindexed;
    float scale, eps, inv_cols;
    HopMask mask;
    const void *x, *b, *z;
    int64_t ldx, ldb, ldz;
    const float *post, *pre, *gate;
    int64_t post_stride, pre_stride, gate_stride;
    void *y, *h;                   // forward
    int64_t ldy, ldh;
    const void *dy, *dh;           // gradient (y: read)
    void *dx, *db, *dz;
    int64_t lddy, lddh, lddx, lddb, lddz;
    float *dpost, *dpre, *dgate;
    int64_t dpost_stride, dpre_stride, dgate_stride;
    float* partial;                // sums of dpost, dpre, dgate over the rows of a chunk: [chunk][3][cols]
    int32_t shift;                 // rows of a chunk: 1 << shift
};

// Kernel launchers; each returns a hipError_t as int.
HopProductPlan hopl_product_plan(const HopProductTask& t, int dtype, int transposed);
HopProductPlan hopl_product_grad_plan(const HopProductGradTask& t, int dtype);
int hopl_product(const HopProductTask& t, const HopProductPlan& p, int dtype, int transposed, const HopIndex& index, void* stream);
int hopl_product_grad(const HopProductGradTask& t, const HopProductPlan& p, int dtype, const HopIndex& index, void* stream);
int hopl_dropout(int dtype, const void* x, int64_t ldx, void* y, int64_t ldy, int64_t rows, int64_t cols, const HopMask& m, void* stream);
int hopl_residual(HopResidualTask t, int dtype, const HopIndex& index, void* stream);
int hopl_residual_grad(HopResidualTask t, int dtype, const HopIndex& index, const HopIndex& dindex, void* stream);

// Rows of a chunk of the gradient (as a power of two) and how many chunks its partial sums need room for.
int hopl_grad_shift(int64_t rows, int64_t cols);
int64_t hopl_grad_chunks(int64_t rows, int G, int64_t cols);
