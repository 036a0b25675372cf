// C ABI of include/hop_layers.h: checks of arguments and their translation into what the kernels take.
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstring>

#include "hop_internal.h"
#include "hop_layers_checks.h"

using namespace hopl;

namespace {

constexpr uint64_t STREAM_DROPOUT = 8;         // beside hoprng's streams
constexpr int64_t kMostDropCols = 1 << 29;     // a place in a row is a 32-bit number of bytes
constexpr int64_t kMostCols = 1 << 21;         // a tile's lines, up to 2^20 elements apart, end within the 31 bits of a buffer's places
constexpr int64_t kMostResults = (int64_t)1 << 40;             // elements of a product's result: tiles are counted in 31 bits

bool drop_ok(const hop_drop* d) {
    return !d || (d->p >= 0.f && d->p <= 1.f && d->first_row >= 0 && d->first_row <= INT64_MAX - kMostRows);
}
HopMask mask_of(const hop_drop* d) {
    HopMask m = {0, 0, 0, 0, 0, 1.f};
    if (!d) return m;
    const uint64_t key = hoprng::mix(d->seed, STREAM_DROPOUT, (uint64_t)(int64_t)d->worker, (uint64_t)(int64_t)d->iter, (uint64_t)(int64_t)d->site);
    m.k0 = (uint32_t)key;
    m.k1 = (uint32_t)(key >> 32);
    m.first_row = d->first_row;
    const uint32_t threshold = (uint32_t)std::floor((double)d->p * 65536.0 + 0.5);
    m.none = threshold > 65535u;
    m.threshold = m.none ? 0xFFFFFFFFu : threshold << 16;
    m.factor = m.none ? 0.f : (float)(65536.0 / (65536.0 - threshold));
    return m;
}

bool product_ok(const hop_product_args* a) {
    if (!a || !groups_ok(a->groups, a->w_index != nullptr) || a->in < 1 || a->in > kMostCols || a->out < 1 || a->out > kMostCols) return false;
    if (a->groups.rows > kMostResults / a->out) return false;
    const size_t e = type_bytes(a->groups.dtype);
    return matrix_ok(a->w, a->ldw, a->transposed ? a->out : a->in, e) && vectors_ok(nullptr, a->w_stride) && index_ok(a->w_index, a->groups.G) &&
           (a->groups.rows == 0 || (matrix_ok(a->x, a->ldx, a->in, e) && matrix_ok(a->y, a->ldy, a->out, e)));
}
HopProductTask product_task(const hop_product_args* a) {
    HopProductTask t;
    t.rows = rows_of(a->groups);
    t.x = a->x; t.w = a->w; t.y = a->y;
    t.ldx = a->ldx; t.ldw = a->ldw; t.w_stride = a->w_stride; t.ldy = a->ldy;
    t.in = (int32_t)a->in; t.out = (int32_t)a->out; t.indexed = a->w_index != nullptr;
    t.partial = nullptr;
    return t;
}

bool product_grad_ok(const hop_product_grad_args* a) {
    if (!a || !groups_ok(a->groups, a->dw_index != nullptr) || a->in < 1 || a->in > kMostCols || a->out < 1 || a->out > kMostCols) return false;
    if (a->groups.G > kMostResults / a->out / a->in) return false;
    const size_t e = type_bytes(a->groups.dtype);
    return matrix_ok(a->dw, a->lddw, a->in, 4) && vectors_ok(nullptr, a->dw_stride) && index_ok(a->dw_index, a->groups.G) &&
           distinct(a->dw_index, a->groups.G) && apart(a->dw_index, a->groups.G, a->dw_stride, a->out, a->lddw, a->in) &&
           (a->groups.rows == 0 || (matrix_ok(a->dy, a->lddy, a->out, e) && matrix_ok(a->x, a->ldx, a->in, e)));
}

HopProductGradTask product_grad_task(const hop_product_grad_args* a) {
    HopProductGradTask t;
    t.rows = rows_of(a->groups);
    t.dy = a->dy; t.x = a->x; t.dw = a->dw;
    t.lddy = a->lddy; t.ldx = a->ldx; t.lddw = a->lddw; t.dw_stride = a->dw_stride;
    t.in = (int32_t)a->in; t.out = (int32_t)a->out; t.indexed = a->dw_index != nullptr;
    t.partial = nullptr;
    return t;
}

bool residual_ok(const hop_residual_args* a) {
    if (!a || !groups_ok(a->groups, a->index != nullptr) || a->cols < 1 || a->cols > HOP_MAX_NORM_COLS) return false;
    if (a->norm < HOP_NORM_NONE || a->norm > HOP_NORM_CENTRED || a->next_norm < HOP_NORM_NONE || a->next_norm > HOP_NORM_CENTRED) return false;
    if (!(a->eps >= 0.f) || std::isinf(a->eps) || !std::isfinite(a->scale) || !drop_ok(a->drop) || !index_ok(a->index, a->groups.G)) return false;
    if (!vectors_ok(a->post, a->post_stride) || !vectors_ok(a->pre, a->pre_stride) || !vectors_ok(a->gate, a->gate_stride)) return false;
    const size_t e = type_bytes(a->groups.dtype);
    const bool rows = a->groups.rows > 0;
    if (a->gate_kind == HOP_GATE_VECTOR) {
        if (!a->gate || a->z) return false;
    } else if (a->gate_kind == HOP_GATE_ELEMENT) {
        if (a->gate || (rows && !matrix_ok(a->z, a->ldz, a->cols, e))) return false;
    } else if (a->gate_kind != HOP_GATE_NONE || a->gate || a->z) {
        return false;
    }
    if (!a->b) {                       // a norm by itself; without rows there need be no address
        const bool branch = a->norm || a->post || a->gate_kind || (a->drop && a->drop->p > 0.f);
        if (branch ? rows : !a->next_norm) return false;
    } else if (rows && !matrix_ok(a->b, a->ldb, a->cols, e)) {
        return false;
    }
    return !a->pre || a->next_norm;
}
HopResidualTask residual_task(const hop_residual_args* a) {
    HopResidualTask t;
    std::memset(&t, 0, sizeof(t));
    t.rows = rows_of(a->groups);
    t.cols = (int32_t)a->cols;
    t.norm = a->norm; t.next_norm = a->next_norm; t.gate_kind = a->gate_kind;
    t.indexed = a->index != nullptr;
    t.scale = a->scale; t.eps = a->eps; t.inv_cols = (float)(1.0 / (double)a->cols);
    t.mask = mask_of(a->drop);
    t.b = a->b; t.z = a->z; t.ldb = a->ldb; t.ldz = a->ldz;
    t.post = a->post; t.pre = a->pre; t.gate = a->gate;
    t.post_stride = a->post_stride; t.pre_stride = a->pre_stride; t.gate_stride = a->gate_stride;
    return t;
}
bool grads_ok(const hop_residual_args* a, const hop_residual_grads* g) {
    if (!residual_ok(a) || !g) return false;
    const size_t e = type_bytes(a->groups.dtype);
    const int64_t d = a->cols;
    auto opt = [&](const void* p, int64_t ld) { return !p || matrix_ok(p, ld, d, e); };
    if (!opt(g->dy, g->lddy) || !opt(g->dh, g->lddh) || !opt(g->y, g->ldy) || !opt(g->dx, g->lddx) || !opt(g->db, g->lddb) || !opt(g->dz, g->lddz))
        return false;
    if (!vectors_ok(g->dpost, g->dpost_stride) || !vectors_ok(g->dpre, g->dpre_stride) || !vectors_ok(g->dgate, g->dgate_stride)) return false;
    const bool rows = a->groups.rows > 0;
    if (rows && ((!g->dy && !g->dh) || (g->dh && (!a->next_norm || !g->y)))) return false;
    if (rows && !a->b && (g->db || g->dpost || g->dgate || g->dz)) return false;
    if ((g->dpost && !a->post) || (g->dpre && !a->pre) || (g->dgate && !a->gate) || (g->dz && a->gate_kind != HOP_GATE_ELEMENT)) return false;
    if (g->index && a->groups.G > HOP_MAX_INDEXED) return false;
    if (!index_ok(g->index, a->groups.G) || !distinct(g->index, a->groups.G)) return false;
    auto vectors_apart = [&](const float* p, int64_t stride) { return !p || apart(g->index, a->groups.G, stride, 1, d, d); };
    return vectors_apart(g->dpost, g->dpost_stride) && vectors_apart(g->dpre, g->dpre_stride) && vectors_apart(g->dgate, g->dgate_stride);
}

}  // namespace

extern "C" {

size_t hop_product_scratch_bytes(const hop_product_args* a) {
    if (!product_ok(a) || a->groups.rows == 0) return 0;
    const HopProductPlan p = hopl_product_plan(product_task(a), a->groups.dtype, a->transposed != 0);
    return p.parts > 1 ? (size_t)p.parts * (size_t)a->groups.rows * (size_t)a->out * 4 : 0;
}

int hop_product(const hop_product_args* a, void* scratch, size_t scratch_bytes, void* stream) {
    if (!product_ok(a)) return HOP_ERR_INVALID_ARG;
    if (a->groups.rows == 0) return HOP_OK;
    HopProductTask t = product_task(a);
    const HopProductPlan p = hopl_product_plan(t, a->groups.dtype, a->transposed != 0);
    if (p.parts > 1) {
        if (scratch_bytes < (size_t)p.parts * (size_t)t.rows.rows * (size_t)t.out * 4) return HOP_ERR_ARENA_TOO_SMALL;
        if (!scratch || ((uintptr_t)scratch & 15u)) return HOP_ERR_INVALID_ARG;
        t.partial = (float*)scratch;
    }
    HopIndex index = {};
    hop_index_fill(&index, a->w_index, a->groups.G);
    const int rc = hopl_product(t, p, a->groups.dtype, a->transposed != 0, index, stream);
    return rc ? hip_fail((hipError_t)rc, "product launch") : HOP_OK;
}

size_t hop_product_grad_scratch_bytes(const hop_product_grad_args* a) {
    if (!product_grad_ok(a)) return 0;
    const HopProductPlan p = hopl_product_grad_plan(product_grad_task(a), a->groups.dtype);
    return p.parts > 1 ? (size_t)p.parts * (size_t)a->groups.G * (size_t)a->out * (size_t)a->in * 4 : 0;
}

int hop_product_grad(const hop_product_grad_args* a, void* scratch, size_t scratch_bytes, void* stream) {
    if (!product_grad_ok(a)) return HOP_ERR_INVALID_ARG;
    HopProductGradTask t = product_grad_task(a);
    const HopProductPlan p = hopl_product_grad_plan(t, a->groups.dtype);
    if (p.parts > 1) {
        if (scratch_bytes < (size_t)p.parts * (size_t)t.rows.G * (size_t)t.out * (size_t)t.in * 4) return HOP_ERR_ARENA_TOO_SMALL;
        if (!scratch || ((uintptr_t)scratch & 15u)) return HOP_ERR_INVALID_ARG;
        t.partial = (float*)scratch;
    }
    HopIndex index = {};
    hop_index_fill(&index, a->dw_index, a->groups.G);
    const int rc = hopl_product_grad(t, p, a->groups.dtype, index, stream);
    return rc ? hip_fail((hipError_t)rc, "product gradient launch") : HOP_OK;
}

int hop_dropout(int32_t dtype, const void* x, int64_t ldx, void* y, int64_t ldy, int64_t rows, int64_t cols, const hop_drop* drop, void* stream) {
    if (!known_type(dtype) || !drop || !drop_ok(drop) || rows < 0 || rows > kMostRows || cols < 1 || cols > kMostDropCols) return HOP_ERR_INVALID_ARG;
    if (rows == 0) return HOP_OK;
    const size_t e = type_bytes(dtype);
    if (!matrix_ok(x, ldx, cols, e) || !matrix_ok(y, ldy, cols, e) || (x == y && ldx != ldy)) return HOP_ERR_INVALID_ARG;
    const int rc = hopl_dropout(dtype, x, ldx, y, ldy, rows, cols, mask_of(drop), stream);
    return rc ? hip_fail((hipError_t)rc, "dropout launch") : HOP_OK;
}

int hop_residual(const hop_residual_args* a, const void* x, int64_t ldx, void* y, int64_t ldy, void* h, int64_t ldh, void* stream) {
    if (!residual_ok(a)) return HOP_ERR_INVALID_ARG;
    if (a->groups.rows == 0) return HOP_OK;
    const size_t e = type_bytes(a->groups.dtype);
    if (!matrix_ok(x, ldx, a->cols, e) || (a->b ? !matrix_ok(y, ldy, a->cols, e) : y != nullptr) ||
        (a->next_norm ? !matrix_ok(h, ldh, a->cols, e) : h != nullptr))
        return HOP_ERR_INVALID_ARG;
    // in place, row by row: at another distance a row would be written before another workgroup has read the row that lies there
    if (a->groups.rows > 1 && y && ((y == x && ldy != ldx) || (y == a->b && ldy != a->ldb))) return HOP_ERR_INVALID_ARG;
    HopResidualTask t = residual_task(a);
    t.x = x; t.ldx = ldx;
    t.y = y; t.ldy = ldy;
    t.h = h; t.ldh = ldh;
    HopIndex index = {};
    hop_index_fill(&index, a->index, a->groups.G);
    const int rc = hopl_residual(t, a->groups.dtype, index, stream);
    return rc ? hip_fail((hipError_t)rc, "residual launch") : HOP_OK;
}

size_t hop_residual_grad_scratch_bytes(const hop_residual_args* a, const hop_residual_grads* g) {
    if (!grads_ok(a, g) || !(g->dpost || g->dpre || g->dgate)) return 0;
    return (size_t)hopl_grad_chunks(a->groups.rows, a->groups.G, a->cols) * 3 * (size_t)a->cols * 4;
}

int hop_residual_grad(const hop_residual_args* a, const hop_residual_grads* g, void* scratch, size_t scratch_bytes, void* stream) {
    if (!grads_ok(a, g)) return HOP_ERR_INVALID_ARG;
    const size_t need = hop_residual_grad_scratch_bytes(a, g);
    if (scratch_bytes < need) return HOP_ERR_ARENA_TOO_SMALL;
    if (need && (!scratch || ((uintptr_t)scratch & 15u))) return HOP_ERR_INVALID_ARG;
    HopResidualTask t = residual_task(a);
    t.dy = g->dy; t.dh = g->dh; t.y = const_cast<void*>(g->y);
    t.dx = g->dx; t.db = g->db; t.dz = g->dz;
    t.lddy = g->lddy; t.lddh = g->lddh; t.ldy = g->ldy; t.lddx = g->lddx; t.lddb = g->lddb; t.lddz = g->lddz;
    t.dpost = g->dpost; t.dpre = g->dpre; t.dgate = g->dgate;
    t.dpost_stride = g->dpost_stride; t.dpre_stride = g->dpre_stride; t.dgate_stride = g->dgate_stride;
    t.dindexed = g->index != nullptr;
    t.partial = need ? (float*)scratch : nullptr;
    HopIndex index = {}, dindex = {};
    hop_index_fill(&index, a->index, a->groups.G);
    hop_index_fill(&dindex, g->index, a->groups.G);
    const int rc = hopl_residual_grad(t, a->groups.dtype, index, dindex, stream);
    return rc ? hip_fail((hipError_t)rc, "residual gradient launch") : HOP_OK;
}

}  // extern "C"
