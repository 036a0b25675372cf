// C ABI of include/hop_attention.h: checks of arguments and their translation into what the kernels take.
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstring>

#include "hop_attention_internal.h"
#include "hop_internal.h"
#include "hop_layers_checks.h"

using namespace hopl;

namespace {

constexpr int64_t kMostPairs = 1 << 30;         // rows times heads: pairs are counted in 31 bits
constexpr double kTwoPi = 6.283185307179586476925286766559;

bool table_ok(const int32_t* begin, int S) { return (begin || S == 1) && ((uintptr_t)begin & 3u) == 0; }
// a matrix of rows with heads: as matrix_ok, and not too far apart
bool heads_ok(const void* p, int64_t ld, int64_t cols, size_t elem) { return matrix_ok(p, ld, cols, elem) && ld <= kHopaMostDistance; }

bool rotate_ok(const hop_rotate_args* a) {
    if (!a || !groups_ok(a->groups, a->index != nullptr) || !index_ok(a->index, a->groups.G)) return false;
    if (a->S < 1 || a->S > HOP_MAX_GROUPS || !table_ok(a->seq_begin, a->S) || ((uintptr_t)a->positions & 3u)) return false;
    if (a->q_heads < 0 || a->k_heads < 0 || a->q_heads > HOP_MAX_HEADS || a->k_heads > HOP_MAX_HEADS || a->q_heads + a->k_heads < 1) return false;
    if (a->cols < 1 || a->cols > HOP_MAX_HEAD_COLS || a->rotary < 0 || a->rotary > a->cols || (a->rotary & 1) || a->adjacent < 0 || a->adjacent > 1) return false;
    if (a->norm < HOP_NORM_NONE || a->norm > HOP_NORM_CENTRED || !(a->eps >= 0.f) || std::isinf(a->eps)) return false;
    if (a->rotary && !(a->base > 0.0 && std::isfinite(a->base))) return false;
    return vectors_ok(a->q_weight, a->q_weight_stride) && vectors_ok(a->k_weight, a->k_weight_stride);
}
HopRotateTask rotate_task(const hop_rotate_args* a) {
    HopRotateTask t;
    std::memset(&t, 0, sizeof(t));
    t.rows = rows_of(a->groups);
    t.sequences = HopRows{a->seq_begin, a->S, (int32_t)a->groups.rows};
    t.positions = a->positions;
    t.q_heads = a->q_heads;
    t.heads = a->q_heads + a->k_heads;
    t.cols = a->cols; t.rotary = a->rotary; t.adjacent = a->adjacent; t.norm = a->norm;
    t.indexed = a->index != nullptr;
    t.eps = a->eps;
    t.inv_cols = (float)(1.0 / a->cols);
    t.q_weight = a->q_weight; t.k_weight = a->k_weight;
    t.q_stride = a->q_weight_stride; t.k_stride = a->k_weight_stride;
    // base^(-2 i / rotary) as products of eight and eight powers, a rounding more of 64 bits: 64 powers are 0.3 us of a call of 9.7
    double near[8], far[8];
    for (int i = 0; i < 8 && i < a->rotary / 2; ++i) near[i] = std::pow(a->base, -2.0 * i / a->rotary) / kTwoPi;
    for (int i = 0; 8 * i < a->rotary / 2; ++i) far[i] = std::pow(a->base, -16.0 * i / a->rotary);
    for (int i = 0; i < a->rotary / 2; ++i) t.turns[i] = near[i % 8] * far[i / 8];
    return t;
}
bool rotate_grads_ok(const hop_rotate_args* a, const hop_rotate_grads* g) {
    if (!rotate_ok(a) || !g) return false;
    const int64_t d = (int64_t)(a->q_heads + a->k_heads) * a->cols;
    const size_t e = type_bytes(a->groups.dtype);
    const int G = a->groups.G;
    if (a->groups.rows > 0 && (!matrix_ok(g->dy, g->lddy, d, e) || !matrix_ok(g->x, g->ldx, d, e) || (g->dx && !matrix_ok(g->dx, g->lddx, d, e)))) return false;
    if (a->groups.rows > 1 && g->dx && ((g->dx == g->dy && g->lddx != g->lddy) || (g->dx == g->x && g->lddx != g->ldx))) return false;
    if ((g->dq_weight && !a->q_weight) || (g->dk_weight && !a->k_weight)) return false;
    if (!vectors_ok(g->dq_weight, g->dq_weight_stride) || !vectors_ok(g->dk_weight, g->dk_weight_stride)) return false;
    if ((g->index && G > HOP_MAX_INDEXED) || !index_ok(g->index, G) || !distinct(g->index, G)) return false;
    return (!g->dq_weight || apart(g->index, G, g->dq_weight_stride, 1, a->cols, a->cols)) &&
           (!g->dk_weight || apart(g->index, G, g->dk_weight_stride, 1, a->cols, a->cols));
}

bool attention_ok(const hop_attention_args* a) {
    if (!a || !known_type(a->dtype) || a->q_rows < 0 || a->q_rows > kMostRows || a->k_rows < 0 || a->k_rows > kMostRows) return false;
    if (a->S < 1 || a->S > HOP_MAX_GROUPS || !table_ok(a->q_begin, a->S) || !table_ok(a->k_begin, a->S)) return false;
    if (a->q_heads < 1 || a->q_heads > HOP_MAX_HEADS || a->k_heads < 1 || a->q_heads % a->k_heads || a->cols < 1 || a->cols > HOP_MAX_HEAD_COLS) return false;
    if (a->q_rows * a->q_heads >= kMostPairs || a->k_rows * a->k_heads >= kMostPairs) return false;
    if (a->causal < 0 || a->causal > 1 || !(a->scale > 0.f) || std::isinf(a->scale)) return false;
    const size_t e = type_bytes(a->dtype);
    const int64_t wide = (int64_t)a->q_heads * a->cols, narrow = (int64_t)a->k_heads * a->cols;
    return (a->q_rows == 0 || heads_ok(a->q, a->ldq, wide, e)) && (a->k_rows == 0 || (heads_ok(a->k, a->ldk, narrow, e) && heads_ok(a->v, a->ldv, narrow, e)));
}
HopAttentionTask attention_task(const hop_attention_args* a) {
    HopAttentionTask t;
    std::memset(&t, 0, sizeof(t));
    t.q_begin = a->q_begin; t.k_begin = a->k_begin;
    t.S = a->S;
    t.q_rows = (int32_t)a->q_rows; t.k_rows = (int32_t)a->k_rows;
    t.k_heads = a->k_heads; t.group = a->q_heads / a->k_heads; t.cols = a->cols;
    t.group_inverse = hopa_group_inverse(t.group);
    t.group_shift = hopa_group_shift(t.group);
    t.causal = a->causal; t.parts = 1;
    t.scale = a->scale;
    t.scale_log2 = (float)(a->scale * 1.4426950408889634074);
    t.q = a->q; t.k = a->k; t.v = a->v;
    t.ldq = a->ldq; t.ldk = a->ldk; t.ldv = a->ldv;
    return t;
}
bool attention_grads_ok(const hop_attention_args* a, const hop_attention_grads* g) {
    if (!attention_ok(a) || !g) return false;
    const size_t e = type_bytes(a->dtype);
    const int64_t wide = (int64_t)a->q_heads * a->cols, narrow = (int64_t)a->k_heads * a->cols;
    if (a->q_rows && (!heads_ok(g->grad, g->ldgrad, wide, e) || !heads_ok(g->o, g->ldo, wide, e) || !heads_ok(g->dq, g->lddq, wide, e) || !g->lse ||
                      ((uintptr_t)g->lse & 3u)))
        return false;
    return a->k_rows == 0 || (heads_ok(g->dk, g->lddk, narrow, e) && heads_ok(g->dv, g->lddv, narrow, e));
}
HopAttentionTask gradient_task(const hop_attention_args* a, const hop_attention_grads* g) {
    HopAttentionTask t = attention_task(a);
    t.grad = g->grad; t.ldgrad = g->ldgrad;
    t.o = const_cast<void*>(g->o); t.ldo = g->ldo;
    t.lse = const_cast<float*>(g->lse);
    t.dq = g->dq; t.dk = g->dk; t.dv = g->dv;
    t.lddq = g->lddq; t.lddk = g->lddk; t.lddv = g->lddv;
    return t;
}

}  // namespace

extern "C" {

int hop_rotate(const hop_rotate_args* a, const void* x, int64_t ldx, void* y, int64_t ldy, void* stream) {
    if (!rotate_ok(a)) return HOP_ERR_INVALID_ARG;
    if (a->groups.rows == 0) return HOP_OK;
    const int64_t d = (int64_t)(a->q_heads + a->k_heads) * a->cols;
    const size_t e = type_bytes(a->groups.dtype);
    if (!matrix_ok(x, ldx, d, e) || !matrix_ok(y, ldy, d, e) || (a->groups.rows > 1 && x == y && ldx != ldy)) return HOP_ERR_INVALID_ARG;
    HopRotateTask t = rotate_task(a);
    t.x = x; t.ldx = ldx;
    t.y = y; t.ldy = ldy;
    HopIndex index = {};
    hop_index_fill(&index, a->index, a->groups.G);
    const int rc = hopa_rotate(t, a->groups.dtype, index, stream);
    return rc ? hip_fail((hipError_t)rc, "rotation launch") : HOP_OK;
}

size_t hop_rotate_grad_scratch_bytes(const hop_rotate_args* a, const hop_rotate_grads* g) {
    if (!rotate_grads_ok(a, g) || !(g->dq_weight || g->dk_weight)) return 0;
    return (size_t)hopa_rotate_chunks(a->groups.rows, a->groups.G) * 2 * (size_t)a->cols * 4;
}

int hop_rotate_grad(const hop_rotate_args* a, const hop_rotate_grads* g, void* scratch, size_t scratch_bytes, void* stream) {
    if (!rotate_grads_ok(a, g)) return HOP_ERR_INVALID_ARG;
    const size_t need = hop_rotate_grad_scratch_bytes(a, g);
    if (scratch_bytes < need) return HOP_ERR_ARENA_TOO_SMALL;
    if (need && (!scratch || ((uintptr_t)scratch & 15u))) return HOP_ERR_INVALID_ARG;
    HopRotateTask t = rotate_task(a);
    t.x = g->x; t.dy = g->dy; t.dx = g->dx;
    t.ldx = g->ldx; t.lddy = g->lddy; t.lddx = g->lddx;
    t.dq_weight = g->dq_weight; t.dk_weight = g->dk_weight;
    t.dq_stride = g->dq_weight_stride; t.dk_stride = g->dk_weight_stride;
    t.dindexed = g->index != nullptr;
    t.partial = need ? (float*)scratch : nullptr;
    if (!t.dx && !need) return HOP_OK;
    HopIndex index = {}, dindex = {};
    hop_index_fill(&index, a->index, a->groups.G);
    hop_index_fill(&dindex, g->index, a->groups.G);
    const int rc = hopa_rotate_grad(t, a->groups.dtype, index, dindex, stream);
    return rc ? hip_fail((hipError_t)rc, "rotation gradient launch") : HOP_OK;
}

size_t hop_attention_scratch_bytes(const hop_attention_args* a) {
    if (!attention_ok(a) || a->q_rows == 0) return 0;
    HopAttentionTask t = attention_task(a);
    return hopa_forward_plan(&t, a->dtype, nullptr).bytes;
}

int hop_attention(const hop_attention_args* a, void* o, int64_t ldo, float* lse, void* scratch, size_t scratch_bytes, void* stream) {
    if (!attention_ok(a) || ((uintptr_t)lse & 3u)) return HOP_ERR_INVALID_ARG;
    if (a->q_rows == 0) return HOP_OK;
    if (!heads_ok(o, ldo, (int64_t)a->q_heads * a->cols, type_bytes(a->dtype))) return HOP_ERR_INVALID_ARG;
    HopAttentionTask t = attention_task(a);
    t.o = o; t.ldo = ldo;
    t.lse = lse;
    const HopAttentionPlan p = hopa_forward_plan(&t, a->dtype, (char*)scratch);
    if (scratch_bytes < p.bytes) return HOP_ERR_ARENA_TOO_SMALL;
    if (p.bytes && (!scratch || ((uintptr_t)scratch & 15u))) return HOP_ERR_INVALID_ARG;
    const int rc = hopa_forward(t, a->dtype, p, stream);
    return rc ? hip_fail((hipError_t)rc, "attention launch") : HOP_OK;
}

size_t hop_attention_grad_scratch_bytes(const hop_attention_args* a, const hop_attention_grads* g) {
    if (!attention_grads_ok(a, g) || (a->q_rows == 0 && a->k_rows == 0)) return 0;
    HopAttentionTask t = gradient_task(a, g);
    return hopa_grad_plan(&t, a->dtype, nullptr).bytes;
}

int hop_attention_grad(const hop_attention_args* a, const hop_attention_grads* g, void* scratch, size_t scratch_bytes, void* stream) {
    if (!attention_grads_ok(a, g)) return HOP_ERR_INVALID_ARG;
    if (a->q_rows == 0 && a->k_rows == 0) return HOP_OK;
    HopAttentionTask t = gradient_task(a, g);
    const HopAttentionPlan p = hopa_grad_plan(&t, a->dtype, (char*)scratch);
    if (scratch_bytes < p.bytes) return HOP_ERR_ARENA_TOO_SMALL;
    if (!scratch || ((uintptr_t)scratch & 15u)) return HOP_ERR_INVALID_ARG;
    const int rc = hopa_grad(t, a->dtype, p, stream);
    return rc ? hip_fail((hipError_t)rc, "attention gradient launch") : HOP_OK;
}

}  // extern "C"
