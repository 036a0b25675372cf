// The host code of hop_attention.cpp under the sanitizers: kernel launchers are stubs that check what they are given.  Walks grids of arguments,
// good and bad ones; prints how many calls of each there were.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>
#include <vector>

#include "hop_attention_internal.h"

namespace {
int launches = 0;
void require(bool ok, const char* what) {
    if (!ok) {
        std::printf("broken: %s\n", what);
        std::exit(1);
    }
}
void attention_ok(const HopAttentionTask& t) {
    require(t.S >= 1 && t.S <= HOP_MAX_GROUPS && (t.S == 1 || (t.q_begin && t.k_begin)), "sequences");
    require(t.group >= 1 && t.k_heads >= 1 && t.cols >= 1 && t.cols <= HOP_MAX_HEAD_COLS && t.scale > 0.f && t.scale_log2 > 0.f, "sizes");
    require((int64_t)t.q_rows * t.group * t.k_heads < 1 << 30 && (t.group == 1) == (t.group_inverse == 0), "pairs");
    for (int64_t x : {int64_t(0), int64_t(t.group) - 1, (int64_t)t.q_rows * t.group - 1, (int64_t)t.q_rows * t.group / 2})       // the kernels' quotient
        if (x >= 0 && t.group > 1) require((int64_t)(((uint64_t)x * t.group_inverse) >> 32) == x / t.group, "inverse");
    require(!t.q_rows || (t.q && t.ldq >= (int64_t)t.group * t.k_heads * t.cols), "queries");
    require(!t.k_rows || (t.k && t.v && t.ldk >= t.k_heads * t.cols && t.ldv >= t.k_heads * t.cols), "keys");
}
void rotate_ok(const HopRotateTask& t) {
    require(t.heads >= 1 && t.cols >= 1 && t.cols <= HOP_MAX_HEAD_COLS && t.rotary >= 0 && t.rotary <= t.cols && t.rotary % 2 == 0, "rotation");
    for (int i = 0; i < t.rotary / 2; ++i) require(t.turns[i] > 0 && t.turns[i] < std::numeric_limits<double>::infinity(), "turns");
}
}  // namespace

HopAttentionPlan hopa_forward_plan(HopAttentionTask* t, int, char* scratch) {
    HopAttentionPlan p = {};
    t->parts = t->k_rows > 64 ? 3 : 1;
    p.bytes = t->parts > 1 ? 512 : 0;
    t->partial = t->parts > 1 ? (float*)scratch : nullptr;
    return p;
}
int hopa_forward(const HopAttentionTask& t, int, const HopAttentionPlan&, void*) {
    attention_ok(t);
    require(t.q_rows > 0 && t.o && (t.parts == 1) == !t.partial, "attention");
    return ++launches, 0;
}
HopAttentionPlan hopa_grad_plan(HopAttentionTask* t, int, char* scratch) {
    HopAttentionPlan p = {};
    p.bytes = 256;
    t->terms = (float*)scratch;
    return p;
}
int hopa_grad(const HopAttentionTask& t, int, const HopAttentionPlan&, void*) {
    attention_ok(t);
    require((!t.q_rows || (t.grad && t.o && t.lse && t.dq)) && (!t.k_rows || (t.dk && t.dv)) && t.terms, "attention's gradient");
    return ++launches, 0;
}
int hopa_rotate(const HopRotateTask& t, int, const HopIndex&, void*) {
    rotate_ok(t);
    require(t.x && t.y && t.rows.rows > 0, "rotation");
    return ++launches, 0;
}
int hopa_rotate_grad(const HopRotateTask& t, int, const HopIndex&, const HopIndex&, void*) {
    rotate_ok(t);
    require(!(t.dq_weight || t.dk_weight) || t.partial, "rotation's gradient");
    return ++launches, 0;
}
int64_t hopa_rotate_chunks(int64_t rows, int G, int32_t) { return rows / 2 + G; }

int main() {
    std::vector<float> room(1 << 12);
    std::vector<int32_t> index(HOP_MAX_GROUPS + 1);
    for (int g = 0; g <= HOP_MAX_GROUPS; ++g) index[g] = g * 3;
    void* at = room.data();
    const float nan = std::numeric_limits<float>::quiet_NaN(), inf = std::numeric_limits<float>::infinity();
    int good = 0, bad = 0, small = 0;
    auto count = [&](int rc) { rc == HOP_OK ? ++good : rc == HOP_ERR_ARENA_TOO_SMALL ? ++small : ++bad; };
    const int32_t most = std::numeric_limits<int32_t>::max();
    for (int S : {-1, 0, 1, 3, HOP_MAX_GROUPS, HOP_MAX_GROUPS + 1})
        for (int64_t rows : {int64_t(-1), int64_t(0), int64_t(1), int64_t(100), int64_t(1) << 29, std::numeric_limits<int64_t>::max()})
            for (int dtype : {0, 1, 7})
                for (int heads : {-3, 0, 1, 6, HOP_MAX_HEADS, most})
                    for (int cols : {-1, 0, 1, 17, 64, HOP_MAX_HEAD_COLS, HOP_MAX_HEAD_COLS + 1, most})
                        for (int kind : {0, 1, 2}) {
                            const int k_heads = kind == 1 && heads > 0 && heads % 2 == 0 ? heads / 2 : kind == 2 ? 4 : heads;
                            const int64_t ld = kind == 2 ? 1 << 23 : (int64_t)(heads > 0 ? heads : 1) * (cols > 0 ? cols : 1);
                            const float scale = kind == 2 && S == 3 ? nan : kind == 2 && S == 1 ? inf : 0.5f;
                            hop_attention_args a = {rows, rows, S == 1 ? nullptr : index.data(), S == 1 ? nullptr : index.data(), S, dtype, at, ld, at, ld, at, ld, heads, k_heads, cols, kind & 1, scale, 0};
                            const size_t need = hop_attention_scratch_bytes(&a);
                            count(hop_attention(&a, at, ld, room.data(), at, need, nullptr));
                            if (need) count(hop_attention(&a, at, ld, nullptr, at, need - 1, nullptr)), count(hop_attention(&a, at, ld, nullptr, nullptr, need, nullptr));
                            hop_attention_grads g = {at, ld, at, ld, room.data(), at, ld, at, ld, at, ld};
                            const size_t wanted = hop_attention_grad_scratch_bytes(&a, &g);
                            count(hop_attention_grad(&a, &g, at, wanted, nullptr));
                            if (wanted) count(hop_attention_grad(&a, &g, at, wanted - 1, nullptr));
                            const hop_groups groups = {rows, S == 1 ? nullptr : index.data(), S, dtype};
                            for (double base : {10000.0, 0.0, (double)nan})
                                for (int rotary : {0, 16, 64, -2}) {
                                    hop_rotate_args r = {groups, nullptr, nullptr, 1, heads, k_heads, cols, rotary, kind & 1, room.data(), cols, kind ? room.data() : nullptr, cols,
                                                         kind == 1 ? index.data() : nullptr, base, kind == 2 ? inf : 1e-5f, kind};
                                    const int64_t wide = (int64_t)(heads + (int64_t)k_heads) * cols;
                                    count(hop_rotate(&r, at, wide, at, wide, nullptr));
                                    hop_rotate_grads d = {at, wide, at, wide, at, wide, room.data(), cols, kind ? room.data() : nullptr, cols, kind == 1 ? index.data() : nullptr};
                                    const size_t room_for = hop_rotate_grad_scratch_bytes(&r, &d);
                                    count(hop_rotate_grad(&r, &d, at, room_for, nullptr));
                                    if (room_for) count(hop_rotate_grad(&r, &d, at, room_for - 1, nullptr));
                                }
                        }
    count(hop_rotate(nullptr, nullptr, 0, nullptr, 0, nullptr));
    count(hop_rotate_grad(nullptr, nullptr, nullptr, 0, nullptr));
    count(hop_attention(nullptr, nullptr, 0, nullptr, nullptr, 0, nullptr));
    count(hop_attention_grad(nullptr, nullptr, nullptr, 0, nullptr));
    std::printf("ok good=%d bad=%d small=%d launches=%d\n", good, bad, small, launches);
    return 0;
}
