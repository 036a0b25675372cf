// The host code of hop_layers.cpp under the sanitizers: kernel launchers are stubs that check what they are given.  Walks grids of arguments,
// good and bad ones; prints how many calls of each there were.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>
#include <vector>

#include "hop_layers_internal.h"

namespace {
int launches = 0;
void require(bool ok, const char* what) {
    if (!ok) {
        std::printf("broken: %s\n", what);
        std::exit(1);
    }
}
void rows_ok(const HopRows& r) { require(r.G >= 1 && r.G <= HOP_MAX_GROUPS && r.rows >= 0 && (r.begin || r.G == 1), "rows"); }
HopProductPlan plan(int parts) { return HopProductPlan{HOPL_ANY, parts, 1}; }
}  // namespace

HopProductPlan hopl_product_plan(const HopProductTask& t, int, int) { return plan(t.in > 64 ? 4 : 1); }
HopProductPlan hopl_product_grad_plan(const HopProductGradTask& t, int) { return plan(t.rows.rows > 64 ? 2 : 1); }
int hopl_product(const HopProductTask& t, const HopProductPlan& p, int dtype, int transposed, const HopIndex& index, void*) {
    rows_ok(t.rows);
    require(t.rows.rows > 0 && t.x && t.w && t.y && t.ldx >= t.in && t.ldy >= t.out && t.ldw >= (transposed ? t.out : t.in), "product");
    require((dtype == HOP_F32 || dtype == HOP_BF16) && (p.parts == 1) == !t.partial, "product's parts");
    for (int g = 0; t.indexed && g < t.rows.G; ++g) require(index.at[g] >= 0, "index");
    return ++launches, 0;
}
int hopl_product_grad(const HopProductGradTask& t, const HopProductPlan& p, int, const HopIndex&, void*) {
    rows_ok(t.rows);
    require(t.dw && t.lddw >= t.in && (p.parts == 1) == !t.partial, "product's gradient");
    return ++launches, 0;
}
int hopl_dropout(int, const void* x, int64_t ldx, void* y, int64_t ldy, int64_t rows, int64_t cols, const HopMask& m, void*) {
    require(x && y && rows > 0 && cols > 0 && ldx >= cols && ldy >= cols && m.factor >= 0.f && (m.none ? m.factor == 0.f : m.factor >= 1.f), "dropout");
    return ++launches, 0;
}
int hopl_residual(HopResidualTask t, int, const HopIndex&, void*) {
    rows_ok(t.rows);
    require(t.x && (t.b ? t.y != nullptr : !t.y) && (t.next_norm ? t.h != nullptr : !t.h) && !(t.gate && t.z), "residual");
    return ++launches, 0;
}
int hopl_residual_grad(HopResidualTask t, int, const HopIndex&, const HopIndex&, void*) {
    rows_ok(t.rows);
    require(t.rows.rows == 0 || t.dy || t.dh, "residual's gradient");
    require((t.dpost || t.dpre || t.dgate) || !t.partial, "partial sums");
    return ++launches, 0;
}
int hopl_grad_shift(int64_t rows, int64_t) { return rows > 100 ? 2 : 0; }
int64_t hopl_grad_chunks(int64_t rows, int G, int64_t) { return rows / 2 + G; }

int main() {
    std::vector<float> room(1 << 16);
    std::vector<int32_t> begin(HOP_MAX_GROUPS + 1), index(HOP_MAX_GROUPS);
    for (int g = 0; g < HOP_MAX_GROUPS; ++g) index[g] = g * 3;
    void* at = room.data();
    const float nan = std::numeric_limits<float>::quiet_NaN(), inf = std::numeric_limits<float>::infinity();
    int good = 0, bad = 0, small = 0;
    auto count = [&](int rc) { rc == HOP_OK ? ++good : rc == HOP_ERR_ARENA_TOO_SMALL ? ++small : ++bad; };
    for (int G : {-1, 0, 1, 3, HOP_MAX_INDEXED, HOP_MAX_INDEXED + 1, HOP_MAX_GROUPS, HOP_MAX_GROUPS + 1})
        for (int64_t rows : {int64_t(-1), int64_t(0), int64_t(1), int64_t(100), int64_t(1) << 29, int64_t(1) << 31, std::numeric_limits<int64_t>::max()})
            for (int dtype : {0, 1, 7})
                for (int64_t cols : {int64_t(0), int64_t(1), int64_t(65), int64_t(1) << 21, int64_t(1) << 40, std::numeric_limits<int64_t>::min()})
                    for (int indexed : {0, 1}) {
                        const hop_groups groups = {rows, indexed && G == 1 ? nullptr : begin.data(), G, dtype};
                        for (int transposed : {0, 1}) {
                            hop_product_args a = {groups, at, cols, at, cols < 7 ? 7 : cols, 7, indexed ? index.data() : nullptr, at, 7, cols, 7, transposed, 0};
                            const size_t need = hop_product_scratch_bytes(&a);
                            count(hop_product(&a, nullptr, 0, nullptr));
                            if (need) count(hop_product(&a, at, need, nullptr)), count(hop_product(&a, at, need - 1, nullptr)), count(hop_product(&a, nullptr, need, nullptr));
                        }
                        hop_product_grad_args b = {groups, at, 7, at, cols, room.data(), cols, 9, indexed ? index.data() : nullptr, cols, 7};
                        const size_t need = hop_product_grad_scratch_bytes(&b);
                        count(hop_product_grad(&b, at, need, nullptr));
                        if (need) count(hop_product_grad(&b, at, need - 1, nullptr));
                        for (float p : {0.f, 0.3f, 1.f, 1.5f, nan, -inf}) {
                            const hop_drop drop = {~0ull, indexed ? std::numeric_limits<int64_t>::max() : 5, -1, std::numeric_limits<int32_t>::min(), 3, p};
                            count(hop_dropout(dtype, at, cols, at, cols, rows, cols, &drop, nullptr));
                            for (int kind : {-1, 0, 1, 2})
                                for (int norm : {0, 2, 3}) {
                                    hop_residual_args r;
                                    std::memset(&r, 0, sizeof(r));
                                    r.groups = groups;
                                    r.cols = cols;
                                    r.b = norm ? at : nullptr;
                                    r.ldb = r.ldz = cols;
                                    r.z = kind == 2 ? at : nullptr;
                                    r.gate = kind == 1 ? room.data() : nullptr;
                                    r.post = norm ? room.data() : nullptr;
                                    r.pre = room.data();
                                    r.index = indexed ? index.data() : nullptr;
                                    r.drop = &drop;
                                    r.norm = norm;
                                    r.next_norm = 1;
                                    r.gate_kind = kind;
                                    r.scale = 1.f;
                                    r.eps = p == 0.3f ? 1e-5f : p;
                                    count(hop_residual(&r, at, cols, norm ? at : nullptr, cols, at, cols, nullptr));
                                    hop_residual_grads g;
                                    std::memset(&g, 0, sizeof(g));
                                    g.dy = g.dh = g.y = at;
                                    g.dx = at;
                                    g.db = norm ? at : nullptr;
                                    g.lddy = g.lddh = g.ldy = g.lddx = g.lddb = cols;
                                    g.dpre = room.data();
                                    g.dgate = kind == 1 ? room.data() : nullptr;
                                    g.index = indexed ? index.data() : nullptr;
                                    const size_t wanted = hop_residual_grad_scratch_bytes(&r, &g);
                                    count(hop_residual_grad(&r, &g, at, wanted, nullptr));
                                    if (wanted) count(hop_residual_grad(&r, &g, at, wanted - 1, nullptr));
                                }
                        }
                    }
    count(hop_product(nullptr, nullptr, 0, nullptr));
    count(hop_product_grad(nullptr, nullptr, 0, nullptr));
    count(hop_residual(nullptr, nullptr, 0, nullptr, 0, nullptr, 0, nullptr));
    count(hop_residual_grad(nullptr, nullptr, nullptr, 0, nullptr));
    std::printf("ok good=%d bad=%d small=%d launches=%d\n", good, bad, small, launches);
    return 0;
}
