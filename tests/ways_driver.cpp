// Which way the library computes products: reads lines "rows groups in out", prints for each of them "size" and the plans of the product, of the
// transposed one and of the gradient to the weights, in both types, for rows that are tensors of their own and for rows at an odd address, three
// elements further apart:  type(f32|bf16) call(y|dx|dw) kind tile parts
#include <cstdio>
#include <initializer_list>

#include "hop_layers_internal.h"

namespace {
int32_t begin[2];
char place[64];

void tell(const char* type, const char* call, const HopProductPlan& p) { std::printf("%s %s %d %d %d\n", type, call, p.kind, p.tile, p.parts); }
}  // namespace

int main() {
    long long rows, groups, in, out;
    while (std::scanf("%lld %lld %lld %lld", &rows, &groups, &in, &out) == 4) {
        std::printf("size\n");
        const HopRows r = {begin, (int32_t)groups, (int32_t)rows};
        for (int dtype : {HOP_F32, HOP_BF16})
            for (int aligned : {1, 0}) {
                const char* type = dtype == HOP_F32 ? "f32" : "bf16";
                const char* at = place + (aligned ? 0 : dtype == HOP_F32 ? 4 : 2);
                const int64_t pad = aligned ? 0 : 3;
                for (int transposed : {0, 1}) {
                    HopProductTask t = {};
                    t.rows = r;
                    t.x = at;
                    t.w = place;
                    t.in = (int32_t)(transposed ? out : in);
                    t.out = (int32_t)(transposed ? in : out);
                    t.ldx = t.in + pad;
                    t.ldw = in;
                    t.w_stride = in * out;
                    tell(type, transposed ? "dx" : "y", hopl_product_plan(t, dtype, transposed));
                }
                HopProductGradTask t = {};
                t.rows = r;
                t.dy = at;
                t.x = at;
                t.lddy = out + pad;
                t.ldx = in + pad;
                t.in = (int32_t)in;
                t.out = (int32_t)out;
                tell(type, "dw", hopl_product_grad_plan(t, dtype));
            }
    }
    return 0;
}
