// hop_layers.cpp under the sanitizers with gradients of parameters that lie apart, behind each other and side by side, in index lists of every
// kind; the launchers and checks are layers_driver.cpp's.
#define main grids_of_arguments
#include "layers_driver.cpp"
#undef main
#include <algorithm>

int main() {
    std::vector<float> room(1 << 10);
    std::vector<int32_t> begin(HOP_MAX_GROUPS + 1);
    void* at = room.data();
    int good = 0, bad = 0;
    const int64_t far = (int64_t)1 << 40;
    for (int G : {1, 2, HOP_MAX_INDEXED, HOP_MAX_GROUPS})
        for (int order : {0, 1, 2, 3}) {                    // none, ascending, descending, with gaps as far as a list can say
            if (order && G > HOP_MAX_INDEXED) continue;
            std::vector<int32_t> index(G);
            for (int g = 0; g < G; ++g) index[g] = order == 3 ? (g ? std::numeric_limits<int32_t>::max() - g : 0) : order == 2 ? G - 1 - g : g;
            const int64_t span = order == 3 && G > 1 ? std::numeric_limits<int32_t>::max() - 1 : G - 1;
            for (int64_t in : {1, 8, 65, 1 << 21})
                for (int64_t out : {1, 7, 1 << 21})
                    for (int64_t ld : {in, in + 5, std::min(far + 1, in * (span + 1)), std::min(far, in * (span + 1) - 1), far})
                        for (int64_t stride : {int64_t(0), in - 1, in, -in, (out - 1) * ld + in, 1 - (out - 1) * ld - in, far, -far, std::numeric_limits<int64_t>::min()}) {
                            const hop_groups groups = {100, begin.data(), G, HOP_F32};
                            hop_product_grad_args a = {groups, at, out, at, in, room.data(), ld, stride, order ? index.data() : nullptr, in, out};
                            const size_t need = hop_product_grad_scratch_bytes(&a);
                            const int rc = hop_product_grad(&a, at, need, nullptr);
                            const int64_t s = stride == std::numeric_limits<int64_t>::min() ? far + 1 : std::abs(stride);        // too far in any case
                            const bool taken = ld >= in && ld <= far && s <= far && (double)G * out * in <= 1099511627776.0 &&
                                               (G == 1 || s >= (out - 1) * ld + in || (s >= in && ((double)span * s + in <= ld || out == 1)));
                            require((rc == HOP_OK) == taken, "product's gradient");
                            rc == HOP_OK ? ++good : ++bad;
                            if (in > HOP_MAX_NORM_COLS) continue;
                            hop_residual_args r;
                            std::memset(&r, 0, sizeof(r));
                            r.groups = groups;
                            r.cols = r.ldb = in;
                            r.b = at;
                            r.post = r.gate = room.data();
                            r.gate_kind = HOP_GATE_VECTOR;
                            r.scale = 1.f;
                            hop_residual_grads g;
                            std::memset(&g, 0, sizeof(g));
                            g.dy = g.dx = at;
                            g.lddy = g.lddx = in;
                            g.dpost = g.dgate = room.data();
                            g.dpost_stride = in;
                            g.dgate_stride = stride;
                            g.index = order ? index.data() : nullptr;
                            const size_t wanted = hop_residual_grad_scratch_bytes(&r, &g);
                            const bool apart = s <= far && (G == 1 || s >= in);
                            require((wanted > 0) == apart && (hop_residual_grad(&r, &g, at, wanted, nullptr) == HOP_OK) == apart, "vectors' gradients");
                            apart ? ++good : ++bad;
                        }
        }
    std::printf("ok good=%d bad=%d launches=%d\n", good, bad, launches);
    return 0;
}
