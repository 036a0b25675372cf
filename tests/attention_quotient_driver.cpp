// Rows of pairs: the quotient that hop_attention.cpp prepares and the kernels take, for every group there may be, through the C entries (kernel launchers are stubs that
// check it).  Prints how many launches there were and how many quotients were looked at.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "hop_attention_internal.h"

namespace {
int64_t launches = 0, looked = 0;
void look(const HopAttentionTask& t, int64_t x) {
    if (x < 0 || x >= (int64_t)1 << 31) return;
    ++looked;
    if (hopa_divide((int)x, t.group_inverse, t.group_shift) == x / t.group) return;
    std::printf("broken: %lld / %d\n", (long long)x, t.group);
    std::exit(1);
}
// What is rounded up in the inverse weighs most in front of a multiple of the group, and the more the larger the number: multiples near every power of two, many
// in between, and the largest ones, of pairs and below 2^31.
void task_ok(const HopAttentionTask& t) {
    ++launches;
    const int64_t g = t.group;
    for (int bit = 0; bit <= 31; ++bit)
        for (int64_t k = ((int64_t)1 << bit) / g - 2; k <= ((int64_t)1 << bit) / g + 2; ++k)
            for (int64_t more : {int64_t(-1), int64_t(0), int64_t(1), g / 2}) look(t, k * g + more);
    const int64_t most = ((int64_t)1 << 31) / g, step = most / 4096 + 1;
    for (int64_t k = 0; k <= most; k += step) look(t, k * g - 1), look(t, k * g);
    for (int64_t x = ((int64_t)1 << 31) - 2 * g; x < (int64_t)1 << 31; ++x) look(t, x);
    const int64_t pairs = (int64_t)t.q_rows * g;
    look(t, pairs - 1), look(t, pairs), look(t, pairs + 127);
}
}  // namespace

HopAttentionPlan hopa_forward_plan(HopAttentionTask*, int, char*) { return {}; }
int hopa_forward(const HopAttentionTask& t, int, const HopAttentionPlan&, void*) { return task_ok(t), 0; }
HopAttentionPlan hopa_grad_plan(HopAttentionTask*, int, char*) { return {}; }
int hopa_grad(const HopAttentionTask& t, int, const HopAttentionPlan&, void*) { return task_ok(t), 0; }
int hopa_rotate(const HopRotateTask&, int, const HopIndex&, void*) { return 0; }
int hopa_rotate_grad(const HopRotateTask&, int, const HopIndex&, const HopIndex&, void*) { return 0; }

int main() {
    std::vector<float> room(64);
    void* at = room.data();
    for (int group = 1; group <= HOP_MAX_HEADS; ++group)
        for (int k_heads : {1, HOP_MAX_HEADS / group}) {
            const int64_t most = std::min((((int64_t)1 << 30) - 1) / (group * k_heads), ((int64_t)1 << 30) - 65536);
            const hop_attention_args a = {most, 5, nullptr, nullptr, 1, 1, at, group * k_heads, at, k_heads, at, k_heads, group * k_heads, k_heads, 1, 1, 1.f, 0};
            const hop_attention_grads g = {at, group * k_heads, at, group * k_heads, room.data(), at, group * k_heads, at, k_heads, at, k_heads};
            if (hop_attention(&a, at, group * k_heads, room.data(), nullptr, 0, nullptr) || hop_attention_grad(&a, &g, at, 256, nullptr)) {
                std::printf("broken: %d heads a group refused\n", group);
                return 1;
            }
        }
    std::printf("ok launches=%lld looked=%lld\n", (long long)launches, (long long)looked);
    return 0;
}
