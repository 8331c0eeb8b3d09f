// Drives the validation layer of gradient norms and clipping through calls that are taken
// and calls that are refused, with launchers that only note what they were given.
#include <stdio.h>
#include <stdlib.h>

#include <vector>

#include "clip_launch.h"
#include "cpdp.h"

extern int g_launches;
static cpdp::Gradients seen;
static bool seen_mean;

namespace cpdp {
int launch_grad_norm(const Gradients& g, bool mean, float*, void*, void*) {
    seen = g;
    seen_mean = mean;
    return ++g_launches, 0;
}
int launch_clip_grads(const Gradients& g, bool mean, float, float*, void*, void*) {
    return launch_grad_norm(g, mean, nullptr, nullptr, nullptr);
}
}  // namespace cpdp

#define CHECK(x)                                              \
    do {                                                      \
        if (!(x)) {                                           \
            printf("line %d: %s\n", __LINE__, #x);            \
            exit(1);                                          \
        }                                                     \
    } while (0)

static char* at(int k) { return reinterpret_cast<char*>(((uintptr_t)1 << 40) * (k + 1)); }

int main() {
    float* norm = reinterpret_cast<float*>(at(1));
    void* ws = at(2);
    // launches hold one block a part at most
    for (int64_t W : {1, 2, 3, 7, 100, 2047, 2048, 2049, 1 << 23})
        for (int64_t P : {0, 1, 1024, 1025, 1 << 20, 1 << 30}) {
            const int64_t need = cpdp_grad_norm_workspace((int)W, P), ld = (P + 7) / 8 * 8;
            CHECK(need >= 8 * W || P == 0);
            for (unsigned flags : {0u, 1u}) {
                const int before = g_launches;
                CHECK(cpdp_grad_norm(at(0), (int)W, P, ld, 0, flags, norm, ws, need, nullptr) ==
                      (W * ld * 4 > (int64_t)1 << 40 ? CPDP_ERR_OVERLAP : CPDP_OK));
                if (W * ld * 4 > (int64_t)1 << 40) continue;
                CHECK(cpdp_clip_grads(at(0), (int)W, P, ld, 1, 1.0f, flags, norm, ws, need,
                                      nullptr) == CPDP_OK);
                CHECK(g_launches == before + 2);
                CHECK(seen.base == at(0) && seen.ld == ld && seen.P == P && seen.bf16 &&
                      seen.plan == nullptr && seen.W == W && seen_mean == (flags == 1));
                const int64_t parts = cpdp::norm_parts(W, seen.chunks);
                CHECK(parts >= 1 && (parts <= seen.chunks || parts == 1));
                CHECK(parts * W * 256 < (int64_t)1 << 32 && parts * W * 8 <= need);
                CHECK(cpdp::norm_parts(1, seen.chunks) * 8 <= need);
                if (need > 0)
                    CHECK(cpdp_grad_norm(at(0), (int)W, P, ld, 0, flags, norm, ws, need - 1,
                                         nullptr) == CPDP_ERR_INVALID_ARG);
            }
        }
    // gradients of nothing need no address
    CHECK(cpdp_grad_norm(nullptr, 2, 0, 8, 0, 0, norm, ws, 16, nullptr) == CPDP_OK);

    // a plan: its own sizes, and only as it was built
    std::vector<int64_t> table(4096);
    const int64_t numel[2] = {3000, 0};
    void* params[4] = {at(3), nullptr, at(4), nullptr};
    void* mom[4] = {at(5), nullptr, at(6), nullptr};
    void* grads[4] = {at(7), nullptr, at(8), nullptr};
    cpdp_plan plan{};
    plan.table = table.data();
    CHECK(cpdp_plan_build(&plan, 4096 * 8, 2, 2, numel, params, mom, nullptr, grads, nullptr,
                          nullptr, 0) == CPDP_OK);
    const int64_t need = cpdp_grad_norm_plan_workspace(&plan);
    CHECK(need == cpdp_grad_norm_workspace(2, 3000));
    CHECK(cpdp_clip_grads_plan(&plan, 1.0f, 1, norm, ws, need, nullptr) == CPDP_OK);
    CHECK(seen.plan == table.data() && seen.n == 2 && seen.W == 2 && seen_mean);
    CHECK(cpdp_grad_norm_plan(&plan, 0, norm, ws, need, nullptr) == CPDP_OK && !seen_mean);
    const int before = g_launches;
    CHECK(cpdp_grad_norm_plan(&plan, 4, norm, ws, need, nullptr) == CPDP_ERR_INVALID_ARG);
    CHECK(cpdp_grad_norm_plan(&plan, 0, norm, ws, need - 1, nullptr) == CPDP_ERR_INVALID_ARG);
    CHECK(cpdp_grad_norm_plan(&plan, 0, nullptr, ws, need, nullptr) == CPDP_ERR_NULL);
    CHECK(cpdp_clip_grads_plan(&plan, 1.0f, 0, norm, at(2) + 8, need, nullptr) ==
          CPDP_ERR_MISALIGNED);
    CHECK(cpdp_clip_grads_plan(&plan, 0.0f, 0, norm, ws, need, nullptr) == CPDP_ERR_INVALID_ARG);
    CHECK(cpdp_clip_grads_plan(&plan, 1.0f, 0, norm, norm, need, nullptr) == CPDP_ERR_OVERLAP);
    plan.W = 1;
    CHECK(cpdp_grad_norm_plan(&plan, 0, norm, ws, need, nullptr) == CPDP_ERR_INVALID_ARG);
    CHECK(cpdp_grad_norm_plan_workspace(&plan) == 0);
    CHECK(g_launches == before);
    printf("OK\n");
    return 0;
}
