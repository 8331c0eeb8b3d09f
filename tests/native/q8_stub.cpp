// Host-only stand-ins for the launchers of the 8-bit path, so its validation
// layer (q8_api.cpp) builds with g++ under sanitizers.
#include "q8_launch.h"

int g_launches = 0;

namespace cpdp {
namespace q8 {
int launch_rows(Mat, int64_t, int64_t, Held, Mat, void*) { return ++g_launches, 0; }
int launch_values(Held, int64_t, int64_t, Mat, void*) { return ++g_launches, 0; }
int launch_norm(Mat, Mat, const void*, bool, float, int64_t, int64_t, Mat, Held, float*, Mat,
                void*) {
    return ++g_launches, 0;
}
int64_t norm_bwd_workspace(int64_t, int64_t D) { return D * 4; }
int launch_norm_bwd(Mat, Mat, Mat, const void*, bool, const float*, int64_t, int64_t, Mat, void*,
                    bool, void*, void*) {
    return ++g_launches, 0;
}
int launch_act(Act, Mat, Mat, int64_t, int64_t, Held, Mat, Held, Held, void*) {
    return ++g_launches, 0;
}
int launch_act_bwd(Act, Mat, Held, Held, int64_t, int64_t, Mat, Mat, void*) {
    return ++g_launches, 0;
}
int64_t matmul_workspace(int64_t M, int64_t, int64_t) { return M * 16; }
int launch_matmul(Held, Held, int64_t, int64_t, int64_t, Mat, void*, void*) {
    return ++g_launches, 0;
}
int64_t grad_input_workspace(int64_t T, int64_t, int64_t, bool, bool) { return T * 16; }
int launch_grad_input(Mat, Held, int64_t, int64_t, int64_t, Mat, void*, void*) {
    return ++g_launches, 0;
}
int64_t grad_weight_workspace(int64_t T, int64_t, int64_t, bool, bool) { return T * 16; }
int launch_grad_weight(Mat, Held, int64_t, int64_t, int64_t, Mat, void*, void*) {
    return ++g_launches, 0;
}
}  // namespace q8
}  // namespace cpdp
