// Internal interface between the C ABI of the loss (q8_xent_api.cpp: validation) and
// its gfx950 kernels (q8_xent*.hip), as q8_launch.h is for the other operators.
#pragma once
#include "q8_launch.h"

namespace cpdp {
namespace q8 {

// The rows and weights of a loss, and its targets.
struct Loss {
    Held x, w;
    const int64_t* target;
    int64_t T, V, K;
};

int64_t xent_workspace(int64_t T, int64_t V, int64_t K);
int launch_xent(const Loss& l, float* loss, float* lse, void* workspace, void* stream);

// dx.p or dw.p may be null; the workspace is that of the types of both.
int64_t xent_bwd_workspace(int64_t T, int64_t V, int64_t K, bool dx_bf16, bool dw_bf16);
int launch_xent_bwd(const Loss& l, const float* lse, const float* g, Mat dx, Mat dw,
                    void* workspace, void* stream);

// The same for up to 64 tokens (q8_xent_few.hip).
int64_t few_xent_workspace(int64_t T, int64_t V, int64_t K);
int launch_few_xent(const Loss& l, float* loss, float* lse, void* workspace, void* stream);
int64_t few_xent_bwd_workspace(int64_t T, int64_t V, int64_t K, bool dx_bf16, bool dw_bf16);
int launch_few_xent_bwd(const Loss& l, const float* lse, const float* g, Mat dx, Mat dw,
                        void* workspace, void* stream);

}  // namespace q8
}  // namespace cpdp
