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

// Of each token; miss, 1 - exp(-loss), may be null.
struct LossOut {
    float* loss;
    float* lse;
    float* miss;
};

int64_t xent_workspace(int64_t T, int64_t V, int64_t K);
int launch_xent(const Loss& l, const LossOut& to, void* workspace, void* stream);

// What the gradients have of each token; without miss, a target's p - 1 is exp(z - lse) - 1.
struct LossIn {
    const float* lse;
    const float* miss;
    const float* g;
};

// dx.p or dw.p may be null; the workspace is that of the types of both.
int64_t xent_bwd_workspace(int64_t T, int64_t V, int64_t K, bool dx_bf16, bool dw_bf16);
int launch_xent_bwd(const Loss& l, const LossIn& in, Mat dx, Mat dw, void* workspace,
                    void* stream);

// Whether a loss' logits are made by q8_xent_few.hip, whose blocks read 16 classes' weights
// and all tokens.  Loss in us, here and in tiles:
//   classes x channels   tokens 1             8              16             32
//   32768 x 4096         30.9   27.0          34.3   26.6    37.9   26.7    54.9   27.2
//   116960 x 3264        70.5   81.0          90.4   83.0    115    85.9    145    91.7
//   118416 x 119         16.9   22.6          18.2   22.9    20.3   23.7    41.4   23.6
//   32003 x 257          9.3    11.1          10.0   12.4    9.8    12.3    15.5   12.3
//   8192 x 1024          8.0    8.5           8.3    9.5     8.4    8.8     9.9    8.8
// (32768 x 4096 from the memory-side cache; from memory 31.9 and 36.2 for one token)
inline bool few_logits(int64_t T, int64_t K) { return T <= 16 && T * K <= 16384; }

// The loss of few tokens, and the gradients of up to 64 (q8_xent_few.hip).
int64_t few_xent_workspace(int64_t T, int64_t V);
int launch_few_xent(const Loss& l, const LossOut& to, void* workspace, void* stream);
int64_t few_xent_bwd_workspace(int64_t T, int64_t V, int64_t K, bool dx_bf16, bool dw_bf16);
int launch_few_xent_bwd(const Loss& l, const LossIn& in, Mat dx, Mat dw, void* workspace,
                        void* stream);
// The logits' gradient of classes first to first + n, in tiles (q8_xent.hip): d [T x n], fp32,
// ld a multiple of 4, and the tokens' scales, 0 for those that do not count.
int launch_few_slopes(const Loss& l, int64_t first, int64_t n, const LossIn& in, float* d,
                      int64_t ld, float* scale, void* stream);

}  // namespace q8
}  // namespace cpdp
