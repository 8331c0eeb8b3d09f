// Internal interface between the C ABI of the 8-bit activation path
// (q8_api.cpp: validation) and its gfx950 kernels (q8_*.hip).  Plain C++ types
// only, so the validation layer builds with any host compiler.  Launchers assume
// validated arguments and return 0 or the HIP error code of a failed launch.
#pragma once
#include <stdint.h>

namespace cpdp {
namespace q8 {

// A matrix argument: base, row stride in elements, and whether it is bf16 (else
// fp32).  base == nullptr: absent.
struct Mat {
    void* p;
    int64_t ld;
    bool bf16;
};

// 8-bit rows: base, row stride in bytes, one scale a row.
struct Held {
    int8_t* q;
    int64_t ld;
    float* scale;
};

enum class Act { GELU, SWIGLU };

int launch_rows(Mat x, int64_t T, int64_t D, Held out, Mat y, void* stream);
int launch_values(Held in, int64_t T, int64_t D, Mat y, void* stream);

int launch_norm(Mat x, Mat residual, const void* w, bool w_bf16, float eps, int64_t T, int64_t D,
                Mat h, Held out, float* rstd, Mat y, void* stream);

int64_t norm_bwd_workspace(int64_t T, int64_t D);
int launch_norm_bwd(Mat dy, Mat h, Mat dres, const void* w, bool w_bf16, const float* rstd,
                    int64_t T, int64_t D, Mat dx, void* dw, bool dw_bf16, void* workspace,
                    void* stream);

int launch_act(Act kind, Mat g, Mat u, int64_t T, int64_t F, Held out, Mat y, Held cg, Held cu,
               void* stream);
int launch_act_bwd(Act kind, Mat da, Held cg, Held cu, int64_t T, int64_t F, Mat dg, Mat du,
                   void* stream);

int64_t matmul_workspace(int64_t M, int64_t N, int64_t K);
int launch_matmul(Held a, Held b, int64_t M, int64_t N, int64_t K, Mat y, void* workspace,
                  void* stream);

int64_t grad_input_workspace(int64_t T, int64_t N, int64_t K, bool dy_bf16, bool out_bf16);
int launch_grad_input(Mat dy, Held b, int64_t T, int64_t N, int64_t K, Mat dx, void* workspace,
                      void* stream);
int64_t grad_weight_workspace(int64_t T, int64_t N, int64_t K, bool dy_bf16, bool out_bf16);
int launch_grad_weight(Mat dy, Held a, int64_t T, int64_t N, int64_t K, Mat dw, void* workspace,
                       void* stream);

}  // namespace q8
}  // namespace cpdp
