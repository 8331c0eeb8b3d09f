// C ABI of the loss on 8-bit rows: argument validation on the host, then the kernel
// launches on the caller's stream.  No HIP call is made before every argument has been
// checked.  The contract is documented in include/cpdp_q8.h.
#include <cstdint>

#include "q8_check.h"
#include "q8_xent_launch.h"

namespace {

using cpdp::q8::LossIn;
using cpdp::q8::LossOut;

bool sizes_ok(int64_t T, int64_t V, int64_t K) {
    return T >= 0 && V >= 1 && T <= CPDP_Q8_MAX_T && V <= kMaxRows && K >= 1 &&
           K <= CPDP_Q8_MAX_K;
}

void inputs(Buffers& b, const int8_t* x, int64_t ldx, const float* x_scale, const int8_t* w,
            int64_t ldw, const float* w_scale, const int64_t* target, int64_t T, int64_t V,
            int64_t K) {
    b.in(x, ldx, T, K, 1);
    b.in(x_scale, T, 4, 4);
    // (without rows nothing is read)
    b.in(w, ldw, T == 0 ? 0 : V, K, 1);
    b.in(w_scale, T == 0 ? 0 : V, 4, 4);
    b.in(target, T, 8, 8);
}

// `with_miss`: the call has the argument
int loss(const int8_t* x, int64_t ldx, const float* x_scale, const int8_t* w, int64_t ldw,
         const float* w_scale, const int64_t* target, int64_t T, int64_t V, int64_t K,
         const LossOut& to, bool with_miss, void* workspace, int64_t workspace_bytes,
         void* stream) {
    if (!sizes_ok(T, V, K)) return CPDP_ERR_INVALID_ARG;
    const int64_t need = cpdp_q8_xent_workspace(T, V, K);
    if (workspace_bytes < need) return CPDP_ERR_INVALID_ARG;
    Buffers b;
    inputs(b, x, ldx, x_scale, w, ldw, w_scale, target, T, V, K);
    b.out(to.loss, T, 4, 4);
    b.out(to.lse, T, 4, 4);
    if (with_miss) b.out(to.miss, T, 4, 4);
    if (need > 0) b.out(workspace, need, 1, 16);
    if (int s = b.status()) return s;
    if (ldx > kMaxTileLd || ldw > kMaxTileLd) return CPDP_ERR_TOO_LARGE;
    if (T == 0) return CPDP_OK;
    return hip_status(cpdp::q8::launch_xent({held(x, ldx, x_scale), held(w, ldw, w_scale), target,
                                             T, V, K},
                                            to, workspace, stream));
}

int gradients(const int8_t* x, int64_t ldx, const float* x_scale, const int8_t* w, int64_t ldw,
              const float* w_scale, const int64_t* target, const LossIn& in, bool with_miss,
              int64_t T, int64_t V, int64_t K, void* dx, int64_t lddx, int dx_dt, void* dw,
              int64_t lddw, int dw_dt, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!sizes_ok(T, V, K)) return CPDP_ERR_INVALID_ARG;
    if (!is_dtype(dx_dt) || !is_dtype(dw_dt)) return CPDP_ERR_DTYPE;
    if (dx == nullptr && dw == nullptr && T > 0) return CPDP_ERR_NULL;
    const int64_t need = cpdp_q8_xent_bwd_workspace(T, V, K, dx_dt, dw_dt);
    if (workspace_bytes < need) return CPDP_ERR_INVALID_ARG;
    Buffers b;
    inputs(b, x, ldx, x_scale, w, ldw, w_scale, target, T, V, K);
    b.in(in.lse, T, 4, 4);
    if (with_miss) b.in(in.miss, T, 4, 4);
    b.in(in.g, T, 4, 4);
    if (dx != nullptr) b.out(dx, lddx, T, K, esize(dx_dt == CPDP_BF16));
    if (dw != nullptr) b.out(dw, lddw, V, K, esize(dw_dt == CPDP_BF16));
    if (need > 0) b.out(workspace, need, 1, 16);
    if (int s = b.status()) return s;
    if (ldx > kMaxTileLd || ldw > kMaxTileLd) return CPDP_ERR_TOO_LARGE;
    if (T == 0 && dw == nullptr) return CPDP_OK;
    return hip_status(cpdp::q8::launch_xent_bwd({held(x, ldx, x_scale), held(w, ldw, w_scale),
                                                 target, T, V, K},
                                                in, mat(dx, lddx, dx_dt), mat(dw, lddw, dw_dt),
                                                workspace, stream));
}

}  // namespace

extern "C" {

int64_t cpdp_q8_xent_workspace(int64_t T, int64_t V, int64_t K) {
    return sizes_ok(T, V, K) && T > 0 ? cpdp::q8::xent_workspace(T, V, K) : 0;
}

int cpdp_q8_xent(const int8_t* x, int64_t ldx, const float* x_scale, const int8_t* w, int64_t ldw,
                 const float* w_scale, const int64_t* target, int64_t T, int64_t V, int64_t K,
                 float* loss_out, float* lse, void* workspace, int64_t workspace_bytes,
                 void* stream) {
    return loss(x, ldx, x_scale, w, ldw, w_scale, target, T, V, K, {loss_out, lse, nullptr}, false,
                workspace, workspace_bytes, stream);
}

int cpdp_q8_xent_miss(const int8_t* x, int64_t ldx, const float* x_scale, const int8_t* w,
                      int64_t ldw, const float* w_scale, const int64_t* target, int64_t T,
                      int64_t V, int64_t K, float* loss_out, float* lse, float* miss,
                      void* workspace, int64_t workspace_bytes, void* stream) {
    return loss(x, ldx, x_scale, w, ldw, w_scale, target, T, V, K, {loss_out, lse, miss}, true,
                workspace, workspace_bytes, stream);
}

int64_t cpdp_q8_xent_bwd_workspace(int64_t T, int64_t V, int64_t K, int dx_dt, int dw_dt) {
    return sizes_ok(T, V, K) && T > 0 && is_dtype(dx_dt) && is_dtype(dw_dt)
               ? cpdp::q8::xent_bwd_workspace(T, V, K, dx_dt == CPDP_BF16, dw_dt == CPDP_BF16)
               : 0;
}

int cpdp_q8_xent_bwd(const int8_t* x, int64_t ldx, const float* x_scale, const int8_t* w,
                     int64_t ldw, const float* w_scale, const int64_t* target, const float* lse,
                     const float* g, int64_t T, int64_t V, int64_t K, void* dx, int64_t lddx,
                     int dx_dt, void* dw, int64_t lddw, int dw_dt, void* workspace,
                     int64_t workspace_bytes, void* stream) {
    return gradients(x, ldx, x_scale, w, ldw, w_scale, target, {lse, nullptr, g}, false, T, V, K,
                     dx, lddx, dx_dt, dw, lddw, dw_dt, workspace, workspace_bytes, stream);
}

int cpdp_q8_xent_miss_bwd(const int8_t* x, int64_t ldx, const float* x_scale, const int8_t* w,
                          int64_t ldw, const float* w_scale, const int64_t* target,
                          const float* lse, const float* miss, const float* g, int64_t T,
                          int64_t V, int64_t K, void* dx, int64_t lddx, int dx_dt, void* dw,
                          int64_t lddw, int dw_dt, void* workspace, int64_t workspace_bytes,
                          void* stream) {
    return gradients(x, ldx, x_scale, w, ldw, w_scale, target, {lse, miss, g}, true, T, V, K, dx,
                     lddx, dx_dt, dw, lddw, dw_dt, workspace, workspace_bytes, stream);
}

}  // extern "C"
