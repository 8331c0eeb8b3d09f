// C ABI of the 8-bit activation path: argument validation on the host, then
// the kernel launches on the caller's stream.  No HIP call is made before every
// argument has been checked.  The contract is documented in
// include/cpdp_q8.h.
#include "cpdp_q8.h"

#include <cmath>
#include <cstdint>

#include "q8_check.h"

extern "C" {

int cpdp_q8_rows(const void* x, int64_t ldx, int x_dt, int64_t T, int64_t D, int8_t* q,
                 int64_t ldq, float* scale, void* y, int64_t ldy, int y_dt, void* stream) {
    if (!rows_ok(T, D)) return CPDP_ERR_INVALID_ARG;
    if (!is_dtype(x_dt) || (y != nullptr && !is_dtype(y_dt))) return CPDP_ERR_DTYPE;
    Buffers b;
    b.in(x, ldx, T, D, esize(x_dt == CPDP_BF16));
    b.out(q, ldq, T, D, 1);
    b.out(scale, T, 4, 4);
    if (y != nullptr) b.out(y, ldy, T, D, esize(y_dt == CPDP_BF16));
    if (int s = b.status()) return s;
    if (T == 0) return CPDP_OK;
    return hip_status(cpdp::q8::launch_rows(mat(x, ldx, x_dt), T, D, held(q, ldq, scale),
                                            mat(y, ldy, y_dt), stream));
}

int cpdp_q8_values(const int8_t* q, int64_t ldq, const float* scale, int64_t T, int64_t D, void* y,
                   int64_t ldy, int y_dt, void* stream) {
    if (!rows_ok(T, D)) return CPDP_ERR_INVALID_ARG;
    if (!is_dtype(y_dt)) return CPDP_ERR_DTYPE;
    Buffers b;
    b.in(q, ldq, T, D, 1);
    b.in(scale, T, 4, 4);
    b.out(y, ldy, T, D, esize(y_dt == CPDP_BF16));
    if (int s = b.status()) return s;
    if (T == 0) return CPDP_OK;
    return hip_status(
        cpdp::q8::launch_values(held(q, ldq, scale), T, D, mat(y, ldy, y_dt), stream));
}

int cpdp_q8_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, int act_dt,
                 const void* w, int w_dt, float eps, int64_t T, int64_t D, void* h, int64_t ldh,
                 int8_t* q, int64_t ldq, float* scale, float* rstd, void* y, int64_t ldy, int y_dt,
                 void* stream) {
    if (!rows_ok(T, D)) return CPDP_ERR_INVALID_ARG;
    if (!(std::isfinite(eps) && eps >= 0.0f)) return CPDP_ERR_INVALID_ARG;
    if (!is_dtype(act_dt) || !is_dtype(w_dt) || (y != nullptr && !is_dtype(y_dt)))
        return CPDP_ERR_DTYPE;
    if ((residual == nullptr) != (h == nullptr)) return CPDP_ERR_NULL;
    const int64_t e = esize(act_dt == CPDP_BF16);
    Buffers b;
    b.in(x, ldx, T, D, e);
    const int bx = b.last();
    b.in(w, D, esize(w_dt == CPDP_BF16), 16);
    b.out(q, ldq, T, D, 1);
    b.out(scale, T, 4, 4);
    if (rstd != nullptr) b.out(rstd, T, 4, 4);
    if (y != nullptr) b.out(y, ldy, T, D, esize(y_dt == CPDP_BF16));
    if (residual != nullptr) {
        b.in(residual, ldr, T, D, e);
        const int br = b.last();
        b.out(h, ldh, T, D, e);
        b.may_be(bx);
        b.may_be(br);
    }
    if (int s = b.status()) return s;
    if (T == 0) return CPDP_OK;
    return hip_status(cpdp::q8::launch_norm(
        mat(x, ldx, act_dt), mat(residual, ldr, act_dt), w, w_dt == CPDP_BF16, eps, T, D,
        mat(h, ldh, act_dt), held(q, ldq, scale), rstd, mat(y, ldy, y_dt), stream));
}

int64_t cpdp_q8_norm_bwd_workspace(int64_t T, int64_t D) {
    return rows_ok(T, D) ? cpdp::q8::norm_bwd_workspace(T, D) : 0;
}

int cpdp_q8_norm_bwd(const void* dy, int64_t lddy, const void* h, int64_t ldh, const void* dres,
                     int64_t lddres, int act_dt, const void* w, int w_dt, const float* rstd,
                     int64_t T, int64_t D, void* dx, int64_t lddx, void* dw, int dw_dt,
                     void* workspace, int64_t workspace_bytes, void* stream) {
    if (!rows_ok(T, D)) return CPDP_ERR_INVALID_ARG;
    if (!is_dtype(act_dt) || !is_dtype(w_dt) || !is_dtype(dw_dt)) return CPDP_ERR_DTYPE;
    const int64_t e = esize(act_dt == CPDP_BF16), need = cpdp::q8::norm_bwd_workspace(T, D);
    if (workspace_bytes < need) return CPDP_ERR_INVALID_ARG;
    Buffers b;
    b.in(dy, lddy, T, D, e);
    b.in(h, ldh, T, D, e);
    if (dres != nullptr) b.in(dres, lddres, T, D, e);
    b.in(w, D, esize(w_dt == CPDP_BF16), 16);
    b.in(rstd, T, 4, 4);
    b.out(dx, lddx, T, D, e);
    b.out(dw, D, esize(dw_dt == CPDP_BF16), 16);
    if (need > 0) b.out(workspace, need, 1, 16);
    if (int s = b.status()) return s;
    return hip_status(cpdp::q8::launch_norm_bwd(
        mat(dy, lddy, act_dt), mat(h, ldh, act_dt), mat(dres, lddres, act_dt), w,
        w_dt == CPDP_BF16, rstd, T, D, mat(dx, lddx, act_dt), dw, dw_dt == CPDP_BF16, workspace,
        stream));
}

int64_t cpdp_q8_matmul_workspace(int64_t M, int64_t N, int64_t K) {
    if (M < 1 || N < 1 || M > kMaxRows || N > kMaxRows || K < 1 || K > CPDP_Q8_MAX_K) return 0;
    return cpdp::q8::matmul_workspace(M, N, K);
}

int cpdp_q8_matmul(const int8_t* a, int64_t lda, const float* a_scale, const int8_t* b,
                   int64_t ldb, const float* b_scale, int64_t M, int64_t N, int64_t K, void* y,
                   int64_t ldy, int y_dt, void* workspace, int64_t workspace_bytes,
                   void* stream) {
    if (M < 0 || N < 0 || M > kMaxRows || N > kMaxRows || K < 1 || K > CPDP_Q8_MAX_K)
        return CPDP_ERR_INVALID_ARG;
    if (!is_dtype(y_dt)) return CPDP_ERR_DTYPE;
    const int64_t need = cpdp_q8_matmul_workspace(M, N, K);
    if (workspace_bytes < need) return CPDP_ERR_INVALID_ARG;
    Buffers s;
    s.in(a, lda, M, K, 1);
    s.in(a_scale, M, 4, 4);
    s.in(b, ldb, N, K, 1);
    s.in(b_scale, N, 4, 4);
    s.out(y, ldy, M, N, esize(y_dt == CPDP_BF16));
    if (need > 0) s.out(workspace, need, 1, 16);
    if (int e = s.status()) return e;
    if (lda > kMaxTileLd || ldb > kMaxTileLd) return CPDP_ERR_TOO_LARGE;
    if (M == 0 || N == 0) return CPDP_OK;
    return hip_status(cpdp::q8::launch_matmul(held(a, lda, a_scale), held(b, ldb, b_scale), M, N,
                                              K, mat(y, ldy, y_dt), workspace, stream));
}

int cpdp_q8_act(int kind, const void* g, const void* u, int64_t ldg, int act_dt, int64_t T,
                int64_t F, int8_t* q, int64_t ldq, float* scale, void* y, int64_t ldy, int y_dt,
                int8_t* cg, float* cg_scale, int8_t* cu, float* cu_scale, int64_t ldc,
                void* stream) {
    if (kind != CPDP_ACT_GELU && kind != CPDP_ACT_SWIGLU) return CPDP_ERR_INVALID_ARG;
    if (!rows_ok(T, F)) return CPDP_ERR_INVALID_ARG;
    if (!is_dtype(act_dt) || (y != nullptr && !is_dtype(y_dt))) return CPDP_ERR_DTYPE;
    const bool gated = kind == CPDP_ACT_SWIGLU;
    const bool keep = cg != nullptr || cg_scale != nullptr ||
                      (gated && (cu != nullptr || cu_scale != nullptr));
    const int64_t e = esize(act_dt == CPDP_BF16);
    Buffers b;
    b.in(g, ldg, T, F, e);
    if (gated) b.in(u, ldg, T, F, e);
    b.out(q, ldq, T, F, 1);
    b.out(scale, T, 4, 4);
    if (y != nullptr) b.out(y, ldy, T, F, esize(y_dt == CPDP_BF16));
    if (keep) {
        b.out(cg, ldc, T, F, 1);
        b.out(cg_scale, T, 4, 4);
        if (gated) {
            b.out(cu, ldc, T, F, 1);
            b.out(cu_scale, T, 4, 4);
        }
    }
    if (int s = b.status()) return s;
    if (T == 0) return CPDP_OK;
    return hip_status(cpdp::q8::launch_act(
        gated ? Act::SWIGLU : Act::GELU, mat(g, ldg, act_dt), mat(gated ? u : nullptr, ldg, act_dt),
        T, F, held(q, ldq, scale), mat(y, ldy, y_dt), held(keep ? cg : nullptr, ldc, cg_scale),
        held(keep && gated ? cu : nullptr, ldc, cu_scale), stream));
}

int cpdp_q8_act_bwd(int kind, const void* da, int64_t ldda, int act_dt, const int8_t* cg,
                    const float* cg_scale, const int8_t* cu, const float* cu_scale, int64_t ldc,
                    int64_t T, int64_t F, void* dg, void* du, int64_t lddg, void* stream) {
    if (kind != CPDP_ACT_GELU && kind != CPDP_ACT_SWIGLU) return CPDP_ERR_INVALID_ARG;
    if (!rows_ok(T, F)) return CPDP_ERR_INVALID_ARG;
    if (!is_dtype(act_dt)) return CPDP_ERR_DTYPE;
    const bool gated = kind == CPDP_ACT_SWIGLU;
    const int64_t e = esize(act_dt == CPDP_BF16);
    Buffers b;
    b.in(da, ldda, T, F, e);
    b.in(cg, ldc, T, F, 1);
    b.in(cg_scale, T, 4, 4);
    b.out(dg, lddg, T, F, e);
    if (gated) {
        b.in(cu, ldc, T, F, 1);
        b.in(cu_scale, T, 4, 4);
        b.out(du, lddg, T, F, e);
    }
    if (int s = b.status()) return s;
    if (T == 0) return CPDP_OK;
    return hip_status(cpdp::q8::launch_act_bwd(
        gated ? Act::SWIGLU : Act::GELU, mat(da, ldda, act_dt), held(cg, ldc, cg_scale),
        held(gated ? cu : nullptr, ldc, cu_scale), T, F, mat(dg, lddg, act_dt),
        mat(gated ? du : nullptr, lddg, act_dt), stream));
}

// Sizes of the two gradients: the reduced size R is rounded up to whole tiles in
// the workspace, whose rows a product then reads.
static bool grad_sizes_ok(int64_t T, int64_t N, int64_t K) {
    return T >= 0 && N >= 0 && K >= 1 && T <= kMaxRows && N <= kMaxRows && K <= kMaxRows;
}
static bool grad_too_large(int64_t reduced) { return reduced > kMaxTileLd / 2 - 64; }

int64_t cpdp_q8_grad_input_workspace(int64_t T, int64_t N, int64_t K, int dy_dt, int out_dt) {
    if (!grad_sizes_ok(T, N, K) || T == 0 || N == 0 || !is_dtype(dy_dt) || !is_dtype(out_dt) ||
        grad_too_large(N))
        return 0;
    return cpdp::q8::grad_input_workspace(T, N, K, dy_dt == CPDP_BF16, out_dt == CPDP_BF16);
}

int cpdp_q8_grad_input(const void* dy, int64_t lddy, int dy_dt, const int8_t* b, int64_t ldb,
                       const float* b_scale, int64_t T, int64_t N, int64_t K, void* dx,
                       int64_t lddx, int out_dt, void* workspace, int64_t workspace_bytes,
                       void* stream) {
    if (!grad_sizes_ok(T, N, K)) return CPDP_ERR_INVALID_ARG;
    if (!is_dtype(dy_dt) || !is_dtype(out_dt)) return CPDP_ERR_DTYPE;
    const int64_t need = cpdp_q8_grad_input_workspace(T, N, K, dy_dt, out_dt);
    if (workspace_bytes < need) return CPDP_ERR_INVALID_ARG;
    Buffers s;
    if (N > 0) {
        s.in(dy, lddy, T, N, esize(dy_dt == CPDP_BF16));
        s.in(b, ldb, N, K, 1);
        s.in(b_scale, N, 4, 4);
    }
    s.out(dx, lddx, T, K, esize(out_dt == CPDP_BF16));
    if (need > 0) s.out(workspace, need, 1, 16);
    if (int e = s.status()) return e;
    if (grad_too_large(N) || lddy > kMaxTileLd / 2 || ldb > kMaxTileLd) return CPDP_ERR_TOO_LARGE;
    if (T == 0) return CPDP_OK;
    return hip_status(cpdp::q8::launch_grad_input(mat(dy, lddy, dy_dt), held(b, ldb, b_scale), T, N,
                                                  K, mat(dx, lddx, out_dt), workspace, stream));
}

int64_t cpdp_q8_grad_weight_workspace(int64_t T, int64_t N, int64_t K, int dy_dt, int out_dt) {
    if (!grad_sizes_ok(T, N, K) || T == 0 || N == 0 || !is_dtype(dy_dt) || !is_dtype(out_dt) ||
        grad_too_large(T))
        return 0;
    return cpdp::q8::grad_weight_workspace(T, N, K, dy_dt == CPDP_BF16, out_dt == CPDP_BF16);
}

int cpdp_q8_grad_weight(const void* dy, int64_t lddy, int dy_dt, const int8_t* a, int64_t lda,
                        const float* a_scale, int64_t T, int64_t N, int64_t K, void* dw,
                        int64_t lddw, int out_dt, void* workspace, int64_t workspace_bytes,
                        void* stream) {
    if (!grad_sizes_ok(T, N, K)) return CPDP_ERR_INVALID_ARG;
    if (!is_dtype(dy_dt) || !is_dtype(out_dt)) return CPDP_ERR_DTYPE;
    const int64_t need = cpdp_q8_grad_weight_workspace(T, N, K, dy_dt, out_dt);
    if (workspace_bytes < need) return CPDP_ERR_INVALID_ARG;
    Buffers s;
    if (T > 0) {
        s.in(dy, lddy, T, N, esize(dy_dt == CPDP_BF16));
        s.in(a, lda, T, K, 1);
        s.in(a_scale, T, 4, 4);
    }
    s.out(dw, lddw, N, K, esize(out_dt == CPDP_BF16));
    if (need > 0) s.out(workspace, need, 1, 16);
    if (int e = s.status()) return e;
    if (grad_too_large(T) || lddy > kMaxTileLd / 2 || lda > kMaxTileLd) return CPDP_ERR_TOO_LARGE;
    if (N == 0) return CPDP_OK;
    return hip_status(cpdp::q8::launch_grad_weight(mat(dy, lddy, dy_dt), held(a, lda, a_scale), T,
                                                   N, K, mat(dw, lddw, out_dt), workspace,
                                                   stream));
}

}  // extern "C"
