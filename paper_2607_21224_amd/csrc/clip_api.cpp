// C ABI of gradient norms and clipping: argument validation on the host, then the
// kernel launches on the caller's stream.  No HIP call is made before every argument
// has been checked.  The contract is documented in include/cpdp.h.
#include <cmath>
#include <cstdint>

#include "clip_launch.h"
#include "cpdp.h"
#include "cpdp_launch.h"
#include "plan_check.h"

namespace {

// Replicas at most: each is a block of a launch at least, which holds fewer than 2^32
// work items.
constexpr int kMaxRows = 1 << 23;
// (as the other entry points: byte sizes stay far from the address space's end)
constexpr int64_t kMaxElems = (int64_t)1 << 57;

struct Range {
    uintptr_t lo, hi;
};
Range range(const void* p, int64_t bytes) {
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
    return {lo, lo + (uintptr_t)bytes};
}
bool wraps(const Range& r) { return r.hi < r.lo; }
bool overlap(const Range& a, const Range& b) {
    return a.lo < a.hi && b.lo < b.hi && a.lo < b.hi && b.lo < a.hi;
}
bool aligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

int64_t chunks_of(int64_t P) {
    const int64_t each = cpdp::coords_per_block();
    return (P + each - 1) / each;
}

bool shape_ok(int W, int64_t P, int64_t ld) {
    return W >= 1 && W <= kMaxRows && P >= 0 && ld >= P && ld <= kMaxElems &&
           (int64_t)(W - 1) <= kMaxElems / (ld > 0 ? ld : 1);
}

// norm and workspace of a call over W replicas; `grads`: the gradients' range, if known
int check_results(const float* norm, const void* workspace, int64_t workspace_bytes, int W,
                  bool mean, int64_t chunks, Range grads) {
    const int64_t need = cpdp::norm_bytes(W, chunks);
    if (workspace_bytes < need) return CPDP_ERR_INVALID_ARG;
    if (norm == nullptr || workspace == nullptr) return CPDP_ERR_NULL;
    const Range n = range(norm, mean ? 4 : 4 * (int64_t)W), w = range(workspace, need);
    if (wraps(n) || wraps(w) || wraps(grads)) return CPDP_ERR_INVALID_ARG;
    if (!aligned(norm, 4) || !aligned(workspace, 16)) return CPDP_ERR_MISALIGNED;
    if (overlap(n, w) || overlap(n, grads) || overlap(w, grads)) return CPDP_ERR_OVERLAP;
    return CPDP_OK;
}

int check_flat(const void* grads, int W, int64_t P, int64_t ld, int grad_dt, unsigned flags,
               const float* norm, const void* workspace, int64_t workspace_bytes) {
    if (!shape_ok(W, P, ld) || (flags & ~(unsigned)CPDP_NORM_MEAN) != 0)
        return CPDP_ERR_INVALID_ARG;
    if (grad_dt != CPDP_F32 && grad_dt != CPDP_BF16) return CPDP_ERR_DTYPE;
    const int64_t es = grad_dt == CPDP_BF16 ? 2 : 4;
    if (P > 0 && grads == nullptr) return CPDP_ERR_NULL;
    const Range g = range(grads, P == 0 ? 0 : ((int64_t)(W - 1) * ld + P) * es);
    if (int s = check_results(norm, workspace, workspace_bytes, W, flags & CPDP_NORM_MEAN,
                              chunks_of(P), g))
        return s;
    if (P > 0 && (!aligned(grads, 16) || ld * es % 16 != 0)) return CPDP_ERR_MISALIGNED;
    return CPDP_OK;
}

int check_plan(const cpdp_plan* plan, unsigned flags, const float* norm, const void* workspace,
               int64_t workspace_bytes) {
    if (int s = cpdp::check_plan_handle(plan)) return s;
    if ((flags & ~(unsigned)CPDP_NORM_MEAN) != 0) return CPDP_ERR_INVALID_ARG;
    return check_results(norm, workspace, workspace_bytes, plan->W, flags & CPDP_NORM_MEAN,
                         plan->total_chunks, Range{0, 0});
}

bool max_norm_ok(float x) { return std::isfinite(x) && x > 0.0f; }
int hip_status(int err) { return err == 0 ? CPDP_OK : CPDP_ERR_HIP; }

cpdp::Gradients flat(const void* grads, int W, int64_t P, int64_t ld, int grad_dt) {
    return {const_cast<void*>(grads), ld, P, grad_dt == CPDP_BF16, nullptr, 0, chunks_of(P), W};
}
cpdp::Gradients of_plan(const cpdp_plan* plan) {
    return {nullptr, 0, 0, false, static_cast<const int64_t*>(plan->table), plan->n_tensors,
            plan->total_chunks, plan->W};
}

}  // namespace

extern "C" {

int64_t cpdp_grad_norm_workspace(int W, int64_t P) {
    return shape_ok(W, P, P) ? cpdp::norm_bytes(W, chunks_of(P)) : 0;
}

int cpdp_grad_norm(const void* grads, int W, int64_t P, int64_t ld, int grad_dt, unsigned flags,
                   float* norm, void* workspace, int64_t workspace_bytes, void* stream) {
    if (int s = check_flat(grads, W, P, ld, grad_dt, flags, norm, workspace, workspace_bytes))
        return s;
    return hip_status(cpdp::launch_grad_norm(flat(grads, W, P, ld, grad_dt),
                                             flags & CPDP_NORM_MEAN, norm, workspace, stream));
}

int cpdp_clip_grads(void* grads, int W, int64_t P, int64_t ld, int grad_dt, float max_norm,
                    unsigned flags, float* norm, void* workspace, int64_t workspace_bytes,
                    void* stream) {
    if (!max_norm_ok(max_norm)) return CPDP_ERR_INVALID_ARG;
    if (int s = check_flat(grads, W, P, ld, grad_dt, flags, norm, workspace, workspace_bytes))
        return s;
    return hip_status(cpdp::launch_clip_grads(flat(grads, W, P, ld, grad_dt),
                                              flags & CPDP_NORM_MEAN, max_norm, norm, workspace,
                                              stream));
}

int64_t cpdp_grad_norm_plan_workspace(const cpdp_plan* plan) {
    return cpdp::check_plan_handle(plan) == CPDP_OK
               ? cpdp::norm_bytes(plan->W, plan->total_chunks)
               : 0;
}

int cpdp_grad_norm_plan(const cpdp_plan* plan, unsigned flags, float* norm, void* workspace,
                        int64_t workspace_bytes, void* stream) {
    if (int s = check_plan(plan, flags, norm, workspace, workspace_bytes)) return s;
    return hip_status(cpdp::launch_grad_norm(of_plan(plan), flags & CPDP_NORM_MEAN, norm,
                                             workspace, stream));
}

int cpdp_clip_grads_plan(const cpdp_plan* plan, float max_norm, unsigned flags, float* norm,
                         void* workspace, int64_t workspace_bytes, void* stream) {
    if (!max_norm_ok(max_norm)) return CPDP_ERR_INVALID_ARG;
    if (int s = check_plan(plan, flags, norm, workspace, workspace_bytes)) return s;
    return hip_status(cpdp::launch_clip_grads(of_plan(plan), flags & CPDP_NORM_MEAN, max_norm,
                                              norm, workspace, stream));
}

}  // extern "C"
