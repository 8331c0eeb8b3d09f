// Internal interface between the C ABI of gradient clipping (clip_api.cpp:
// validation) and its gfx950 kernels (kernels_clip.hip).  Plain C++ types only, so
// the validation layer builds with any host compiler.  Launchers assume validated
// arguments and return 0 or the HIP error code of a failed launch.
#pragma once
#include <stdint.h>

#include "cpdp.h"

namespace cpdp {

// The gradients of W replicas: flat rows (plan == nullptr), or the gradient tensors
// of a multi-tensor plan's table (fp32).
struct Gradients {
    void* base;
    int64_t ld, P;
    bool bf16;
    const int64_t* plan;
    int n;           // tensors
    int64_t chunks;  // of a replica, coords_per_block() coordinates each at most
    int W;
};

// Parts that each of `rows` rows of `chunks` chunks is taken in, one block each; a
// workspace holds the fp64 sum of each part.  2048 blocks of 256 threads are all that
// the card holds at once.
inline int64_t norm_parts(int64_t rows, int64_t chunks) {
    const int64_t most = rows < 2048 ? 2048 / rows : 1;
    return chunks < 1 ? 1 : chunks < most ? chunks : most;
}

inline int64_t norm_bytes(int64_t W, int64_t chunks) {
    // (the mean is one row)
    const int64_t rows = W * norm_parts(W, chunks), mean = norm_parts(1, chunks);
    return 8 * (rows > mean ? rows : mean);
}

int launch_grad_norm(const Gradients& g, bool mean, float* norm, void* workspace, void* stream);
int launch_clip_grads(const Gradients& g, bool mean, float max_norm, float* norm, void* workspace,
                      void* stream);

}  // namespace cpdp
