// Products of few tokens' 8-bit rows with 8-bit weights: the weights are what is read, once.
#pragma once

#include "q8_gemm.h"

namespace cpdp {
namespace q8 {
namespace {

// For M <= 16 MT tokens, U steps of a wavefront on their way together.  A block takes 16
// channels, from n0 on; its wavefronts take the steps of K in turn, each lane 32
// consecutive bytes of a weight row, so a step reads 128 bytes of 16 rows.  Those go to the matrix cores as they are: a
// sum does not depend on which of its terms an instruction takes together, as
// long as the tokens' bytes, read from L2, are dealt alike.  The wavefronts'
// sums meet in LDS, as whole numbers, so their order does not matter: `sums` [wavefront]
// has element e, of token e / 16 and channel e % 16, at [e / 4][e % 4].
template <int MT>
using FewSums = i32x4[16][MT * 64];
template <int MT, int U>
__device__ __forceinline__ void few_sums(const int8_t* a, int64_t lda, const int8_t* b,
                                         int64_t ldb, int M, int64_t N, int K, int64_t n0,
                                         FewSums<MT>& sums) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const char* bp = reinterpret_cast<const char*>(b) + (n0 + r < N ? n0 + r : N - 1) * ldb + g * 32;
    const char* ap[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
        ap[i] = reinterpret_cast<const char*>(a) + (i * 16 + r < M ? i * 16 + r : M - 1) * lda +
                g * 32;
    i32x4 acc[MT] = {};
    const int steps = K / kStep;
    for (int k = wave; k < steps; k += waves * U) {
        u32x4 w[U][2], x[U][MT][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (k + u * waves >= steps) break;
            const int64_t at = (int64_t)(k + u * waves) * kStep;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                w[u][h] = *reinterpret_cast<const u32x4*>(bp + at + h * 16);
#pragma unroll
                for (int i = 0; i < MT; ++i)
                    x[u][i][h] = *reinterpret_cast<const u32x4*>(ap[i] + at + h * 16);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (k + u * waves >= steps) break;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < MT; ++i) acc[i] = Int8::mfma(w[u][h], x[u][i][h], acc[i]);
        }
    }
    if (K % kStep != 0 && wave == steps % waves) {
        const int64_t at = (int64_t)steps * kStep;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int n = K - (int)at - g * 32 - h * 16, before = (int)at + g * 32 + h * 16;
            const u32x4 w = load_tail(bp + at + h * 16, n, before);
#pragma unroll
            for (int i = 0; i < MT; ++i)
                acc[i] = Int8::mfma(w, load_tail(ap[i] + at + h * 16, n, before), acc[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) sums[wave][i * 64 + r * 4 + g] = acc[i];
    __syncthreads();
}
// an element's sum over the wavefronts
template <int MT>
__device__ __forceinline__ int32_t few_sum(const FewSums<MT>& sums, int e, int waves) {
    int32_t s = 0;
    for (int w = 0; w < waves; ++w) s += sums[w][e / 4][e % 4];
    return s;
}
// wavefronts of a block: each takes at least two steps where there are enough
inline int few_waves(int64_t K) {
    const int64_t steps = up(K, kStep);
    return steps >= 32 ? 16 : steps >= 16 ? 8 : steps >= 8 ? 4 : 2;
}

}  // namespace
}  // namespace q8
}  // namespace cpdp
