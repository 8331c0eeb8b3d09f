// Product of 8-bit rows with 8-bit weights, scaled by token and channel.
//
// From 65 tokens on a tile kernel takes it (q8_gemm.h).  With fewer, the weights
// are what is read, once, and nothing is worth staging in LDS: the few kernel.
#include "q8_gemm.h"

namespace cpdp {
namespace q8 {
namespace {

// y [M x N] for M <= 16 MT tokens.  A block takes 16 channels; its wavefronts take
// the steps of K in turn, each lane 32 consecutive bytes of a weight row, so a
// step reads 128 bytes of 16 rows.  Those go to the matrix cores as they are: a
// sum does not depend on which of its terms an instruction takes together, as
// long as the tokens' bytes, read from L2, are dealt alike.  The wavefronts'
// sums meet in LDS, as whole numbers, so their order does not matter.
template <int MT>
__global__ __launch_bounds__(1024) void few_kernel(const int8_t* a, int64_t lda, const int8_t* b,
                                                   int64_t ldb, int M, int64_t N, int K,
                                                   Target t) {
    __shared__ i32x4 sums[16][MT * 64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const char* bp = reinterpret_cast<const char*>(b) + (n0 + r < N ? n0 + r : N - 1) * ldb + g * 32;
    const char* ap[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
        ap[i] = reinterpret_cast<const char*>(a) + (i * 16 + r < M ? i * 16 + r : M - 1) * lda +
                g * 32;
    i32x4 acc[MT] = {};
    // U steps are on their way together
    constexpr int U = MT == 1 ? 4 : 2;
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
    // element e: token e / 16, channel e % 16
    for (int e = threadIdx.x; e < MT * 256; e += blockDim.x) {
        const int m = e / 16;
        const int64_t n = n0 + e % 16;
        if (m >= M || n >= N) continue;
        int32_t s = 0;
        for (int w = 0; w < waves; ++w) s += sums[w][e / 4][e % 4];
        const float v = (float)s * t.row_scale[m] * t.col_scale[n];
        if (t.bf16) narrow(v, static_cast<uint16_t*>(t.c) + m * t.ldc + n);
        else static_cast<float*>(t.c)[m * t.ldc + n] = v;
    }
}

constexpr int64_t kFewTokens = 64;

template <int MT>
int launch_few(Held a, Held b, int64_t M, int64_t N, int64_t K, const Target& t, void* stream) {
    // a wavefront takes at least two steps where there are enough
    const int64_t steps = up(K, kStep);
    const int waves = steps >= 32 ? 16 : steps >= 16 ? 8 : steps >= 8 ? 4 : 2;
    // rows of C in one launch: fewer than 2^32 work items
    const int64_t most = (int64_t)1 << 25;
    for (int64_t n = 0; n < N; n += most) {
        const int64_t now = N - n < most ? N - n : most;
        Target part = t;
        part.c = static_cast<char*>(t.c) + n * (t.bf16 ? 2 : 4);
        part.col_scale = t.col_scale + n;
        if (int e = launch(few_kernel<MT>, dim3((uint32_t)up(now, 16)), 64 * waves, stream, a.q,
                           a.ld, b.q + n * b.ld, b.ld, M, now, K, part))
            return e;
    }
    return 0;
}

}  // namespace

int64_t matmul_workspace(int64_t M, int64_t N, int64_t K) {
    return M <= kFewTokens ? 0 : slices_bytes(M, N, shape_of(M, N, up(K, kStep)));
}

int launch_matmul(Held a, Held b, int64_t M, int64_t N, int64_t K, Mat y, void* workspace,
                  void* stream) {
    Target t{};
    t.c = y.p;
    t.ldc = y.ld;
    t.bf16 = y.bf16;
    t.row_scale = a.scale;
    t.col_scale = b.scale;
    if (M <= 16) return launch_few<1>(a, b, M, N, K, t, stream);
    if (M <= 32) return launch_few<2>(a, b, M, N, K, t, stream);
    if (M <= kFewTokens) return launch_few<4>(a, b, M, N, K, t, stream);
    Operands o{};
    o.a = reinterpret_cast<const char*>(a.q);
    o.b = reinterpret_cast<const char*>(b.q);
    o.lda = a.ld;
    o.ldb = b.ld;
    o.M = M;
    o.N = N;
    o.row = (int)K;
    return launch_gemm<Int8>(o, t, workspace, stream);
}

}  // namespace q8
}  // namespace cpdp
