// Product of 8-bit rows with 8-bit weights, scaled by token and channel.
//
// From 65 tokens on a tile kernel takes it (q8_gemm.h).  With fewer, the weights
// are what is read, once, and nothing is worth staging in LDS: the few kernel.
#include "q8_few.h"

namespace cpdp {
namespace q8 {
namespace {

// y [M x N] for M <= 16 MT tokens (see few_sums).
template <int MT>
__global__ __launch_bounds__(1024) void few_kernel(const int8_t* a, int64_t lda, const int8_t* b,
                                                   int64_t ldb, int M, int64_t N, int K,
                                                   Target t) {
    __shared__ FewSums<MT> sums;
    const int waves = blockDim.x >> 6;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    few_sums<MT, MT == 1 ? 4 : 2>(a, lda, b, ldb, M, N, K, n0, sums);
    // element e: token e / 16, channel e % 16
    for (int e = threadIdx.x; e < MT * 256; e += blockDim.x) {
        const int m = e / 16;
        const int64_t n = n0 + e % 16;
        if (m >= M || n >= N) continue;
        const float v = (float)few_sum<MT>(sums, e, waves) * t.row_scale[m] * t.col_scale[n];
        if (t.bf16) narrow(v, static_cast<uint16_t*>(t.c) + m * t.ldc + n);
        else static_cast<float*>(t.c)[m * t.ldc + n] = v;
    }
}

constexpr int64_t kFewTokens = 64;

template <int MT>
int launch_few(Held a, Held b, int64_t M, int64_t N, int64_t K, const Target& t, void* stream) {
    const int waves = few_waves(K);
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
