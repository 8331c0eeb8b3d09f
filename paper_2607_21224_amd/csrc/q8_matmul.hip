// Product of 8-bit rows with 8-bit weights, scaled by token and channel.
#include "q8_gemm.h"

namespace cpdp {
namespace q8 {

int64_t matmul_workspace(int64_t M, int64_t N, int64_t K) { return slices_bytes(M, N, K / kStep); }

int launch_matmul(Held a, Held b, int64_t M, int64_t N, int64_t K, Mat y, void* workspace,
                  void* stream) {
    Operands o{};
    o.a = reinterpret_cast<const char*>(a.q);
    o.b = reinterpret_cast<const char*>(b.q);
    o.lda = a.ld;
    o.ldb = b.ld;
    o.M = M;
    o.N = N;
    o.row = (int)K;
    o.parts = 1;
    Target t{};
    t.c = y.p;
    t.ldc = y.ld;
    t.bf16 = y.bf16;
    t.row_scale = a.scale;
    t.col_scale = b.scale;
    return launch_gemm<Int8>(o, t, workspace, stream);
}

}  // namespace q8
}  // namespace cpdp
