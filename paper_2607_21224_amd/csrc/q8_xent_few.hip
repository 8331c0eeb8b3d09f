// The loss of few tokens (see few_logits), and the gradients of up to 64.  What they cost is
// reading the weights: once for the loss, and for the gradients once for the logits'
// gradient, which is small and kept in fp32, and once more for dx.
#include "q8_few.h"
#include "q8_xent_stats.h"

namespace cpdp {
namespace q8 {
namespace {

constexpr int kClasses = 16;  // of a block (see few_sums)

// A block's classes: each token's largest logit and sum of exp's, part [token][block], and
// the target's logit of the tokens that have it here.
__global__ __launch_bounds__(1024, 8) void xent_few_stats_kernel(Held x, Held w,
                                                                 const int64_t* target, int M,
                                                                 int64_t V, int K, int64_t first,
                                                                 int64_t blocks, Stats* part,
                                                                 float* hit) {
    __shared__ FewSums<1> sums;
    const int waves = blockDim.x >> 6;
    const int64_t block = first + blockIdx.x, n0 = block * kClasses;
    few_sums<1, 2>(x.q, x.ld, w.q, w.ld, M, V, K, n0, sums);
    const int64_t n = n0 + threadIdx.x % kClasses, from = n < V ? n : V - 1;
    const float ws = w.scale[from];
    for (int e = threadIdx.x; e < 256; e += blockDim.x) {
        const int m = e / kClasses, at = m < M ? m : M - 1;
        float z = (float)few_sum<1>(sums, e, waves) * x.scale[at] * ws;
        if (n >= V) z = -__builtin_inff();
        if (m < M && n < V && n == target[m]) hit[m] = z;
        Stats s = {z, exp_of(z - pivot(z))};
#pragma unroll
        for (int off = 1; off < kClasses; off <<= 1)
            s = join(s, {__shfl_xor(s.top, off), __shfl_xor(s.sum, off)});
        if (m < M && threadIdx.x % kClasses == 0) part[m * blocks + block] = s;
    }
}

// A block joins a token's parts.
__global__ __launch_bounds__(1024) void xent_few_join_kernel(const Stats* part, int64_t blocks,
                                                             const float* hit, int64_t V,
                                                             const int64_t* target, LossOut to) {
    __shared__ Stats words[16];
    const int64_t t = blockIdx.x;
    Stats s = {-__builtin_inff(), 0.0f};
    for (int64_t j = threadIdx.x; j < blocks; j += 1024) s = join(s, part[t * blocks + j]);
#pragma unroll
    for (int off = 1; off < 64; off <<= 1)
        s = join(s, {__shfl_xor(s.top, off), __shfl_xor(s.sum, off)});
    if (threadIdx.x % 64 == 0) words[threadIdx.x / 64] = s;
    __syncthreads();
    if (threadIdx.x != 0) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) s = join(s, words[i]);
    write_loss(s, hit[t], target[t], V, to, t);
}

// The logits' gradient, d [M x N] for N classes from `first` on, and the tokens' scales
// with 0 for those that do not count.
__global__ __launch_bounds__(1024) void xent_few_slopes_kernel(Held x, Held w,
                                                               const int64_t* target, int M,
                                                               int64_t N, int K, int64_t first,
                                                               int64_t V, LossIn in, float* d,
                                                               int64_t ld, float* scale) {
    __shared__ FewSums<1> sums;
    const int waves = blockDim.x >> 6;
    const int64_t n0 = (int64_t)blockIdx.x * kClasses;
    few_sums<1, 2>(x.q, x.ld, w.q, w.ld, M, N, K, n0, sums);
    if (blockIdx.x == 0 && (int)threadIdx.x < M)
        scale[threadIdx.x] = target[threadIdx.x] < 0 ? 0.0f : x.scale[threadIdx.x];
    const int64_t n = n0 + threadIdx.x % kClasses;
    if (n >= N) return;
    const float ws = w.scale[n];
    for (int e = threadIdx.x; e < 256; e += blockDim.x) {
        const int m = e / kClasses;
        if (m >= M) break;
        const int64_t y = target[m];
        const float z = (float)few_sum<1>(sums, e, waves) * x.scale[m] * ws;
        const float l = y >= V ? __builtin_nanf("") : in.lse[m];
        float p = exp_of(z - l);
        if (first + n == y) p = in.miss != nullptr ? -in.miss[m] : p - 1.0f;
        const float v = in.g[m] * p;
        d[m * ld + n] = y < 0 ? 0.0f : v;
    }
}

// sum <- sum + part, to dx after the last piece
__global__ __launch_bounds__(256) void xent_few_add_kernel(float* sum, const float* part,
                                                           int64_t ld, int64_t K, int first,
                                                           int last, Target out) {
    const int64_t t = blockIdx.x;
    for (int64_t k = threadIdx.x; k < K; k += 256) {
        const int64_t i = t * ld + k;
        const float x = first ? part[i] : sum[i] + part[i];
        if (!last) sum[i] = x;
        else if (out.bf16) narrow(x, static_cast<uint16_t*>(out.c) + t * out.ldc + k);
        else static_cast<float*>(out.c)[t * out.ldc + k] = x;
    }
}

struct ForwardRoom : Room {
    int64_t blocks, part, hit;
};
ForwardRoom forward_room(int64_t T, int64_t V) {
    ForwardRoom r;
    r.blocks = up(V, kClasses);
    r.part = r.take(T * r.blocks * (int64_t)sizeof(Stats));
    r.hit = r.take(T * 4);
    return r;
}

// Classes of a piece: 2^25 logits at most, so that their gradient takes 128 MB.
int64_t piece_of(int64_t T, int64_t V) {
    return piece_size(V, up(V, ((int64_t)1 << 25) / T / kClasses * kClasses), kClasses);
}
// Classes of a piece that a product for dx takes: where it lays their weights out, 120 MB of them
// at most, which the memory-side cache holds until they are multiplied (64 x 151936 x 4096 whole,
// 1.2 GB, and so: fp32 1505 and 1465 us, bf16 1300 and 1395, whose terms are then held in three
// numbers; 64 x 116960 x 3264 fp32 1048 and 968, bf16 857 and 901; in 60 MB 1709 at the first).
int64_t part_of(int64_t T, int64_t piece, int64_t K) {
    constexpr int64_t kRoom = (int64_t)120 << 20;
    for (int64_t parts = 1;;) {
        const int64_t n = piece_size(piece, parts, kClasses);
        const int64_t room = grad_input_workspace(T, n, K, false, false);
        if (room <= kRoom || n <= 1024) return n;
        parts = up(parts * room, kRoom);
    }
}

struct BackwardRoom : Room {
    int64_t piece, part;  // classes of a piece, and of its product for dx
    int64_t ld, ldk;      // row strides of d and of dx' sums
    int64_t d, scale, sum, term, product;
};
BackwardRoom backward_room(int64_t T, int64_t V, int64_t K, bool dx_bf16, bool dw_bf16) {
    BackwardRoom r;
    r.piece = piece_of(T, V);
    r.part = part_of(T, r.piece, K);
    r.ld = up(r.piece, 4) * 4;
    r.ldk = up(K, 4) * 4;
    r.d = r.take(T * r.ld * 4);
    r.scale = r.take(T * 4);
    const bool several = r.part < V;
    if (several) {
        r.sum = r.take(T * r.ldk * 4);
        r.term = r.take(T * r.ldk * 4);
    }
    int64_t most = 0;
    const auto need = [&](int64_t bytes) { most = bytes > most ? bytes : most; };
    const int64_t pieces[] = {r.piece, V - (V - 1) / r.piece * r.piece};
    for (const int64_t n : pieces) {
        need(grad_weight_workspace(T, n, K, false, dw_bf16));
        const int64_t whole = r.part < n ? r.part : n, last = n - (n - 1) / whole * whole;
        need(grad_input_workspace(T, whole, K, false, dx_bf16 && !several));
        need(grad_input_workspace(T, last, K, false, dx_bf16 && !several));
    }
    r.product = r.take(most);
    return r;
}

}  // namespace

int64_t few_xent_workspace(int64_t T, int64_t V) { return forward_room(T, V).bytes; }

int launch_few_xent(const Loss& l, const LossOut& to, void* ws, void* stream) {
    const ForwardRoom r = forward_room(l.T, l.V);
    const int waves = few_waves(l.K);
    // (a launch holds fewer than 2^32 work items)
    const int64_t most = (int64_t)1 << 21;
    for (int64_t b = 0; b < r.blocks; b += most) {
        const int64_t n = r.blocks - b < most ? r.blocks - b : most;
        if (int e = launch(xent_few_stats_kernel, dim3((uint32_t)n), 64 * waves, stream, l.x, l.w,
                           l.target, (int)l.T, l.V, (int)l.K, b, r.blocks, at<Stats>(ws, r.part),
                           at<float>(ws, r.hit)))
            return e;
    }
    return launch(xent_few_join_kernel, dim3((uint32_t)l.T), 1024, stream, at<Stats>(ws, r.part),
                  r.blocks, at<float>(ws, r.hit), l.V, l.target, to);
}

int64_t few_xent_bwd_workspace(int64_t T, int64_t V, int64_t K, bool dx_bf16, bool dw_bf16) {
    return backward_room(T, V, K, dx_bf16, dw_bf16).bytes;
}

int launch_few_xent_bwd(const Loss& l, const LossIn& in, Mat dx, Mat dw, void* ws,
                        void* stream) {
    const BackwardRoom r = backward_room(l.T, l.V, l.K, dx.bf16, dw.bf16);
    const Mat d{at<float>(ws, r.d), r.ld, false}, term{at<float>(ws, r.term), r.ldk, false};
    const Held x{l.x.q, l.x.ld, at<float>(ws, r.scale)};
    char* room = at<char>(ws, r.product);
    for (int64_t v = 0; v < l.V; v += r.piece) {
        const int64_t n = l.V - v < r.piece ? l.V - v : r.piece;
        const Held w{l.w.q + v * l.w.ld, l.w.ld, l.w.scale + v};
        auto* scale = at<float>(ws, r.scale);
        const int e = few_logits(l.T, l.K)
                          ? launch(xent_few_slopes_kernel, dim3((uint32_t)up(n, kClasses)),
                                   64 * few_waves(l.K), stream, l.x, w, l.target, (int)l.T, n,
                                   (int)l.K, v, l.V, in, static_cast<float*>(d.p), r.ld, scale)
                          : launch_few_slopes(l, v, n, in, static_cast<float*>(d.p), r.ld, scale,
                                              stream);
        if (e) return e;
        for (int64_t i = 0; i < n && dx.p != nullptr; i += r.part) {
            const int64_t m = n - i < r.part ? n - i : r.part;
            const Mat some{static_cast<float*>(d.p) + i, r.ld, false};
            const Held of{w.q + i * w.ld, w.ld, w.scale + i};
            const bool first = v + i == 0, last = v + i + m == l.V;
            if (int s = launch_grad_input(some, of, l.T, m, l.K, first && last ? dx : term, room,
                                          stream))
                return s;
            if (first && last) continue;
            Target out{};
            out.c = dx.p;
            out.ldc = dx.ld;
            out.bf16 = dx.bf16;
            if (int s = launch(xent_few_add_kernel, dim3((uint32_t)l.T), 256, stream,
                               at<float>(ws, r.sum), static_cast<const float*>(term.p), r.ldk,
                               l.K, (int)first, (int)last, out))
                return s;
        }
        if (dw.p != nullptr) {
            const Mat rows{static_cast<char*>(dw.p) + v * dw.ld * (dw.bf16 ? 2 : 4), dw.ld,
                           dw.bf16};
            if (int s = launch_grad_weight(d, x, l.T, n, l.K, rows, room, stream)) return s;
        }
    }
    return 0;
}

}  // namespace q8
}  // namespace cpdp
