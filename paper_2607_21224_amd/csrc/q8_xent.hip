// Softmax cross entropy of 8-bit rows over the classes of 8-bit weights, and its
// gradients, without the logits being kept: the classes are taken in pieces, whose
// logits are made, used and overwritten by the next piece's.
#include <initializer_list>

#include "q8_gemm.h"
#include "q8_xent_launch.h"

namespace cpdp {
namespace q8 {
namespace {

// Logits of a piece: 2^25 at most (128 MB), whole steps of 256 classes.
int64_t piece_of(int64_t T, int64_t V) {
    int64_t n = ((int64_t)1 << 25) / (T < 1 ? 1 : T) / 256 * 256;
    if (n < 256) n = 256;
    return n < V ? n : V;
}

// What is known of a row after some of the pieces.
struct Stats {
    float top, sum, hit;  // maximum, sum of exp(z - top), the target's logit
};

int64_t up256(int64_t n) { return (n + 255) / 256 * 256; }

struct Room {
    int64_t piece, ld;  // classes of a piece; its logits' row stride
    int64_t logits, stats, scale, sum, part, product;  // where each begins
    int64_t bytes;
};
Room room_of(int64_t T, int64_t V, int64_t K, bool bwd, bool dx_bf16, bool dw_bf16) {
    Room r{};
    r.piece = piece_of(T, V);
    r.ld = (r.piece + 15) / 16 * 16;
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += up256(bytes);
        return here;
    };
    r.logits = take(T * r.ld * 4);
    r.stats = take(T * (int64_t)sizeof(Stats));
    int64_t product = matmul_workspace(T, r.piece, K);
    const int64_t last = V - (V - 1) / r.piece * r.piece;
    for (const int64_t n : {r.piece, last}) {
        const int64_t need[] = {matmul_workspace(T, n, K),
                                bwd ? grad_input_workspace(T, n, K, false, false) : 0,
                                bwd ? grad_weight_workspace(T, n, K, false, dw_bf16) : 0};
        for (const int64_t b : need) product = b > product ? b : product;
    }
    if (bwd) {
        r.scale = take(T * 4);
        const int64_t ldk = (K + 15) / 16 * 16;
        r.sum = take(T * ldk * 4);
        r.part = take(T * ldk * 4);
    }
    r.product = take(product);
    r.bytes = at;
    return r;
}

struct Add2 {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct Max2 {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

template <class Op>
__device__ __forceinline__ float over_block(float x, Op op, float* words) {
    x = wave_reduce(x, op);
    if (threadIdx.x % 64 == 0) words[threadIdx.x / 64] = x;
    __syncthreads();
    x = words[0];
#pragma unroll
    for (int w = 1; w < 4; ++w) x = op(x, words[w]);
    return x;
}

// exp(z - top), where top is the largest of some logits; nothing but -infinities: 0
__device__ __forceinline__ float weight(float z, float top) {
    return top == -__builtin_inff() ? (z == top ? 0.0f : z) : expf(z - top);
}

// A block takes a row of a piece's logits.
__global__ __launch_bounds__(256) void xent_stats_kernel(const float* z, int64_t ld, int64_t v0,
                                                         int n, const int64_t* target,
                                                         Stats* stats, int first, int last,
                                                         float* loss, float* lse) {
    __shared__ float words[2][4];
    const int64_t t = blockIdx.x;
    const float* row = z + t * ld;
    float top = -__builtin_inff();
    for (int v = threadIdx.x; v < n; v += 256) top = fmaxf(top, row[v]);
    top = over_block(top, Max2(), words[0]);
    float sum = 0.0f;
    for (int v = threadIdx.x; v < n; v += 256) sum += weight(row[v], top);
    sum = over_block(sum, Add2(), words[1]);
    if (threadIdx.x != 0) return;
    Stats s = {-__builtin_inff(), 0.0f, __builtin_nanf("")};
    if (!first) s = stats[t];
    const float both = fmaxf(s.top, top);
    s.sum = s.sum * weight(s.top, both) + sum * weight(top, both);
    s.top = both;
    const int64_t at = target[t] - v0;
    if (at >= 0 && at < n) s.hit = row[at];
    stats[t] = s;
    if (last) {
        const float l = s.top + logf(s.sum);
        lse[t] = l;
        loss[t] = target[t] < 0 ? 0.0f : l - s.hit;
    }
}

// The logits' gradient takes the logits' place.  Rows that do not count have none.
__global__ __launch_bounds__(256) void xent_grad_kernel(float* z, int64_t ld, int64_t v0, int n,
                                                        int64_t V, const int64_t* target,
                                                        const float* lse, const float* g) {
    const int64_t t = blockIdx.x;
    const int64_t y = target[t];
    const float l = y >= V ? __builtin_nanf("") : lse[t], f = g[t];
    for (int v = threadIdx.x; v < n; v += 256) {
        float* p = z + t * ld + v;
        const float d = f * (expf(*p - l) - (v0 + v == y ? 1.0f : 0.0f));
        *p = y < 0 ? 0.0f : d;
    }
}

__global__ __launch_bounds__(256) void xent_scale_kernel(const float* scale, const int64_t* target,
                                                         int64_t T, float* out) {
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t < T) out[t] = target[t] < 0 ? 0.0f : scale[t];
}

// sum <- sum + part, to dx after the last piece
__global__ __launch_bounds__(256) void xent_add_kernel(float* sum, const float* part, int64_t ld,
                                                       int64_t K, const int64_t* target, int first,
                                                       int last, Target out) {
    const int64_t t = blockIdx.x;
    for (int64_t k = threadIdx.x; k < K; k += 256) {
        const int64_t i = t * ld + k;
        const float x = target[t] < 0 ? 0.0f : first ? part[i] : sum[i] + part[i];
        if (!last) sum[i] = x;
        else if (out.bf16) narrow(x, static_cast<uint16_t*>(out.c) + t * out.ldc + k);
        else static_cast<float*>(out.c)[t * out.ldc + k] = x;
    }
}

}  // namespace

int64_t xent_workspace(int64_t T, int64_t V, int64_t K) {
    return room_of(T, V, K, false, false, false).bytes;
}

int launch_xent(const Loss& l, float* loss, float* lse, void* workspace, void* stream) {
    const Room r = room_of(l.T, l.V, l.K, false, false, false);
    char* ws = static_cast<char*>(workspace);
    auto* z = reinterpret_cast<float*>(ws + r.logits);
    for (int64_t v = 0; v < l.V; v += r.piece) {
        const int64_t n = l.V - v < r.piece ? l.V - v : r.piece;
        const Held w{l.w.q + v * l.w.ld, l.w.ld, l.w.scale + v};
        if (int e = launch_matmul(l.x, w, l.T, n, l.K, Mat{z, r.ld, false}, ws + r.product, stream))
            return e;
        if (int e = launch(xent_stats_kernel, dim3((uint32_t)l.T), 256, stream, z, r.ld, v, (int)n,
                           l.target, reinterpret_cast<Stats*>(ws + r.stats), (int)(v == 0),
                           (int)(v + n == l.V), loss, lse))
            return e;
    }
    return 0;
}

int64_t xent_bwd_workspace(int64_t T, int64_t V, int64_t K, bool dx_bf16, bool dw_bf16) {
    return room_of(T, V, K, true, dx_bf16, dw_bf16).bytes;
}

int launch_xent_bwd(const Loss& l, const float* lse, const float* g, Mat dx, Mat dw,
                    void* workspace, void* stream) {
    const Room r = room_of(l.T, l.V, l.K, true, dx.bf16, dw.bf16);
    char* ws = static_cast<char*>(workspace);
    if (l.T == 0)
        return launch_grad_weight(Mat{nullptr, 0, false}, l.x, 0, l.V, l.K, dw, ws, stream);
    auto* z = reinterpret_cast<float*>(ws + r.logits);
    auto* scale = reinterpret_cast<float*>(ws + r.scale);
    const int64_t ldk = (l.K + 15) / 16 * 16;
    if (int e = launch(xent_scale_kernel, dim3((uint32_t)((l.T + 255) / 256)), 256, stream,
                       l.x.scale, l.target, l.T, scale))
        return e;
    for (int64_t v = 0; v < l.V; v += r.piece) {
        const int64_t n = l.V - v < r.piece ? l.V - v : r.piece;
        const Held w{l.w.q + v * l.w.ld, l.w.ld, l.w.scale + v};
        const Mat d{z, r.ld, false};
        if (int e = launch_matmul(l.x, w, l.T, n, l.K, d, ws + r.product, stream)) return e;
        if (int e = launch(xent_grad_kernel, dim3((uint32_t)l.T), 256, stream, z, r.ld, v, (int)n,
                           l.V, l.target, lse, g))
            return e;
        if (dx.p != nullptr) {
            const Mat part{ws + r.part, ldk, false};
            if (int e = launch_grad_input(d, w, l.T, n, l.K, part, ws + r.product, stream))
                return e;
            Target out{};
            out.c = dx.p;
            out.ldc = dx.ld;
            out.bf16 = dx.bf16;
            if (int e = launch(xent_add_kernel, dim3((uint32_t)l.T), 256, stream,
                               reinterpret_cast<float*>(ws + r.sum),
                               reinterpret_cast<const float*>(ws + r.part), ldk, l.K, l.target,
                               (int)(v == 0), (int)(v + n == l.V), out))
                return e;
        }
        if (dw.p != nullptr) {
            const int64_t e = dw.bf16 ? 2 : 4;
            const Mat part{static_cast<char*>(dw.p) + v * dw.ld * e, dw.ld, dw.bf16};
            if (int s = launch_grad_weight(d, Held{l.x.q, l.x.ld, scale}, l.T, n, l.K, part,
                                           ws + r.product, stream))
                return s;
        }
    }
    return 0;
}

}  // namespace q8
}  // namespace cpdp
