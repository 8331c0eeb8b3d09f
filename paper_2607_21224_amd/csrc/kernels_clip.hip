// The global norm of a replica's gradient, and clipping by it.
//   norm_i = sqrt(sum over p of g_i[p]^2), or of the replicas' mean gradient;
//   c_i = min(1, max_norm / (norm_i + 1e-6));  g_i <- c_i g_i
//
// Both are bound by HBM.  A first launch gives each block a run of chunks of one
// replica (of all replicas for the mean) and leaves one sum for each; a second one adds
// them up, and a third scales.  Where the gradients are small, the second is left out:
// every block of the last adds its replica's sums up by itself, in the same order; and a
// replica of up to 80 KB is one block's, in one launch.  Squares and sums are fp64: they
// cannot overflow or lose small values, and cost nothing beside the memory (2 instructions a
// coordinate of 4 bytes).  There are no atomics; the order of a sum is fixed by the sizes.
#include "cpdp_device.h"

#include "clip_launch.h"

namespace cpdp {
namespace {

constexpr int kThreads = 256, kRowThreads = 1024;  // of a part's block, of a whole row's
constexpr int64_t kCoords = (int64_t)kBlock * kVec;  // of a chunk

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

// 16 bytes of gradients as they lie in memory
struct F32Piece {
    using T = float;
    static constexpr int N = 4;
    u32x4 v;
    __device__ __forceinline__ float get(int k) const { return __uint_as_float(v[k]); }
    __device__ __forceinline__ void set(const float (&x)[N]) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = __float_as_uint(x[k]);
    }
    static __device__ __forceinline__ float one(T x) { return x; }
    static __device__ __forceinline__ T narrow(float x) { return x; }
};
struct BF16Piece {
    using T = uint16_t;
    static constexpr int N = 8;
    u32x4 v;
    __device__ __forceinline__ float get(int k) const {
        return __uint_as_float(k % 2 == 0 ? v[k / 2] << 16 : v[k / 2] & 0xFFFF0000u);
    }
    __device__ __forceinline__ void set(const float (&x)[N]) {
#pragma unroll
        for (int k = 0; k < N / 2; ++k)
            v[k] = bf16_bits(x[2 * k]) | (bf16_bits(x[2 * k + 1]) << 16);
    }
    static __device__ __forceinline__ float one(T x) { return bf16_value(x); }
    static __device__ __forceinline__ T narrow(float x) { return (T)bf16_bits(x); }
};

// Where replica i's coordinates lie.  runs(c0, c1, f) calls f(t, e, count) for each run
// of `count` coordinates, from e on, of a tensor t that chunks c0 to c1 cover.
template <class G>
struct FlatRows {
    typename G::T* base;
    int64_t ld, P;
    __device__ __forceinline__ typename G::T* row(int64_t i, int64_t) const {
        return base + i * ld;
    }
    template <class F>
    __device__ __forceinline__ void runs(int64_t c0, int64_t c1, F f) const {
        const int64_t e = c0 * kCoords;
        f((int64_t)0, e, min(c1 * kCoords, P) - e);
    }
};
struct PlanRows {
    const int64_t* plan;
    int W, n;
    __device__ __forceinline__ float* row(int64_t i, int64_t t) const {
        return global_ptr<float>(plan_view(plan, W, n).grads[i * n + t]);
    }
    template <class F>
    __device__ __forceinline__ void runs(int64_t c0, int64_t c1, F f) const {
        const PlanView v = plan_view(plan, W, n);
        int64_t t = plan_tensor_scalar(v, n, c0);
        for (int64_t c = c0; c < c1; ++t) {
            const int64_t start = v.chunk_start[t], end = min(v.chunk_start[t + 1], c1);
            if (end <= c) continue;  // an empty tensor
            const int64_t e = (c - start) * kCoords;
            f(t, e, min((end - start) * kCoords, v.numel[t]) - e);
            c = end;
        }
    }
};

// body(whole, at, first) for the thread's pieces of `count` coordinates, U of them at a
// time, and the rest together (at, first: arrays of them): a piece is read at `at`, and
// its coordinates from `first` on are the thread's.  whole: all of them are, and pieces
// are aligned.  (A piece that the end cuts short is read as the last N coordinates,
// wherever they start.)  count >= N.
template <int THREADS, int N, int U, class Body>
__device__ __forceinline__ void pieces(int64_t count, Body body) {
    constexpr int64_t kRound = (int64_t)THREADS * N;
    const int64_t lane = (int64_t)threadIdx.x * N;
    int64_t r = 0;
    for (; r + U * kRound <= count; r += U * kRound) {
        int64_t at[U];
        int first[U];
#pragma unroll
        for (int u = 0; u < U; ++u) at[u] = r + u * kRound + lane, first[u] = 0;
        body(std::true_type(), at, first);
    }
    const auto rest = [&](auto some) {
        int64_t at[some];
        int first[some];
#pragma unroll
        for (int u = 0; u < some; ++u) {
            const int64_t i = r + u * kRound + lane, last = count - N;
            at[u] = i < last ? i : last;
            first[u] = (int)min(i - at[u], (int64_t)N);
        }
        body(std::false_type(), at, first);
    };
    const int64_t left = count - r;
    if (left <= 0) return;
    if (left <= kRound) rest(std::integral_constant<int, 1>());
    else if (left <= 2 * kRound) rest(std::integral_constant<int, 2>());
    else if (left <= 4 * kRound) rest(std::integral_constant<int, 4>());
    else rest(std::integral_constant<int, 8>());
}
// a piece that is read once more, if at all, long after (nontemporal, 8 at a time: the
// norms of 8 x 21.3 M fp32 107 us; ordinary 121)
template <bool WHOLE>
__device__ __forceinline__ u32x4 read_once(const void* p) {
    if constexpr (WHOLE) return __builtin_nontemporal_load(static_cast<const u32x4*>(p));
    else return *static_cast<const u32x4_any*>(p);
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
    return x;
}
// the sum over the block's threads, in every thread
template <int THREADS>
__device__ __forceinline__ double block_sum(double x) {
    __shared__ double words[THREADS / 64];
    x = wave_sum(x);
    if (threadIdx.x % 64 == 0) words[threadIdx.x / 64] = x;
    __syncthreads();
    x = words[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) x += words[w];
    return x;
}

// A part of the sum of squares of a row, or (MEAN) of the mean of W rows: the rows'
// coordinates are added up in fp32, in their order, as a synchronisation step does.
template <int THREADS, class G, bool MEAN, class Src>
__device__ __forceinline__ double part_sum(const Src& src, int64_t row, int W, float inv_w,
                                           int64_t c0, int64_t c1) {
    using T = typename G::T;
    constexpr int N = G::N;
    double acc[4] = {0.0, 0.0, 0.0, 0.0};
    src.runs(c0, c1, [&](int64_t t, int64_t e, int64_t count) {
        if (count < N) {
            if ((int64_t)threadIdx.x >= count) return;
            const int64_t at = e + threadIdx.x;
            float x;
            if constexpr (MEAN) {
                x = 0.0f;
                for (int i = 0; i < W; ++i) x += G::one(src.row(i, t)[at]);
                x *= inv_w;
            } else {
                x = G::one(src.row(row, t)[at]);
            }
            acc[0] = fma((double)x, (double)x, acc[0]);
            return;
        }
        pieces<THREADS, N, MEAN ? 1 : 8>(count, [&](auto whole, const auto& at, const auto& first) {
            constexpr int U = sizeof(at) / sizeof(at[0]);
            const auto load = [&](int64_t i, int64_t at) {
                return G{read_once<whole>(static_cast<const T*>(src.row(i, t)) + e + at)};
            };
            if constexpr (MEAN) {
                float s[N] = {};
                const auto add = [&](int i, auto rows) {
                    G g[rows];
#pragma unroll
                    for (int j = 0; j < rows; ++j) g[j] = load(i + j, at[0]);
#pragma unroll
                    for (int j = 0; j < rows; ++j)
#pragma unroll
                        for (int k = 0; k < N; ++k) s[k] += g[j].get(k);
                };
                int i = 0;
                for (; i + 8 <= W; i += 8) add(i, std::integral_constant<int, 8>());
                for (; i + 2 <= W; i += 2) add(i, std::integral_constant<int, 2>());
                if (i < W) add(i, std::integral_constant<int, 1>());
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const float x = !whole && k < first[0] ? 0.0f : s[k] * inv_w;
                    acc[k % 4] = fma((double)x, (double)x, acc[k % 4]);
                }
            } else {
                G g[U];
#pragma unroll
                for (int u = 0; u < U; ++u) g[u] = load(row, at[u]);
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        const float x = !whole && k < first[u] ? 0.0f : g[u].get(k);
                        acc[k % 4] = fma((double)x, (double)x, acc[k % 4]);
                    }
            }
        });
    });
    return (acc[0] + acc[1]) + (acc[2] + acc[3]);
}

// first chunk of part k of `parts`
__device__ __forceinline__ int64_t part_start(int64_t chunks, int64_t parts, int64_t k) {
    return chunks / parts * k + min(chunks % parts, k);
}

template <class G, bool MEAN, class Src>
__global__ __launch_bounds__(kThreads) void norm_part_kernel(Src src, int W, float inv_w,
                                                             int64_t chunks, int parts,
                                                             double* sums) {
    const int64_t row = blockIdx.x / parts, k = blockIdx.x % parts;
    const double s = block_sum<kThreads>(part_sum<kThreads, G, MEAN>(src, row, W, inv_w,
                                                           part_start(chunks, parts, k),
                                                           part_start(chunks, parts, k + 1)));
    if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

// the norm of a row from its parts, in every thread
__device__ __forceinline__ float row_norm(const double* sums, int parts) {
    double s = 0.0;
    for (int k = threadIdx.x; k < parts; k += kThreads) s += sums[k];
    return (float)sqrt(block_sum<kThreads>(s));
}

__global__ __launch_bounds__(kThreads) void norm_join_kernel(const double* sums, int parts,
                                                             float* norm) {
    const float x = row_norm(sums + (int64_t)blockIdx.x * parts, parts);
    if (threadIdx.x == 0) norm[blockIdx.x] = x;
}

// 1 where the norm is not longer; a NaN stays one
__device__ __forceinline__ float clip_scale(float norm, float max_norm) {
    const float c = max_norm / (norm + 1e-6f);
    return c >= 1.0f ? 1.0f : c;
}

// Scales chunks c0 to c1 of a row by c.
template <int THREADS, class G, class Src>
__device__ __forceinline__ void scale(const Src& src, int64_t row, int64_t c0, int64_t c1,
                                      float c) {
    using T = typename G::T;
    constexpr int N = G::N;
    src.runs(c0, c1, [&](int64_t t, int64_t e, int64_t count) {
        T* const p = src.row(row, t) + e;
        if (count < N) {
            if ((int64_t)threadIdx.x < count)
                p[threadIdx.x] = G::narrow(G::one(p[threadIdx.x]) * c);
            return;
        }
        pieces<THREADS, N, 4>(count, [&](auto whole, const auto& at, const auto& first) {
            constexpr int U = sizeof(at) / sizeof(at[0]);
            G g[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if constexpr (whole) g[u].v = *reinterpret_cast<const u32x4*>(p + at[u]);
                else g[u].v = *reinterpret_cast<const u32x4_any*>(p + at[u]);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float y[N];
#pragma unroll
                for (int j = 0; j < N; ++j) y[j] = g[u].get(j) * c;
                if constexpr (whole) {
                    g[u].set(y);
                    *reinterpret_cast<u32x4*>(p + at[u]) = g[u].v;
                } else if (first[u] == 0) {
                    g[u].set(y);
                    *reinterpret_cast<u32x4_any*>(p + at[u]) = g[u].v;
                } else {
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        if (j >= first[u]) p[at[u] + j] = G::narrow(y[j]);
                }
            }
        });
    });
}

// Part k of `parts` of a row (mean: every row's norm is the first's), whose norm is the
// sum of `of_sums` parts, or, with 0 of them, there already.  Rows that are not longer
// than max_norm are not read.
template <class G, class Src>
__global__ __launch_bounds__(kThreads) void clip_kernel(Src src, int64_t chunks, int parts,
                                                        const double* sums, int of_sums, int mean,
                                                        float max_norm, float* norm) {
    const int64_t row = blockIdx.x / parts, k = blockIdx.x % parts, of = mean ? 0 : row;
    float x;
    if (of_sums > 0) {
        x = row_norm(sums + of * of_sums, of_sums);
        if (k == 0 && row == of && threadIdx.x == 0) norm[of] = x;
    } else {
        x = norm[of];
    }
    const float c = clip_scale(x, max_norm);
    if (c != 1.0f)
        scale<kThreads, G>(src, row, part_start(chunks, parts, k),
                           part_start(chunks, parts, k + 1), c);
}

// A block's whole row (or the mean of all rows): its norm, and (clip) the row scaled.  In a
// block of its own a small row's sum needs no other's: 2 x 10007 fp32, clipping calls after
// each other, 8.5 us in two launches, 5.7 in one.
template <class G, bool MEAN, class Src>
__global__ __launch_bounds__(kRowThreads) void norm_row_kernel(Src src, int W, float inv_w,
                                                               int64_t chunks, int clip,
                                                               float max_norm, float* norm) {
    const int64_t row = blockIdx.x;
    const float x = (float)sqrt(block_sum<kRowThreads>(
        part_sum<kRowThreads, G, MEAN>(src, row, W, inv_w, (int64_t)0, chunks)));
    if (threadIdx.x == 0) norm[row] = x;
    if constexpr (!MEAN) {
        const float c = clip_scale(x, max_norm);
        if (clip && c != 1.0f) scale<kRowThreads, G>(src, row, 0, chunks, c);
    }
}

template <int THREADS = kThreads, class... Args>
int launch_blocks(void (*kernel)(Args...), int64_t blocks, void* stream,
                  typename same_type<Args>::type... args) {
    void* argv[] = {static_cast<void*>(&args)...};
    return (int)hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((uint32_t)blocks),
                                dim3(THREADS), argv, 0, static_cast<hipStream_t>(stream));
}

// Whether a block takes a row by itself: few enough for a CU each (1000 x 5000 fp32 13.3 us
// so, 11.1 in parts), and small (clipped, 20000 fp32 9.1 and 10.4; 32768 10.1 and 9.5).  (Not
// the mean's W rows where they are clipped: each would need the norm of all of them.)
template <class G>
bool small_rows(const Gradients& g, bool mean) {
    const int64_t bytes = g.chunks * kCoords * (int64_t)sizeof(typename G::T);
    return bytes * (mean ? g.W : 1) <= 81920 && (mean || g.W <= 256);
}

template <class G, class Src>
int norm_parts_of(const Gradients& g, Src src, bool mean, int parts, double* sums, void* stream) {
    const float inv_w = 1.0f / (float)g.W;
    return mean ? launch_blocks(norm_part_kernel<G, true, Src>, parts, stream, src, g.W, inv_w,
                                g.chunks, parts, sums)
                : launch_blocks(norm_part_kernel<G, false, Src>, (int64_t)parts * g.W, stream, src,
                                g.W, inv_w, g.chunks, parts, sums);
}

// f(piece type, source)
template <class F>
int with_source(const Gradients& g, F f) {
    if (g.plan != nullptr) return f(F32Piece(), PlanRows{g.plan, g.W, g.n});
    if (g.bf16)
        return f(BF16Piece(), FlatRows<BF16Piece>{static_cast<uint16_t*>(g.base), g.ld, g.P});
    return f(F32Piece(), FlatRows<F32Piece>{static_cast<float*>(g.base), g.ld, g.P});
}

}  // namespace

int launch_grad_norm(const Gradients& g, bool mean, float* norm, void* workspace, void* stream) {
    return with_source(g, [&](auto piece, auto src) {
        using G = decltype(piece);
        const int rows = mean ? 1 : g.W, parts = (int)norm_parts(rows, g.chunks);
        const float inv_w = 1.0f / (float)g.W;
        if (small_rows<G>(g, mean))
            return launch_blocks<kRowThreads>(mean ? norm_row_kernel<G, true, decltype(src)>
                                                   : norm_row_kernel<G, false, decltype(src)>,
                                              rows, stream, src, g.W, inv_w, g.chunks, 0, 0.0f,
                                              norm);
        auto* sums = static_cast<double*>(workspace);
        if (int e = norm_parts_of<G>(g, src, mean, parts, sums, stream)) return e;
        return launch_blocks(norm_join_kernel, rows, stream, sums, parts, norm);
    });
}

int launch_clip_grads(const Gradients& g, bool mean, float max_norm, float* norm, void* workspace,
                      void* stream) {
    return with_source(g, [&](auto piece, auto src) {
        using G = decltype(piece);
        if (!mean && small_rows<G>(g, false))
            return launch_blocks<kRowThreads>(norm_row_kernel<G, false, decltype(src)>, g.W,
                                              stream, src, g.W, 1.0f, g.chunks, 1, max_norm, norm);
        const int rows = mean ? 1 : g.W, of_sums = (int)norm_parts(rows, g.chunks);
        auto* sums = static_cast<double*>(workspace);
        if (int e = norm_parts_of<G>(g, src, mean, of_sums, sums, stream)) return e;
        // Past 64 MB the norms get a launch of their own, and the blocks that scale are of 32 KB
        // in the order they lie in memory: 8 x 21.3 M fp32 scaled by 2048 blocks 240 us, by
        // 42,000 214.  (Of 16 KB they take 10 us where there is nothing to scale, of 32 KB 6;
        // the norm alone 108 to 112, clipped 325, read from memory.)
        constexpr int64_t kRun = 32768 / (kCoords * (int64_t)sizeof(typename G::T));
        const int64_t fine = (g.chunks + kRun - 1) / kRun;
        const bool large = g.W * g.chunks * kCoords * (int64_t)sizeof(typename G::T) > (64 << 20) &&
                           fine * g.W * kThreads < (int64_t)1 << 32;
        if (large)
            if (int e = launch_blocks(norm_join_kernel, rows, stream, sums, of_sums, norm))
                return e;
        const int parts = (int)(large ? fine : norm_parts(g.W, g.chunks));
        return launch_blocks(clip_kernel<G, decltype(src)>, (int64_t)parts * g.W, stream, src,
                             g.chunks, parts, sums, large ? 0 : of_sums, (int)mean, max_norm,
                             norm);
    });
}

}  // namespace cpdp
