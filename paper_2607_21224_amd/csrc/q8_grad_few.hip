// The gradients of a product over up to 64 tokens.
//
// There the weights (dx) or their gradient (dw) are nearly all that is moved, and
// neither is worth laying out anew first: the operands go from memory to the
// matrix cores through registers.  An instruction wants, in each lane, 8 values of
// one row of its operand that follow each other along the sum, and the sum runs
// down the columns of what is read.  So a lane reads 8 such rows, a few bytes of
// each at the same columns, and takes its columns one after the other: column c of
// the 8 words is its operand of instruction c.  Lane r of 16 then stands for
// columns r, r + 1, .. of W, W columns a lane, instruction c for column W r + c,
// and the results of a lane lie next to each other.
#include "q8_grad.h"

namespace cpdp {
namespace q8 {
namespace {

constexpr int kSum = 32;  // values of the sum that one instruction takes

// 8 rows of int8, W columns (4 or 8) a lane.  Rows that are past the last one repeat
// it (their partners are zeros), and so do columns past the last piece (what they come
// to is not stored): no load is behind a branch, and all are on their way together.
template <int W>
struct Octet {
    uint32_t w[8][W / 4];
    __device__ __forceinline__ void load(const int8_t* p, int64_t ld, int64_t row, int64_t rows,
                                         int64_t col, int64_t cols) {
        const int64_t last = (cols - 1) / W * W, c = col < last ? col : last;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int8_t* q = p + (row + i < rows ? row + i : rows - 1) * ld + c;
#pragma unroll
            for (int k = 0; k < W / 4; ++k) w[i][k] = reinterpret_cast<const uint32_t*>(q)[k];
        }
    }
    // column c of the 8 rows (exact: a number of 8 bits has no bits past a bf16's)
    __device__ __forceinline__ u32x4 column(int c) const {
        u32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float a = (float)(int8_t)(w[2 * k][c / 4] >> (8 * (c % 4)));
            const float b = (float)(int8_t)(w[2 * k + 1][c / 4] >> (8 * (c % 4)));
            v[k] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
        }
        return v;
    }
};

// 8 values in P parts, each part as an operand
template <int P>
__device__ __forceinline__ void operand(const float (&x)[8], u32x4 (&v)[P]) {
    uint16_t part[8][P];
#pragma unroll
    for (int k = 0; k < 8; ++k) split<P>(x[k], part[k]);
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            v[p][k] = (uint32_t)part[2 * k][p] | (uint32_t)part[2 * k + 1][p] << 16;
}

__device__ __forceinline__ int least(int64_t a, int b) { return a < b ? (int)a : b; }

// dx [T x K], T <= 16 MT.  A block takes 128 columns and one of `slices` parts of
// the sum over N; its wavefronts take 32 rows of b in turn and add up in LDS, half
// of them to the other half at a time.
template <class E, int P, int MT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void few_input_kernel(
    const typename E::T* dy, int64_t lddy, const int8_t* b, int64_t ldb, const float* scale, int T,
    int64_t N, int64_t K, int slices, Target t) {
    __shared__ f32x4 sums[WAVES / 2][8 * MT][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int64_t k0 = (int64_t)(blockIdx.x / slices) * 128;
    const int slice = blockIdx.x % slices;
    const int64_t steps = (N + kSum - 1) / kSum;
    const int64_t s1 = steps * (slice + 1) / slices;
    f32x4 acc[8][MT] = {};
    for (int64_t s = steps * slice / slices + wave; s < s1; s += WAVES) {
        const int64_t n = s * kSum + g * 8;
        Octet<8> w;
        w.load(b, ldb, n, N, k0 + r * 8, K);
        // (past the last row the last piece of the scales, as with b: not used)
        const int64_t n_there = n < N ? n : (N - 1) / 8 * 8;
        float f[8];
        load8(scale + n_there, least(N - n_there, 8), least(n_there, 8), f);
        u32x4 d[MT][P];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int m = i * 16 + r;
            float x[8] = {};
            if (m < T && n < N)
                load8(dy + m * lddy + n, least(N - n, 8), n < 8 ? (int)n : 8, x);
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = n + k < N ? x[k] * f[k] : 0.0f;
            operand<P>(x, d[i]);
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const u32x4 col = w.column(c);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int p = 0; p < P; ++p) acc[c][i] = Bf16::mfma(col, d[i][p], acc[c][i]);
        }
    }
#pragma unroll
    for (int half = WAVES / 2; half > 0; half /= 2) {
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int c = 0; c < 8; ++c)
#pragma unroll
                for (int i = 0; i < MT; ++i) sums[wave - half][c * MT + i][lane] = acc[c][i];
        }
        __syncthreads();
        if (wave < half) {
#pragma unroll
            for (int c = 0; c < 8; ++c)
#pragma unroll
                for (int i = 0; i < MT; ++i) acc[c][i] += sums[wave][c * MT + i][lane];
        }
        __syncthreads();
    }
    if (wave != 0) return;
    // lane: token r, columns 32 g to 32 g + 31
    const int64_t c0 = k0 + g * 32;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int m = i * 16 + r;
        float v[32];
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] = acc[k % 8][i][k / 8];
        if (m >= T) continue;
        if (slices > 1) {
            float* p = static_cast<float*>(t.ws) + slice * t.slice + m * t.ldws + c0;
#pragma unroll
            for (int k = 0; k < 32; k += 4)
                *reinterpret_cast<f32x4*>(p + k) = f32x4{v[k], v[k + 1], v[k + 2], v[k + 3]};
        } else if (c0 < K) {
            store_cols<32>(t, m, c0, least(K - c0, 32), v);
        }
    }
}

constexpr int kFewWaves = 4;

int few_input_slices(int64_t N, int64_t K) {
    // two blocks a CU, as long as each wavefront has a step
    const int64_t steps = up(N, kSum), across = up(K, 128);
    int slices = 1;
    while (across * slices < 512 && steps >= 2 * kFewWaves * slices && slices < 64) slices *= 2;
    return slices;
}

template <class E, int P, int MT>
int few_input(Mat dy, Held b, int64_t T, int64_t N, int64_t K, const Target& t, int slices,
              void* stream) {
    constexpr int WAVES = kFewWaves;
    return launch(few_input_kernel<E, P, MT, WAVES>, dim3((uint32_t)(up(K, 128) * slices)),
                  64 * WAVES, stream, static_cast<const typename E::T*>(dy.p), dy.ld, b.q, b.ld,
                  b.scale, T, N, K, slices, t);
}
template <class E, int P>
int few_input_rows(Mat dy, Held b, int64_t T, int64_t N, int64_t K, const Target& t, int slices,
                   void* stream) {
    if (T <= 16) return few_input<E, P, 1>(dy, b, T, N, K, t, slices, stream);
    static_assert(kFewInput == 32, "two tiles of tokens");
    return few_input<E, P, 2>(dy, b, T, N, K, t, slices, stream);
}

// Stores 16 rows of COLS columns that lie in LDS to rows m0, m0 + apart, .. of C.
template <class E, int COLS>
__device__ __forceinline__ void store_tile(const float (&tile)[16][COLS + 4], const Target& t,
                                           int64_t m0, int apart, int64_t M, int64_t k0, int64_t K,
                                           int lane) {
    constexpr int kEach = 16 / sizeof(E);
    constexpr int kLanes = COLS / kEach, kRows = 64 / kLanes;  // of one store
#pragma unroll
    for (int i = 0; i < 16; i += kRows) {
        const int row = i + lane / kLanes, col = lane % kLanes * kEach;
        float v[kEach];
#pragma unroll
        for (int h = 0; h < kEach; h += 4) {
            const f32x4 x = *reinterpret_cast<const f32x4*>(&tile[row][col + h]);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[h + k] = x[k];
        }
        const int64_t m = m0 + row * apart, c = k0 + col;
        if (m >= M || c >= K) continue;
        E* at = static_cast<E*>(t.c) + m * t.ldc + c;
        if (K - c >= kEach) {
            u32x4 p;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (sizeof(E) == 2) p[k] = narrow2(v[2 * k], v[2 * k + 1]);
                else p[k] = __float_as_uint(v[k]);
            }
            // past the caches: the weights' gradients are read when a step is due, long
            // after (4096 x 4096 fp32 of 64 tokens 27.5 us otherwise, and 22 so)
            __builtin_nontemporal_store(p, reinterpret_cast<u32x4*>(at));
        } else {
#pragma unroll
            for (int k = 0; k < kEach - 1; ++k)
                if (k < K - c) narrow(v[k], at + k);
        }
    }
}

// dw [N x K], a sum over at most 64 tokens.  A wavefront takes 16 WN rows and 16 WK
// columns: each lane WN columns of dy and WK of a.
template <class E, int P, int WN, int WK>
__global__ __launch_bounds__(256) void few_weight_kernel(const typename E::T* dy, int64_t lddy,
                                                         const int8_t* a, int64_t lda,
                                                         const float* scale, int T, int64_t N,
                                                         int64_t K, int64_t across, Target t) {
    constexpr int kCols = 16 * WK;
    __shared__ float turn[4][16][kCols + 4];
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int64_t at = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n0 = at / across * 16 * WN, k0 = at % across * kCols;
    if (n0 >= N) return;
    // columns of dy past the last piece repeat it (what they come to is not stored)
    const int64_t last = (N - 1) / WN * WN, n = n0 + r * WN, n_there = n < last ? n : last;
    f32x4 acc[WK][WN] = {};
    for (int t0 = 0; t0 < T; t0 += kSum) {
        const int row = t0 + g * 8;
        Octet<WK> w;
        w.load(a, lda, row, T, k0 + r * WK, K);
        float x[8][WN];
        // (as with a: no branch; a token that is not there is zeros, whatever the last one
        // holds)
        typename E::T e[8][WN];
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int t = row + i < T ? row + i : T - 1;
            const typename E::T* p = dy + t * lddy + n_there;
            __builtin_memcpy(e[i], __builtin_assume_aligned(p, sizeof(e[i])), sizeof(e[i]));
            f[i] = scale[t];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int k = 0; k < WN; ++k) x[i][k] = row + i < T ? widen(e[i][k]) * f[i] : 0.0f;
        u32x4 d[WN][P];
#pragma unroll
        for (int c = 0; c < WN; ++c) {
            float col[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) col[i] = x[i][c];
            operand<P>(col, d[c]);
        }
#pragma unroll
        for (int c = 0; c < WK; ++c) {
            const u32x4 col = w.column(c);
#pragma unroll
            for (int j = 0; j < WN; ++j)
#pragma unroll
                for (int p = 0; p < P; ++p) acc[c][j] = Bf16::mfma(col, d[j][p], acc[c][j]);
        }
    }
    // A lane holds rows WN r to WN r + WN - 1, columns 4 WK g to 4 WK g + 4 WK - 1.
    // Its wavefront turns them over in LDS, 16 rows at a time, so that a store
    // covers whole rows of the tile, 16 bytes a lane: straight from the registers, 16
    // bytes here and there, 4096 x 4096 took 10 to 15 us more.
    float(*mine)[16][kCols + 4] = &turn[threadIdx.x >> 6];
#pragma unroll
    for (int j = 0; j < WN; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < WK; c += 4)
                *reinterpret_cast<f32x4*>(&(*mine)[r][g * 4 * WK + i * WK + c]) =
                    f32x4{acc[c][j][i], acc[c + 1][j][i], acc[c + 2][j][i], acc[c + 3][j][i]};
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (t.bf16) store_tile<uint16_t, kCols>(*mine, t, n0 + j, WN, N, k0, K, lane);
        else store_tile<float, kCols>(*mine, t, n0 + j, WN, N, k0, K, lane);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

template <class E, int P, int WN, int WK>
int few_weight_tiles(Mat dy, Held a, int64_t T, int64_t N, int64_t K, const Target& t,
                     void* stream) {
    const int64_t across = up(K, 16 * WK), blocks = up(up(N, 16 * WN) * across, 4);
    if (blocks * 256 >= (int64_t)1 << 32) return (int)hipErrorInvalidValue;
    return launch(few_weight_kernel<E, P, WN, WK>, dim3((uint32_t)blocks), 256, stream,
                  static_cast<const typename E::T*>(dy.p), dy.ld, a.q, a.ld, a.scale, T, N, K,
                  across, t);
}

// Wider tiles take a's columns once for more of dw, where there are enough of them for
// most SIMDs (bf16, T = 1 and 64, 4096 x 4096: 9 and 12.4 us, narrow ones 11 and 16.7;
// 40 x 2000 x 2000 6.8 and 7.4); narrow ones are done sooner (fp32, 1536 x 384: 4.2 us,
// wide ones 5.2).
template <class E, int P>
int few_weight(Mat dy, Held a, int64_t T, int64_t N, int64_t K, const Target& t, void* stream) {
    return up(N, 32) * up(K, 128) >= 768 ? few_weight_tiles<E, P, 2, 8>(dy, a, T, N, K, t, stream)
                                         : few_weight_tiles<E, P, 2, 4>(dy, a, T, N, K, t, stream);
}

}  // namespace

int64_t few_input_workspace(int64_t T, int64_t N, int64_t K) {
    const int slices = few_input_slices(N, K);
    return slices == 1 ? 0 : slices * T * up(K, 128) * 128 * 4;
}

int launch_few_input(Mat dy, Held b, int64_t T, int64_t N, int64_t K, Mat dx, void* workspace,
                     void* stream) {
    const int slices = few_input_slices(N, K);
    Target t{};
    t.c = dx.p;
    t.ldc = dx.ld;
    t.bf16 = dx.bf16;
    t.ws = workspace;
    t.ldws = up(K, 128) * 128;
    t.slice = T * t.ldws;
    const int parts = parts_of(N, dy.bf16, dx.bf16);
    const int e = dy.bf16 ? parts == 1
                                ? few_input_rows<BF16, 1>(dy, b, T, N, K, t, slices, stream)
                                : few_input_rows<BF16, 2>(dy, b, T, N, K, t, slices, stream)
                  : parts == 1 ? few_input_rows<F32, 1>(dy, b, T, N, K, t, slices, stream)
                               : few_input_rows<F32, 3>(dy, b, T, N, K, t, slices, stream);
    if (e || slices == 1) return e;
    return launch_join<Bf16>(t, T, K, slices, stream);
}

int launch_few_weight(Mat dy, Held a, int64_t T, int64_t N, int64_t K, Mat dw, void* stream) {
    Target t{};
    t.c = dw.p;
    t.ldc = dw.ld;
    t.bf16 = dw.bf16;
    // (a sum of at most 64 values takes all parts: kFewWeight is kFew)
    static_assert(kFewWeight == kFew, "short sums");
    return dy.bf16 ? few_weight<BF16, 2>(dy, a, T, N, K, t, stream)
                   : few_weight<F32, 3>(dy, a, T, N, K, t, stream);
}

}  // namespace q8
}  // namespace cpdp
