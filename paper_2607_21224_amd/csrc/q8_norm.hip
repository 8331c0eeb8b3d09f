// Root-mean-square norm with the residual's addition and 8-bit output, and its
// backward pass.
#include "q8_device.h"

namespace cpdp {
namespace q8 {
namespace {

__device__ __forceinline__ void load_w(const void* w, bool bf16, int c, int n, float (&x)[kPiece]) {
    if (bf16) load8(static_cast<const uint16_t*>(w) + c, n, c, x);
    else load8(static_cast<const float*>(w) + c, n, c, x);
}

// h and p = h w of one piece; h is stored where there is a residual
template <class E>
__device__ __forceinline__ void norm_piece(const typename E::T* x, const typename E::T* r,
                                           typename E::T* h, const void* w, bool w_bf16, int c,
                                           int n, float& sum, uint32_t& top, float (&p)[kPiece]) {
    float a[kPiece], b[kPiece];
    load8(x, n, c, a);
    load_w(w, w_bf16, c, n, p);
    if (r != nullptr) {
        load8(r, n, c, b);
#pragma unroll
        for (int k = 0; k < kPiece; ++k) a[k] = stored<E>(a[k] + b[k]);
        store8(h, n, a);
    }
#pragma unroll
    for (int k = 0; k < kPiece; ++k) {
        sum = fmaf(a[k], a[k], sum);
        p[k] = a[k] * p[k];
        top = max(top, magnitude(p[k]));
    }
}

// 1 / sqrt(mean + eps) and the scale of the row v = p rstd.  Rounding keeps
// order, so max |v| is max |p| times rstd, rounded: the sum and the maximum come
// out of one pass over the row.
struct NormScale {
    float rstd;
    RowScale r;
};
__device__ __forceinline__ NormScale norm_scale(float sum, uint32_t top, int D, float eps) {
    const float rstd = 1.0f / sqrtf(sum / (float)D + eps);
    return {rstd, row_scale(__uint_as_float(top) * rstd)};
}

// Bound by HBM: with a residual and the values in bf16, 9 bytes an element in
// bf16 and 15 in fp32, each moved once.
template <class E, class Y, int TPR, int CH>
__global__ __launch_bounds__(block_of(TPR)) void norm_kernel(
    const typename E::T* x, int64_t ldx, const typename E::T* res, int64_t ldr, const void* w,
    bool w_bf16, float eps, int64_t T, int D, typename E::T* h, int64_t ldh, int8_t* q,
    int64_t ldq, float* scale, float* rstd, typename Y::T* y, int64_t ldy) {
    __shared__ RowWords<TPR, 1> words;
    const int64_t row = (int64_t)blockIdx.x * rows_of(TPR) + (int)threadIdx.x / TPR;
    const int lane = (int)threadIdx.x % TPR;
    if (row >= T) return;  // a whole wavefront, in the one-wavefront form only
    float p[CH][kPiece], sum = 0.0f;
    uint32_t top[1] = {0};
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int c = (j * TPR + lane) * kPiece;
        if (c < D)
            norm_piece<E>(x + row * ldx + c, res == nullptr ? res : res + row * ldr + c,
                          h + row * ldh + c, w, w_bf16, c, D - c, sum, top[0], p[j]);
    }
    row_reduce<TPR, true, 1>(sum, top, words);
    const NormScale s = norm_scale(sum, top[0], D, eps);
    if (lane == 0) {
        scale[row] = s.r.s;
        if (rstd != nullptr) rstd[row] = s.rstd;
    }
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int c = (j * TPR + lane) * kPiece;
        if (c < D) {
#pragma unroll
            for (int k = 0; k < kPiece; ++k) p[j][k] *= s.rstd;
            write_piece<Y>(p[j], s.r, q + row * ldq + c, y == nullptr ? y : y + row * ldy + c,
                           D - c);
        }
    }
}

// A row too long to be held: h is read again, as it was stored.
template <class E, class Y>
__global__ __launch_bounds__(1024) void norm_long_kernel(
    const typename E::T* x, int64_t ldx, const typename E::T* res, int64_t ldr, const void* w,
    bool w_bf16, float eps, int D, typename E::T* h, int64_t ldh, int8_t* q, int64_t ldq,
    float* scale, float* rstd, typename Y::T* y, int64_t ldy) {
    __shared__ RowWords<1024, 1> words;
    const int64_t row = blockIdx.x;
    float p[kPiece], v[kPiece], sum = 0.0f;
    uint32_t top[1] = {0};
    for (int c = (int)threadIdx.x * kPiece; c < D; c += 1024 * kPiece)
        norm_piece<E>(x + row * ldx + c, res == nullptr ? res : res + row * ldr + c,
                      h + row * ldh + c, w, w_bf16, c, D - c, sum, top[0], p);
    row_reduce<1024, true, 1>(sum, top, words);
    const NormScale s = norm_scale(sum, top[0], D, eps);
    if (threadIdx.x == 0) {
        scale[row] = s.r.s;
        if (rstd != nullptr) rstd[row] = s.rstd;
    }
    // every thread reads back what it wrote itself
    const typename E::T* hr = res == nullptr ? x + row * ldx : h + row * ldh;
    for (int c = (int)threadIdx.x * kPiece; c < D; c += 1024 * kPiece) {
        load8(hr + c, D - c, c, v);
        load_w(w, w_bf16, c, D - c, p);
#pragma unroll
        for (int k = 0; k < kPiece; ++k) p[k] = v[k] * p[k] * s.rstd;
        write_piece<Y>(p, s.r, q + row * ldq + c, y == nullptr ? y : y + row * ldy + c, D - c);
    }
}

template <class E, class Y>
int norm_typed(Mat x, Mat res, const void* w, bool w_bf16, float eps, int64_t T, int D, Mat h,
               Held out, float* rstd, Mat y, void* stream) {
    using ET = typename E::T;
    using YT = typename Y::T;
    return with_row_shape(T, D, [&](auto tpr, auto ch) {
        return in_parts(T, 1024, [&](int64_t t, int64_t n) {
            const ET* xt = static_cast<const ET*>(x.p) + t * x.ld;
            const ET* rt = res.p == nullptr ? nullptr : static_cast<const ET*>(res.p) + t * res.ld;
            ET* ht = res.p == nullptr ? nullptr : static_cast<ET*>(h.p) + t * h.ld;
            YT* yt = y.p == nullptr ? nullptr : static_cast<YT*>(y.p) + t * y.ld;
            float* st = rstd == nullptr ? nullptr : rstd + t;
            if constexpr (tpr == 0)
                return launch(norm_long_kernel<E, Y>, dim3((uint32_t)n), 1024, stream, xt, x.ld, rt,
                              res.ld, w, w_bf16, eps, D, ht, h.ld, out.q + t * out.ld, out.ld,
                              out.scale + t, st, yt, y.ld);
            else
                return launch(norm_kernel<E, Y, tpr, ch>,
                              dim3((uint32_t)((n + rows_of(tpr) - 1) / rows_of(tpr))),
                              block_of(tpr), stream, xt, x.ld, rt, res.ld, w, w_bf16, eps, n, D, ht,
                              h.ld, out.q + t * out.ld, out.ld, out.scale + t, st, yt, y.ld);
        });
    });
}

// ---- backward ---------------------------------------------------------------------
//
// dx = rstd (dy w - n mean(dy w n)) + dres with n = h rstd, a row at a time, and
// dw = sum over rows of dy n.  A block takes every G-th row and keeps its
// columns' part of dw in registers (where a wavefront holds a row, the block's four
// meet in LDS); the G parts go to the workspace and are added in their order by a
// second launch, so the result does not depend on which block ran first (few and short
// rows: norm_bwd_one_kernel).  Joining the wavefronts' own parts, four times as many,
// made 1576 x 384 fp32 9.4 us and 16384 x 512 bf16 22, now 7.1 and 15.5 (calls that
// follow each other, as in the figures below).

// Floats from part to part: whole 16-byte pieces.
__host__ __device__ constexpr int64_t parts_ld(int64_t D) { return (D + 3) / 4 * 4; }

template <class E, int TPR, int CH>
__global__ __launch_bounds__(block_of(TPR)) void norm_bwd_kernel(
    const typename E::T* dy, int64_t lddy, const typename E::T* h, int64_t ldh,
    const typename E::T* dres, int64_t lddres, const void* w, bool w_bf16, const float* rstd,
    int64_t T, int D, typename E::T* dx, int64_t lddx, float* parts) {
    __shared__ RowWords<TPR, 0> words[2];
    const int64_t group = (int64_t)blockIdx.x * rows_of(TPR) + (int)threadIdx.x / TPR;
    const int64_t groups = (int64_t)gridDim.x * rows_of(TPR);
    const int lane = (int)threadIdx.x % TPR;
    float acc[CH][kPiece] = {}, wv[CH][kPiece];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int c = (j * TPR + lane) * kPiece;
        load_w(w, w_bf16, c < D ? c : 0, c < D ? D - c : 0, wv[j]);
    }
    // a row's dy and h are sent for while the row before is worked on
    Raw<E> g[CH], n[CH], r[CH];
    const auto fetch = [&](int64_t row) {
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int c = (j * TPR + lane) * kPiece;
            if (c < D) {
                g[j].load(dy + row * lddy + c, D - c, c);
                n[j].load(h + row * ldh + c, D - c, c);
            }
        }
    };
    if (group < T) fetch(group);
    int turn = 0;
    for (int64_t row = group; row < T; row += groups, turn ^= 1) {
        const float rs = rstd[row];
        float sum = 0.0f;
        uint32_t none[1];
        Raw<E> g0[CH], n0[CH];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int c = (j * TPR + lane) * kPiece;
            g0[j] = g[j];
            n0[j] = n[j];
            if (c < D && dres != nullptr) r[j].load(dres + row * lddres + c, D - c, c);
        }
        if (row + groups < T) fetch(row + groups);
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            if ((j * TPR + lane) * kPiece < D) {
#pragma unroll
                for (int k = 0; k < kPiece; ++k) {
                    const float nk = n0[j][k] * rs;
                    acc[j][k] = fmaf(g0[j][k], nk, acc[j][k]);
                    sum = fmaf(g0[j][k] * wv[j][k], nk, sum);
                }
            }
        }
        row_reduce<TPR, true, 0>(sum, none, words[turn]);
        const float mean = sum / (float)D;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int c = (j * TPR + lane) * kPiece;
            if (c < D) {
                float d[kPiece];
#pragma unroll
                for (int k = 0; k < kPiece; ++k)
                    d[k] = fmaf(fmaf(-(n0[j][k] * rs), mean, g0[j][k] * wv[j][k]), rs,
                                dres != nullptr ? r[j][k] : 0.0f);
                store8(dx + row * lddx + c, D - c, d);
            }
        }
    }
    float* part = parts + blockIdx.x * parts_ld(D);
    if constexpr (TPR == 64) {
        static_assert(CH == 1, "one piece a lane");
        __shared__ f32x4 others[3][2][64];
        const int wave = (int)threadIdx.x / 64;
        if (wave > 0) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                others[wave - 1][h][lane] =
                    f32x4{acc[0][4 * h], acc[0][4 * h + 1], acc[0][4 * h + 2], acc[0][4 * h + 3]};
        }
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int i = 0; i < 3; ++i)
#pragma unroll
            for (int k = 0; k < kPiece; ++k) acc[0][k] += others[i][k / 4][lane][k % 4];
    }
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int c = (j * TPR + lane) * kPiece;
        if (c < D) store8(part + c, D - c, acc[j]);
    }
}

// Both in one launch, for few and short rows: the first blocks take 8 columns of dw
// each, over all rows, the others a row of dx (four, where a wavefront holds one).  dy
// and h are read twice, by the first blocks a piece here and there, which costs less
// than a second launch as long as they are small (bwd_one).
template <class E, int TPR, int CH>
__global__ __launch_bounds__(block_of(TPR)) void norm_bwd_one_kernel(
    const typename E::T* dy, int64_t lddy, const typename E::T* h, int64_t ldh,
    const typename E::T* dres, int64_t lddres, const void* w, bool w_bf16, const float* rstd,
    int T, int D, typename E::T* dx, int64_t lddx, void* dw, bool dw_bf16, int dw_blocks) {
    constexpr int kThreads = block_of(TPR), kWaves = kThreads / 64;
    if ((int)blockIdx.x < dw_blocks) {
        __shared__ float sums[kWaves][kPiece];
        const int c = (int)blockIdx.x * kPiece;
        float acc[kPiece] = {};
        constexpr int U = 4;  // rows on their way
        for (int row = (int)threadIdx.x; row < T; row += U * kThreads) {
            Raw<E> g[U], n[U];
            float rs[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = row + u * kThreads < T ? row + u * kThreads : row;
                g[u].load(dy + at * lddy + c, D - c, c);
                n[u].load(h + at * ldh + c, D - c, c);
                rs[u] = rstd[at];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool there = row + u * kThreads < T;
#pragma unroll
                for (int k = 0; k < kPiece; ++k)
                    acc[k] = there ? fmaf(g[u][k], n[u][k] * rs[u], acc[k]) : acc[k];
            }
        }
#pragma unroll
        for (int k = 0; k < kPiece; ++k) acc[k] = wave_reduce(acc[k], Add());
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < kPiece; ++k) sums[threadIdx.x >> 6][k] = acc[k];
        }
        __syncthreads();
        const int k = (int)threadIdx.x;
        if (k >= kPiece || c + k >= D) return;
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) s += sums[i][k];
        if (dw_bf16) narrow(s, static_cast<uint16_t*>(dw) + c + k);
        else static_cast<float*>(dw)[c + k] = s;
        return;
    }
    __shared__ RowWords<TPR, 0> words;
    const int row =
        ((int)blockIdx.x - dw_blocks) * rows_of(TPR) + (int)threadIdx.x / TPR;
    const int lane = (int)threadIdx.x % TPR;
    if (row >= T) return;  // a whole wavefront, in the one-wavefront form only
    const float rs = rstd[row];
    float sum = 0.0f, gw[CH][kPiece], nv[CH][kPiece], r[CH][kPiece] = {};
    uint32_t none[1];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int c = (j * TPR + lane) * kPiece;
        if (c < D) {
            float wv[kPiece];
            load8(dy + row * lddy + c, D - c, c, gw[j]);
            load8(h + row * ldh + c, D - c, c, nv[j]);
            load_w(w, w_bf16, c, D - c, wv);
            if (dres != nullptr) load8(dres + row * lddres + c, D - c, c, r[j]);
#pragma unroll
            for (int k = 0; k < kPiece; ++k) {
                nv[j][k] *= rs;
                gw[j][k] *= wv[k];
                sum = fmaf(gw[j][k], nv[j][k], sum);
            }
        }
    }
    row_reduce<TPR, true, 0>(sum, none, words);
    const float mean = sum / (float)D;
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int c = (j * TPR + lane) * kPiece;
        if (c < D) {
            float d[kPiece];
#pragma unroll
            for (int k = 0; k < kPiece; ++k)
                d[k] = fmaf(fmaf(-nv[j][k], mean, gw[j][k]), rs, r[j][k]);
            store8(dx + row * lddx + c, D - c, d);
        }
    }
}

// A row too long to be held: dx reads it twice, dw takes it column by column.
template <class E>
__global__ __launch_bounds__(1024) void norm_bwd_long_kernel(
    const typename E::T* dy, int64_t lddy, const typename E::T* h, int64_t ldh,
    const typename E::T* dres, int64_t lddres, const void* w, bool w_bf16, const float* rstd, int D,
    typename E::T* dx, int64_t lddx) {
    __shared__ RowWords<1024, 0> words;
    const int64_t row = blockIdx.x;
    const float rs = rstd[row];
    float sum = 0.0f, g[kPiece], n[kPiece], v[kPiece];
    uint32_t none[1];
    for (int c = (int)threadIdx.x * kPiece; c < D; c += 1024 * kPiece) {
        load8(dy + row * lddy + c, D - c, c, g);
        load8(h + row * ldh + c, D - c, c, n);
        load_w(w, w_bf16, c, D - c, v);
#pragma unroll
        for (int k = 0; k < kPiece; ++k) sum = fmaf(g[k] * v[k], n[k] * rs, sum);
    }
    row_reduce<1024, true, 0>(sum, none, words);
    const float mean = sum / (float)D;
    for (int c = (int)threadIdx.x * kPiece; c < D; c += 1024 * kPiece) {
        float d[kPiece] = {};
        load8(dy + row * lddy + c, D - c, c, g);
        load8(h + row * ldh + c, D - c, c, n);
        load_w(w, w_bf16, c, D - c, v);
        if (dres != nullptr) load8(dres + row * lddres + c, D - c, c, d);
#pragma unroll
        for (int k = 0; k < kPiece; ++k)
            d[k] = fmaf(fmaf(-(n[k] * rs), mean, g[k] * v[k]), rs, d[k]);
        store8(dx + row * lddx + c, D - c, d);
    }
}

template <class E>
__global__ __launch_bounds__(256) void norm_dw_kernel(const typename E::T* dy, int64_t lddy,
                                                      const typename E::T* h, int64_t ldh,
                                                      const float* rstd, int64_t T, int D,
                                                      float* parts) {
    const int c = ((int)blockIdx.x * 256 + (int)threadIdx.x) * kPiece;
    if (c >= D) return;
    float acc[kPiece] = {}, g[kPiece], n[kPiece];
    for (int64_t row = blockIdx.y; row < T; row += gridDim.y) {
        const float rs = rstd[row];
        load8(dy + row * lddy + c, D - c, c, g);
        load8(h + row * ldh + c, D - c, c, n);
#pragma unroll
        for (int k = 0; k < kPiece; ++k) acc[k] = fmaf(g[k], n[k] * rs, acc[k]);
    }
    store8(parts + blockIdx.y * parts_ld(D) + c, D - c, acc);
}

// dw <- the sum of `groups` parts: 32 columns a block, 32 threads a column, each
// with 8 parts on their way at a time.
template <class W>
__global__ __launch_bounds__(1024) void norm_dw_join_kernel(const float* parts, int groups, int D,
                                                            typename W::T* dw) {
    __shared__ float sums[32][33];
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int64_t c0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 32;
    const int64_t c = c0 + lane, ld = parts_ld(D);
    float s = 0.0f;
    if (c < D) {
        const float* p = parts + part * ld + c;
        int left = (groups - part + 31) / 32;
        for (; left >= 8; left -= 8, p += 8 * 32 * ld) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = p[32 * i * ld];
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];
        }
        if (left > 0) {
            float v[7];
#pragma unroll
            for (int i = 0; i < 7; ++i) v[i] = p[(i < left ? 32 * i : 0) * ld];
#pragma unroll
            for (int i = 0; i < 7; ++i) s += i < left ? v[i] : 0.0f;
        }
    }
    sums[part][lane] = s;
    __syncthreads();
    // a wavefront's half takes a column: its 32 sums, added pairwise
    s = sums[lane][part];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) s += __shfl_xor(s, off);
    const int64_t col = c0 + part;
    if (lane == 0 && col < D) narrow(s, dw + col);
}

// How the backward pass holds a row (it keeps three numbers a column, so fewer
// columns a thread than the forward pass).
template <class F>
int with_bwd_shape(int64_t D, F f) {
    if (D <= 512) return f(Int<64>(), Int<1>());
    if (D <= 2048) return f(Int<256>(), Int<1>());
    if (D <= 4096) return f(Int<256>(), Int<2>());
    if (D <= 8192) return f(Int<512>(), Int<2>());
    if (D <= 16384) return f(Int<1024>(), Int<2>());
    return f(Int<0>(), Int<0>());
}

// Blocks of the backward pass, each with one part of dw: four a CU,
// and as many as there are rows for where they are fewer.
int64_t bwd_blocks(int64_t T, int rows) {
    const int64_t blocks = (T + rows - 1) / rows;
    return blocks < 1 ? 1 : blocks > 1024 ? 1024 : blocks;
}

// Whether one launch takes both: as long as a thread has two turns of four rows, a
// block's 256 threads suffice for a row, and dy is so small that reading it and h again
// is nothing.  In us, two launches and one: 256 x 384 fp32 7.3 and 5.0, 1576 x 384 bf16
// 7.4 and 5.5; but 1576 x 384 fp32 (2.4 MB) 7.3 and 9.7, 3000 x 96 7.3 and 8.5.  Rows
// past 4096 columns, for which a block has 512 threads and dw's blocks most of them idle,
// go either way (64 x 7264 bf16 7.6 and 6.2, 5 x 8191 fp32 7.7 and 8.7) and take two.
bool bwd_one(int64_t T, int64_t D, int64_t element) {
    return T <= 2048 && D <= 4096 && T * D * element <= 3 << 19;
}

template <class E>
int norm_bwd_typed(Mat dy, Mat h, Mat dres, const void* w, bool w_bf16, const float* rstd,
                   int64_t T, int D, Mat dx, void* dw, bool dw_bf16, float* parts, void* stream) {
    using ET = typename E::T;
    const ET *dyp = static_cast<const ET*>(dy.p), *hp = static_cast<const ET*>(h.p),
             *rp = static_cast<const ET*>(dres.p);
    ET* dxp = static_cast<ET*>(dx.p);
    int groups = 0;
    bool done = false;
    int e = with_bwd_shape(D, [&](auto tpr, auto ch) {
        if constexpr (tpr == 0) {
            groups = (int)bwd_blocks(T, 4);
            if (int f = in_parts(T, 1024, [&](int64_t t, int64_t n) {
                    return launch(norm_bwd_long_kernel<E>, dim3((uint32_t)n), 1024, stream,
                                  dyp + t * dy.ld, dy.ld, hp + t * h.ld, h.ld,
                                  rp == nullptr ? rp : rp + t * dres.ld, dres.ld, w, w_bf16,
                                  rstd + t, D, dxp + t * dx.ld, dx.ld);
                }))
                return f;
            return launch(norm_dw_kernel<E>,
                          dim3((uint32_t)((D + 256 * kPiece - 1) / (256 * kPiece)),
                               (uint32_t)groups),
                          256, stream, dyp, dy.ld, hp, h.ld, rstd, T, D, parts);
        } else {
            if constexpr (tpr <= 256) {  // (rows of up to 4096)
                if (bwd_one(T, D, sizeof(ET))) {
                    done = true;
                    const int dw_blocks = (D + kPiece - 1) / kPiece;
                    const int64_t rows = (T + rows_of(tpr) - 1) / rows_of(tpr);
                    return launch(norm_bwd_one_kernel<E, tpr, ch>,
                                  dim3((uint32_t)(dw_blocks + rows)), block_of(tpr), stream, dyp,
                                  dy.ld, hp, h.ld, rp, dres.ld, w, w_bf16, rstd, (int)T, D, dxp,
                                  dx.ld, dw, dw_bf16, dw_blocks);
                }
            }
            groups = (int)bwd_blocks(T, rows_of(tpr));
            return launch(norm_bwd_kernel<E, tpr, ch>, dim3((uint32_t)groups), block_of(tpr),
                          stream, dyp, dy.ld, hp, h.ld, rp, dres.ld, w, w_bf16, rstd, T, D, dxp,
                          dx.ld, parts);
        }
    });
    if (e || done) return e;
    // (fewer than 2^32 work items in a direction of the grid)
    const int64_t across = ((int64_t)D + 31) / 32, most = 1 << 21;
    const dim3 grid((uint32_t)(across < most ? across : most),
                    (uint32_t)((across + most - 1) / most));
    return dw_bf16 ? launch(norm_dw_join_kernel<BF16>, grid, 1024, stream, parts, groups, D,
                            static_cast<uint16_t*>(dw))
                   : launch(norm_dw_join_kernel<F32>, grid, 1024, stream, parts, groups, D,
                            static_cast<float*>(dw));
}

}  // namespace

int launch_norm(Mat x, Mat residual, const void* w, bool w_bf16, float eps, int64_t T, int64_t D,
                Mat h, Held out, float* rstd, Mat y, void* stream) {
    const int d = (int)D;
    if (x.bf16)
        return y.bf16
                   ? norm_typed<BF16, BF16>(x, residual, w, w_bf16, eps, T, d, h, out, rstd, y,
                                            stream)
                   : norm_typed<BF16, F32>(x, residual, w, w_bf16, eps, T, d, h, out, rstd, y,
                                           stream);
    return y.bf16 ? norm_typed<F32, BF16>(x, residual, w, w_bf16, eps, T, d, h, out, rstd, y,
                                          stream)
                  : norm_typed<F32, F32>(x, residual, w, w_bf16, eps, T, d, h, out, rstd, y,
                                         stream);
}

int64_t norm_bwd_workspace(int64_t T, int64_t D) {
    int64_t groups = 0;
    with_bwd_shape(D, [&](auto tpr, auto) {
        groups = bwd_blocks(T, tpr == 0 ? 4 : rows_of(tpr));
        return 0;
    });
    return groups * parts_ld(D) * 4;
}

int launch_norm_bwd(Mat dy, Mat h, Mat dres, const void* w, bool w_bf16, const float* rstd,
                    int64_t T, int64_t D, Mat dx, void* dw, bool dw_bf16, void* workspace,
                    void* stream) {
    float* parts = static_cast<float*>(workspace);
    return dy.bf16 ? norm_bwd_typed<BF16>(dy, h, dres, w, w_bf16, rstd, T, (int)D, dx, dw, dw_bf16,
                                          parts, stream)
                   : norm_bwd_typed<F32>(dy, h, dres, w, w_bf16, rstd, T, (int)D, dx, dw, dw_bf16,
                                         parts, stream);
}

}  // namespace q8
}  // namespace cpdp
