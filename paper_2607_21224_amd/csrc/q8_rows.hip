// 8-bit rows of a matrix, and their values read back.
#include "q8_device.h"

namespace cpdp {
namespace q8 {
namespace {

// Both kernels are bound by HBM: each element is read once and written once
// (4 + 1 or 2 + 1 bytes to write a row, 1 + 2 or 1 + 4 to read it back).

template <class E, class Y, int TPR, int CH>
__global__ __launch_bounds__(block_of(TPR)) void rows_kernel(const typename E::T* x, int64_t ldx,
                                                             int64_t T, int D, int8_t* q,
                                                             int64_t ldq, float* scale,
                                                             typename Y::T* y, int64_t ldy) {
    __shared__ RowWords<TPR, 1> words;
    const int64_t row = (int64_t)blockIdx.x * rows_of(TPR) + (int)threadIdx.x / TPR;
    const int lane = (int)threadIdx.x % TPR;
    if (row >= T) return;  // a whole wavefront, in the one-wavefront form only
    float v[CH][kPiece];
    float none;
    uint32_t top[1] = {0};
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int c = (j * TPR + lane) * kPiece;
        if (c < D) {
            load8(x + row * ldx + c, D - c, c, v[j]);
#pragma unroll
            for (int k = 0; k < kPiece; ++k) top[0] = max(top[0], magnitude(v[j][k]));
        }
    }
    row_reduce<TPR, false, 1>(none, top, words);
    const RowScale r = row_scale(__uint_as_float(top[0]));
    if (lane == 0) scale[row] = r.s;
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int c = (j * TPR + lane) * kPiece;
        if (c < D)
            write_piece<Y>(v[j], r, q + row * ldq + c, y == nullptr ? y : y + row * ldy + c, D - c);
    }
}

// A row too long to be held: read twice.
template <class E, class Y>
__global__ __launch_bounds__(1024) void rows_long_kernel(const typename E::T* x, int64_t ldx, int D,
                                                         int8_t* q, int64_t ldq, float* scale,
                                                         typename Y::T* y, int64_t ldy) {
    __shared__ RowWords<1024, 1> words;
    const int64_t row = blockIdx.x;
    float none;
    uint32_t top[1] = {0};
    float v[kPiece];
    for (int c = (int)threadIdx.x * kPiece; c < D; c += 1024 * kPiece) {
        load8(x + row * ldx + c, D - c, c, v);
#pragma unroll
        for (int k = 0; k < kPiece; ++k) top[0] = max(top[0], magnitude(v[k]));
    }
    row_reduce<1024, false, 1>(none, top, words);
    const RowScale r = row_scale(__uint_as_float(top[0]));
    if (threadIdx.x == 0) scale[row] = r.s;
    for (int c = (int)threadIdx.x * kPiece; c < D; c += 1024 * kPiece) {
        load8(x + row * ldx + c, D - c, c, v);
        write_piece<Y>(v, r, q + row * ldq + c, y == nullptr ? y : y + row * ldy + c, D - c);
    }
}

template <class E, class Y>
int rows_typed(Mat x, int64_t T, int D, Held out, Mat y, void* stream) {
    auto* xp = static_cast<const typename E::T*>(x.p);
    auto* yp = static_cast<typename Y::T*>(y.p);
    return with_row_shape(T, D, [&](auto tpr, auto ch) {
        return in_parts(T, 1024, [&](int64_t t, int64_t n) {
            const auto* xt = xp + t * x.ld;
            auto* yt = yp == nullptr ? yp : yp + t * y.ld;
            if constexpr (tpr == 0)
                return launch(rows_long_kernel<E, Y>, dim3((uint32_t)n), 1024, stream, xt, x.ld, D,
                              out.q + t * out.ld, out.ld, out.scale + t, yt, y.ld);
            else
                return launch(rows_kernel<E, Y, tpr, ch>,
                              dim3((uint32_t)((n + rows_of(tpr) - 1) / rows_of(tpr))),
                              block_of(tpr), stream, xt, x.ld, n, D, out.q + t * out.ld, out.ld,
                              out.scale + t, yt, y.ld);
        });
    });
}

// One piece a thread; a block covers 4 rows of 64 pieces.
template <class Y>
__global__ __launch_bounds__(256) void values_kernel(const int8_t* q, int64_t ldq,
                                                     const float* scale, int64_t T, int D,
                                                     int blocks_across, typename Y::T* y,
                                                     int64_t ldy) {
    const int64_t row = (int64_t)(blockIdx.x / blocks_across) * 4 + (threadIdx.x >> 6);
    const int c = ((int)(blockIdx.x % blocks_across) * 64 + (int)(threadIdx.x & 63)) * kPiece;
    if (row >= T || c >= D) return;
    float v[kPiece];
    const float s = scale[row];
    load8(q + row * ldq + c, D - c, c, v);
#pragma unroll
    for (int k = 0; k < kPiece; ++k) v[k] *= s;
    store8(y + row * ldy + c, D - c, v);
}

template <class Y>
int values_typed(Held in, int64_t T, int D, Mat y, void* stream) {
    const int64_t across = (D + 64 * kPiece - 1) / (64 * kPiece);
    return in_parts(T, across * 64, [&](int64_t t, int64_t n) {
        return launch(values_kernel<Y>, dim3((uint32_t)((n + 3) / 4 * across)), 256, stream,
                      in.q + t * in.ld, in.ld, in.scale + t, n, D, (int)across,
                      static_cast<typename Y::T*>(y.p) + t * y.ld, y.ld);
    });
}

}  // namespace

int launch_rows(Mat x, int64_t T, int64_t D, Held out, Mat y, void* stream) {
    const int d = (int)D;
    if (x.bf16)
        return y.bf16 ? rows_typed<BF16, BF16>(x, T, d, out, y, stream)
                      : rows_typed<BF16, F32>(x, T, d, out, y, stream);
    return y.bf16 ? rows_typed<F32, BF16>(x, T, d, out, y, stream)
                  : rows_typed<F32, F32>(x, T, d, out, y, stream);
}

int launch_values(Held in, int64_t T, int64_t D, Mat y, void* stream) {
    return y.bf16 ? values_typed<BF16>(in, T, (int)D, y, stream)
                  : values_typed<F32>(in, T, (int)D, y, stream);
}

}  // namespace q8
}  // namespace cpdp
