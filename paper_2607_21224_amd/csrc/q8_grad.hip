// The two gradients of a product from its 8-bit operands, on the bf16 matrix
// cores.
//
// Both sums run over an index along which the operands' rows do not lie (dx over
// output channels, dw over tokens), and over which the scale of the 8-bit operand
// varies, so it cannot be taken out of the sum.  A first launch per operand lays
// it out with that index contiguous, as bf16 numbers, scale applied; the product
// kernel then reads both from memory straight into LDS.  The extra traffic is
// that of the operands, small beside the product: 2 T N K operations.
//
// A value that one bf16 number cannot hold is laid out as several, each the
// rounding of what the ones before it left, and the product runs over them as
// over a longer sum.  It is the gradient that is scaled and taken apart, q being
// exact in one part: an infinity in it is one part's and meets each q once.
//   bf16 dy   dy * s has 16 significant bits: two parts, exactly
//   fp32 dy   dy * s has 24: three parts
// With bf16 results one part is kept where the sum is long: its relative error, up
// to 2^-8 a value and independent from value to value, averages out to that of
// one rounding of the result.  A sum of few values has nothing to average over,
// and costs as much as a launch does either way: it takes all parts.
#include "q8_gemm.h"

namespace cpdp {
namespace q8 {
namespace {

constexpr int kRound = kStep / 2;  // bf16 numbers in a step: rows are padded to whole steps

// x in P bf16 parts
template <int P>
__device__ __forceinline__ void split(float x, uint16_t (&part)[P]) {
    uint32_t b = narrow2(x, x) << 16;
    if constexpr (P > 1) {
        // a number past the largest bf16 keeps its first bits; nothing is left of
        // an infinity or a NaN
        if ((b & 0x7f800000u) == 0x7f800000u && magnitude(x) < 0x7f800000u)
            b = __float_as_uint(x) & 0xffff0000u;
    }
    part[0] = (uint16_t)(b >> 16);
    const bool finite = magnitude(x) < 0x7f800000u;
    float left = x;
#pragma unroll
    for (int p = 1; p < P; ++p) {
        left = finite ? left - widen(part[p - 1]) : 0.0f;
        part[p] = (uint16_t)narrow2(left, left);
    }
}

// in [R x C] -> out [P][C][Rp], scaled by row, zeros from R to Rp.  A block takes
// 64 x 64 elements through LDS; rows of the LDS tile are 66 numbers long, so that
// neither direction meets one bank with more than two lanes at a time.
template <class In, int P>
__global__ __launch_bounds__(256) void transpose_kernel(const In* in, int64_t ld,
                                                        const float* scale, int64_t R, int64_t C,
                                                        uint16_t* out, int64_t Rp,
                                                        int64_t tiles_r) {
    __shared__ uint16_t tile[P][64][66];
    const int64_t r0 = (int64_t)(blockIdx.x % tiles_r) * 64, c0 = (int64_t)(blockIdx.x / tiles_r) * 64;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = h * 32 + (int)threadIdx.x / 8, c = (int)threadIdx.x % 8 * kPiece;
        const int64_t n = r0 + r < R ? C - c0 - c : 0;
        float x[kPiece] = {};
        if (n > 0) {
            load8(in + (r0 + r) * ld + c0 + c, n < kPiece ? (int)n : kPiece, (int)c0 + c, x);
            if (scale != nullptr) {
                const float s = scale[r0 + r];
#pragma unroll
                for (int k = 0; k < kPiece; ++k) x[k] = k < n ? x[k] * s : 0.0f;
            }
        }
#pragma unroll
        for (int k = 0; k < kPiece; ++k) {
            uint16_t part[P];
            split<P>(x[k], part);
#pragma unroll
            for (int p = 0; p < P; ++p) tile[p][c + k][r] = part[p];
        }
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c = h * 32 + (int)threadIdx.x / 8, r = (int)threadIdx.x % 8 * kPiece;
            if (c0 + c >= C) continue;
            u32x4 v;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                v[k] = *reinterpret_cast<const uint32_t*>(&tile[p][c][r + 2 * k]);
            *reinterpret_cast<u32x4*>(out + ((int64_t)p * C + c0 + c) * Rp + r0 + r) = v;
        }
}

// in [R x C] -> out [P][R][Cp], scaled by column, zeros from C to Cp
template <class In, int P>
__global__ __launch_bounds__(256) void spread_kernel(const In* in, int64_t ld, const float* scale,
                                                     int64_t R, int64_t C, uint16_t* out,
                                                     int64_t Cp) {
    const int64_t across = Cp / kPiece;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t r = i / across, c = i % across * kPiece;
    if (r >= R) return;
    float x[kPiece] = {};
    const int64_t n = C - c;
    if (n > 0) load8(in + r * ld + c, n < kPiece ? (int)n : kPiece, (int)c, x);
    uint16_t part[kPiece][P];
#pragma unroll
    for (int k = 0; k < kPiece; ++k) {
        if (scale != nullptr && k < n) x[k] *= scale[c + k];
        split<P>(x[k], part[k]);
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
        u32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            v[k] = (uint32_t)part[2 * k][p] | (uint32_t)part[2 * k + 1][p] << 16;
        *reinterpret_cast<u32x4*>(out + ((int64_t)p * R + r) * Cp + c) = v;
    }
}

__global__ __launch_bounds__(256) void zero_rows_kernel(char* p, int64_t ld, int64_t R,
                                                        int64_t row) {
    // elements are 2 or 4 bytes: 2 at a time
    const int64_t across = row / 2;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i / across >= R) return;
    *reinterpret_cast<uint16_t*>(p + i / across * ld + i % across * 2) = 0;
}

constexpr int64_t kMostItems = ((int64_t)1 << 32) - 4096;

template <class In, int P>
int transpose(const In* in, int64_t ld, const float* scale, int64_t R, int64_t C, uint16_t* out,
              int64_t Rp, void* stream) {
    const int64_t tiles_r = Rp / 64, blocks = tiles_r * up(C, 64);
    if (blocks > kMostItems / 256) return (int)hipErrorInvalidValue;
    return launch(transpose_kernel<In, P>, dim3((uint32_t)blocks), 256, stream, in, ld, scale, R, C,
                  out, Rp, tiles_r);
}
template <class In>
int transpose_parts(int parts, const In* in, int64_t ld, const float* scale, int64_t R, int64_t C,
                    uint16_t* out, int64_t Rp, void* stream) {
    if (parts == 1) return transpose<In, 1>(in, ld, scale, R, C, out, Rp, stream);
    if (parts == 2) return transpose<In, 2>(in, ld, scale, R, C, out, Rp, stream);
    return transpose<In, 3>(in, ld, scale, R, C, out, Rp, stream);
}

template <class In, int P>
int spread(const In* in, int64_t ld, const float* scale, int64_t R, int64_t C, uint16_t* out,
           int64_t Cp, void* stream) {
    const int64_t items = R * (Cp / kPiece);
    if (items > kMostItems) return (int)hipErrorInvalidValue;
    return launch(spread_kernel<In, P>, dim3((uint32_t)up(items, 256)), 256, stream, in, ld, scale,
                  R, C, out, Cp);
}

template <class In>
int spread_parts(int parts, const In* in, int64_t ld, const float* scale, int64_t R, int64_t C,
                 uint16_t* out, int64_t Cp, void* stream) {
    if (parts == 1) return spread<In, 1>(in, ld, scale, R, C, out, Cp, stream);
    if (parts == 2) return spread<In, 2>(in, ld, scale, R, C, out, Cp, stream);
    return spread<In, 3>(in, ld, scale, R, C, out, Cp, stream);
}

int zero_rows(Mat c, int64_t R, int64_t C, void* stream) {
    const int64_t e = c.bf16 ? 2 : 4;
    return in_parts(R, up(C * e / 2, 1), [&](int64_t r, int64_t n) {
        return launch(zero_rows_kernel, dim3((uint32_t)up(n * (C * e / 2), 256)), 256, stream,
                      static_cast<char*>(c.p) + r * c.ld * e, c.ld * e, n, C * e);
    });
}

// A sum of at most so many values (one step) is taken with all parts.
constexpr int64_t kFew = 64;

// How the operands of a gradient are laid out.  One part: a bf16 gradient stays as
// it is and the 8-bit operand is scaled; otherwise dy is scaled.
struct Layout {
    int parts;         // of dy
    bool held_scaled;  // the 8-bit operand takes the scale
    int64_t Rp;        // reduced size, padded
    bool dy_in_place;  // dy is read where it is
    int64_t dy_bytes, held_bytes;
};
Layout layout(int64_t rows_dy, int64_t rows_held, int64_t R, bool dy_bf16, bool out_bf16,
              bool dy_rows_run_along) {
    Layout l;
    const bool one = out_bf16 && R > kFew;
    l.parts = one ? 1 : dy_bf16 ? 2 : 3;
    l.held_scaled = one && dy_bf16;
    l.Rp = up(R, kRound) * kRound;
    l.dy_in_place = l.held_scaled && dy_rows_run_along && l.Rp == R;
    l.dy_bytes = l.dy_in_place ? 0 : l.parts * rows_dy * l.Rp * 2;
    l.held_bytes = rows_held * l.Rp * 2;
    return l;
}
int64_t workspace_of(const Layout& l, int64_t M, int64_t N) {
    return l.dy_bytes + l.held_bytes + slices_bytes(M, N, l.Rp * 2 / kStep * l.parts);
}

// c [M x N] = sum over the laid-out index of dy and the 8-bit operand
int product(const Layout& l, const void* dy, int64_t ld_dy, int64_t M, const void* held, int64_t N,
            Mat c, void* slices, void* stream) {
    Operands o{};
    o.a = static_cast<const char*>(dy);
    o.b = static_cast<const char*>(held);
    o.lda = ld_dy * 2;
    o.ldb = l.Rp * 2;
    o.a_part = M * l.Rp * 2;
    o.M = M;
    o.N = N;
    o.row = (int)(l.Rp * 2);
    o.parts = l.parts;
    Target t{};
    t.c = c.p;
    t.ldc = c.ld;
    t.bf16 = c.bf16;
    return launch_gemm<Bf16>(o, t, slices, stream);
}

}  // namespace

int64_t grad_input_workspace(int64_t T, int64_t N, int64_t K, bool dy_bf16, bool out_bf16) {
    return workspace_of(layout(T, K, N, dy_bf16, out_bf16, true), T, K);
}

int launch_grad_input(Mat dy, Held b, int64_t T, int64_t N, int64_t K, Mat dx, void* workspace,
                      void* stream) {
    if (N == 0) return zero_rows(dx, T, K, stream);
    const Layout l = layout(T, K, N, dy.bf16, dx.bf16, true);
    char* ws = static_cast<char*>(workspace);
    uint16_t* dyw = reinterpret_cast<uint16_t*>(ws);
    uint16_t* bw = reinterpret_cast<uint16_t*>(ws + l.dy_bytes);
    const float* dy_scale = l.held_scaled ? nullptr : b.scale;
    int e = 0;
    if (!l.dy_in_place)
        e = dy.bf16 ? spread_parts(l.parts, static_cast<const uint16_t*>(dy.p), dy.ld, dy_scale, T,
                                   N, dyw, l.Rp, stream)
                    : spread_parts(l.parts, static_cast<const float*>(dy.p), dy.ld, dy_scale, T, N,
                                   dyw, l.Rp, stream);
    if (e) return e;
    if (int f = transpose<int8_t, 1>(b.q, b.ld, l.held_scaled ? b.scale : nullptr, N, K, bw, l.Rp,
                                     stream))
        return f;
    return product(l, l.dy_in_place ? dy.p : dyw, l.dy_in_place ? dy.ld : l.Rp, T, bw, K, dx,
                   ws + l.dy_bytes + l.held_bytes, stream);
}

int64_t grad_weight_workspace(int64_t T, int64_t N, int64_t K, bool dy_bf16, bool out_bf16) {
    return workspace_of(layout(N, K, T, dy_bf16, out_bf16, false), N, K);
}

int launch_grad_weight(Mat dy, Held a, int64_t T, int64_t N, int64_t K, Mat dw, void* workspace,
                       void* stream) {
    if (T == 0) return zero_rows(dw, N, K, stream);
    const Layout l = layout(N, K, T, dy.bf16, dw.bf16, false);
    char* ws = static_cast<char*>(workspace);
    uint16_t* dyw = reinterpret_cast<uint16_t*>(ws);
    uint16_t* aw = reinterpret_cast<uint16_t*>(ws + l.dy_bytes);
    const float* dy_scale = l.held_scaled ? nullptr : a.scale;
    const int e = dy.bf16 ? transpose_parts(l.parts, static_cast<const uint16_t*>(dy.p), dy.ld,
                                            dy_scale, T, N, dyw, l.Rp, stream)
                          : transpose_parts(l.parts, static_cast<const float*>(dy.p), dy.ld,
                                            dy_scale, T, N, dyw, l.Rp, stream);
    if (e) return e;
    if (int f = transpose<int8_t, 1>(a.q, a.ld, l.held_scaled ? a.scale : nullptr, T, K, aw, l.Rp,
                                     stream))
        return f;
    return product(l, dyw, l.Rp, N, aw, K, dw, ws + l.dy_bytes + l.held_bytes, stream);
}

}  // namespace q8
}  // namespace cpdp
