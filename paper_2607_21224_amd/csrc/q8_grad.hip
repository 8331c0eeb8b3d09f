// The two gradients of a product from its 8-bit operands, on the bf16 matrix
// cores.
//
// Both sums run over an index along which the operands' rows do not lie (dx over
// output channels, dw over tokens), and over which the scale of the 8-bit operand
// varies, so it cannot be taken out of the sum.  A first launch lays
// both out with that index contiguous, as bf16 numbers (dy in parts), scale
// applied; the product kernel then reads them from memory straight into LDS.  The
// extra traffic is that of the operands, small beside the product's 2 T N K
// operations.
#include "q8_grad_f32.h"
#include "q8_grad_gemm.h"

namespace cpdp {
namespace q8 {
namespace {

constexpr int kRound = kStep / 2;  // bf16 numbers in a step: rows are padded to whole steps

// What is laid out: [R x C], with a scale per row (transposed) or per column, or
// null.
struct Source {
    const void* p;
    int64_t ld;
    const float* scale;
    int64_t R, C;
    uint16_t* out;
    int64_t pad;     // the output's row length, a multiple of 64
    int64_t blocks;  // that lay it out
};

// Columns of a block of the transposing layout: 8 threads across, 16 bytes or more
// of a row each.
template <class In>
constexpr int tile_cols() {
    return sizeof(In) == 1 ? 128 : 64;
}

// LDS of one: columns of 32 pairs of rows, a word more, so that the 64 lanes of a
// wavefront, 8 pairs of rows and 8 columns 8 apart, write to 64 banks.
template <int P, int COLS>
using Tile = uint32_t[P][COLS][33];

// in [R x C] -> out [P][C][pad], scaled by row, zeros from R to pad.  A block takes
// 64 rows through LDS, two neighbouring ones a thread.  All that a thread reads is
// sent for before any of it is used (WHOLE: and without a branch, as all of the
// block's rows and columns are there): one after the other, its rows and their scales
// were 8 waits for memory, and the layout of 1576 x 1536 fp32 took 11 us.
template <class E, int P, bool WHOLE>
__device__ __forceinline__ void turn(const Source& s, int64_t r0, int64_t c0,
                                     Tile<P, tile_cols<typename E::T>()>& tile) {
    constexpr int H = tile_cols<typename E::T>() / 64;
    const int pair = (int)threadIdx.x / 8, col = (int)threadIdx.x % 8 * kPiece;
    const int64_t r = r0 + 2 * pair;
    Raw<E> x[H][2] = {};
    float f[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bool there = WHOLE || r + i < s.R;
        // (rows that are not there are zeros, whatever the scales)
        f[i] = !there ? 0.0f : s.scale == nullptr ? 1.0f : s.scale[r + i];
#pragma unroll
        for (int h = 0; h < H; ++h) {
            const int64_t c = c0 + h * 64 + col;
            const int n = WHOLE || s.C - c > kPiece ? kPiece : (int)(s.C - c);
            if (there && n > 0)
                x[h][i].load(static_cast<const typename E::T*>(s.p) + (r + i) * s.ld + c, n,
                             (int)(c < 8 ? c : 8));
        }
    }
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
        for (int k = 0; k < kPiece; ++k) {
            uint16_t lo[P], hi[P];
            split<P>(x[h][0][k] * f[0], lo);
            split<P>(x[h][1][k] * f[1], hi);
#pragma unroll
            for (int p = 0; p < P; ++p)
                tile[p][h * 64 + col + k][pair] = (uint32_t)lo[p] | (uint32_t)hi[p] << 16;
        }
}
template <class E, int P>
__device__ void transpose(const Source& s, uint32_t block,
                          Tile<P, tile_cols<typename E::T>()>& tile) {
    constexpr int COLS = tile_cols<typename E::T>();
    const uint32_t tiles_r = (uint32_t)(s.pad / 64);
    const int64_t r0 = (int64_t)(block % tiles_r) * 64, c0 = (int64_t)(block / tiles_r) * COLS;
    if (r0 + 64 <= s.R && c0 + COLS <= s.C) turn<E, P, true>(s, r0, c0, tile);
    else turn<E, P, false>(s, r0, c0, tile);
    __syncthreads();
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int h = 0; h < COLS; h += 32) {
            const int c = h + (int)threadIdx.x / 8, w = (int)threadIdx.x % 8 * 4;
            if (c0 + c >= s.C) continue;
            const u32x4 v = {tile[p][c][w], tile[p][c][w + 1], tile[p][c][w + 2],
                             tile[p][c][w + 3]};
            *reinterpret_cast<u32x4*>(s.out + ((int64_t)p * s.C + c0 + c) * s.pad + r0 + 2 * w) = v;
        }
}

// in [R x C] -> out [P][R][pad], scaled by column, zeros from C to pad
template <class E, int P>
__device__ void spread(const Source& s, uint32_t block) {
    // (a launch holds fewer than 2^32 work items)
    const uint32_t across = (uint32_t)(s.pad / kPiece), i = block * 256u + threadIdx.x;
    const int64_t r = i / across, c = (int64_t)(i % across) * kPiece;
    if (r >= s.R) return;
    Raw<E> x = {};
    Raw<F32> f = {};
    const int n = s.C - c < kPiece ? (int)(s.C - c) : kPiece, before = (int)(c < 8 ? c : 8);
    if (n > 0) {
        x.load(static_cast<const typename E::T*>(s.p) + r * s.ld + c, n, before);
        if (s.scale != nullptr) f.load(s.scale + c, n, before);
    }
    uint16_t part[kPiece][P];
#pragma unroll
    for (int k = 0; k < kPiece; ++k) split<P>(s.scale != nullptr ? x[k] * f[k] : x[k], part[k]);
#pragma unroll
    for (int p = 0; p < P; ++p) {
        u32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            v[k] = (uint32_t)part[2 * k][p] | (uint32_t)part[2 * k + 1][p] << 16;
        *reinterpret_cast<u32x4*>(s.out + ((int64_t)p * s.R + r) * s.pad + c) = v;
    }
}

// One launch lays out what has to be: the first blocks the 8-bit operand, the
// others dy.
template <class E, int P, bool ALONG>
__global__ __launch_bounds__(256) void layout_kernel(Source held, Source dy) {
    __shared__ union {
        Tile<1, tile_cols<int8_t>()> held;
        Tile<ALONG ? 1 : P, tile_cols<typename E::T>()> dy;
    } tile;
    if (blockIdx.x < held.blocks)
        transpose<I8, 1>(held, blockIdx.x, tile.held);
    else if constexpr (ALONG)
        spread<E, P>(dy, blockIdx.x - (uint32_t)held.blocks);
    else
        transpose<E, P>(dy, blockIdx.x - (uint32_t)held.blocks, tile.dy);
}

__global__ __launch_bounds__(256) void zero_rows_kernel(char* p, int64_t ld, int64_t R,
                                                        int64_t row) {
    // elements are 2 or 4 bytes: 2 at a time
    const int64_t across = row / 2;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i / across >= R) return;
    *reinterpret_cast<uint16_t*>(p + i / across * ld + i % across * 2) = 0;
}

int zero_rows(Mat c, int64_t R, int64_t C, void* stream) {
    const int64_t e = c.bf16 ? 2 : 4;
    return in_parts(R, up(C * e / 2, 1), [&](int64_t r, int64_t n) {
        return launch(zero_rows_kernel, dim3((uint32_t)up(n * (C * e / 2), 256)), 256, stream,
                      static_cast<char*>(c.p) + r * c.ld * e, c.ld * e, n, C * e);
    });
}

// How a gradient takes its operands.  With dy in one part, bf16 dy stays as it is
// and the 8-bit operand takes the scale; else dy is laid out, scaled, in parts.
struct Layout {
    int parts;
    bool held_scaled;
    bool dy_as_is, held_as_is;
    bool f32;  // fp32 dy as it is, taken apart on its way (q8_grad_f32.h)
    int64_t Rp;  // summed size, padded to whole steps,
    int64_t steps;
    Shape shape;  // of the product
    int64_t dy_bytes, held_bytes;
};

// Laying an operand out costs its size, reading it as it is part of the product's
// time, so few rows of C a value, or few values a sum, are taken as they are.
// Measured with bf16 and 4096 x 4096 weights: dx of 128 tokens 32 us laid out and
// 28 as it is, of 256 37 and 40; dw of 128 tokens 22 and 18, of 1024 47 and 42, of
// 2048 (2048 x 2048) 40 and 48.
constexpr int64_t kHeldInput = 128, kHeldWeight = 1024;

// fp32 dy in three parts: written at about 2.2 TB/s where that is much of the time
// there is.  dx laid out, and taken apart on its way: 1576 x 1536 x 384 26 and 20 us,
// 1000^3 18.8 and 17.1, 4000 x 600 x 600 33 and 24, 2048^3 57 and 69.
constexpr double kLayoutNs = 6 / 2200.0;

Layout layout(int64_t M, int64_t N, int64_t R, bool dy_bf16, bool out_bf16, bool along) {
    Layout l{};
    l.parts = parts_of(R, dy_bf16, out_bf16);
    l.held_scaled = l.parts == 1 && dy_bf16;
    l.Rp = up(R, kRound) * kRound;
    l.steps = l.Rp / kRound;
    l.held_as_is = l.held_scaled && (along ? M <= kHeldInput : R <= kHeldWeight);
    l.shape = grad_shape(M, N, l.steps, l.parts, l.held_as_is);
    if (l.parts == 3) {
        const Shape s = f32_shape(M, N, l.steps);
        l.f32 = s.ns >= 0 && s.ns < l.shape.ns + (double)M * (double)l.Rp * kLayoutNs;
        if (l.f32) l.shape = s;
    }
    // a step of dx reads 128 bytes of a row of dy, which have to be there
    l.dy_as_is = l.f32 || (along ? l.held_scaled && l.Rp == R : l.held_as_is);
    l.dy_bytes = l.dy_as_is ? 0 : l.parts * M * l.Rp * 2;
    l.held_bytes = l.held_as_is ? 0 : N * l.Rp * 2;
    return l;
}
int64_t workspace_of(const Layout& l, int64_t M, int64_t N) {
    return l.dy_bytes + l.held_bytes + slices_bytes(M, N, l.shape);
}

// c [M x N] = the sum over R of dy, which has its rows, and the 8-bit operand,
// which has its columns.  ALONG: dy's rows lie along the sum.
template <bool ALONG>
int gradient(Mat dy, Held held, int64_t R, int64_t M, int64_t N, Mat c, void* workspace,
             void* stream) {
    const Layout l = layout(M, N, R, dy.bf16, c.bf16, ALONG);
    char* ws = static_cast<char*>(workspace);
    Source h{held.q, held.ld, l.held_scaled ? held.scale : nullptr, R, N,
             reinterpret_cast<uint16_t*>(ws + l.dy_bytes), l.Rp, 0};
    Source d{dy.p, dy.ld, l.held_scaled ? nullptr : held.scale, ALONG ? M : R, ALONG ? R : M,
             reinterpret_cast<uint16_t*>(ws), l.Rp, 0};
    if (!l.held_as_is) h.blocks = l.Rp / 64 * up(N, tile_cols<int8_t>());
    if (!l.dy_as_is) d.blocks = ALONG ? up(M * (l.Rp / kPiece), 256) : l.Rp / 64 * up(M, 64);
    if (h.blocks + d.blocks > 0) {
        if ((h.blocks + d.blocks) * 256 >= (int64_t)1 << 32) return (int)hipErrorInvalidValue;
        const dim3 grid((uint32_t)(h.blocks + d.blocks));
        const int e =
            dy.bf16
                ? l.parts == 1 ? launch(layout_kernel<BF16, 1, ALONG>, grid, 256, stream, h, d)
                               : launch(layout_kernel<BF16, 2, ALONG>, grid, 256, stream, h, d)
            : l.parts == 1 ? launch(layout_kernel<F32, 1, ALONG>, grid, 256, stream, h, d)
                           : launch(layout_kernel<F32, 3, ALONG>, grid, 256, stream, h, d);
        if (e) return e;
    }
    Target t{};
    t.c = c.p;
    t.ldc = c.ld;
    t.bf16 = c.bf16;
    void* slices = ws + l.dy_bytes + l.held_bytes;
    if (l.f32) {
        const F32Operands o{static_cast<const char*>(dy.p), dy.ld * 4, ws, l.Rp * 2,
                            held.scale, R, M, N, (int)l.steps};
        return launch_grad_f32<!ALONG>(o, t, l.shape.slices, slices, stream);
    }
    GradOperands o{};
    o.a = l.dy_as_is ? static_cast<const char*>(dy.p) : ws;
    o.lda = (l.dy_as_is ? dy.ld : l.Rp) * 2;
    o.a_part = M * l.Rp * 2;
    o.b = l.held_as_is ? reinterpret_cast<const char*>(held.q) : ws + l.dy_bytes;
    o.ldb = l.held_as_is ? held.ld : l.Rp * 2;
    o.scale = held.scale;
    o.R = R;
    o.M = M;
    o.N = N;
    o.steps = (int)l.steps;
    o.parts = l.parts;
    if (l.held_as_is) return launch_grad_gemm<!ALONG, true, 1>(o, t, l.shape, slices, stream);
    if (l.parts == 1) return launch_grad_gemm<false, false, 1>(o, t, l.shape, slices, stream);
    return l.parts == 2 ? launch_grad_gemm<false, false, 2>(o, t, l.shape, slices, stream)
                        : launch_grad_gemm<false, false, 3>(o, t, l.shape, slices, stream);
}

}  // namespace

int64_t grad_input_workspace(int64_t T, int64_t N, int64_t K, bool dy_bf16, bool out_bf16) {
    if (T <= kFewInput) return few_input_workspace(T, N, K);
    return workspace_of(layout(T, K, N, dy_bf16, out_bf16, true), T, K);
}

int launch_grad_input(Mat dy, Held b, int64_t T, int64_t N, int64_t K, Mat dx, void* workspace,
                      void* stream) {
    if (N == 0) return zero_rows(dx, T, K, stream);
    if (T <= kFewInput) return launch_few_input(dy, b, T, N, K, dx, workspace, stream);
    return gradient<true>(dy, b, N, T, K, dx, workspace, stream);
}

int64_t grad_weight_workspace(int64_t T, int64_t N, int64_t K, bool dy_bf16, bool out_bf16) {
    if (T <= kFewWeight) return 0;
    return workspace_of(layout(N, K, T, dy_bf16, out_bf16, false), N, K);
}

int launch_grad_weight(Mat dy, Held a, int64_t T, int64_t N, int64_t K, Mat dw, void* workspace,
                       void* stream) {
    if (T == 0) return zero_rows(dw, N, K, stream);
    if (T <= kFewWeight) return launch_few_weight(dy, a, T, N, K, dw, stream);
    return gradient<false>(dy, a, T, N, K, dw, workspace, stream);
}

}  // namespace q8
}  // namespace cpdp
