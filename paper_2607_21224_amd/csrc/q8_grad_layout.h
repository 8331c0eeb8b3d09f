// Operands of a gradient's product laid out with the index that is summed over
// contiguous, as bf16 numbers.
#pragma once

#include "q8_grad.h"

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

}  // namespace
}  // namespace q8
}  // namespace cpdp
