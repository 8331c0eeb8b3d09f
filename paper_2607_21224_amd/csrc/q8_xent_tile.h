// The logits of a loss by tiles, made by Gemm's loop (q8_gemm.h) and used where they
// are, in registers: nothing of them goes to memory but what the loss needs of each row
// of a tile, or their gradient.
//
// A lane has, for MT rows of the tile, 4 NT consecutive classes; the four lanes g of a row
// and the WN wavefronts beside each other have the rest of its classes.
#pragma once

#include "q8_grad_gemm.h"
#include "q8_xent_launch.h"

namespace cpdp {
namespace q8 {
namespace {

// Logits' operands, scales and targets; a tile's classes are counted from `first` on.
struct Logits {
    Operands o;
    const float* x_scale;
    const float* w_scale;
    const int64_t* target;
    int64_t first;
};

// Where the logits' gradient goes, laid out for the gradients' products.
struct Slopes {
    uint16_t* by_row;    // [parts][rows][row_ld]
    uint16_t* by_class;  // [parts][classes][class_ld]
    int64_t row_ld, row_part, class_ld, class_part;  // row lengths are whole steps
    const float* lse;
    const float* g;
    int64_t classes;  // of the loss
};

// What is known of a row's logits after some of the classes: the largest, and the sum of
// exp(z - top).
struct Stats {
    float top, sum;
};

// exp(x) for x <= 0 or NaN, as 2^(x log2 e): v_exp is within a unit of the last place,
// what its argument's rounding adds is |x| 2^-24 at most.  Results below 2^-126 are 0.
__device__ __forceinline__ float exp_of(float x) {
    return __builtin_amdgcn_exp2f(x * 1.44269504f);
}

// `top` to subtract: with nothing but -infinities, 0 (their exp is then 0)
__device__ __forceinline__ float pivot(float top) { return top == -__builtin_inff() ? 0.0f : top; }

__device__ __forceinline__ Stats join(Stats a, Stats b) {
    const float top = fmaxf(a.top, b.top), p = pivot(top);
    return {top, a.sum * exp_of(a.top - p) + b.sum * exp_of(b.top - p)};
}

template <int BM, int BN, int WM, int WN, int S>
struct LogitTile {
    using G = Gemm<Int8, BM, BN, WM, WN, S>;
    static constexpr int MT = G::MT, NT = G::NT, COLS = 4 * NT;
    static constexpr int kThreads = G::kThreads;
    static constexpr int kLds = S * G::kBuffer;

    struct Place {
        TileAt tile;
        int wave, lane, wm, wn, r, g;
        int64_t n0;  // the lane's first class
    };
    static __device__ __forceinline__ Place place(int64_t tiles_m, int64_t tiles_n) {
        Place p;
        p.tile = tile_at(tiles_m, tiles_n, BM, BN);
        p.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        p.lane = threadIdx.x & 63;
        p.wm = p.wave / WN;
        p.wn = p.wave % WN;
        p.r = p.lane & 15;
        p.g = p.lane >> 4;
        p.n0 = p.tile.n + p.wn * NT * 16 + p.g * COLS;
        return p;
    }
    static __device__ __forceinline__ int64_t row(const Place& p, int i) {
        return p.tile.m + (p.wm * MT + i) * 16 + p.r;
    }

    static __device__ __forceinline__ void sums(const Logits& l, const Place& p, char* lds,
                                                i32x4 (&acc)[MT][NT]) {
        const Operands& o = l.o;
        const auto at = G::loads(o, p.tile.m, p.tile.n, p.wave, p.lane);
        const char* a0 = o.a + p.tile.m * o.lda;
        const char* b0 = o.b + p.tile.n * o.ldb;
        const int steps = o.row / kStep, tail = o.row % kStep;
        typename G::Tail last;
        if constexpr (G::kEarly)
            if (tail != 0)
                G::load(last, a0 + (int64_t)steps * kStep, b0 + (int64_t)steps * kStep, at, p.wave,
                        p.lane, tail, steps * kStep);
        G::sums(o, at, a0, b0, 0, steps, tail, last, lds, p.wave, p.lane, acc);
    }

    // f(i, row, z, hot) for each of the lane's rows with its logits; hot: which of them is
    // the target's, in [0, COLS) if any.  Classes that are not there have -infinity.
    template <class F>
    static __device__ __forceinline__ void for_rows(const Logits& l, const Place& p,
                                                    const i32x4 (&acc)[MT][NT], F f) {
        float ws[COLS], xs[MT];
        int64_t y[MT];
#pragma unroll
        for (int k = 0; k < COLS; ++k) {
            const int64_t c = p.n0 + k;
            ws[k] = l.w_scale[c < l.o.N ? c : l.o.N - 1];
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int64_t m = row(p, i), at = m < l.o.M ? m : l.o.M - 1;
            xs[i] = l.x_scale[at];
            y[i] = l.target[at];
        }
        const bool whole = p.tile.n + BN <= l.o.N;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            float z[COLS];
#pragma unroll
            for (int k = 0; k < COLS; ++k) z[k] = (float)acc[i][k / 4][k % 4] * xs[i] * ws[k];
            if (!whole) {
#pragma unroll
                for (int k = 0; k < COLS; ++k)
                    z[k] = p.n0 + k < l.o.N ? z[k] : -__builtin_inff();
            }
            // (a negative target is before every class)
            const int64_t hot = y[i] - l.first - p.n0;
            f(i, row(p, i), z, hot >= 0 && hot < COLS && p.n0 + hot < l.o.N ? (int)hot : -1, xs[i],
              ws, y[i]);
        }
    }

    // Each row's largest logit and sum of exp's over the tile's classes, and its target's
    // logit where the tile has it.
    static __device__ __forceinline__ void stats(const Logits& l, Stats* part, float* hit,
                                                 int64_t tiles_m, int64_t tiles_n,
                                                 int64_t first_tile) {
        __shared__ __attribute__((aligned(1024))) char lds[kLds];
        const Place p = place(tiles_m, tiles_n);
        i32x4 acc[MT][NT] = {};
        sums(l, p, lds, acc);
        Stats of[MT];
        for_rows(l, p, acc, [&](int i, int64_t m, const float(&z)[COLS], int hot, float,
                                const float(&)[COLS], int64_t) {
            // a lane's classes against their own largest: the lanes' sums are joined after
            // that, at two exp's a row and not a maximum over the lanes first
            float top = z[0];
#pragma unroll
            for (int k = 1; k < COLS; ++k) top = fmaxf(top, z[k]);
            const float q = pivot(top);
            float sum = 0.0f;
#pragma unroll
            for (int k = 0; k < COLS; ++k) sum += exp_of(z[k] - q);
            of[i] = {top, sum};
            if (__any(hot >= 0)) {
#pragma unroll
                for (int k = 0; k < COLS; ++k)
                    if (k == hot && m < l.o.M) hit[m] = z[k];
            }
        });
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int off = 16; off < 64; off <<= 1)
                of[i] = join(of[i], {__shfl_xor(of[i].top, off), __shfl_xor(of[i].sum, off)});
        __syncthreads();
        auto* words = reinterpret_cast<Stats(*)[BM]>(lds);  // [WN][BM]
        if (p.g == 0) {
#pragma unroll
            for (int i = 0; i < MT; ++i) words[p.wn][(p.wm * MT + i) * 16 + p.r] = of[i];
        }
        __syncthreads();
        if ((int)threadIdx.x >= BM) return;
        Stats s = words[0][threadIdx.x];
#pragma unroll
        for (int w = 1; w < WN; ++w) s = join(s, words[w][threadIdx.x]);
        const int64_t m = p.tile.m + threadIdx.x;
        if (m < l.o.M) part[(first_tile + p.tile.n / BN) * l.o.M + m] = s;
    }

    // The gradient of the logits, times g, twice: by rows, each class scaled by w_scale, for
    // the gradient of x, and by classes, each row scaled by x_scale, for that of w; bf16
    // numbers in PX and PW parts (0: not wanted), with zeros up to the end of a step.
    template <int PX, int PW>
    static __device__ __forceinline__ void grads(const Logits& l, const Slopes& to,
                                                 int64_t tiles_m, int64_t tiles_n) {
        __shared__ __attribute__((aligned(1024))) char lds[kLds];
        const Place p = place(tiles_m, tiles_n);
        i32x4 acc[MT][NT] = {};
        sums(l, p, lds, acc);
        // the wavefront's own rows and classes, to be turned
        constexpr int kRow = NT * 32;  // bytes
        static_assert(G::kWaves * MT * 16 * kRow <= kLds, "room to turn a part");
        char* room = lds + p.wave * MT * 16 * kRow;
        float turn[MT][COLS];  // (in the sums' place)
        for_rows(l, p, acc, [&](int i, int64_t m, const float(&z)[COLS], int hot, float xs,
                                const float(&ws)[COLS], int64_t y) {
            const int64_t at = m < l.o.M ? m : l.o.M - 1;
            const float lse = y >= to.classes ? __builtin_nanf("") : to.lse[at], g = to.g[at];
            float e[COLS];
#pragma unroll
            for (int k = 0; k < COLS; ++k) e[k] = exp_of(z[k] - lse);
            if (__any(hot >= 0)) {
#pragma unroll
                for (int k = 0; k < COLS; ++k) e[k] = k == hot ? e[k] - 1.0f : e[k];
            }
#pragma unroll
            for (int k = 0; k < COLS; ++k) {
                e[k] *= g;
                turn[i][k] = e[k] * xs;
                e[k] *= ws[k];
            }
            const bool counts = y >= 0 && m < l.o.M;
            if (__any(!counts) || p.tile.n + BN > l.o.N) {
                // what is not there is 0, whatever was computed for it
#pragma unroll
                for (int k = 0; k < COLS; ++k) {
                    const bool there = counts && p.n0 + k < l.o.N;
                    turn[i][k] = there ? turn[i][k] : 0.0f;
                    e[k] = there ? e[k] : 0.0f;
                }
            }
            const int64_t m0 = p.tile.m + (p.wm * MT + i) * 16, c0 = p.tile.n + p.wn * NT * 16;
#pragma unroll
            for (int q = 0; q < PX; ++q) {
                u32x4 v[COLS / 8];
#pragma unroll
                for (int k = 0; k < COLS; k += 2)
                    v[k / 8][k % 8 / 2] =
                        q + 1 < PX ? take2(e[k], e[k + 1]) : narrow2(e[k], e[k + 1]);
                store_turned(v, to.by_row + q * to.row_part + m0 * to.row_ld + c0, to.row_ld,
                             l.o.M - m0, to.row_ld - c0, p.r, p.g);
            }
        });
        if constexpr (PW > 0) {
            __syncthreads();  // (all have read the last step)
#pragma unroll
            for (int q = 0; q < PW; ++q) {
                // rows of the tile into LDS, their 16-byte pieces exchanged so that the 16
                // lanes of a row's piece touch all banks
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < COLS / 8; ++j) {
                        u32x4 v;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            float &a = turn[i][8 * j + 2 * k], &b = turn[i][8 * j + 2 * k + 1];
                            v[k] = q + 1 < PW ? take2(a, b) : narrow2(a, b);
                        }
                        const int at = i * 16 + p.r, piece = p.g * (COLS / 8) + j;
                        *reinterpret_cast<u32x4*>(room + at * kRow + ((piece ^ swap(at)) << 4)) = v;
                    }
                __syncthreads();
                // and out of it by classes: 16 lanes read 4 rows of 16 classes, and each gets
                // one class' 4 rows; two reads are 8 rows, 16 bytes
#pragma unroll
                for (int c = 0; c < NT; ++c)
#pragma unroll
                    for (int i = 0; i < MT / 2; ++i) {
                        const int at = i * 32 + p.g * 8;
                        const u32x2 lo = turned(room, at, c, p.r);
                        const u32x2 hi = turned(room, at + 4, c, p.r);
                        const int64_t v = p.tile.n + (p.wn * NT + c) * 16 + p.r;
                        const int64_t t = p.tile.m + p.wm * MT * 16 + at;
                        if (v < l.o.N && t < to.class_ld)
                            *reinterpret_cast<u32x4*>(to.by_class + q * to.class_part +
                                                      v * to.class_ld + t) =
                                u32x4{lo[0], lo[1], hi[0], hi[1]};
                    }
                if (q + 1 < PW) __syncthreads();
            }
        }
    }
    // The first of the parts that a and b are still to be held in (see split), which is
    // taken off them.
    static __device__ __forceinline__ uint32_t take2(float& a, float& b) {
        uint32_t v = narrow2(a, b);
        float x[2] = {a, b};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint32_t bits = k == 0 ? v << 16 : v & 0xffff0000u;
            const bool finite = magnitude(x[k]) < 0x7f800000u;
            // a number past the largest bf16 keeps its first bits
            if (finite && (bits & 0x7f800000u) == 0x7f800000u) {
                bits = __float_as_uint(x[k]) & 0xffff0000u;
                v = k == 0 ? (v & 0xffff0000u) | bits >> 16 : (v & 0xffffu) | bits;
            }
            x[k] = finite ? x[k] - __uint_as_float(bits) : 0.0f;
        }
        a = x[0];
        b = x[1];
        return v;
    }
    static __device__ __forceinline__ int swap(int row) {
        return NT == 4 ? (row >> 1) & 7 : (row >> 1) & 3;
    }
    // 4 rows, from `row` on, of class 16 c + r
    static __device__ __forceinline__ u32x2 turned(const char* room, int row, int c, int r) {
        const int at = row + (r >> 2), piece = 2 * c + (r >> 1 & 1);
        const char* from = room + at * NT * 32 + ((piece ^ swap(at)) << 4) + (r & 1) * 8;
        return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                             (__attribute__((address_space(3))) i16x4*)(from)));
    }
};

template <int BM, int BN, int WM, int WN, int S>
__global__ __launch_bounds__(64 * WM * WN) void xent_stats_kernel(Logits l, Stats* part, float* hit,
                                                                  int64_t tiles_m, int64_t tiles_n,
                                                                  int64_t first_tile) {
    LogitTile<BM, BN, WM, WN, S>::stats(l, part, hit, tiles_m, tiles_n, first_tile);
}
template <int BM, int BN, int WM, int WN, int S, int PX, int PW>
__global__ __launch_bounds__(64 * WM * WN) void xent_slopes_kernel(Logits l, Slopes to,
                                                                   int64_t tiles_m,
                                                                   int64_t tiles_n) {
    LogitTile<BM, BN, WM, WN, S>::template grads<PX, PW>(l, to, tiles_m, tiles_n);
}

// Rows and classes of the tile that some logits are made in: 256, 128 or 64.
inline int logit_tile(int64_t M, int64_t N, int64_t steps) {
    struct {
        int tile, alone, each, end;  // ns of a step, and of what follows the last
    } const tiles[] = {{256, 1800, 1800, 6000}, {128, 540, 620, 3000}, {64, 280, 220, 1500}};
    double best = -1;
    int tile = 0;
    for (const auto& t : tiles) {
        const int64_t n = up(M, t.tile) * up(N, t.tile);
        const double time = n <= kCus ? steps * (double)t.alone + t.end
                                      : (double)up(n, kCus) * (steps * (double)t.each + t.end / 2);
        if (best < 0 || time < best) {
            best = time;
            tile = t.tile;
        }
    }
    return tile;
}

}  // namespace
}  // namespace q8
}  // namespace cpdp
