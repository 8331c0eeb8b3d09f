// The logits of a loss by tiles, made by Gemm's loop (q8_gemm.h) and used where they
// are, in registers: nothing of them goes to memory but what the loss needs of each row
// of a tile, or their gradient.
//
// A lane has, for MT rows of the tile, 4 NT consecutive classes; the four lanes g of a row
// and the WN wavefronts beside each other have the rest of its classes.
#pragma once

#include "q8_xent_stats.h"

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

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Products of fp16 numbers, with fp32 sums (see Gemm).
struct Half {
    using Acc = f32x4;
    using Sum = float;
    static __device__ __forceinline__ Acc mfma(u32x4 a, u32x4 b, Acc c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                      __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};

// two fp32 values as fp16, rounded to nearest-even (the low half is the first)
__device__ __forceinline__ uint32_t halves(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, f16x2));
}

constexpr float kSecond = 4096.0f;  // (see Slopes)
constexpr int kLargest = 32;

// the power of two that brings x into [2^14, 2^15), as far as that and its inverse are
// normal numbers
__device__ __forceinline__ float scale_for(float x) {
    if (x == 0.0f) return 1.0f;
    const int e = (int)(__float_as_uint(x) >> 23) - 127;  // (below 2^-126: -127)
    const int up = 14 - e;
    return __uint_as_float((uint32_t)((up > 126 ? 126 : up) + 127) << 23);
}

// Where the logits' gradient e = exp(z - lse) - [target] goes, laid out for the gradients'
// products, in fp16 numbers: one for a bf16 result, 11 bits of it; two for an fp32 one, 22
// bits, the second as a part of its own after the first and 2^12 times as large, so that
// what is too small for the first is still in it.  8-bit numbers, the other operands, are
// exact in fp16, and so are they over 2^12, which the second part is multiplied by.
//   by_row    e w_scale[v] * scale[0]          [rows][parts][row_ld]
//   by_class  e g[t] x_scale[t] * scale[1]     [classes][parts][class_ld]
// scale are powers of two that bring the largest |w_scale| and |g x_scale| there are, found
// from those of up to 32 parts, to 2^14 or more and below 2^15.  What fp16 keeps of a number ends at 2^-24: at 2^-38 of that,
// 2^-50 with two parts, where e itself has an error of 2^-24 or more at the target (from miss:
// that of the loss; else lse's, 2^-24 |lse|).  (In bfloat16
// numbers, which do not end there, an fp32 result needs three, and its product is half as
// long again: loss and gradients of 4096 x 65536 x 1024 with fp32 dw 2820 us, and 2400 when
// this was all that changed.)
// What the products are then scaled by: rows[t] = g[t] / scale[0], classes[v] = 1 / scale[1].
struct Slopes {
    uint16_t* by_row;
    uint16_t* by_class;
    int64_t row_ld, class_ld;  // of a part; whole steps
    LossIn in;
    const float* largest;  // [2][kLargest]
    float* rows;
    float* classes;
    int64_t V;  // classes of the loss
};

// Where it goes for few tokens: d[t, v] = e g[t], fp32, 0 for tokens that do not count, and
// their scales, 0 for those.
struct FewSlopes {
    float* d;
    int64_t ld;
    LossIn in;
    float* scale;
    int64_t V;  // classes of the loss
};

// Where a tile's findings go: its part of each row's statistics [tile][row] and the
// targets' logits; or, without parts, the loss.
struct Found {
    Stats* part;
    float* hit;
    LossOut out;
};

// Tiles of TILE rows and classes by 2 x WN wavefronts, with S LDS buffers.
template <int TILE, int WN, int S>
struct LogitTile {
    using G = Gemm<Int8, TILE, TILE, 2, WN, S>;
    static constexpr int MT = G::MT, NT = G::NT, COLS = 4 * NT;
    static constexpr int kThreads = G::kThreads, kWaves = G::kWaves;
    static constexpr int kBuffers = S * G::kBuffer;

    struct Place {
        TileAt tile;
        int wave, lane, wm, wn, r, g;
        int row;    // of the tile, the lane's first (16 apart)
        int first;  // class of the tile, the lane's first
    };
    static __device__ __forceinline__ Place place(int64_t tiles_m, int64_t tiles_n) {
        Place p;
        p.tile = tile_at(tiles_m, tiles_n, TILE, TILE);
        p.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        p.lane = threadIdx.x & 63;
        p.wm = p.wave / WN;
        p.wn = p.wave % WN;
        p.r = p.lane & 15;
        p.g = p.lane >> 4;
        p.row = p.wm * MT * 16 + p.r;
        p.first = p.wn * NT * 16 + p.g * COLS;
        return p;
    }

    // What the end needs of each row and class of the tile, sent for into LDS before the
    // sums' loads, so that it is there when they are done.  (Held in registers from the
    // start, or loaded at the end, it made the large tile's kernels spill; in an LDS array of
    // its own it made the compiler wait for all loads in the loop, 1945 -> 2275 us for the
    // logits of 8192 x 131072 x 2048.)
    struct Vectors {
        float x_scale[TILE], w_scale[TILE];
        uint32_t target[2][TILE];  // halves
        float lse[TILE], g[TILE], miss[TILE];
        float largest[2 * kLargest];
    };
    static_assert(2 * kLargest == 64, "a load of a wavefront");
    // (without SLOPES nothing of `in`; `largest` may be null)
    template <bool SLOPES>
    static __device__ __forceinline__ void send(const Logits& l, const LossIn& in,
                                                const float* largest, const Place& p, Vectors& v) {
        if constexpr (SLOPES)
            if (p.wave == 0 && largest != nullptr)
                __builtin_amdgcn_global_load_lds(
                    (__attribute__((address_space(1))) void*)(largest + p.lane),
                    (__attribute__((address_space(3))) void*)(v.largest), 4, 0, 0);
        constexpr int kEach = TILE / 64;
        constexpr int count = (SLOPES ? 7 : 4) * kEach;
#pragma unroll
        for (int j = 0; j < (count + kWaves - 1) / kWaves; ++j) {
            const int k = j * kWaves + p.wave;
            if (k >= count) break;
            const int what = k / kEach, at = k % kEach * 64;
            // rows and classes that are not there take the last one's
            const int64_t m = p.tile.m + at + p.lane < l.o.M ? p.tile.m + at + p.lane : l.o.M - 1;
            const int64_t n = p.tile.n + at + p.lane < l.o.N ? p.tile.n + at + p.lane : l.o.N - 1;
            const auto* half = reinterpret_cast<const uint32_t*>(l.target + m);
            const void* from = what == 0   ? static_cast<const void*>(l.x_scale + m)
                               : what == 1 ? static_cast<const void*>(l.w_scale + n)
                               : what == 2 ? static_cast<const void*>(half)
                               : !SLOPES || what == 3 ? static_cast<const void*>(half + 1)
                               : what == 4            ? static_cast<const void*>(in.lse + m)
                               : what == 5            ? static_cast<const void*>(in.g + m)
                               // (something, where there is none)
                               : in.miss != nullptr ? static_cast<const void*>(in.miss + m)
                                                    : static_cast<const void*>(in.lse + m);
            __builtin_amdgcn_global_load_lds(
                (__attribute__((address_space(1))) void*)(from),
                (__attribute__((address_space(3))) void*)(reinterpret_cast<char*>(&v) +
                                                          (what * TILE + at) * 4),
                4, 0, 0);
        }
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
        // all have read the last step, and the vectors are there
        wait_loads<0>();
        barrier();
    }

    // the target of a row of the tile
    static __device__ __forceinline__ int64_t target(const Vectors& v, int row) {
        return (int64_t)((uint64_t)v.target[1][row] << 32 | v.target[0][row]);
    }
    // which of the lane's COLS classes it is, or something else (a negative target is
    // before every class)
    static __device__ __forceinline__ int hot(const Logits& l, const Place& p, int64_t y) {
        const int64_t at = y - l.first - p.tile.n - p.first;
        return at >= 0 && at < COLS ? (int)at : -1;
    }

    // p of the target less 1: what its loss leaves of it, where that is known
    static __device__ __forceinline__ void less_one(float (&e)[COLS], int at, const LossIn& in,
                                                    float miss) {
#pragma unroll
        for (int k = 0; k < COLS; ++k)
            if (k == at) e[k] = in.miss != nullptr ? -miss : e[k] - 1.0f;
    }

    // Each row's largest logit and sum of exp's over the tile's classes, and its target's
    // logit where the tile has it; the loss, if these are all the classes.
    static __device__ __forceinline__ void stats(const Logits& l, const Found& to, int64_t tiles_m,
                                                 int64_t tiles_n, int64_t first_tile) {
        __shared__ __attribute__((aligned(1024))) char lds[kBuffers + sizeof(Vectors)];
        Vectors& v = *reinterpret_cast<Vectors*>(lds + kBuffers);
        const Place p = place(tiles_m, tiles_n);
        send<false>(l, LossIn{}, nullptr, p, v);
        i32x4 acc[MT][NT] = {};
        sums(l, p, lds, acc);
        float ws[COLS];
#pragma unroll
        for (int k = 0; k < COLS; ++k) ws[k] = v.w_scale[p.first + k];
        const bool whole = p.tile.n + TILE <= l.o.N;
        const int64_t n0 = p.tile.n + p.first;
        auto* words = reinterpret_cast<Stats(*)[TILE]>(lds);  // [WN][TILE]
        float* hit = v.g;  // (free here)
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const float xs = v.x_scale[p.row + i * 16];
            float z[COLS];
#pragma unroll
            for (int k = 0; k < COLS; ++k) z[k] = (float)acc[i][k / 4][k % 4] * xs * ws[k];
            if (!whole) {
#pragma unroll
                for (int k = 0; k < COLS; ++k) z[k] = n0 + k < l.o.N ? z[k] : -__builtin_inff();
            }
            // a lane's classes against their own largest: the lanes' sums are joined after
            // that, at two exp's a row and not a maximum over the lanes first
            float top = z[0];
#pragma unroll
            for (int k = 1; k < COLS; ++k) top = fmaxf(top, z[k]);
            const float q = pivot(top);
            float sum[2] = {0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < COLS; ++k) sum[k % 2] += exp_of(z[k] - q);
            const int at = hot(l, p, target(v, p.row + i * 16));
            if (__any(at >= 0)) {
#pragma unroll
                for (int k = 0; k < COLS; ++k)
                    if (k == at) hit[p.row + i * 16] = z[k];
            }
            Stats s = {top, sum[0] + sum[1]};
#pragma unroll
            for (int off = 16; off < 64; off <<= 1)
                s = join(s, {__shfl_xor(s.top, off), __shfl_xor(s.sum, off)});
            if (p.g == 0) words[p.wn][p.row + i * 16] = s;
        }
        __syncthreads();
        if ((int)threadIdx.x >= TILE) return;
        Stats s = words[0][threadIdx.x];
#pragma unroll
        for (int w = 1; w < WN; ++w) s = join(s, words[w][threadIdx.x]);
        const int64_t m = p.tile.m + threadIdx.x, y = target(v, (int)threadIdx.x);
        if (m >= l.o.M) return;
        const int64_t at = y - l.first - p.tile.n;
        const bool here = at >= 0 && at < TILE && p.tile.n + at < l.o.N;
        if (to.part == nullptr) {
            write_loss(s, hit[threadIdx.x], y, here ? y + 1 : 0, to.out, m);
            return;
        }
        to.part[(first_tile + p.tile.n / TILE) * l.o.M + m] = s;
        if (here) to.hit[m] = hit[threadIdx.x];
    }

    // The gradient of the logits by rows, for the gradient of x, and by classes, for that of
    // w, in PX and PW parts (0: not wanted), with zeros up to the end of a step.
    template <int PX, int PW>
    static __device__ __forceinline__ void grads(const Logits& l, const Slopes& to,
                                                 int64_t tiles_m, int64_t tiles_n) {
        __shared__ __attribute__((aligned(1024))) char lds[kBuffers + sizeof(Vectors)];
        Vectors& v = *reinterpret_cast<Vectors*>(lds + kBuffers);
        const Place p = place(tiles_m, tiles_n);
        send<true>(l, to.in, to.largest, p, v);
        i32x4 acc[MT][NT] = {};
        sums(l, p, lds, acc);
        const int64_t n0 = p.tile.n + p.first;
        float largest = v.largest[p.lane];
#pragma unroll
        for (int off = 1; off < kLargest; off <<= 1)
            largest = fmaxf(largest, __shfl_xor(largest, off));
        const float other = __shfl_xor(largest, kLargest);  // (the first lane's: of g x_scale)
        const float scale_w = scale_for(__uint_as_float(
            __builtin_amdgcn_readfirstlane(__float_as_uint(largest))));
        const float scale_x = scale_for(__uint_as_float(
            __builtin_amdgcn_readfirstlane(__float_as_uint(other))));
        if ((int)threadIdx.x < TILE) {
            const int64_t m = p.tile.m + threadIdx.x, n = p.tile.n + threadIdx.x;
            if (p.tile.n == 0 && m < l.o.M)
                to.rows[m] = target(v, (int)threadIdx.x) < 0 ? 0.0f : v.g[threadIdx.x] / scale_w;
            if (p.tile.m == 0 && n < l.o.N) to.classes[n] = 1.0f / scale_x;
        }
        float ws[COLS];
#pragma unroll
        for (int k = 0; k < COLS; ++k) ws[k] = v.w_scale[p.first + k];
        float turn[PW > 0 ? MT : 1][COLS];  // (in the sums' place)
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int row = p.row + i * 16;
            const int64_t y = target(v, row), m = p.tile.m + row;
            const int at = hot(l, p, y);
            const float xs = v.x_scale[row], gx = v.g[row] * xs * scale_x;
            const float lse = y >= to.V ? __builtin_nanf("") : v.lse[row];
            float e[COLS], t[COLS];
#pragma unroll
            for (int k = 0; k < COLS; ++k)
                e[k] = exp_of((float)acc[i][k / 4][k % 4] * xs * ws[k] - lse);
            if (__any(at >= 0)) less_one(e, at, to.in, v.miss[row]);
#pragma unroll
            for (int k = 0; k < COLS; ++k) {
                t[k] = e[k] * gx;
                e[k] *= ws[k] * scale_w;
            }
            const bool counts = y >= 0 && m < l.o.M;
            if (__any(!counts) || p.tile.n + TILE > l.o.N) {
                // what is not there is 0, whatever was computed for it
#pragma unroll
                for (int k = 0; k < COLS; ++k) {
                    const bool there = counts && n0 + k < l.o.N;
                    t[k] = there ? t[k] : 0.0f;
                    e[k] = there ? e[k] : 0.0f;
                }
            }
            if constexpr (PW > 0) {
#pragma unroll
                for (int k = 0; k < COLS; ++k) turn[i][k] = t[k];
            }
            if constexpr (PX > 0) {
                const int64_t m0 = m - p.r, c0 = p.tile.n + p.wn * NT * 16;
                const bool finite = is_finite<PX>(e);
#pragma unroll
                for (int q = 0; q < PX; ++q) {
                    u32x4 x[COLS / 8];
#pragma unroll
                    for (int k = 0; k < COLS; k += 2)
                        x[k / 8][k % 8 / 2] = take2<PX>(q, e[k], e[k + 1], finite);
                    if (c0 < to.row_ld)
                        store_whole(x, to.by_row + (m0 * PX + q) * to.row_ld + c0,
                                    PX * to.row_ld, l.o.M - m0, p);
                }
            }
        }
        if constexpr (PW > 0) {
            // The wavefront's rows go into LDS, of which it has a part to itself and whose
            // reads and writes are done in order, their 16-byte pieces exchanged so that
            // the 16 lanes of a piece touch all banks.
            constexpr int kRow = NT * 32;  // bytes
            static_assert(kWaves * MT * 16 * kRow <= kBuffers, "room to turn a part");
            char* room = lds + p.wave * MT * 16 * kRow;
            bool finite = true;
#pragma unroll
            for (int i = 0; i < MT; ++i) finite = finite && is_finite<PW>(turn[i]);
#pragma unroll
            for (int q = 0; q < PW; ++q) {
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < COLS / 8; ++j) {
                        u32x4 x;
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            x[k] = take2<PW>(q, turn[i][8 * j + 2 * k], turn[i][8 * j + 2 * k + 1],
                                             finite);
                        const int at = i * 16 + p.r, piece = p.g * (COLS / 8) + j;
                        *reinterpret_cast<u32x4*>(room + at * kRow + ((piece ^ swap(at)) << 4)) = x;
                    }
                asm volatile("" ::: "memory");
                by_classes(l, to, p, room, to.by_class + q * to.class_ld, PW * to.class_ld);
                asm volatile("" ::: "memory");
            }
        }
    }

    // The gradient of few tokens' logits.
    static __device__ __forceinline__ void few_grads(const Logits& l, const FewSlopes& to,
                                                     int64_t tiles_m, int64_t tiles_n) {
        __shared__ __attribute__((aligned(1024))) char lds[kBuffers + sizeof(Vectors)];
        Vectors& v = *reinterpret_cast<Vectors*>(lds + kBuffers);
        const Place p = place(tiles_m, tiles_n);
        send<true>(l, to.in, nullptr, p, v);
        i32x4 acc[MT][NT] = {};
        sums(l, p, lds, acc);
        if (p.tile.n == 0 && (int)threadIdx.x < TILE && p.tile.m + threadIdx.x < l.o.M)
            to.scale[p.tile.m + threadIdx.x] =
                target(v, (int)threadIdx.x) < 0 ? 0.0f : v.x_scale[threadIdx.x];
        const int64_t n0 = p.tile.n + p.first;
        float ws[COLS];
#pragma unroll
        for (int k = 0; k < COLS; ++k) ws[k] = v.w_scale[p.first + k];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int row = p.row + i * 16;
            const int64_t y = target(v, row), m = p.tile.m + row;
            const int at = hot(l, p, y);
            const float xs = v.x_scale[row], g = v.g[row];
            const float lse = y >= to.V ? __builtin_nanf("") : v.lse[row];
            float e[COLS];
#pragma unroll
            for (int k = 0; k < COLS; ++k)
                e[k] = exp_of((float)acc[i][k / 4][k % 4] * xs * ws[k] - lse);
            if (__any(at >= 0)) less_one(e, at, to.in, v.miss[row]);
            if (m >= l.o.M) continue;
            float* d = to.d + m * to.ld + n0;
#pragma unroll
            for (int k = 0; k < COLS; k += 4) {
                const float a = g * e[k], b = g * e[k + 1], c = g * e[k + 2], h = g * e[k + 3];
                // (rows are whole pieces)
                if (n0 + k < l.o.N)
                    *reinterpret_cast<f32x4*>(d + k) =
                        y < 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : f32x4{a, b, c, h};
            }
        }
    }

    // Stores a part by classes.  16 lanes read 4 rows of 16 classes, and each gets one
    // class' 4 rows; two reads are 8 rows, 16 bytes.  With 64 rows, the lanes exchange
    // pieces (see Turn), so that a store covers 128 bytes of 8 classes and not 64 of 16.
    static __device__ __forceinline__ void by_classes(const Logits& l, const Slopes& to,
                                                      const Place& p, const char* room,
                                                      uint16_t* out, int64_t ld) {
        constexpr int PIECES = MT % 4 == 0 ? 2 : 1;
        const int64_t t0 = p.tile.m + p.wm * MT * 16;
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            const int64_t v0 = p.tile.n + (p.wn * NT + c) * 16;
#pragma unroll
            for (int i = 0; i < MT / 2 / PIECES; ++i) {
                u32x4 x[PIECES];
#pragma unroll
                for (int j = 0; j < PIECES; ++j) {
                    const int at = i * 32 * PIECES + (p.g * PIECES + j) * 8;
                    const u32x2 lo = turned(room, at, c, p.r), hi = turned(room, at + 4, c, p.r);
                    x[j] = u32x4{lo[0], lo[1], hi[0], hi[1]};
                }
                const int64_t t = t0 + i * 32 * PIECES;
                if (t < to.class_ld)
                    store_whole(x, out + v0 * ld + t, ld, l.o.N - v0, p);
            }
        }
    }
    // store_turned where all of a row's pieces are there: `ld` is whole steps.  Past the
    // caches, which do not hold what the products read next: gradients of 2048 x 32768 x 1024
    // bf16 468 -> 434 us, of 7426 x 35888 x 96 fp32 1226 -> 1134, of 997 x 12345 x 385 as before.
    template <int PIECES>
    static __device__ __forceinline__ void store_whole(u32x4 (&x)[PIECES], uint16_t* c, int64_t ld,
                                                       int64_t rows, const Place& p) {
        Turn<PIECES>::run(x, p.r);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int row = Turn<PIECES>::row_of(i, p.r);
            if (row < rows)
                __builtin_nontemporal_store(
                    x[i],
                    reinterpret_cast<u32x4*>(c + row * ld + Turn<PIECES>::place_of(p.g, p.r) * 8));
        }
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

    // Whether none of the wavefront's numbers is an infinity (asked for numbers that are
    // to be taken apart).
    template <int P>
    static __device__ __forceinline__ bool is_finite(const float (&x)[COLS]) {
        if constexpr (P == 1) return true;
        float most = 0.0f;
#pragma unroll
        for (int k = 0; k < COLS; ++k) most = fmaxf(most, fabsf(x[k]));
        return !__any(most == __builtin_inff());
    }
    // Part q of P of two numbers, which is taken off them; nothing is left of an infinity.
    template <int P>
    static __device__ __forceinline__ uint32_t take2(int q, float& a, float& b, bool finite) {
        const uint32_t part = halves(a, b);
        if (q + 1 < P) {
            const f16x2 h = __builtin_bit_cast(f16x2, part);
            const float x = a, y = b;
            a = (a - (float)h[0]) * kSecond;
            b = (b - (float)h[1]) * kSecond;
            if (!finite) {
                a = magnitude(x) == 0x7f800000u ? 0.0f : a;
                b = magnitude(y) == 0x7f800000u ? 0.0f : b;
            }
        }
        return part;
    }
};

template <int TILE, int WN, int S>
__global__ __launch_bounds__(128 * WN) void xent_stats_kernel(Logits l, Found to,
                                                              int64_t tiles_m, int64_t tiles_n,
                                                              int64_t first_tile) {
    LogitTile<TILE, WN, S>::stats(l, to, tiles_m, tiles_n, first_tile);
}
template <int TILE, int WN, int S, int PX, int PW>
__global__ __launch_bounds__(128 * WN) void xent_slopes_kernel(Logits l, Slopes to,
                                                               int64_t tiles_m, int64_t tiles_n) {
    LogitTile<TILE, WN, S>::template grads<PX, PW>(l, to, tiles_m, tiles_n);
}

template <int TILE, int WN, int S>
__global__ __launch_bounds__(128 * WN) void xent_few_grads_kernel(Logits l, FewSlopes to,
                                                                  int64_t tiles_m,
                                                                  int64_t tiles_n) {
    LogitTile<TILE, WN, S>::few_grads(l, to, tiles_m, tiles_n);
}

// Rows and classes of the tile that some logits are made in: 256, 128 or 64, whichever
// should take least.  `join`: ns that more than one tile of classes costs; `parts`: in
// which their gradient is written (0: the loss).  Measured on one card, us:
//                              loss                  gradients, bf16 (2 parts)
//   tokens, classes, channels  256   128   64        256   128   64
//   128 x 100 x 384            14.5  8.3   7.3       27.5  19.0  13.6
//   512 x 4096 x 384           16.2  10.4  8.4       40.8  31.4  28.7
//   997 x 12345 x 385          21.2  24.4  34.9      78.5  81.0  89.2
//   256 x 32768 x 1024         21.8  17.9  26.9      111   107   112
//   2048 x 32768 x 1024        78.4  91.5  152       424   423   481
//   100 x 50000 x 2048         33.2  26.6  36.7      241   235   242
//   4096 x 4096 x 2048         35.8  43.6  62.2      177   182   200
struct TileTime {
    int tile;
    double ns;
};
inline TileTime logit_tile(int64_t M, int64_t N, int64_t steps, int join, int parts) {
    struct {
        int tile, alone, each;  // ns of a step: one tile a CU, and several
        int end, more;          // and of what follows the last
    } const tiles[] = {{256, 1650, 1650, 7000 + 4500 * parts, 5500 + 4500 * parts},
                       {128, 540, 620, 4200 + 1700 * parts, 1300 + 1100 * parts},
                       {64, 280, 220, 300 + 750 * parts, 1100 + 300 * parts}};
    TileTime best{0, 0.0};
    for (const auto& t : tiles) {
        const int64_t tn = up(N, t.tile), n = up(M, t.tile) * tn;
        const double time = (n <= kCus ? steps * (double)t.alone + t.end
                                       : (double)up(n, kCus) * (steps * (double)t.each + t.more)) +
                            (tn > 1 ? join : 0);
        if (best.tile == 0 || time < best.ns) best = {t.tile, time};
    }
    return best;
}

// The same in two launches, where a last turn of the CUs would find work for few: as many
// classes in tiles of 256 as whole turns hold, and the rest in what takes least
// (1003 x 50001 x 1025, 784 tiles of 256: 96.5 us in one launch, and 84.6; 2600 x 8200 x
// 1030 49.6 and 46.6).
struct TwoTiles {
    int64_t first;  // classes of the first launch, in tiles of 256; 0: there is none
    int tile;       // of the rest
};
inline TwoTiles logit_tiles(int64_t M, int64_t N, int64_t steps, int join, int parts) {
    const TileTime one = logit_tile(M, N, steps, join, parts);
    const int64_t tm = up(M, 256), turns = tm * up(N, 256) / kCus;
    const int64_t first = turns * kCus / tm * 256;
    if (first == 0 || first >= N) return {0, one.tile};
    const TileTime rest = logit_tile(M, N - first, steps, 0, parts);
    const double whole = (double)turns * ((double)steps * 1650 + 5500 + 4500 * parts);
    if (whole + rest.ns + 2500 + join < one.ns) return {first, rest.tile};
    return {0, one.tile};
}

}  // namespace
}  // namespace q8
}  // namespace cpdp
