// The product of a gradient on the bf16 matrix cores:
//   C[m, n] = sum over r of A[m, r] B[n, r]
// Each operand is laid out, bf16 with r contiguous, or read as it is, its rows
// running across the sum (DOWN):
//   A   a bf16 matrix [R x M]; or laid out in `parts`, whose sum is A: P of them
//       taken in one pass, all P by the same B, or one a pass
//   B   the 8-bit operand [R x N], scaled by row and rounded to bf16 on its way; or
//       laid out, the same for every part
//
// The loop is that of Gemm (q8_gemm.h): steps of 64 values of r go from memory
// straight into one of S LDS buffers, half a step is in registers, one barrier a
// step.  What differs is how a DOWN operand leaves LDS, where r runs down the
// buffer and an instruction wants 8 values of r from each lane, for one row of its
// operand.
//   A   The transposing read does it: 16 lanes read 4 rows of 16 columns, 4 columns
//       a lane, and each gets one column's 4 rows.
//   B   A lane reads 4 neighbouring columns of 8 rows and takes them one after the
//       other: column c of the 8 is its part of instruction c, which so stands for
//       columns 4 i + c, i the lane's place among 16.  Bytes become floats, are
//       scaled and rounded: 2.5 instructions a value beside the matrix cores', which
//       costs more than it saves where the product is large.
//
// The 16-byte pieces of a row are permuted in LDS so that the rows one read touches
// fall on different banks; B's rows lie in the order (r / 32, r % 8, r / 8 % 4), so
// that the four groups of 16 lanes read neighbouring ones.
#pragma once

#include "q8_grad.h"

namespace cpdp {
namespace q8 {
namespace {

typedef short i16x4 __attribute__((ext_vector_type(4)));

struct GradOperands {
    const char* a;
    int64_t lda;     // bytes, as the other strides
    int64_t a_part;  // from pass to pass
    const char* b;
    int64_t ldb;
    const float* scale;  // of the rows of a DOWN B
    int64_t R, M, N;
    int steps, parts;  // steps of one pass: R / 64, rounded up
};

// The tile of such a product (see shape_of).  A step with several parts of A takes them
// one after the other (256), or together, with the loads of B once; one whose 8-bit
// operand is converted on its way takes about as long as one of three parts, by the
// kernels with a wavefront a SIMD.
inline Shape grad_shape(int64_t M, int64_t N, int64_t steps, int parts, bool down) {
    const int p = down ? 3 : parts, each = 230 + 390 * p;
    const TileCost tiles[] = {
        {256, 256, p * 1800, p * 1800, 0},
        {256, 128, p * 1100, p * 1100, 0},
        {128, 128, down ? each : 310 + 290 * p, each, down ? 0 : 800},
        {64, 64, 250 + 100 * p, 105 + 115 * p, 0}};
    return least_of(tiles, M, N, steps);
}

template <int BM, int BN, int WM, int WN, bool ADOWN, bool BDOWN, int P, int S, int KS = 1>
struct GradGemm {
    using G = Gemm<Bf16, BM, BN, WM, WN, 2>;
    static constexpr int kWaves = WM * WN * KS;
    static constexpr int MT = BM / WM / 16, NT = BN / WN / 16;
    static_assert(!BDOWN || NT == 4, "4 columns of B a lane");
    static_assert(BDOWN || !ADOWN, "as it is, A meets B as it is");
    static_assert(P == 1 || !BDOWN, "parts are laid out");
    static_assert(KS == 1 || !BDOWN, "halves of laid out steps");
    static constexpr int kRows = kStep / 2;  // of a step
    static constexpr int kPart = BM * kStep, kA = P * kPart, kB = BDOWN ? kRows * BN : BN * kStep;
    static constexpr int kBuffer = kA + kB + (BDOWN ? 256 : 0);
    static constexpr int kLoadsA = kPart / 1024 / kWaves, kLoadsB = kB / 1024 / kWaves;
    static_assert(kLoadsA * kWaves * 1024 == kPart && kLoadsB * kWaves * 1024 == kB, "whole loads");

    // B: the row of a step at place s of LDS, and the exchange of its pieces.  A read
    // takes 64 bytes of each of 4 places: they have to fill 256 bytes together.
    static __device__ __forceinline__ int row_at(int s) {
        return (s & 32) | (s & 3) << 3 | (s >> 2 & 7);
    }
    static __device__ __forceinline__ int place_b(int s) {
        return BN == 256 ? (s & 3) << 2 : BN == 128 ? (s >> 1 & 1) << 2 : 0;
    }
    // A: half the lanes read 32 bytes of rows r to r + 3 and r + 8 to r + 11
    static __device__ __forceinline__ int place_a(int r) {
        return BM >= 128 ? ((r & 3) | (r >> 3 & 1) << 2) << 1
                         : ((r >> 1 & 1) | (r >> 3 & 1) << 1) << 1;
    }

    struct Half {
        u32x4 a[P][MT], b[NT];  // operands
        uint32_t q[8];          // DOWN B, as it is: 8 rows of 4 columns,
        f32x4 s[2];             // and their scales
    };
    // 32-bit offsets of a lane's loads from the tile's first row (DOWN: the step's
    // first row, the tile's first column).  Rows of C, and DOWN pieces of columns,
    // that are not there repeat the last one.
    struct Offsets {
        uint32_t a[kLoadsA], b[kLoadsB];
    };
    static __device__ __forceinline__ Offsets offsets(const GradOperands& o, const TileAt& tile,
                                                      int wave, int lane) {
        Offsets l;
#pragma unroll
        for (int j = 0; j < kLoadsA; ++j) {
            if constexpr (ADOWN) {
                const int row = row_a(j, wave, lane);
                const int piece = lane % (BM / 8) ^ place_a(row);
                const int64_t last = (o.M - 1 - tile.m) / 8;
                l.a[j] = (uint32_t)(row * o.lda) + ((piece < last ? piece : (int)last) << 4);
            } else {
                const int row = (j * kWaves + wave) * 8 + (lane >> 3);
                const int64_t m = tile.m + row < o.M ? row : o.M - 1 - tile.m;
                l.a[j] = (uint32_t)(m * o.lda) + (((lane & 7) ^ G::place_a(row)) << 4);
            }
        }
#pragma unroll
        for (int j = 0; j < kLoadsB; ++j) {
            if constexpr (BDOWN) {
                const int s = place_of_b(j, wave, lane);
                const int piece = lane % (BN / 16) ^ place_b(s);
                const int64_t last = (o.N - 1 - tile.n) / 16;
                l.b[j] = (uint32_t)(row_at(s) * o.ldb) + ((piece < last ? piece : (int)last) << 4);
            } else {
                const int row = (j * kWaves + wave) * 8 + (lane >> 3);
                const int64_t n = tile.n + row < o.N ? row : o.N - 1 - tile.n;
                l.b[j] = (uint32_t)(n * o.ldb) + (((lane & 7) ^ G::place_b(row)) << 4);
            }
        }
        return l;
    }
    // row of A, and place of B, that a lane's load j fills
    static __device__ __forceinline__ int row_a(int j, int wave, int lane) {
        return (j * kWaves + wave) * 512 / BM + lane / (BM / 8);
    }
    static __device__ __forceinline__ int place_of_b(int j, int wave, int lane) {
        return (j * kWaves + wave) * (1024 / BN) + lane / (BN / 16);
    }

    // Sends for a step that begins at a, b and `scale`; `rows` of its 64 rows are
    // there, all of them unless LAST.
    template <bool LAST>
    static __device__ __forceinline__ void fetch(const char* a, int64_t a_part, const char* b,
                                                 const float* scale, int64_t rows,
                                                 const Offsets& l, char* lds, int wave, int lane) {
        const char* nothing = reinterpret_cast<const char*>(kNothing);
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int j = 0; j < kLoadsA; ++j) {
                const bool there = !LAST || !ADOWN || row_a(j, wave, lane) < rows;
                to_lds(there ? a + p * a_part + l.a[j] : nothing,
                       lds + p * kPart + (j * kWaves + wave) * 1024);
            }
#pragma unroll
        for (int j = 0; j < kLoadsB; ++j) {
            const bool there = !LAST || !BDOWN || row_at(place_of_b(j, wave, lane)) < rows;
            to_lds(there ? b + l.b[j] : nothing, lds + kA + (j * kWaves + wave) * 1024);
        }
        if constexpr (BDOWN) {
            if (wave == 0) {
                const char* p = reinterpret_cast<const char*>(scale + lane);
                __builtin_amdgcn_global_load_lds(
                    (__attribute__((address_space(1))) void*)(!LAST || lane < rows ? p : nothing),
                    (__attribute__((address_space(3))) void*)(lds + kA + kB), 4, 0, 0);
            }
        }
    }

    // lane's places in a buffer
    struct At {
        int a, b, s;
        int swap;  // laid out operands
    };
    static __device__ __forceinline__ At at(int wave, int lane) {
        At t;
        const int wm = wave / WN % WM, wn = wave % WN, r = lane & 15, g = lane >> 4;
        t.swap = (g ^ (r >> 1)) << 4;
        if constexpr (ADOWN) {
            // row 8 g + r / 4, columns 4 (r % 4) on
            const int row = g * 8 + (r >> 2), byte = wm * MT * 32 + (r & 3) * 8;
            t.a = row * BM * 2 + ((byte >> 4 ^ place_a(row)) << 4) + (byte & 15);
        } else {
            t.a = (wm * MT * 16 + r) * kStep;
        }
        const int byte = wn * 64 + r * 4;
        t.b = kA + (BDOWN ? g * BN + ((byte >> 4 ^ place_b(g)) << 4) + (byte & 15)
                          : (wn * NT * 16 + (r >> 2) * 4 * NT + (r & 3)) * kStep);
        t.s = kA + kB + g * 32;
        return t;
    }

    static __device__ __forceinline__ void read(Half& h, const char* lds, const At& t, int half) {
        if constexpr (BDOWN) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                h.q[i] = *reinterpret_cast<const uint32_t*>(lds + t.b + (half * 32 + i * 4) * BN);
#pragma unroll
            for (int i = 0; i < 2; ++i)
                h.s[i] = *reinterpret_cast<const f32x4*>(lds + t.s + half * 128 + i * 16);
        } else {
#pragma unroll
            for (int j = 0; j < NT; ++j)
                h.b[j] = *reinterpret_cast<const u32x4*>(lds + t.b + j * 4 * kStep +
                                                         (t.swap ^ (half << 6)));
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            if constexpr (ADOWN) {
                // (a tile of 16 columns is 2 pieces on: the exchange flips bits of
                // that count, so it is flipped in rather than added)
                const char* p = lds + (t.a ^ i << 5) + half * 32 * BM * 2;
                const u32x2 lo = read_down(p), hi = read_down(p + 4 * BM * 2);
                h.a[0][i] = u32x4{lo[0], lo[1], hi[0], hi[1]};
            } else {
#pragma unroll
                for (int p = 0; p < P; ++p)
                    h.a[p][i] = *reinterpret_cast<const u32x4*>(
                        lds + p * kPart + t.a + i * 16 * kStep + (t.swap ^ (half << 6)));
            }
        }
    }
    // 4 rows of the lane's column
    static __device__ __forceinline__ u32x2 read_down(const char* p) {
        return __builtin_bit_cast(
            u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                       (__attribute__((address_space(3))) i16x4*)(p)));
    }

    // a DOWN B's 4 columns as operands
    static __device__ __forceinline__ void convert(Half& h) {
        if constexpr (BDOWN) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float x = (float)(int8_t)(h.q[2 * k] >> (8 * c));
                    const float y = (float)(int8_t)(h.q[2 * k + 1] >> (8 * c));
                    h.b[c][k] =
                        narrow2(x * h.s[k / 2][2 * k % 4], y * h.s[k / 2][2 * k % 4 + 1]);
                }
        }
    }

    static __device__ __forceinline__ void multiply(const Half& h, f32x4 (&acc)[MT][NT]) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int p = 0; p < P; ++p)
                    acc[i][j] = Bf16::mfma(h.b[j], h.a[p][i], acc[i][j]);
    }

    // (see Gemm) spreads the reads, and LOADS loads, over the matrix instructions
    template <int LOADS>
    static __device__ __forceinline__ void spread() {
        if constexpr (BDOWN) return;
        constexpr int kReads = P * MT + NT;
        constexpr int kEach = P * MT * NT / kReads > 0 ? P * MT * NT / kReads : 1;
#pragma unroll
        for (int i = 0; i < kReads; ++i) {
            if (i < LOADS) __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);  // a load
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);                 // an LDS read
            __builtin_amdgcn_sched_group_barrier(0x008, kEach, 0);             // multiplies
        }
    }

    static __device__ __forceinline__ void run(const GradOperands& o, const Target& t, int64_t tiles_m,
                               int64_t tiles_n, int slices) {
        __shared__ __attribute__((aligned(1024))) char lds[S * kBuffer];
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int lane = threadIdx.x & 63;
        const TileAt tile = tile_at(tiles_m, tiles_n, BM, BN);
        const Offsets l = offsets(o, tile, wave, lane);
        // DOWN: a step is 64 rows on, and the tile's columns begin at its first
        const char* a0 = o.a + (ADOWN ? tile.m * 2 : tile.m * o.lda);
        const char* b0 = o.b + (BDOWN ? tile.n : tile.n * o.ldb);
        const int64_t a_step = ADOWN ? kRows * o.lda : kStep;
        const int64_t b_step = BDOWN ? kRows * o.ldb : kStep;
        const int passes = o.parts / P, steps = o.steps * passes;
        const int k0 = (int)((int64_t)steps * tile.slice / slices);
        const int k1 = (int)((int64_t)steps * (tile.slice + 1) / slices);
        int pass = k0 / o.steps, in_pass = k0 - pass * o.steps;
        // sends for the next step; LAST: it may be the last one, of fewer rows
        const auto send = [&](char* buffer, auto last) {
            fetch<last>(a0 + pass * o.a_part + in_pass * a_step, o.a_part, b0 + in_pass * b_step,
                        o.scale + (int64_t)in_pass * kRows, o.R - (int64_t)in_pass * kRows, l,
                        buffer, wave, lane);
            const bool wrap = ++in_pass == o.steps;
            in_pass = wrap ? 0 : in_pass;
            pass += wrap;
        };

        const At at_ = at(wave, lane);
        const int wk = KS == 1 ? 0 : wave / (WM * WN);  // (see Gemm)
        f32x4 acc[MT][NT] = {};
        Half h0, h1;
        // loads of a step; the first wavefront has the scales too
        constexpr int kLoads = P * kLoadsA + kLoadsB;
        const auto wait = [&](auto steps) {
            if (BDOWN && wave == 0) wait_loads<steps * (kLoads + 1)>();
            else wait_loads<steps * kLoads>();
        };
        if (k0 < k1) {
#pragma unroll
            for (int i = 0; i < S; ++i)
                if (k0 + i < k1) send(lds + i * kBuffer, std::true_type());
            if (BDOWN && wave == 0) wait_steps<S - 1, kLoads + 1>(k1 - k0 - 1);
            else wait_steps<S - 1, kLoads>(k1 - k0 - 1);
            barrier();
            read(h0, lds, at_, wk);
            convert(h0);
        }
        // one step; `ahead` steps (S: or more) come after it, S + 1: the step S on may
        // be the last, of fewer rows
        const auto step = [&](int k, auto ahead) {
            constexpr int kAhead = ahead;
            char* now = lds + (k - k0) % S * kBuffer;
            char* then = lds + (k - k0 + 1) % S * kBuffer;
            if constexpr (KS == 1) {
                read(h1, now, at_, 1);
                multiply(h0, acc);
                spread<0>();
                convert(h1);
            }
            wait(Int<(kAhead >= S ? S - 2 : kAhead >= 2 ? kAhead - 1 : 0)>());
            barrier();
            if constexpr (kAhead >= S) send(now, std::integral_constant<bool, (kAhead > S)>());
            if constexpr (KS == 2) {
                if constexpr (kAhead >= 1) read(h1, then, at_, wk);
                multiply(h0, acc);
                if constexpr (kAhead >= 1) {
                    spread<kAhead >= S ? kLoads : 0>();
                    h0 = h1;
                }
                return;
            }
            if constexpr (kAhead >= 1) read(h0, then, at_, 0);
            multiply(h1, acc);
            if constexpr (kAhead >= 1) {
                spread<kAhead >= S ? kLoads : 0>();
                convert(h0);
            }
        };
        int k = k0;
        if constexpr (ADOWN || BDOWN) {
            for (; k < k1 - S - 1; ++k) step(k, Int<S>());
            if (k < k1 - S) step(k++, Int<S + 1>());
        } else {
            for (; k < k1 - S; ++k) step(k, Int<S>());
        }
        if constexpr (S > 3)
            if (k < k1 - 3) step(k++, Int<3>());
        if constexpr (S > 2)
            if (k < k1 - 2) step(k++, Int<2>());
        if (k < k1 - 1) step(k++, Int<1>());
        if (k < k1) step(k, Int<0>());

        constexpr int MO = MT / KS;
        f32x4 sum[MO][NT];
        if constexpr (KS == 1) {
#pragma unroll
            for (int i = 0; i < MO; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) sum[i][j] = acc[i][j];
        } else {
            static_assert(kWaves * MO * NT * 1024 <= S * kBuffer, "the sums' room");
            join_halves<WM * WN>(acc, sum, lds, wave, lane);
        }

        // lane: 4 NT columns of MO rows
        const int wm = wave / WN % WM, wn = wave % WN, r = lane & 15, g = lane >> 4;
        const int64_t n = tile.n + wn * NT * 16;
#pragma unroll
        for (int i = 0; i < MO; ++i) {
            const int64_t m = tile.m + (wm * MT + wk * MO + i) * 16;
            float v[4 * NT];
#pragma unroll
            for (int c = 0; c < 4 * NT; ++c)
                v[c] = BDOWN ? sum[i][c % 4][c / 4] : sum[i][c / 4][c % 4];
            if (slices > 1) {
                u32x4 p[NT];
#pragma unroll
                for (int c = 0; c < 4 * NT; ++c) p[c / 4][c % 4] = __float_as_uint(v[c]);
                // (the workspace has rows of whole tiles)
                store_turned(p, static_cast<uint32_t*>(t.ws) + tile.slice * t.slice + m * t.ldws + n,
                             t.ldws, o.M - m, t.ldws - n, r, g);
            } else {
                store_rows<NT>(t, m, n, o.M - m, o.N - n, r, g, v);
            }
        }
    }
};

template <int BM, int BN, int WM, int WN, bool ADOWN, bool BDOWN, int P, int S, int KS>
__global__ __launch_bounds__(64 * WM * WN * KS) void grad_gemm_kernel(GradOperands o, Target t,
                                                                      int64_t tiles_m,
                                                                      int64_t tiles_n,
                                                                      int slices) {
    GradGemm<BM, BN, WM, WN, ADOWN, BDOWN, P, S, KS>::run(o, t, tiles_m, tiles_n, slices);
}

template <int BM, int BN, int WM, int WN, bool ADOWN, bool BDOWN, int P, int S, int KS>
int launch_grad_kernel(const GradOperands& o, const Target& t, int slices, void* stream) {
    const int64_t tm = up(o.M, BM), tn = up(o.N, BN), blocks = tm * tn * slices;
    constexpr int kThreads = 64 * WM * WN * KS;
    if (blocks * kThreads >= ((int64_t)1 << 32)) return (int)hipErrorInvalidValue;
    return launch(grad_gemm_kernel<BM, BN, WM, WN, ADOWN, BDOWN, P, S, KS>, dim3((uint32_t)blocks),
                  kThreads, stream, o, t, tm, tn, slices);
}
template <int BM, int BN, int WM, int WN, bool ADOWN, bool BDOWN, int P>
int launch_grad_tiles(const GradOperands& o, const Target& t, int slices, void* stream) {
    const int64_t blocks = up(o.M, BM) * up(o.N, BN) * slices;
    constexpr int kDeep = 4 * GradGemm<BM, BN, WM, WN, ADOWN, BDOWN, P, 4>::kBuffer;
    // (64 x 64 tiles gain nothing by it)
    if constexpr (BM == 128 && !BDOWN)
        if (blocks <= kCus)
            return launch_grad_kernel<BM, BN, WM, WN, ADOWN, BDOWN, P,
                                      kDeep <= 160 * 1024 ? 4 : 2, 2>(o, t, slices, stream);
    if constexpr ((BM == 64 || (BM == 128 && BDOWN)) && kDeep <= 160 * 1024)
        if (all_at_once(blocks, kDeep))
            return launch_grad_kernel<BM, BN, WM, WN, ADOWN, BDOWN, P, 4, 1>(o, t, slices, stream);
    constexpr int S = BM + BN == 384 ? 3 : 2;
    return launch_grad_kernel<BM, BN, WM, WN, ADOWN, BDOWN, P, S, 1>(o, t, slices, stream);
}

template <bool ADOWN, bool BDOWN, int P>
int launch_grad_gemm(const GradOperands& o, Target t, const Shape& s, void* ws, void* stream) {
    t.ws = ws;
    t.ldws = slices_ld(o.N);
    t.slice = o.M * t.ldws;
    // (as it is, the 8-bit operand of dx meets at most 128 rows: never this tile,
    // whose LDS holds one part)
    if constexpr (ADOWN || !BDOWN)
        if (s.bn == 256) return launch_grad_tiles<256, 256, 2, 4, ADOWN, BDOWN, 1>(o, t, 1, stream);
    // (with more parts than one, two tiles of 128 x 128 take less than this one)
    if constexpr (!BDOWN && P == 1)
        if (s.bm == 256) return launch_grad_tiles<256, 128, 4, 2, false, false, 1>(o, t, 1, stream);
    if (s.bm >= 128) return launch_grad_tiles<128, 128, 2, 2, ADOWN, BDOWN, P>(o, t, 1, stream);
    // (a DOWN B is read 4 columns a lane: 64 a wavefront)
    constexpr int WM = BDOWN ? 4 : 2;
    if (int e = launch_grad_tiles<64, 64, WM, 4 / WM, ADOWN, BDOWN, P>(o, t, s.slices, stream))
        return e;
    if (s.slices == 1) return 0;
    return launch_join<Bf16>(t, o.M, o.N, s.slices, stream);
}

}  // namespace
}  // namespace q8
}  // namespace cpdp
