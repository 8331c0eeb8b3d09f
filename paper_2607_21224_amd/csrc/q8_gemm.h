// Matrix products C[M x N] = A[M x K] B[N x K]^T on the matrix cores, both
// operands with K contiguous: int8 with 32-bit integer sums, or bf16 with fp32
// sums.
//
// A block computes a BM x BN tile of C with WM x WN wavefronts.  It walks K in
// steps of 128 bytes a row; the step's rows of A and B go from memory straight
// into one of S LDS buffers (16 bytes a lane, no registers in between) while the
// matrix cores work on another.  Two buffers do where a CU has several blocks, or a
// step's work takes as long as its loads; with a block a CU or two, small tiles have
// four, so that loads are sent for three steps ahead.  The 16-byte pieces of a row are stored
// permuted (piece p of row r at place p ^ f(r)), so that the 16 lanes that read
// the same piece of 16 rows touch all 64 banks.  The permutation is applied to
// the address that a lane loads from; a row's 128 bytes stay one request.
//
// The 16 x 16 instructions take the rows of B as their first operand, in an
// order that leaves each lane with 4 NT consecutive columns of one row of C:
// row r of instruction tile j is column (r / 4) 4 NT + 4 j + r % 4 of the
// wavefront's 16 NT.  Stores are then 16 bytes and more a lane.
#pragma once

#include "q8_device.h"

namespace cpdp {
namespace q8 {
namespace {

constexpr int kStep = 128;  // bytes of a row in one step

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// The matrix-core instruction of an operand type, its sums and their type.
struct Int8 {
    using Acc = i32x4;
    using Sum = int32_t;
    static __device__ __forceinline__ Acc mfma(u32x4 a, u32x4 b, Acc c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a),
                                                     __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
    }
};
struct Bf16 {
    using Acc = f32x4;
    using Sum = float;
    static __device__ __forceinline__ Acc mfma(u32x4 a, u32x4 b, Acc c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};

// Operands of a product.
struct Operands {
    const char* a;
    const char* b;
    int64_t lda, ldb;  // bytes from row to row, below 2^23
    int64_t M, N;
    int row;  // bytes of a row that are there
};

// Where the sums of a product go: C in its own type, or (slices > 1) the sums of
// one slice of K as they are, at ws[slice][row][column].
struct Target {
    void* c;
    int64_t ldc;
    bool bf16;
    const float* row_scale;  // of the rows and columns of C, or null
    const float* col_scale;
    void* ws;
    int64_t ldws, slice;  // elements
};

__device__ __forceinline__ void to_lds(const char* src, char* dst) {
    __builtin_amdgcn_global_load_lds(
        (__attribute__((address_space(1))) void*)(src),
        (__attribute__((address_space(3))) void*)(dst), 16, 0, 0);
}

// Waits until at most N of the wavefront's loads are on their way, and all that it
// reads from LDS has come.
template <int N>
__device__ __forceinline__ void wait_loads() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | (N >> 4) << 14);
    asm volatile("" ::: "memory");
}
// The same for the loads of `steps` (at most MOST) steps, EACH of a step.
template <int MOST, int EACH>
__device__ __forceinline__ void wait_steps(int steps) {
    if constexpr (MOST == 0) {
        wait_loads<0>();
    } else {
        if (steps >= MOST) wait_loads<MOST * EACH>();
        else wait_steps<MOST - 1, EACH>(steps);
    }
}
// A barrier that waits for no load (the caller has waited for those it needs).
__device__ __forceinline__ void barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// 16 bytes at p, of which the first n exist (n may be negative) and `before` bytes
// of the row come before p.  A piece that is cut short is read as the row's last
// 16 bytes, shifted into place; a row shorter than that, byte by byte.
__device__ __forceinline__ u32x4 load_tail(const char* p, int n, int before) {
    if (n >= 16) return *reinterpret_cast<const u32x4*>(p);
    u32x4 v = {0, 0, 0, 0};
    if (n <= 0) return v;
    if (before + n >= 16) {
        const u32x4 x = *reinterpret_cast<const u32x4_any*>(p + n - 16);
        const unsigned __int128 all = __builtin_bit_cast(unsigned __int128, x);
        return __builtin_bit_cast(u32x4, all >> (8 * (16 - n)));
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (i < n) v[i / 4] |= (uint32_t)(uint8_t)p[i] << (8 * (i % 4));
    return v;
}

// n (at most COLS) consecutive results of one row
template <int COLS>
__device__ __forceinline__ void store_cols(const Target& t, int64_t m, int64_t n0, int n,
                                           const float (&v)[COLS]) {
    static_assert(COLS % 8 == 0 || COLS == 4, "whole pieces");
    if (t.bf16) {
        uint16_t* p = static_cast<uint16_t*>(t.c) + m * t.ldc + n0;
        if (n >= COLS) {
#pragma unroll
            for (int k = 0; k < COLS; k += 4)
                *reinterpret_cast<u32x2*>(p + k) =
                    u32x2{narrow2(v[k], v[k + 1]), narrow2(v[k + 2], v[k + 3])};
        } else {
#pragma unroll
            for (int k = 0; k < COLS; ++k)
                if (k < n) narrow(v[k], p + k);
        }
    } else {
        float* p = static_cast<float*>(t.c) + m * t.ldc + n0;
        if (n >= COLS) {
#pragma unroll
            for (int k = 0; k < COLS; k += 4)
                *reinterpret_cast<f32x4*>(p + k) = f32x4{v[k], v[k + 1], v[k + 2], v[k + 3]};
        } else {
#pragma unroll
            for (int k = 0; k < COLS; ++k)
                if (k < n) p[k] = v[k];
        }
    }
}

// A wavefront's 16 rows of C, as the matrix instructions leave them: lane (g, r) has
// row r, and PIECES pieces of 16 bytes from PIECES g on.  A store of one piece a lane
// would touch every row, and 16 bytes of every 32 or 64.  So the lanes r of 16
// exchange pieces until piece i of a lane is of row row_of(i), its place there
// place_of(): a store then covers whole rows.  Written as they are, 4096 x 4096 x 256
// took 30 us (fp32) and 17 (bf16), and so 18 and 15.  Stores past the caches took 13
// in bf16, but whoever reads the results then pays for it and more (8192 x 8192 x
// 1024 and the rows made 8-bit: 127 us, and 115 so).
template <int PIECES>
struct Turn {
    static_assert(PIECES == 1 || PIECES == 2 || PIECES == 4, "a power of two");
    static __device__ __forceinline__ int row_of(int i, int r) {
        return PIECES == 1 ? r : PIECES == 2 ? (r & 7) | i << 3 : (r & 3) | i << 2;
    }
    static __device__ __forceinline__ int place_of(int g, int r) {
        return PIECES == 1 ? g : PIECES == 2 ? g << 1 | r >> 3 : g << 2 | r >> 2;
    }
    // gives the lower lane's b for the a of the one ACROSS (8 or 4) above it
    template <int ACROSS>
    static __device__ __forceinline__ void swap(u32x4& a, u32x4& b, int r) {
        const bool upper = (r & ACROSS) != 0;
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            uint32_t x = upper ? a[d] : b[d];
            if constexpr (ACROSS == 8) {
                x = __builtin_amdgcn_update_dpp(0, x, 0x128, 15, 15, true);  // row_ror:8
            } else {
                x = __builtin_amdgcn_update_dpp(0, x, 0x141, 15, 15, true);  // row_half_mirror
                x = __builtin_amdgcn_update_dpp(0, x, 0x1b, 15, 15, true);   // quad_perm:[3,2,1,0]
            }
            a[d] = upper ? x : a[d];
            b[d] = upper ? b[d] : x;
        }
    }
    static __device__ __forceinline__ void run(u32x4 (&p)[PIECES], int r) {
        if constexpr (PIECES == 2) {
            swap<8>(p[0], p[1], r);
        }
        if constexpr (PIECES == 4) {
            swap<8>(p[0], p[2], r);
            swap<8>(p[1], p[3], r);
            swap<4>(p[0], p[1], r);
            swap<4>(p[2], p[3], r);
        }
    }
};
// Stores them to the rows at c, E as wide as an element; `rows` and `cols` are there.
template <class E, int PIECES>
__device__ __forceinline__ void store_turned(u32x4 (&p)[PIECES], E* c, int64_t ld, int64_t rows,
                                             int64_t cols, int r, int g) {
    using T = Turn<PIECES>;
    constexpr int kEach = 16 / sizeof(E);
    T::run(p, r);
    const int col = T::place_of(g, r) * kEach;
    const int n = cols - col < kEach ? (int)(cols - col) : kEach;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int row = T::row_of(i, r);
        if (row >= rows) continue;
        E* at = c + row * ld + col;
        if (n == kEach) {
            *reinterpret_cast<u32x4*>(at) = p[i];
        } else {
#pragma unroll
            for (int k = 0; k < kEach - 1; ++k)
                if (k < n)
                    at[k] = (E)(p[i][k * sizeof(E) / 4] >> (sizeof(E) == 2 ? 16 * (k % 2) : 0));
        }
    }
}

// The same for numbers v of C: 4 NT consecutive columns of row m + r a lane.
template <int NT>
__device__ __forceinline__ void store_rows(const Target& t, int64_t m, int64_t n, int64_t rows,
                                           int64_t cols, int r, int g, const float (&v)[4 * NT]) {
    if (t.bf16) {
        u32x4 p[NT / 2];
#pragma unroll
        for (int k = 0; k < 4 * NT; k += 2) p[k / 8][k % 8 / 2] = narrow2(v[k], v[k + 1]);
        store_turned(p, static_cast<uint16_t*>(t.c) + m * t.ldc + n, t.ldc, rows, cols, r, g);
    } else {
        u32x4 p[NT];
#pragma unroll
        for (int k = 0; k < 4 * NT; ++k) p[k / 4][k % 4] = __float_as_uint(v[k]);
        store_turned(p, static_cast<uint32_t*>(t.c) + m * t.ldc + n, t.ldc, rows, cols, r, g);
    }
}

// The tile of a block.  Blocks are dealt to the 8 XCDs in turn; each XCD takes a
// run of consecutive tiles, and those go down 8 rows of tiles before the next
// column, so that the tiles an XCD works on share rows of A and B in its L2.
struct TileAt {
    int64_t m, n;
    int slice;
};
__device__ __forceinline__ TileAt tile_at(int64_t tiles_m, int64_t tiles_n, int BM, int BN) {
    const int64_t tiles = tiles_m * tiles_n;
    const int64_t b = blockIdx.x, slice = b / tiles;
    int64_t t = b % tiles;
    const int64_t each = tiles / 8, rest = tiles % 8, xcd = t % 8;
    t = xcd * each + (xcd < rest ? xcd : rest) + t / 8;
    const int64_t band = t / (8 * tiles_n);
    const int64_t high = tiles_m - band * 8 < 8 ? tiles_m - band * 8 : 8;
    const int64_t in = t - band * 8 * tiles_n;
    return {(band * 8 + in % high) * BM, in / high * BN, (int)slice};
}

// Two groups of WAVES wavefronts have sums of the same rows of C over the two halves of
// the steps: each gives the other its sums of half the rows, and adds what it gets.
template <int WAVES, class Acc, int MT, int NT>
__device__ __forceinline__ void join_halves(const Acc (&acc)[MT][NT], Acc (&sum)[MT / 2][NT],
                                            char* lds, int wave, int lane) {
    const bool second = wave >= WAVES;
    auto* room = reinterpret_cast<Acc(*)[MT / 2][NT][64]>(lds);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MT / 2; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
            room[wave][i][j][lane] = second ? acc[i][j] : acc[MT / 2 + i][j];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MT / 2; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
            sum[i][j] = (second ? acc[MT / 2 + i][j] : acc[i][j]) + room[wave ^ WAVES][i][j][lane];
}

// KS == 2: the wavefronts are two groups, each with one half of every step.  With one
// block a CU a wavefront has a SIMD to itself and waits for what it has sent for; two
// share it, and each reads half as much of LDS for a step (1024 x 4096 x 4096 25 -> 20
// us, 2000^3 16.7 -> 14.8, 256 x 4096 x 4096 11.6 -> 10; with several blocks a CU it
// costs: 1576 x 1536 x 384 5.9 -> 8.4).
template <class Op, int BM, int BN, int WM, int WN, int S, int KS = 1>
struct Gemm {
    static constexpr int kWaves = WM * WN * KS;
    static constexpr int kThreads = 64 * kWaves;
    static constexpr int MT = BM / WM / 16, NT = BN / WN / 16;
    static constexpr int kLoadsA = BM / 8 / kWaves, kLoadsB = BN / 8 / kWaves;
    static constexpr int kBuffer = (BM + BN) * kStep;
    static_assert(kLoadsA * 8 * kWaves == BM && kLoadsB * 8 * kWaves == BN, "whole loads");

    static __device__ __forceinline__ int place_a(int row) { return (row >> 1) & 7; }
    static __device__ __forceinline__ int place_b(int row) {
        return ((row >> 1) & 1) | ((row / (4 * NT) & 3) << 1);
    }

    // 32-bit offsets of a lane's loads from the tile's first row; rows past the
    // matrix take its last one (their sums are not stored)
    struct Loads {
        uint32_t a[kLoadsA], b[kLoadsB];
    };
    static __device__ __forceinline__ Loads loads(const Operands& o, int64_t m0, int64_t n0,
                                                  int wave, int lane) {
        Loads l;
#pragma unroll
        for (int j = 0; j < kLoadsA; ++j) {
            const int row = (j * kWaves + wave) * 8 + (lane >> 3);
            const int64_t at = m0 + row < o.M ? row : o.M - 1 - m0;
            l.a[j] = (uint32_t)(at * o.lda) + (((lane & 7) ^ place_a(row)) << 4);
        }
#pragma unroll
        for (int j = 0; j < kLoadsB; ++j) {
            const int row = (j * kWaves + wave) * 8 + (lane >> 3);
            const int64_t at = n0 + row < o.N ? row : o.N - 1 - n0;
            l.b[j] = (uint32_t)(at * o.ldb) + (((lane & 7) ^ place_b(row)) << 4);
        }
        return l;
    }

    static __device__ __forceinline__ void fetch(const char* a, const char* b, const Loads& l,
                                                 char* lds, int wave) {
#pragma unroll
        for (int j = 0; j < kLoadsA; ++j) to_lds(a + l.a[j], lds + (j * kWaves + wave) * 1024);
#pragma unroll
        for (int j = 0; j < kLoadsB; ++j)
            to_lds(b + l.b[j], lds + BM * kStep + (j * kWaves + wave) * 1024);
    }

    // the last, short step of a row: through registers, zeros past the end
    struct Tail {
        u32x4 a[kLoadsA], b[kLoadsB];
    };
    static __device__ __forceinline__ void load(Tail& t, const char* a, const char* b,
                                                const Loads& l, int wave, int lane, int bytes,
                                                int before) {
#pragma unroll
        for (int j = 0; j < kLoadsA; ++j) {
            const int row = (j * kWaves + wave) * 8 + (lane >> 3);
            const int k = ((lane & 7) ^ place_a(row)) << 4;
            t.a[j] = load_tail(a + l.a[j], bytes - k, before + k);
        }
#pragma unroll
        for (int j = 0; j < kLoadsB; ++j) {
            const int row = (j * kWaves + wave) * 8 + (lane >> 3);
            const int k = ((lane & 7) ^ place_b(row)) << 4;
            t.b[j] = load_tail(b + l.b[j], bytes - k, before + k);
        }
    }
    static __device__ __forceinline__ void store(const Tail& t, char* lds, int wave, int lane) {
#pragma unroll
        for (int j = 0; j < kLoadsA; ++j)
            *reinterpret_cast<u32x4*>(lds + (j * kWaves + wave) * 1024 + (lane << 4)) = t.a[j];
#pragma unroll
        for (int j = 0; j < kLoadsB; ++j)
            *reinterpret_cast<u32x4*>(lds + BM * kStep + (j * kWaves + wave) * 1024 +
                                      (lane << 4)) = t.b[j];
    }

    // the operands of half a step: 64 bytes of the wavefront's rows
    struct Half {
        u32x4 a[MT], b[NT];
    };
    static __device__ __forceinline__ void read(Half& h, const char* at_a, const char* at_b,
                                                int half, int swap) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
            h.b[j] = *reinterpret_cast<const u32x4*>(at_b + j * 4 * kStep + (swap ^ (half << 6)));
#pragma unroll
        for (int i = 0; i < MT; ++i)
            h.a[i] = *reinterpret_cast<const u32x4*>(at_a + i * 16 * kStep + (swap ^ (half << 6)));
    }
    static __device__ __forceinline__ void multiply(const Half& h,
                                                    typename Op::Acc (&acc)[MT][NT]) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = Op::mfma(h.b[j], h.a[i], acc[i][j]);
    }
    // tells the scheduler to spread LOADS loads of a step to come and the reads of
    // the next half over the matrix instructions of this one
    template <int LOADS>
    static __device__ __forceinline__ void spread() {
        constexpr int kReads = MT + NT, kEach = MT * NT / kReads > 0 ? MT * NT / kReads : 1;
#pragma unroll
        for (int i = 0; i < kReads; ++i) {
            if (i < LOADS) __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);  // a load
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);                 // an LDS read
            __builtin_amdgcn_sched_group_barrier(0x008, kEach, 0);             // multiplies
        }
    }

    static __device__ __forceinline__ void run(const Operands& o, const Target& t, int64_t tiles_m,
                               int64_t tiles_n, int slices) {
        __shared__ __attribute__((aligned(1024))) char lds[S * kBuffer];
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int lane = threadIdx.x & 63;
        const TileAt tile = tile_at(tiles_m, tiles_n, BM, BN);
        const Loads l = loads(o, tile.m, tile.n, wave, lane);
        const char* a0 = o.a + tile.m * o.lda;
        const char* b0 = o.b + tile.n * o.ldb;

        // whole steps of this slice: k0 to k1, and the short one at the end of the
        // last slice
        const int steps = o.row / kStep, tail = o.row % kStep;
        const int k0 = (int)((int64_t)steps * tile.slice / slices);
        const int k1 = (int)((int64_t)steps * (tile.slice + 1) / slices);

        typename Op::Acc acc[MT][NT] = {};
        // KS == 2: which half of a step the wavefront takes, and then of its rows of C
        const int wk = KS == 1 ? 0 : wave / (WM * WN);
        const int wm = wave / WN % WM, wn = wave % WN, r = lane & 15, g = lane >> 4;
        const int off_a = (wm * MT * 16 + r) * kStep;
        const int off_b = BM * kStep + (wn * NT * 16 + (r >> 2) * 4 * NT + (r & 3)) * kStep;
        const int swap = (g ^ (r >> 1)) << 4;

        // Up to S steps are on their way or in LDS, and half a step in registers.  A
        // step's first half is multiplied while its second is read; then, its LDS
        // buffer done with, one barrier, and the step S on is sent for into that
        // buffer while the second half is multiplied and the next step's first is
        // read.
        // What the end needs, the short step and the scales, is sent for first where
        // registers are to be had and a block's time short enough for it to show
        // (2000 x 2000 x 2000 18.5 us, and 19.8 with both at the end; 1576 x 1153 x
        // 385 8.1 and 8.4).
        constexpr bool kEarly = BM <= 128;
        constexpr int COLS = 4 * NT, MO = MT / KS;
        const int64_t n0 = tile.n + wn * NT * 16 + g * COLS;
        const bool has_tail = tail != 0 && tile.slice == slices - 1;
        Tail last;
        float cs[COLS], rs[MO];
        const auto scales = [&] {
            if (slices > 1 || t.row_scale == nullptr) return;
#pragma unroll
            for (int k = 0; k < COLS; ++k) {
                const int64_t c = n0 + k;
                cs[k] = t.col_scale[c < o.N ? c : o.N - 1];
            }
#pragma unroll
            for (int i = 0; i < MO; ++i) {
                const int64_t m = tile.m + (wm * MT + wk * MO + i) * 16 + r;
                rs[i] = t.row_scale[m < o.M ? m : o.M - 1];
            }
        };
        if constexpr (kEarly) {
            if (has_tail)
                load(last, a0 + (int64_t)steps * kStep, b0 + (int64_t)steps * kStep, l, wave, lane,
                     tail, steps * kStep);
            scales();
        }

        const char* a_at = a0 + (int64_t)k0 * kStep;
        const char* b_at = b0 + (int64_t)k0 * kStep;
        const auto send = [&](int k) {
            fetch(a_at, b_at, l, lds + (k - k0) % S * kBuffer, wave);
            a_at += kStep;
            b_at += kStep;
        };
        Half h0, h1;
        if (k0 < k1) {
#pragma unroll
            for (int i = 0; i < S; ++i)
                if (k0 + i < k1) send(k0 + i);
            // the first step has come, later ones may be on their way
            wait_steps<S - 1, kLoadsA + kLoadsB>(k1 - k0 - 1);
            barrier();
            read(h0, lds + off_a, lds + off_b, wk, swap);
        }
        // one step; `ahead` steps (S: or more) come after it
        const auto step = [&](int k, auto ahead) {
            constexpr int kAhead = ahead;
            char* now = lds + (k - k0) % S * kBuffer;
            char* then = lds + (k - k0 + 1) % S * kBuffer;
            if constexpr (KS == 1) {
                read(h1, now + off_a, now + off_b, 1, swap);
                multiply(h0, acc);
                spread<0>();
            }
            // the next step has come, and `now` has been read
            wait_loads<(kAhead >= S ? S - 2 : kAhead >= 2 ? kAhead - 1 : 0) *
                       (kLoadsA + kLoadsB)>();
            barrier();
            if constexpr (kAhead >= S) send(k + S);
            if constexpr (KS == 2) {
                if constexpr (kAhead >= 1) read(h1, then + off_a, then + off_b, wk, swap);
                multiply(h0, acc);
                if constexpr (kAhead >= 1) {
                    spread<kAhead >= S ? kLoadsA + kLoadsB : 0>();
                    h0 = h1;
                }
                return;
            }
            if constexpr (kAhead >= 1) read(h0, then + off_a, then + off_b, 0, swap);
            multiply(h1, acc);
            if constexpr (kAhead >= 1) spread<kAhead >= S ? kLoadsA + kLoadsB : 0>();
        };
        int k = k0;
        for (; k < k1 - S; ++k) step(k, Int<S>());
        if constexpr (S > 3)
            if (k < k1 - 3) step(k++, Int<3>());
        if constexpr (S > 2)
            if (k < k1 - 2) step(k++, Int<2>());
        if (k < k1 - 1) step(k++, Int<1>());
        if (k < k1) step(k, Int<0>());
        if (has_tail) {
            // no load is on its way, and all wavefronts are past their reads of every
            // buffer but the last step's
            char* now = lds + (k1 - k0) % S * kBuffer;
            if constexpr (!kEarly)
                load(last, a0 + (int64_t)steps * kStep, b0 + (int64_t)steps * kStep, l, wave, lane,
                     tail, steps * kStep);
            store(last, now, wave, lane);
            __syncthreads();
            read(h0, now + off_a, now + off_b, wk, swap);
            if constexpr (KS == 1) read(h1, now + off_a, now + off_b, 1, swap);
            multiply(h0, acc);
            if constexpr (KS == 1) multiply(h1, acc);
        }
        typename Op::Acc sum[MO][NT];
        if constexpr (KS == 1) {
#pragma unroll
            for (int i = 0; i < MO; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) sum[i][j] = acc[i][j];
        } else {
            static_assert(kWaves * MO * NT * 1024 <= S * kBuffer, "the sums' room");
            join_halves<WM * WN>(acc, sum, lds, wave, lane);
        }

        if constexpr (!kEarly) scales();
        const int64_t n_wave = tile.n + wn * NT * 16;
#pragma unroll
        for (int i = 0; i < MO; ++i) {
            const int64_t m = tile.m + (wm * MT + wk * MO + i) * 16;
            if (slices > 1) {
                u32x4 p[NT];
#pragma unroll
                for (int j = 0; j < NT; ++j) p[j] = __builtin_bit_cast(u32x4, sum[i][j]);
                // (the workspace has rows of whole tiles)
                store_turned(p, static_cast<uint32_t*>(t.ws) + tile.slice * t.slice + m * t.ldws +
                                    n_wave,
                             t.ldws, o.M - m, t.ldws - n_wave, r, g);
                continue;
            }
            float v[COLS];
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) v[4 * j + k] = (float)sum[i][j][k];
            if (t.row_scale != nullptr) {
#pragma unroll
                for (int k = 0; k < COLS; ++k) v[k] = v[k] * rs[i] * cs[k];
            }
            store_rows<NT>(t, m, n_wave, o.M - m, o.N - n_wave, r, g, v);
        }
    }
};

template <class Op, int BM, int BN, int WM, int WN, int S, int KS>
__global__ __launch_bounds__(64 * WM * WN * KS) void gemm_kernel(Operands o, Target t,
                                                                 int64_t tiles_m, int64_t tiles_n,
                                                                 int slices) {
    Gemm<Op, BM, BN, WM, WN, S, KS>::run(o, t, tiles_m, tiles_n, slices);
}

// Joins the slices of a product in their order: 4 columns a thread.
template <class Op>
__global__ __launch_bounds__(256) void join_kernel(Target t, int64_t M, int64_t N, int slices) {
    const int64_t across = (N + 3) / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t m = i / across, n0 = i % across * 4;
    if (m >= M) return;
    const auto* p = static_cast<const typename Op::Sum*>(t.ws) + m * t.ldws + n0;
    // slices are a power of two; up to 8 are on their way together
    typename Op::Acc s = {};
    const auto add = [&](int z, auto count) {
        typename Op::Acc v[count];
#pragma unroll
        for (int i = 0; i < count; ++i)
            v[i] = *reinterpret_cast<const typename Op::Acc*>(p + (z + i) * t.slice);
#pragma unroll
        for (int i = 0; i < count; ++i) s += v[i];
    };
    if (slices == 2) add(0, Int<2>());
    else if (slices == 4) add(0, Int<4>());
    else
        for (int z = 0; z < slices; z += 8) add(z, Int<8>());
    const int n = (int)(N - n0 < 4 ? N - n0 : 4);
    float v[4] = {(float)s[0], (float)s[1], (float)s[2], (float)s[3]};
    if (t.row_scale != nullptr) {
        const float rs = t.row_scale[m];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = v[k] * rs * t.col_scale[n0 + (k < n ? k : 0)];
    }
    store_cols<4>(t, m, n0, n, v);
}

// ---- which tile takes a product ----------------------------------------------------

struct Shape {
    int bm, bn;  // 256 x 256, 256 x 128, 128 x 128, 128 x 64 or 64 x 64
    int slices;  // of K
    double ns;   // it should take
};

inline int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The tile and the slices of K that should take the least time.  A step of a tile's
// block takes `alone` ns while its CU has no other (and `first` before the first and
// after the last), and the CU gets through one such step in `each` ns when it has
// several (0: not taken then; a tile of 128 x 64 is for up to twice as many tiles of
// 64 x 64 as there are CUs).  Measured on int8 products with N = K = 4096 and bf16
// results, calls that follow each other on one card, in us:
//   rows     256 x 256   256 x 128   128 x 128   128 x 64   64 x 64
//   256          43          28          19         13         11
//   512          44          29          20         14         16
//   1024         45          29          21         26         29
//   2048         46          34          38         49         53
//   4096         55          64          72         98        101
// and the rule takes the best of every row.
// Slices are added up by a second launch: its start, and each sum written and read
// again at 3 TB/s.
constexpr int64_t kCus = 256;

struct TileCost {
    int bm, bn, alone, each, first;
};
template <int TILES>
inline Shape least_of(const TileCost (&tiles)[TILES], int64_t M, int64_t N, int64_t steps) {
    Shape best = {256, 256, 1, -1};
    for (const auto& t : tiles) {
        const int64_t n = up(M, t.bm) * up(N, t.bn);
        // (a launch holds fewer than 2^32 work items, at most 512 a block)
        if (t.bm < 256 && n >= (int64_t)1 << 23) continue;
        for (int slices = 1; slices <= 64; slices *= 2) {
            if (slices > 1 && (t.bm != 64 || n * slices > 2048 || steps < 4 * slices)) break;
            const bool alone = n * slices <= kCus;
            if (!alone && t.each == 0) break;
            const double step = alone ? t.alone : (double)up(n * slices, kCus) * t.each;
            const double time = (double)up(steps, slices) * step + (alone ? t.first : 0) +
                                (slices > 1 ? 4500.0 + slices * (double)M * (double)N / 375.0 : 0);
            if (best.ns < 0 || time < best.ns) best = {t.bm, t.bn, slices, time};
        }
    }
    return best;
}
inline Shape shape_of(int64_t M, int64_t N, int64_t steps) {
    const TileCost tiles[] = {{256, 256, 1800, 1800, 0},
                              {256, 128, 1100, 1100, 0},
                              {128, 128, 540, 620, 800},
                              {128, 64, 350, 0, 500},
                              {64, 64, 280, 220, 0}};
    return least_of(tiles, M, N, steps);
}

// Workspace of a product's slices.
inline int64_t slices_ld(int64_t N) { return up(N, 64) * 64; }
inline int64_t slices_bytes(int64_t M, int64_t N, const Shape& s) {
    return s.slices == 1 ? 0 : s.slices * M * slices_ld(N) * 4;
}

// Whether all blocks of a launch are on the card at once, each with `bytes` of LDS.
inline bool all_at_once(int64_t blocks, int bytes) { return blocks <= kCus * (160 * 1024 / bytes); }

template <class Op, int BM, int BN, int WM, int WN, int S, int KS>
int launch_kernel(const Operands& o, const Target& t, int slices, void* stream) {
    const int64_t tm = up(o.M, BM), tn = up(o.N, BN), blocks = tm * tn * slices;
    constexpr int kThreads = 64 * WM * WN * KS;
    if (blocks * kThreads >= ((int64_t)1 << 32)) return (int)hipErrorInvalidValue;
    return launch(gemm_kernel<Op, BM, BN, WM, WN, S, KS>, dim3((uint32_t)blocks), kThreads, stream,
                  o, t, tm, tn, slices);
}
template <class Op, int BM, int BN, int WM, int WN>
int launch_tiles(const Operands& o, const Target& t, int slices, void* stream) {
    const int64_t blocks = up(o.M, BM) * up(o.N, BN) * slices;
    if constexpr (BM < 256)
        if (blocks <= kCus) return launch_kernel<Op, BM, BN, WM, WN, 4, 2>(o, t, slices, stream);
    // (four buffers of larger tiles leave a CU room for one block)
    if constexpr (BM == 64)
        if (all_at_once(blocks, Gemm<Op, BM, BN, WM, WN, 4>::kBuffer * 4))
            return launch_kernel<Op, BM, BN, WM, WN, 4, 1>(o, t, slices, stream);
    constexpr int S = BM + BN == 384 ? 3 : 2;
    return launch_kernel<Op, BM, BN, WM, WN, S, 1>(o, t, slices, stream);
}

template <class Op>
int launch_join(const Target& t, int64_t M, int64_t N, int slices, void* stream) {
    const int64_t items = M * up(N, 4);
    if (items >= ((int64_t)1 << 32) - 256) return (int)hipErrorInvalidValue;
    return launch(join_kernel<Op>, dim3((uint32_t)up(items, 256)), 256, stream, t, M, N, slices);
}

template <class Op>
int launch_gemm(const Operands& o, Target t, void* ws, void* stream) {
    const Shape s = shape_of(o.M, o.N, up(o.row, kStep));
    t.ws = ws;
    t.ldws = slices_ld(o.N);
    t.slice = o.M * t.ldws;
    if (s.bn == 256) return launch_tiles<Op, 256, 256, 2, 4>(o, t, 1, stream);
    if (s.bm == 256) return launch_tiles<Op, 256, 128, 4, 2>(o, t, 1, stream);
    if (s.bn == 128) return launch_tiles<Op, 128, 128, 2, 2>(o, t, 1, stream);
    if (s.bm == 128) return launch_kernel<Op, 128, 64, 2, 2, 4, 2>(o, t, 1, stream);
    if (int e = launch_tiles<Op, 64, 64, 2, 2>(o, t, s.slices, stream)) return e;
    if (s.slices == 1) return 0;
    return launch_join<Op>(t, o.M, o.N, s.slices, stream);
}

}  // namespace
}  // namespace q8
}  // namespace cpdp
