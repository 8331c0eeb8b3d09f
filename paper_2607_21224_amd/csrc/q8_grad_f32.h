// The product of a gradient with fp32 dy, which it takes as it is:
//   C[m, n] = sum over r of A[m, r] s[r] B[n, r]
// A is dy, its rows along the sum, or across it (DOWN); B the 8-bit operand, laid out
// as bf16 with r contiguous, unscaled.  A lane scales 8 values of A and takes them
// apart on their way from LDS to the matrix cores: the 24 significant bits of A s are
// three times 8, so three bf16 numbers hold it exactly.
//
// Laying dy out in three parts first writes 6 bytes a value, at about 2 TB/s from a
// launch this short; here it is work beside the matrix cores', some 9 vector
// instructions a value, which bounds the kernel: with several blocks a CU a step of a
// tile takes 560 ns, one of three parts laid out 450.  So it takes what is not large,
// where the layout's launch is much of the time (1576 x 1536 x 384: dx 26 -> 20 us, dw
// 25 -> 20.6; 2048^3 would take 69 us and not 57).
//
// No value is taken apart twice: a block's 64 x 64 tile is that of 8 wavefronts, each
// with 16 rows, all columns and one half of a step's values of r, and the halves are
// added in LDS at the end.  Two wavefronts a SIMD so have one convert while the other
// multiplies.  (Two 64 x 128 tiles of 4 wavefronts a CU, a wavefront with both halves,
// took 19 us for that dx and this 15; reading a step from LDS while the one before is
// converted and a third multiplied costs 16 moves a step and 2 us.)
//
// Steps of 64 values of r go straight into one of S LDS buffers.  A's rows are 256
// bytes there.  Along the sum a lane reads two 16-byte pieces, piece p of row r at
// place p ^ r % 16; across it, one value of each of 8 rows, the pieces exchanged by
// groups of 8 rows, so that a wavefront's 4 groups of lanes read 4 different 64 bytes.
#pragma once

#include "q8_grad.h"

namespace cpdp {
namespace q8 {
namespace {

struct F32Operands {
    const char* a;  // dy
    int64_t lda;    // bytes
    const char* b;
    int64_t ldb;         // bytes
    const float* scale;  // of r
    int64_t R, M, N;
    int steps;  // R / 64, rounded up
};

template <bool DOWN, int S>
struct F32Gemm {
    static constexpr int kTile = 64, kWaves = 8, kThreads = 512, NT = 4, P = 3;
    using G = Gemm<Bf16, kTile, kTile, 1, 1, 2>;  // (its order of B)
    static constexpr int kSums = kStep / 2;       // values of r in a step
    static constexpr int kRowA = 256, kA = kTile * kRowA, kB = kTile * kStep;
    static constexpr int kBuffer = kA + kB + kWaves * 256;
    static constexpr int kLoadsA = 2, kLoads = kLoadsA + 2;

    // row of A's 64 in LDS (of C along the sum, of the step across it) and piece that a
    // lane's load j fills
    static __device__ __forceinline__ int row_a(int j, int wave, int lane) {
        return (j * kWaves + wave) * 4 + (lane >> 4);
    }
    static __device__ __forceinline__ int piece_a(int j, int wave, int lane) {
        const int row = row_a(j, wave, lane);
        return (lane & 15) ^ (DOWN ? (row >> 3 & 3) << 2 : row & 15);
    }

    struct Offsets {
        uint32_t a[kLoadsA], b;
    };
    // Rows of C, and DOWN pieces of columns, that are not there repeat the last one.
    static __device__ __forceinline__ Offsets offsets(const F32Operands& o, const TileAt& tile,
                                                      int wave, int lane) {
        Offsets l;
#pragma unroll
        for (int j = 0; j < kLoadsA; ++j) {
            const int row = row_a(j, wave, lane), piece = piece_a(j, wave, lane);
            if constexpr (DOWN) {
                const int64_t last = (o.M - 1 - tile.m) / 4;
                l.a[j] = (uint32_t)(row * o.lda) + ((piece < last ? piece : (int)last) << 4);
            } else {
                const int64_t m = tile.m + row < o.M ? row : o.M - 1 - tile.m;
                l.a[j] = (uint32_t)(m * o.lda) + (piece << 4);
            }
        }
        const int row = wave * 8 + (lane >> 3);
        const int64_t n = tile.n + row < o.N ? row : o.N - 1 - tile.n;
        l.b = (uint32_t)(n * o.ldb) + (((lane & 7) ^ G::place_b(row)) << 4);
        return l;
    }

    // Sends for a step that begins at a, b and `scale`, with `sums` of its values there
    // (all of them unless LAST).  What is not there is read as zeros.
    template <bool LAST>
    static __device__ __forceinline__ void fetch(const char* a, const char* b, const float* scale,
                                                 int64_t sums, const Offsets& l, char* lds,
                                                 int wave, int lane) {
        const char* nothing = reinterpret_cast<const char*>(kNothing);
#pragma unroll
        for (int j = 0; j < kLoadsA; ++j) {
            const int first = DOWN ? row_a(j, wave, lane) : piece_a(j, wave, lane) * 4;
            to_lds(!LAST || first < sums ? a + l.a[j] : nothing,
                   lds + (j * kWaves + wave) * 1024);
        }
        to_lds(b + l.b, lds + kA + wave * 1024);
        // (each wavefront its own, so that all wait for as many loads)
        const char* p = reinterpret_cast<const char*>(scale + lane);
        __builtin_amdgcn_global_load_lds(
            (__attribute__((address_space(1))) void*)(!LAST || lane < sums ? p : nothing),
            (__attribute__((address_space(3))) void*)(lds + kA + kB + wave * 256), 4, 0, 0);
    }

    // A wavefront's half of a step
    struct Half {
        float x[kPiece];  // A as it is
        f32x4 s[2];       // and its scales
        u32x4 a[P], b[NT];
    };
    struct At {
        int a, b, s;
    };
    static __device__ __forceinline__ At at(int wave, int lane) {
        const int r = lane & 15, g = lane >> 4, half = wave >> 2, wm = wave & 3;
        At t;
        t.a = DOWN ? (half * 32 + g * 8) * kRowA + (((wm * 4 + (r >> 2)) ^ (g << 2)) << 4) +
                         (r & 3) * 4
                   : (wm * 16 + r) * kRowA + (((half * 8 + g * 2) ^ r) << 4);
        t.b = kA + ((r >> 2) * 4 * NT + (r & 3)) * kStep + (((g ^ (r >> 1)) << 4) ^ (half << 6));
        t.s = kA + kB + wave * 256 + half * 128 + g * 32;
        return t;
    }
    static __device__ __forceinline__ void read(Half& h, const char* lds, const At& t) {
        if constexpr (DOWN) {
#pragma unroll
            for (int i = 0; i < kPiece; ++i)
                h.x[i] = *reinterpret_cast<const float*>(lds + t.a + i * kRowA);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(lds + (t.a ^ (i << 4)));
#pragma unroll
                for (int k = 0; k < 4; ++k) h.x[4 * i + k] = v[k];
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) h.s[i] = *reinterpret_cast<const f32x4*>(lds + t.s + i * 16);
#pragma unroll
        for (int j = 0; j < NT; ++j)
            h.b[j] = *reinterpret_cast<const u32x4*>(lds + t.b + j * 4 * kStep);
    }
    // A s in three parts; the first `sums` of the lane's 8 values are there (LAST)
    template <bool LAST>
    static __device__ __forceinline__ void convert(Half& h, int sums) {
        float x[kPiece], most = 0.0f;
#pragma unroll
        for (int k = 0; k < kPiece; ++k) {
            x[k] = h.x[k] * h.s[k / 4][k % 4];
            if (LAST && !DOWN) x[k] = k < sums ? x[k] : 0.0f;
            most = fmaxf(most, fabsf(x[k]));
        }
        uint32_t part[P][kPiece];
#pragma unroll
        for (int k = 0; k < kPiece; ++k) {
            const float top = __uint_as_float(__float_as_uint(x[k]) & 0xffff0000u);
            const float rest = x[k] - top;
            const float mid = __uint_as_float(__float_as_uint(rest) & 0xffff0000u);
            part[0][k] = __float_as_uint(top);
            part[1][k] = __float_as_uint(mid);
            part[2][k] = __float_as_uint(rest - mid);
        }
        if (__builtin_expect(__any(most == __builtin_inff()), 0)) {
            // nothing is left of an infinity (asked once for the wavefront's 512 values, a
            // comparison and a choice less for each: 20.0 -> 19.3 us; a product that is a
            // NaN is a quiet one, whose first bits are a NaN)
#pragma unroll
            for (int k = 0; k < kPiece; ++k)
#pragma unroll
                for (int p = 1; p < P; ++p)
                    if (magnitude(x[k]) == 0x7f800000u) part[p][k] = 0;
        }
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                h.a[p][k] = __builtin_amdgcn_perm(part[p][2 * k + 1], part[p][2 * k], 0x07060302u);
    }
    static __device__ __forceinline__ void multiply(const Half& h, f32x4 (&acc)[NT]) {
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[j] = Bf16::mfma(h.b[j], h.a[p], acc[j]);
    }

    static __device__ __forceinline__ void run(const F32Operands& o, const Target& t,
                                               int64_t tiles_m, int64_t tiles_n, int slices) {
        __shared__ __attribute__((aligned(1024))) char lds[S * kBuffer];
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
        const TileAt tile = tile_at(tiles_m, tiles_n, kTile, kTile, slices);
        const Offsets l = offsets(o, tile, wave, lane);
        const char* a0 = o.a + (DOWN ? tile.m * 4 : tile.m * o.lda);
        const char* b0 = o.b + tile.n * o.ldb;
        const int64_t a_step = DOWN ? kSums * o.lda : kSums * 4;
        const int k0 = (int)((int64_t)o.steps * tile.slice / slices);
        const int k1 = (int)((int64_t)o.steps * (tile.slice + 1) / slices);
        const auto send = [&](int k, auto last) {
            fetch<last>(a0 + k * a_step, b0 + (int64_t)k * kStep, o.scale + (int64_t)k * kSums,
                        o.R - (int64_t)k * kSums, l, lds + (k - k0) % S * kBuffer, wave, lane);
        };
        // how many values of step k are there, from the lane's first on
        const auto there = [&](int k) {
            return (int)(o.R - (int64_t)k * kSums) - (wave >> 2) * 32 - g * kPiece;
        };

        const At at_ = at(wave, lane);
        f32x4 acc[NT] = {};
        Half h;
        if (k0 < k1) {
#pragma unroll
            for (int i = 0; i < S; ++i)
                if (k0 + i < k1) send(k0 + i, std::true_type());
            wait_steps<S - 1, kLoads>(k1 - k0 - 1);
            barrier();
            read(h, lds, at_);
            convert<true>(h, there(k0));
        }
        // one step, its operands in registers; `ahead` steps (S: or more) come after it,
        // S + 1: the step S on may be the last
        const auto step = [&](int k, auto ahead) {
            constexpr int kAhead = ahead;
            if constexpr (kAhead == 0) {
                multiply(h, acc);
            } else {
                // the next step has come, and all have read this one
                wait_loads<(kAhead >= S ? S - 2 : kAhead - 1) * kLoads>();
                barrier();
                if constexpr (kAhead >= S)
                    send(k + S, std::integral_constant<bool, (kAhead > S)>());
                Half next;
                read(next, lds + (k - k0 + 1) % S * kBuffer, at_);
                multiply(h, acc);
                convert<kAhead == 1>(next, there(k + 1));
                h = next;
            }
        };
        int k = k0;
        for (; k < k1 - S - 1; ++k) step(k, Int<S>());
        if (k < k1 - S) step(k++, Int<S + 1>());
        if constexpr (S > 3)
            if (k < k1 - 3) step(k++, Int<3>());
        if constexpr (S > 2)
            if (k < k1 - 2) step(k++, Int<2>());
        if (k < k1 - 1) step(k++, Int<1>());
        if (k < k1) step(k, Int<0>());

        // the second half's sums join the first's
        __syncthreads();
        f32x4(*sums)[NT][64] = reinterpret_cast<f32x4(*)[NT][64]>(lds);
        if (wave >= 4) {
#pragma unroll
            for (int j = 0; j < NT; ++j) sums[wave - 4][j][lane] = acc[j];
        }
        __syncthreads();
        if (wave >= 4) return;
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[j] += sums[wave][j][lane];
        // lane: 16 columns of row r of the wavefront's 16
        const int64_t m = tile.m + wave * 16;
        if (slices > 1) {
            u32x4 p[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) p[j] = __builtin_bit_cast(u32x4, acc[j]);
            // (the workspace has rows of whole tiles)
            store_turned(p, static_cast<uint32_t*>(t.ws) + tile.slice * t.slice + m * t.ldws +
                                tile.n,
                         t.ldws, o.M - m, t.ldws - tile.n, r, g);
        } else {
            float v[4 * NT];
#pragma unroll
            for (int c = 0; c < 4 * NT; ++c) v[c] = acc[c / 4][c % 4];
            store_rows<NT>(t, m, tile.n, o.M - m, o.N - tile.n, r, g, v);
        }
    }
};

template <bool DOWN, int S>
__global__ __launch_bounds__(512) void grad_f32_kernel(F32Operands o, Target t, int64_t tiles_m,
                                                       int64_t tiles_n, int slices) {
    F32Gemm<DOWN, S>::run(o, t, tiles_m, tiles_n, slices);
}

// Its slices, and its time beside that of shape_of: ns a step with a block a CU, and
// with several.
inline Shape f32_shape(int64_t M, int64_t N, int64_t steps) {
    const TileCost tile[] = {{64, 64, 700, 560, 0}};
    return least_of(tile, M, N, steps);
}

template <bool DOWN>
int launch_grad_f32(const F32Operands& o, Target t, int slices, void* ws, void* stream) {
    constexpr int S = 3;  // (2 leave a step's loads too little time, with 4 a CU has one block)
    const int64_t tm = up(o.M, 64), tn = up(o.N, 64), blocks = tm * tn * slices;
    if (blocks * 512 >= (int64_t)1 << 32) return (int)hipErrorInvalidValue;
    t.ws = ws;
    t.ldws = slices_ld(o.N);
    t.slice = o.M * t.ldws;
    if (int e = launch(grad_f32_kernel<DOWN, S>, dim3((uint32_t)blocks), 512, stream, o, t, tm, tn,
                       slices))
        return e;
    return slices == 1 ? 0 : launch_join<Bf16>(t, o.M, o.N, slices, stream);
}

}  // namespace
}  // namespace q8
}  // namespace cpdp
