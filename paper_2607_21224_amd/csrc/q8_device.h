// Device building blocks of the row kernels of the 8-bit activation path (norm,
// activation, row quantiser and their backward passes).  All of them stream
// rows once: a group of threads holds a row in registers, eight consecutive
// elements a thread and piece (16 bytes of bf16, two times 16 of fp32, 8 of
// int8), so that everything a row's scale depends on is known before its first
// byte is written.
//
// Arithmetic is fp32; the library is built with -ffp-contract=off, so only the
// explicit fmaf calls fuse.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "q8_launch.h"

namespace cpdp {
namespace q8 {
namespace {

constexpr int kPiece = 8;  // elements of one piece

struct F32 {
    using T = float;
};
struct BF16 {
    using T = uint16_t;
};
struct I8 {
    using T = int8_t;
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float widen(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ __forceinline__ float widen(float x) { return x; }

// two fp32 values as bf16, rounded to nearest-even (the low half is the first)
__device__ __forceinline__ uint32_t narrow2(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
__device__ __forceinline__ void narrow(float x, uint16_t* p) { *p = (uint16_t)narrow2(x, x); }
__device__ __forceinline__ void narrow(float x, float* p) { *p = x; }

// the value a storage type keeps of x
template <class E>
__device__ __forceinline__ float stored(float x) {
    if constexpr (sizeof(typename E::T) == 2) return __uint_as_float(narrow2(x, x) << 16);
    else return x;
}

// A piece that the row's end cuts short (n < 8 of its elements exist) is read as
// the row's last 8 elements, wherever they start, and shifted into place; what
// was read of the piece before is dropped.  Only a row of fewer than 8 elements
// is read one by one: a load behind a branch for each element made the last
// wavefront of every row wait for memory up to 7 times.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));

// x[k] <- x[k + 8 - n], zeros past the end
__device__ __forceinline__ void shift_down(float (&x)[kPiece], int n) {
    const int s = kPiece - n;
#pragma unroll
    for (int step = 4; step > 0; step >>= 1)
#pragma unroll
        for (int k = 0; k < kPiece; ++k)
            x[k] = (s & step) == 0 ? x[k] : k + step < kPiece ? x[k + step] : 0.0f;
}

// n elements at p, the column c of their row; the missing ones of 8 are 0
// (8 bytes of bf16 or int8 hold whole elements: a shift of the bits will do)
__device__ __forceinline__ u32x4 bits8(const uint16_t* p, int n, int c) {
    if (n >= kPiece) return *reinterpret_cast<const u32x4*>(p);
    if (c + n >= kPiece) {
        const u32x4 v = *reinterpret_cast<const u32x4_any*>(p + n - kPiece);
        return __builtin_bit_cast(
            u32x4, __builtin_bit_cast(unsigned __int128, v) >> (16 * (kPiece - n)));
    }
    u32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < kPiece; ++k)
        if (k < n) v[k / 2] |= (uint32_t)p[k] << (16 * (k % 2));
    return v;
}
__device__ __forceinline__ u32x2 bits8(const int8_t* p, int n, int c) {
    if (n >= kPiece) return *reinterpret_cast<const u32x2*>(p);
    if (c + n >= kPiece) {
        const u32x2 v = *reinterpret_cast<const u32x2_any*>(p + n - kPiece);
        return __builtin_bit_cast(u32x2, __builtin_bit_cast(uint64_t, v) >> (8 * (kPiece - n)));
    }
    u32x2 v = {0, 0};
#pragma unroll
    for (int k = 0; k < kPiece; ++k)
        if (k < n) v[k / 4] |= (uint32_t)(uint8_t)p[k] << (8 * (k % 4));
    return v;
}
__device__ __forceinline__ void load8(const uint16_t* p, int n, int c, float (&x)[kPiece]) {
    const u32x4 v = bits8(p, n, c);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        x[2 * k] = __uint_as_float(v[k] << 16);
        x[2 * k + 1] = __uint_as_float(v[k] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(const float* p, int n, int c, float (&x)[kPiece]) {
    if (n < kPiece && c + n < kPiece) {
#pragma unroll
        for (int k = 0; k < kPiece; ++k) x[k] = k < n ? p[k] : 0.0f;
        return;
    }
    const float* q = n >= kPiece ? p : p + n - kPiece;
    const u32x4 a = *reinterpret_cast<const u32x4_any*>(q);
    const u32x4 b = *reinterpret_cast<const u32x4_any*>(q + 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        x[k] = __uint_as_float(a[k]);
        x[4 + k] = __uint_as_float(b[k]);
    }
    if (n < kPiece) shift_down(x, n);
}
__device__ __forceinline__ void load8(const int8_t* p, int n, int c, float (&x)[kPiece]) {
    const u32x2 v = bits8(p, n, c);
#pragma unroll
    for (int k = 0; k < kPiece; ++k) x[k] = (float)(int8_t)(v[k / 4] >> (8 * (k % 4)));
}

// A piece as it lies in memory, so that one can be on its way, or waiting, in half
// the registers (bf16) its values take.
template <class E>
struct Raw;
template <>
struct Raw<BF16> {
    u32x4 v;
    __device__ __forceinline__ void load(const uint16_t* p, int n, int c) { v = bits8(p, n, c); }
    __device__ __forceinline__ float operator[](int k) const {
        return __uint_as_float(k % 2 == 0 ? v[k / 2] << 16 : v[k / 2] & 0xffff0000u);
    }
};
template <>
struct Raw<F32> {
    float v[kPiece];
    __device__ __forceinline__ void load(const float* p, int n, int c) { load8(p, n, c, v); }
    __device__ __forceinline__ float operator[](int k) const { return v[k]; }
};

template <>
struct Raw<I8> {
    u32x2 v;
    __device__ __forceinline__ void load(const int8_t* p, int n, int c) { v = bits8(p, n, c); }
    __device__ __forceinline__ float operator[](int k) const {
        return (float)(int8_t)(v[k / 4] >> (8 * (k % 4)));
    }
};

// Results leave as they are made, nontemporal: what a launch leaves in an XCD's
// L2 the next one, whose blocks run on other XCDs, cannot use.  With ordinary
// stores the norm of 16384 x 1024 bf16 took 33 us and not 25, of 16384 x 8192
// 226 and not 219.  (Not the fp32 results, whose two stores a lane fill a line only
// together: 3 % slower that way.)
__device__ __forceinline__ void store8(uint16_t* p, int n, const float (&x)[kPiece]) {
    if (n >= kPiece) {
        __builtin_nontemporal_store(u32x4{narrow2(x[0], x[1]), narrow2(x[2], x[3]),
                                          narrow2(x[4], x[5]), narrow2(x[6], x[7])},
                                    reinterpret_cast<u32x4*>(p));
        return;
    }
#pragma unroll
    for (int k = 0; k < kPiece; ++k)
        if (k < n) narrow(x[k], p + k);
}
__device__ __forceinline__ void store8(float* p, int n, const float (&x)[kPiece]) {
    if (n >= kPiece) {
        *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<f32x4*>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
        return;
    }
#pragma unroll
    for (int k = 0; k < kPiece; ++k)
        if (k < n) p[k] = x[k];
}
__device__ __forceinline__ void store_bytes(int8_t* p, int n, u32x2 v) {
    if (n >= kPiece) {
        __builtin_nontemporal_store(v, reinterpret_cast<u32x2*>(p));
        return;
    }
#pragma unroll
    for (int k = 0; k < kPiece; ++k)
        if (k < n) p[k] = (int8_t)(v[k / 4] >> (8 * (k % 4)));
}

// ---- the scale of a row and its whole numbers ------------------------------------

// |x| as an unsigned number: its order is that of |x|, with infinities and NaN
// on top, so a maximum over it cannot lose them
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

struct RowScale {
    float s, inv;
    uint32_t keep;  // all ones; 0 in a row that is not finite
};

// The smallest bfloat16 number s >= 2^-126 with 127 s >= amax.  The quotient's
// first 16 bits may fall one step short of it, which 127 s (exact: 15 bits)
// tells; 1 / s is a normal number for every s there is.
__device__ __forceinline__ RowScale row_scale(float amax) {
    const uint32_t low = __float_as_uint(amax / 127.0f) & 0xffff0000u;
    float s = __uint_as_float(low);
    if (s * 127.0f < amax) s = __uint_as_float(low + 0x10000u);
    s = fmaxf(s, 0x1p-126f);
    const bool finite = magnitude(amax) < 0x7f800000u;
    if (!finite) s = __uint_as_float(0x7fc00000u);
    return {s, 1.0f / s, finite ? 0xffffffffu : 0u};
}

// x / s rounded to the nearest whole number, plus 1.5 * 2^23: its last byte is
// that number in two's complement.  The quotient is the correctly rounded one
// (the reciprocal is, and one step of Newton's method on the quotient makes it
// so), since bf16 values over a bf16 scale lie exactly half way between two
// whole numbers often: a quotient a bit off there would round the wrong way.
constexpr float kWhole = 12582912.0f;
__device__ __forceinline__ float whole(float x, const RowScale& r) {
    const float t = x * r.inv;
    return fmaf(fmaf(-t, r.s, x), r.inv, t) + kWhole;
}

// the last bytes of four numbers
__device__ __forceinline__ uint32_t bytes4(float a, float b, float c, float d) {
    const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(d), __float_as_uint(c), 0x04000c0cu);
    return lo | hi;
}

// Writes one piece of a row in 8 bits (and, if y is not null, its values) at
// column c of the row's n columns.
template <class Y>
__device__ __forceinline__ void write_piece(const float (&v)[kPiece], const RowScale& r, int8_t* q,
                                            typename Y::T* y, int n) {
    float m[kPiece];
#pragma unroll
    for (int k = 0; k < kPiece; ++k) m[k] = whole(v[k], r);
    store_bytes(q, n, u32x2{bytes4(m[0], m[1], m[2], m[3]) & r.keep,
                            bytes4(m[4], m[5], m[6], m[7]) & r.keep});
    if (y != nullptr) {
#pragma unroll
        for (int k = 0; k < kPiece; ++k) m[k] = (m[k] - kWhole) * r.s;
        store8(y, n, m);
    }
}

// ---- reductions over the threads of a row -----------------------------------------

template <class Op, class V>
__device__ __forceinline__ V wave_reduce(V x, Op op) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x = op(x, __shfl_xor(x, off));
    return x;
}

struct Add {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct Max {
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const {
        return a > b ? a : b;
    }
};

// TPR threads hold the row; every one of them gets the sum of `sum` and the
// maxima of `top`, joined in the order of the wavefronts.  One barrier: a kernel
// calls it once a row, with LDS words that the row before did not use.
template <int TPR, int TOPS>
struct RowWords {
    float sum[TPR / 64];
    uint32_t top[TOPS > 0 ? TOPS : 1][TPR / 64];
};
template <int TPR, bool SUM, int TOPS>
__device__ __forceinline__ void row_reduce(float& sum, uint32_t (&top)[TOPS > 0 ? TOPS : 1],
                                           RowWords<TPR, TOPS>& words) {
    if constexpr (SUM) sum = wave_reduce(sum, Add());
#pragma unroll
    for (int i = 0; i < TOPS; ++i) top[i] = wave_reduce(top[i], Max());
    if constexpr (TPR > 64) {
        const int w = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
            if constexpr (SUM) words.sum[w] = sum;
#pragma unroll
            for (int i = 0; i < TOPS; ++i) words.top[i][w] = top[i];
        }
        __syncthreads();
        if constexpr (SUM) {
            sum = words.sum[0];
#pragma unroll
            for (int j = 1; j < TPR / 64; ++j) sum += words.sum[j];
        }
#pragma unroll
        for (int i = 0; i < TOPS; ++i) {
            top[i] = words.top[i][0];
#pragma unroll
            for (int j = 1; j < TPR / 64; ++j) top[i] = max(top[i], words.top[i][j]);
        }
    }
}

// ---- launches --------------------------------------------------------------------

template <class... P, class... A>
int launch(void (*kernel)(P...), dim3 grid, int block, void* stream, A... args) {
    static_assert(sizeof...(P) == sizeof...(A), "arguments of the kernel");
    return [&](P... p) {
        void* argv[] = {static_cast<void*>(&p)...};
        return (int)hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(block), argv,
                                    0, static_cast<hipStream_t>(stream));
    }(static_cast<P>(args)...);
}

// How a row of D elements is held: `threads` threads, `pieces` pieces each.
// f gets both as compile-time numbers; threads == 0: the row is too long to be
// held and is read again for every step.  A row of up to 2048 elements is one
// wavefront's (no barrier, four rows a block); with few rows there are idle
// CUs, and the whole block takes it from 512 elements on.
template <int N>
using Int = std::integral_constant<int, N>;

template <class F>
int with_row_shape(int64_t T, int64_t D, F f) {
    const bool few = T < 4096;
    if (D <= 512) return f(Int<64>(), Int<1>());
    if (!few && D <= 1024) return f(Int<64>(), Int<2>());
    if (D <= 2048) return few ? f(Int<256>(), Int<1>()) : f(Int<64>(), Int<4>());
    if (D <= 4096) return f(Int<256>(), Int<2>());
    if (D <= 8192) return f(Int<256>(), Int<4>());
    if (D <= 16384) return f(Int<512>(), Int<4>());
    if (D <= 32768) return f(Int<1024>(), Int<4>());
    return f(Int<0>(), Int<0>());
}

// threads of a block and rows it covers
constexpr int block_of(int tpr) { return tpr == 64 ? 256 : tpr; }
constexpr int rows_of(int tpr) { return tpr == 64 ? 4 : 1; }

// f(first row, rows) over parts of T rows, so that each part's launch (`per_row`
// work items a row at most) holds fewer than 2^32 work items
template <class F>
int in_parts(int64_t T, int64_t per_row, F f) {
    int64_t most = ((int64_t)1 << 32) / per_row - 4;
    most = most < 4 ? 4 : most / 4 * 4;
    for (int64_t t = 0; t < T; t += most)
        if (int e = f(t, T - t < most ? T - t : most)) return e;
    return 0;
}

}  // namespace
}  // namespace q8
}  // namespace cpdp
