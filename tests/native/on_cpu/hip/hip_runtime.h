// Stand-in for the HIP runtime's header that lets a host compiler (clang, for its
// vector types) build the 8-bit path's kernels and launchers.  A launch is noted, and
// on request every thread of its grid runs the kernel to its end, one after the other:
// reads and writes of memory and of LDS then happen at the addresses they have on the
// GPU, where AddressSanitizer sees them.  What is computed is not what a GPU computes (the
// matrix instructions mix bits, shuffles and barriers do nothing), and no address depends
// on it.
#pragma once
#include <stdint.h>
#include <string.h>

#include <math.h>

#include <type_traits>

#define __global__
#define __device__
#define __host__
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __shared__ static

struct dim3 {
    uint32_t x, y, z;
    dim3(uint32_t a = 1, uint32_t b = 1, uint32_t c = 1) : x(a), y(b), z(c) {}
};
extern dim3 threadIdx, blockIdx, blockDim, gridDim;

typedef void* hipStream_t;
enum hipError_t { hipSuccess = 0, hipErrorInvalidValue = 1 };

// What a launch does: notes the kernel's address; true: run it.
bool on_launch(const void* kernel, dim3 grid, dim3 block);

template <class... P>
int run_grid(void (*kernel)(P...), dim3 grid, dim3 block, P... p) {
    if (!on_launch(reinterpret_cast<const void*>(kernel), grid, block)) return 0;
    gridDim = grid;
    blockDim = block;
    for (blockIdx.y = 0; blockIdx.y < grid.y; ++blockIdx.y)
        for (blockIdx.x = 0; blockIdx.x < grid.x; ++blockIdx.x)
            for (threadIdx.x = 0; threadIdx.x < block.x; ++threadIdx.x) kernel(p...);
    return 0;
}
// (called where `kernel` and its arguments `p` are in scope)
#define hipLaunchKernel(f, grid, block, argv, lds, stream) \
    ((void)(argv), (void)(stream), run_grid(kernel, grid, block, p...))

template <class To, class From>
inline To bits_as(From f) {
    static_assert(sizeof(To) == sizeof(From), "bits");
    To t;
    memcpy(&t, &f, sizeof(t));
    return t;
}
inline float __uint_as_float(uint32_t x) { return bits_as<float>(x); }
inline uint32_t __float_as_uint(float x) { return bits_as<uint32_t>(x); }
template <class T>
inline T __shfl_xor(T x, int) {
    return x;
}
inline bool __any(bool x) { return x; }
inline void __syncthreads() {}
inline uint32_t max(uint32_t a, uint32_t b) { return a > b ? a : b; }

// 16 (or 4) bytes a lane from memory to LDS, at the wavefront's place there
inline void lds_load(const char* src, char* dst, int size) {
    if (reinterpret_cast<uintptr_t>(src) % size != 0) __builtin_trap();
    memcpy(dst + (threadIdx.x & 63) * size, src, size);
}
typedef short lds_i16x4 __attribute__((ext_vector_type(4)));
inline lds_i16x4 lds_read_tr(const char* p) {
    lds_i16x4 v;
    memcpy(&v, p, sizeof(v));
    return v;
}
// keeps all that a matrix instruction takes, so that no load of it is left out
typedef int mixed __attribute__((ext_vector_type(4)));
template <class A, class B, class C>
inline C mix(A a, B b, C c) {
    return bits_as<C>(bits_as<mixed>(a) ^ bits_as<mixed>(b) ^ bits_as<mixed>(c));
}
#define __builtin_amdgcn_global_load_lds(src, dst, size, offset, aux) \
    lds_load((const char*)(src), (char*)(dst), size)
#define __builtin_amdgcn_ds_read_tr16_b64_v4i16(p) lds_read_tr((const char*)(p))
#define __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, x, y, z) mix(a, b, c)
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, x, y, z) mix(a, b, c)
#define __builtin_amdgcn_readfirstlane(x) (x)
#define __builtin_amdgcn_update_dpp(old, x, ctrl, rows, banks, bound) (x)
#define __builtin_amdgcn_perm(a, b, s) ((a) ^ (b))
#define __builtin_amdgcn_rcpf(x) (1.0f / (x))
#define __builtin_amdgcn_exp2f(x) exp2f(x)
#define __builtin_amdgcn_s_waitcnt(x) ((void)0)
#define __builtin_amdgcn_s_barrier() ((void)0)
#define __builtin_amdgcn_sched_group_barrier(a, b, c) ((void)0)
#define __builtin_amdgcn_fence(...) ((void)0)
#define __builtin_amdgcn_wave_barrier() ((void)0)
