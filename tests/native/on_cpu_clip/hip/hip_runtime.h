// The stand-in of on_cpu, with what the kernels of gradient norms and clipping need beyond it.
#pragma once
#include "../../on_cpu/hip/hip_runtime.h"

// (called where `kernel` and its arguments `args` are in scope)
#undef hipLaunchKernel
#define hipLaunchKernel(f, grid, block, argv, lds, stream) \
    ((void)(argv), (void)(lds), (void)(stream),            \
     static_cast<hipError_t>(run_grid(kernel, grid, block, args...)))

constexpr int warpSize = 64;
inline bool __all(bool x) { return x; }
inline unsigned long long __ballot(bool x) { return x; }
inline int __popcll(unsigned long long x) { return __builtin_popcountll(x); }
inline int64_t min(int64_t a, int64_t b) { return a < b ? a : b; }
inline int min(int a, int b) { return a < b ? a : b; }
#define __builtin_amdgcn_sched_barrier(x) ((void)0)
