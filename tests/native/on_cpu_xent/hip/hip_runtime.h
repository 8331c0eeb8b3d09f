// The loss' kernels need the matrix instruction for fp16 numbers, too.
#pragma once
#include "../../on_cpu/hip/hip_runtime.h"

#define __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, x, y, z) mix(a, b, c)
