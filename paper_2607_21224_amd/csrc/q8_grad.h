// What the two units of a product's gradients share (q8_grad.hip: tiles of many
// tokens, q8_grad_few.hip: up to 64 tokens).
//
// A value that one bf16 number cannot hold is taken as several, each the rounding
// of what the ones before it left, and the product runs over them as over a
// longer sum.  It is the gradient that is scaled and taken apart, q being exact in
// one part: an infinity in it is one part's and meets each q once.
//   bf16 dy   dy * s has 16 significant bits where s has 8, as every scale has that is
//             written here: two parts, exactly (other scales: within 2^-16; a third part
//             would be half as much work again for every caller)
//   fp32 dy   dy * s has 24: three parts
// With bf16 results one part is kept where the sum is long: its relative error, up
// to 2^-8 a value and independent from value to value, averages out to that of
// one rounding of the result.  A sum of few values has nothing to average over,
// and costs as much as a launch does either way: it takes all parts.
#pragma once

#include "q8_gemm.h"

namespace cpdp {
namespace q8 {

// Up to so many tokens go to the kernels of q8_grad_few.hip.
constexpr int64_t kFewInput = 32, kFewWeight = 64;

int64_t few_input_workspace(int64_t T, int64_t N, int64_t K);
int launch_few_input(Mat dy, Held b, int64_t T, int64_t N, int64_t K, Mat dx, void* workspace,
                     void* stream);
int launch_few_weight(Mat dy, Held a, int64_t T, int64_t N, int64_t K, Mat dw, void* stream);

namespace {

// A sum of at most so many values (one step) is taken with all parts.
constexpr int64_t kFew = 64;

// What a lane reads for what is not there.
__device__ __attribute__((aligned(16))) const uint32_t kNothing[4] = {0, 0, 0, 0};

// Parts of the scaled gradient in a sum of R values.
inline int parts_of(int64_t R, bool dy_bf16, bool out_bf16) {
    return out_bf16 && R > kFew ? 1 : dy_bf16 ? 2 : 3;
}

// x in P bf16 parts
template <int P>
__device__ __forceinline__ void split(float x, uint16_t (&part)[P]) {
    uint32_t b = narrow2(x, x) << 16;
    if constexpr (P > 1) {
        // a number past the largest bf16 keeps its first bits; nothing is left of
        // an infinity or a NaN
        if ((b & 0x7f800000u) == 0x7f800000u && magnitude(x) < 0x7f800000u)
            b = __float_as_uint(x) & 0xffff0000u;
    }
    part[0] = (uint16_t)(b >> 16);
    const bool finite = magnitude(x) < 0x7f800000u;
    float left = x;
#pragma unroll
    for (int p = 1; p < P; ++p) {
        left = finite ? left - widen(part[p - 1]) : 0.0f;
        part[p] = (uint16_t)narrow2(left, left);
    }
}

}  // namespace
}  // namespace q8
}  // namespace cpdp
