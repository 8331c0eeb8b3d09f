// What the loss' units share: the statistics of a row's logits, and a workspace's parts.
#pragma once

#include "q8_gemm.h"
#include "q8_xent_launch.h"

namespace cpdp {
namespace q8 {
namespace {

// What is known of a row's logits after some of the classes: the largest, and the sum of
// exp(z - top).
struct Stats {
    float top, sum;
};

// exp(x) for x <= 0 or NaN, as 2^(x log2 e): v_exp is within a unit of the last place,
// what its argument's rounding adds is |x| 2^-24 at most.  Results below 2^-126 are 0.
// (Logits scaled by log2 e from the start would save a product each, 2 % of the loss'
// time, but lse has to be rounded once more then, and with it the probability of a token
// that is near 1: the error of dw of 128 x 100 x 384 was twice as large.)
__device__ __forceinline__ float exp_of(float x) {
    return __builtin_amdgcn_exp2f(x * 1.44269504f);
}

// `top` to subtract: with nothing but -infinities, 0 (their exp is then 0)
__device__ __forceinline__ float pivot(float top) { return top == -__builtin_inff() ? 0.0f : top; }

__device__ __forceinline__ Stats join(Stats a, Stats b) {
    const float top = fmaxf(a.top, b.top), p = pivot(top);
    return {top, a.sum * exp_of(a.top - p) + b.sum * exp_of(b.top - p)};
}

// lse, loss and miss from all of a row's logits; hit: its target's.  (lse - hit would lose of
// log(sum) what lse has no bits for: all of a loss below 2^-24 |lse|.)
__device__ __forceinline__ void write_loss(Stats s, float hit, int64_t y, int64_t V,
                                           const LossOut& to, int64_t t) {
    const float more = logf(s.sum);
    const float l = y < 0 ? 0.0f : (s.top - (y < V ? hit : __builtin_nanf(""))) + more;
    to.lse[t] = s.top + more;
    to.loss[t] = l;
    if (to.miss != nullptr) to.miss[t] = -expm1f(-l);
}

// The gradients are made a piece of the classes at a time: V of them in `pieces`, as even as
// whole `unit`s are.
inline int64_t piece_size(int64_t V, int64_t pieces, int64_t unit) {
    const int64_t n = up(up(V, pieces), unit) * unit;
    return n < V ? n : V;
}

// Takes parts of a workspace, each on a 256-byte boundary.
struct Room {
    int64_t bytes = 0;
    int64_t take(int64_t n) {
        const int64_t at = bytes;
        bytes += up(n, 256) * 256;
        return at;
    }
};
template <class T>
T* at(void* workspace, int64_t offset) {
    return reinterpret_cast<T*>(static_cast<char*>(workspace) + offset);
}

}  // namespace
}  // namespace q8
}  // namespace cpdp
