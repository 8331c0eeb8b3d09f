// Activations with 8-bit output and 8-bit checkpoint, and their backward pass
// from the checkpoint.
#include "q8_device.h"

namespace cpdp {
namespace q8 {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kSqrtHalf = 0.70710678118654752f;
constexpr float kInvSqrt2Pi = 0.39894228040143268f;

// The forward pass rounds its result to one of 255 steps, where a bit decides now
// and then, and a row's largest element its scale: it takes the math library's
// functions and a correctly rounded quotient.  That is one step of Newton's method
// from the hardware's reciprocal (Markstein's theorem: exact rounding for every
// number but one all of whose bits are ones), a fifth of a division's instructions;
// the reciprocal of infinity, where e^-g has no fp32 number, is taken as it is.
__device__ __forceinline__ float reciprocal(float x) {
    const float r = __builtin_amdgcn_rcpf(x);
    const float n = fmaf(fmaf(-x, r, 1.0f), r, r);
    return magnitude(x) < 0x7f800000u ? n : r;
}
template <Act K>
__device__ __forceinline__ float activation(float g, float u) {
    if constexpr (K == Act::GELU) return 0.5f * g * (1.0f + erff(g * kSqrtHalf));
    else return g * reciprocal(1.0f + expf(-g)) * u;
}

// 1 + erf cancels for negative g: far below zero its error, about |g| 2^-25, is no longer
// small beside g Phi(g).  A row whose largest result is large does not show it.  One whose
// results are all small and come from there (known by the two maxima) is computed again
// with the upper tail's function below -2; other rows do not pay for that function, the
// vector instructions being what bounds the fp32 forward pass.
__device__ __forceinline__ bool all_small(uint32_t top_a, uint32_t top_g) {
    return top_a < 0x3e800000u && top_g >= 0x40000000u;  // |a| < 1/4, |g| from 2 on
}
__device__ __forceinline__ float small_gelu(float g, float a) {
    return g < -2.0f ? 0.5f * g * erfcf(-g * kSqrtHalf) : a;
}

// The backward pass has no such steps.  e^x and 1 / x are the hardware's
// instructions, each good to one unit in the last place; e^x also takes the rounding
// of x log2(e), |x| 2^-24 relative.
__device__ __forceinline__ float sigmoid(float x) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -kLog2e));
}

// Phi(x) = e^(-x^2 / 2) Q(1 / (1 + |x| / 4)) for x < 0, and 1 minus that of -x for
// x > 0: one exponential, which the density shares, instead of an error function
// and an exponential.  Q is a polynomial of degree 9 without a constant term,
// fitted to e^(x^2 / 2) Phi(x) on [-14, 0] for the least largest relative error
// (6e-8); in fp32 Phi is within 2e-7, and within a relative 1e-6 down to -4.
struct Normal {
    float cdf, pdf;
};
__device__ __forceinline__ Normal normal(float x) {
    const float e = __builtin_amdgcn_exp2f(x * x * (-0.5f * kLog2e));
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(x), 0.25f, 1.0f));
    float q = 2.572378214e-02f;
    q = fmaf(q, t, -1.528107217e-01f);
    q = fmaf(q, t, 2.961246659e-01f);
    q = fmaf(q, t, -2.057864473e-01f);
    q = fmaf(q, t, 2.017605353e-01f);
    q = fmaf(q, t, 3.292692005e-02f);
    q = fmaf(q, t, 1.037469470e-01f);
    q = fmaf(q, t, 9.851680666e-02f);
    q = fmaf(q, t, 9.979748346e-02f);
    q = q * t * e;
    return {x > 0.0f ? 1.0f - q : q, e * kInvSqrt2Pi};
}

// Bound by HBM: 6 bytes an element for GELU with bf16 values written, 9 for the
// gated one (bf16 inputs); the inputs and the result of a row are held until
// their three scales are known.
template <Act K, class E, class Y, int TPR, int CH>
__global__ __launch_bounds__(block_of(TPR)) void act_kernel(
    const typename E::T* g, const typename E::T* u, int64_t ldg, int64_t T, int F, int8_t* q,
    int64_t ldq, float* scale, typename Y::T* y, int64_t ldy, int8_t* cg, float* cg_scale,
    int8_t* cu, float* cu_scale, int64_t ldc) {
    constexpr bool kGated = K == Act::SWIGLU;
    constexpr int kTops = kGated ? 3 : 2;
    __shared__ RowWords<TPR, kTops> words;
    const int64_t row = (int64_t)blockIdx.x * rows_of(TPR) + (int)threadIdx.x / TPR;
    const int lane = (int)threadIdx.x % TPR;
    if (row >= T) return;  // a whole wavefront, in the one-wavefront form only
    float gv[CH][kPiece], uv[kGated ? CH : 1][kPiece], a[CH][kPiece], none;
    uint32_t top[kTops] = {};
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int c = (j * TPR + lane) * kPiece;
        if (c < F) {
            load8(g + row * ldg + c, F - c, c, gv[j]);
            if constexpr (kGated) load8(u + row * ldg + c, F - c, c, uv[j]);
#pragma unroll
            for (int k = 0; k < kPiece; ++k) {
                a[j][k] = activation<K>(gv[j][k], kGated ? uv[kGated ? j : 0][k] : 0.0f);
                top[0] = max(top[0], magnitude(a[j][k]));
                top[1] = max(top[1], magnitude(gv[j][k]));
                if constexpr (kGated) top[2] = max(top[2], magnitude(uv[j][k]));
            }
        }
    }
    row_reduce<TPR, false, kTops>(none, top, words);
    if constexpr (K == Act::GELU) {
        if (all_small(top[0], top[1])) {  // (all threads of the row)
            __shared__ RowWords<TPR, 1> again;
            uint32_t small[1] = {0};
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                if ((j * TPR + lane) * kPiece < F) {
#pragma unroll
                    for (int k = 0; k < kPiece; ++k) {
                        a[j][k] = small_gelu(gv[j][k], a[j][k]);
                        small[0] = max(small[0], magnitude(a[j][k]));
                    }
                }
            }
            row_reduce<TPR, false, 1>(none, small, again);
            top[0] = small[0];
        }
    }
    RowScale r[kTops];
#pragma unroll
    for (int i = 0; i < kTops; ++i) r[i] = row_scale(__uint_as_float(top[i]));
    if (lane == 0) {
        scale[row] = r[0].s;
        if (cg != nullptr) cg_scale[row] = r[1].s;
        if constexpr (kGated)
            if (cu != nullptr) cu_scale[row] = r[2].s;
    }
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int c = (j * TPR + lane) * kPiece;
        if (c < F) {
            write_piece<Y>(a[j], r[0], q + row * ldq + c, y == nullptr ? y : y + row * ldy + c,
                           F - c);
            if (cg != nullptr) write_piece<F32>(gv[j], r[1], cg + row * ldc + c, nullptr, F - c);
            if constexpr (kGated)
                if (cu != nullptr)
                    write_piece<F32>(uv[j], r[2], cu + row * ldc + c, nullptr, F - c);
        }
    }
}

// A row too long to be held: its inputs are read again.
template <Act K, class E, class Y>
__global__ __launch_bounds__(1024) void act_long_kernel(
    const typename E::T* g, const typename E::T* u, int64_t ldg, int F, int8_t* q, int64_t ldq,
    float* scale, typename Y::T* y, int64_t ldy, int8_t* cg, float* cg_scale, int8_t* cu,
    float* cu_scale, int64_t ldc) {
    constexpr bool kGated = K == Act::SWIGLU;
    __shared__ RowWords<1024, 3> words;
    const int64_t row = blockIdx.x;
    float gv[kPiece], uv[kPiece] = {}, a[kPiece], none;
    uint32_t top[3] = {};
    for (int c = (int)threadIdx.x * kPiece; c < F; c += 1024 * kPiece) {
        load8(g + row * ldg + c, F - c, c, gv);
        if constexpr (kGated) load8(u + row * ldg + c, F - c, c, uv);
#pragma unroll
        for (int k = 0; k < kPiece; ++k) {
            top[0] = max(top[0], magnitude(activation<K>(gv[k], uv[k])));
            top[1] = max(top[1], magnitude(gv[k]));
            top[2] = max(top[2], magnitude(uv[k]));
        }
    }
    row_reduce<1024, false, 3>(none, top, words);
    const bool small = K == Act::GELU && all_small(top[0], top[1]);
    if (small) {
        __shared__ RowWords<1024, 1> again;
        uint32_t most[1] = {0};
        for (int c = (int)threadIdx.x * kPiece; c < F; c += 1024 * kPiece) {
            load8(g + row * ldg + c, F - c, c, gv);
#pragma unroll
            for (int k = 0; k < kPiece; ++k)
                most[0] = max(most[0], magnitude(small_gelu(gv[k], activation<K>(gv[k], 0.0f))));
        }
        row_reduce<1024, false, 1>(none, most, again);
        top[0] = most[0];
    }
    RowScale r[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) r[i] = row_scale(__uint_as_float(top[i]));
    if (threadIdx.x == 0) {
        scale[row] = r[0].s;
        if (cg != nullptr) cg_scale[row] = r[1].s;
        if (kGated && cu != nullptr) cu_scale[row] = r[2].s;
    }
    for (int c = (int)threadIdx.x * kPiece; c < F; c += 1024 * kPiece) {
        load8(g + row * ldg + c, F - c, c, gv);
        if constexpr (kGated) load8(u + row * ldg + c, F - c, c, uv);
#pragma unroll
        for (int k = 0; k < kPiece; ++k) {
            a[k] = activation<K>(gv[k], uv[k]);
            if (small) a[k] = small_gelu(gv[k], a[k]);
        }
        write_piece<Y>(a, r[0], q + row * ldq + c, y == nullptr ? y : y + row * ldy + c, F - c);
        if (cg != nullptr) write_piece<F32>(gv, r[1], cg + row * ldc + c, nullptr, F - c);
        if (kGated && cu != nullptr)
            write_piece<F32>(uv, r[2], cu + row * ldc + c, nullptr, F - c);
    }
}

template <Act K, class E, class Y>
int act_typed(Mat g, Mat u, int64_t T, int F, Held out, Mat y, Held cg, Held cu, void* stream) {
    using ET = typename E::T;
    using YT = typename Y::T;
    return with_row_shape(T, F, [&](auto tpr, auto ch) {
        return in_parts(T, 1024, [&](int64_t t, int64_t n) {
            const ET* gt = static_cast<const ET*>(g.p) + t * g.ld;
            const ET* ut = u.p == nullptr ? nullptr : static_cast<const ET*>(u.p) + t * u.ld;
            YT* yt = y.p == nullptr ? nullptr : static_cast<YT*>(y.p) + t * y.ld;
            int8_t* cgt = cg.q == nullptr ? nullptr : cg.q + t * cg.ld;
            int8_t* cut = cu.q == nullptr ? nullptr : cu.q + t * cu.ld;
            float* cgs = cg.q == nullptr ? nullptr : cg.scale + t;
            float* cus = cu.q == nullptr ? nullptr : cu.scale + t;
            if constexpr (tpr == 0)
                return launch(act_long_kernel<K, E, Y>, dim3((uint32_t)n), 1024, stream, gt, ut,
                              g.ld, F, out.q + t * out.ld, out.ld, out.scale + t, yt, y.ld, cgt,
                              cgs, cut, cus, cg.ld);
            else
                return launch(act_kernel<K, E, Y, tpr, ch>,
                              dim3((uint32_t)((n + rows_of(tpr) - 1) / rows_of(tpr))),
                              block_of(tpr), stream, gt, ut, g.ld, n, F, out.q + t * out.ld, out.ld,
                              out.scale + t, yt, y.ld, cgt, cgs, cut, cus, cg.ld);
        });
    });
}

template <Act K>
int act_kind(Mat g, Mat u, int64_t T, int F, Held out, Mat y, Held cg, Held cu, void* stream) {
    if (g.bf16)
        return y.bf16 ? act_typed<K, BF16, BF16>(g, u, T, F, out, y, cg, cu, stream)
                      : act_typed<K, BF16, F32>(g, u, T, F, out, y, cg, cu, stream);
    return y.bf16 ? act_typed<K, F32, BF16>(g, u, T, F, out, y, cg, cu, stream)
                  : act_typed<K, F32, F32>(g, u, T, F, out, y, cg, cu, stream);
}

// Bound by HBM: 5 bytes an element for GELU, 8 for the gated one (bf16).  One
// piece a thread; a block covers 4 rows of 64 pieces.
template <Act K, class E>
__global__ __launch_bounds__(256) void act_bwd_kernel(const typename E::T* da, int64_t ldda,
                                                      const int8_t* cg, const float* cg_scale,
                                                      const int8_t* cu, const float* cu_scale,
                                                      int64_t ldc, int64_t T, int F,
                                                      int blocks_across, typename E::T* dg,
                                                      typename E::T* du, int64_t lddg) {
    const int64_t row = (int64_t)(blockIdx.x / blocks_across) * 4 + (threadIdx.x >> 6);
    const int c = ((int)(blockIdx.x % blocks_across) * 64 + (int)(threadIdx.x & 63)) * kPiece;
    if (row >= T || c >= F) return;
    const int n = F - c;
    float d[kPiece], G[kPiece], U[kPiece];
    load8(da + row * ldda + c, n, c, d);
    load8(cg + row * ldc + c, n, c, G);
    const float sg = cg_scale[row];
    if constexpr (K == Act::GELU) {
#pragma unroll
        for (int k = 0; k < kPiece; ++k) {
            const float x = G[k] * sg;
            const Normal p = normal(x);
            G[k] = d[k] * fmaf(x, p.pdf, p.cdf);
        }
    } else {
        load8(cu + row * ldc + c, n, c, U);
        const float su = cu_scale[row];
#pragma unroll
        for (int k = 0; k < kPiece; ++k) {
            const float x = G[k] * sg, s = sigmoid(x);
            G[k] = d[k] * (U[k] * su) * s * fmaf(x, 1.0f - s, 1.0f);
            U[k] = d[k] * x * s;
        }
        store8(du + row * lddg + c, n, U);
    }
    store8(dg + row * lddg + c, n, G);
}

template <Act K, class E>
int act_bwd_typed(Mat da, Held cg, Held cu, int64_t T, int F, Mat dg, Mat du, void* stream) {
    using ET = typename E::T;
    const int64_t across = (F + 64 * kPiece - 1) / (64 * kPiece);
    return in_parts(T, across * 64, [&](int64_t t, int64_t n) {
        return launch(act_bwd_kernel<K, E>, dim3((uint32_t)((n + 3) / 4 * across)), 256, stream,
                      static_cast<const ET*>(da.p) + t * da.ld, da.ld, cg.q + t * cg.ld,
                      cg.scale + t, cu.q == nullptr ? cu.q : cu.q + t * cu.ld,
                      cu.q == nullptr ? cu.scale : cu.scale + t, cg.ld, n, F, (int)across,
                      static_cast<ET*>(dg.p) + t * dg.ld,
                      du.p == nullptr ? nullptr : static_cast<ET*>(du.p) + t * du.ld, dg.ld);
    });
}

}  // namespace

int launch_act(Act kind, Mat g, Mat u, int64_t T, int64_t F, Held out, Mat y, Held cg, Held cu,
               void* stream) {
    return kind == Act::GELU ? act_kind<Act::GELU>(g, u, T, (int)F, out, y, cg, cu, stream)
                             : act_kind<Act::SWIGLU>(g, u, T, (int)F, out, y, cg, cu, stream);
}

int launch_act_bwd(Act kind, Mat da, Held cg, Held cu, int64_t T, int64_t F, Mat dg, Mat du,
                   void* stream) {
    const int f = (int)F;
    if (kind == Act::GELU)
        return da.bf16 ? act_bwd_typed<Act::GELU, BF16>(da, cg, cu, T, f, dg, du, stream)
                       : act_bwd_typed<Act::GELU, F32>(da, cg, cu, T, f, dg, du, stream);
    return da.bf16 ? act_bwd_typed<Act::SWIGLU, BF16>(da, cg, cu, T, f, dg, du, stream)
                   : act_bwd_typed<Act::SWIGLU, F32>(da, cg, cu, T, f, dg, du, stream);
}

}  // namespace q8
}  // namespace cpdp
