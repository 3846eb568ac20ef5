// Activations at the end of a layer or a norm, in binary32.
#pragma once
#include <hip/hip_runtime.h>

namespace mixaq {

// GELU(v) = v Phi(v), Phi(v) = 1 / (1 + 2^-t), t = v P(v^2): the logarithm of Phi's odds is odd and smooth, P its fit by weighted least
// squares on 0 < v < 7 (at most 9.4e-8 |v| off; beyond, t only grows).  13 instructions, by Abramowitz and Stegun's erfc, which is as exact,
// 18.  The median keeps the last product at -infinity from being 0 times infinity; a NaN comes through the other factor.
__device__ __forceinline__ float gelu(float v)
{
    const float u = v * v;
    float p = fmaf(u, 0x1.67ab6cp-28f, -0x1.9e7b64p-22f);
    p = fmaf(p, u, 0x1.80c28cp-17f);
    p = fmaf(p, u, -0x1.4e76fep-13f);
    p = fmaf(p, u, -0x1.8fb242p-14f);
    p = fmaf(p, u, 0x1.ad6ad0p-4f);
    p = fmaf(p, u, 0x1.26aebcp+1f);
    float top = INFINITY;
    asm("" : "+v"(top));                                  // (a constant, and the compiler makes two maxima of the median)
    return __builtin_amdgcn_fmed3f(v, -0x1.fffffep+127f, top) * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-v * p));
}

// SiLU(v) = v / (1 + 2^-t), t = v log2(e), with the same median.  The argument of the power is rounded once, so that far below zero (where the result is
// all but 0) the result is off by |t| steps, relative to itself, and nowhere by more than 4e-7 of v.
__device__ __forceinline__ float silu(float v)
{
    float top = INFINITY;
    asm("" : "+v"(top));
    return __builtin_amdgcn_fmed3f(v, -0x1.fffffep+127f, top) * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-0x1.715476p+0f * v));
}

// of the token calls and the group norm
enum Activation { ACT_NONE = 0, ACT_GELU = 1, ACT_SILU = 2, ACT_RELU = 3 };
template <int N>
__device__ __forceinline__ void activate(float (&v)[N], int kind)
{
    if (kind == ACT_GELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = gelu(v[e]);
    } else if (kind == ACT_SILU) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = silu(v[e]);
    } else if (kind == ACT_RELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = v[e] < 0.0f ? 0.0f : v[e];            // (a NaN stays one)
    }
}

}  // namespace mixaq
