// The activations of the gated feed-forward kernels.
#pragma once
#include "../../include/bpt.h"

namespace bpt {

// The special-function unit's 2^x and 1/x (relative error about 2^-22), results below the normal range flushed to zero.
__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float rcp(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// act(g) and, for the backward, its derivative.  The epilogues are bound by instructions per element, so both activations
// cost two special-function calls.  gelu: the normal distribution's integral by Abramowitz and Stegun 7.1.26,
// erfc(z) = (a1 t + .. + a5 t^5) exp(-z^2), t = 1 / (1 + 0.3275911 z), z >= 0, absolute error 1.5e-7, whose exponential with
// z = |g| / sqrt 2 is the density that the derivative needs.  Far in the tail the absolute bound says little: relative to the true
// value erfc is off by 0.05 % at g = -4, 0.16 % at -5, 0.36 % at -6 (about bf16's half step), 1 % at -8, 3 % at -12, where the
// value itself is 6e-9, 5e-15 and 2e-32 (a form by 1 + erf in 32 bits has lost all of it from -5.5 on).
template <int ACT, bool GRAD>
__device__ __forceinline__ float ff_act(float g, float& da) {
    if (ACT == BPT_ACT_SILU) {
        const float s = rcp(1.f + ex2(g * -1.4426950408889634f));
        if (GRAD) da = s * fmaf(g, 1.f - s, 1.f);
        return g * s;
    }
    if (ACT == BPT_ACT_GELU) {
        const float e = ex2(g * g * -0.72134752044448170f);                     // exp(-g^2 / 2)
        const float t = rcp(fmaf(fabsf(g), 0.3275911f * 0.70710678118654752f, 1.f));
        float c = fmaf(fmaf(fmaf(fmaf(1.061405429f, t, -1.453152027f), t, 1.421413741f), t, -0.284496736f), t, 0.254829592f);
        c *= 0.5f * t * e;                                                      // the tail beyond |g|
        c = g < 0.f ? c : 1.f - c;
        if (GRAD) da = fmaf(g * 0.39894228040143268f, e, c);
        return g * c;
    }
    if (GRAD) da = g > 0.f ? 1.f : 0.f;
    return g < 0.f ? 0.f : g;
}

}  // namespace bpt
