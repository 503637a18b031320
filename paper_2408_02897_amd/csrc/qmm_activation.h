// The activations of a gated feed-forward block and their slopes, in binary32.
#pragma once
#include "qmm_device.h"

namespace qmm {

// e^x by the hardware's 2^x: the product x log2(e) is rounded once, so the result is off by |x| 2^-24 relative beside the instruction's own
// last place; above 88.7 infinity, below -87.3 zero.
QMM_DEV float exp_f32(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }
QMM_DEV float logistic(float x) { return __builtin_amdgcn_rcpf(1.0f + exp_f32(-x)); }
// The same to 5 * 2^-24 relative for x > -87, as near as the operations around it round: what the product x log2(e) lost goes into the power to first
// order, and the reciprocal takes a Newton step.  rest: 1 - s as e^-x s to 9 * 2^-24 relative (s being near 1, the subtraction loses up to all of it).  Below -88
// s is zero, above 104 e^-x is.  Gradients take it: their codes are compared with those of values that round once, and one that falls to the other side of a
// tie is off by a whole step (gated gradients of bfloat16 16384 x 4096: 120 us, with logistic() and 1 - s 119).
QMM_DEV float logistic_exact(float x, float& rest)
{
    const float c = __builtin_amdgcn_fmed3f(x, -88.0f, 104.0f), t = c * -1.44269504f;
    const float lost = fmaf(t, 1.90465421e-9f, fmaf(t, -0.693147182f, -c));      // -c - t ln 2
    const float p = __builtin_amdgcn_exp2f(t), e = fmaf(p, lost, p), d = 1.0f + e;
    const float r = __builtin_amdgcn_rcpf(d), s = fmaf(r, fmaf(-d, r, 1.0f), r);
    rest = e * s;
    return x < -88.0f ? 0.0f : s;
}

// e^(-g^2 / 2) to 4 * 2^-24 relative and g^2 2^-29 from the constant, to zero from |g| = 16 on: what the product with log2(e) and (unless SQUARE: g has at most
// 12 bits, its square is exact) the square lose, up to 1.2 g^2 2^-24 together, goes into the power to first order.  Gradients take it, as logistic_exact (of
// bfloat16 16384 x 4096: 122 to 127 us, with exp_f32 121 to 124; 4096 x 1024 13.5 and 13.1).
template <bool SQUARE> QMM_DEV float exp_half_square(float g)
{
    const float z = __builtin_amdgcn_fmed3f(g, -16.0f, 16.0f), half = -0.5f * z, s = z * half, t = s * 1.44269504f;
    float lost = fmaf(t, -0.693147182f, s);                       // -z^2 / 2 - t ln 2
    if constexpr (!SQUARE) lost += fmaf(z, half, -s);
    const float p = __builtin_amdgcn_exp2f(t);
    return fmaf(p, lost, p);
}

// Phi(g), the normal distribution function: with z = |g|, Phi(-z) = exp(-z^2 / 2) q(z) where q(z) = erfcx(z / sqrt 2) / 2 falls slowly, like
// 1 / z.  q as a polynomial of degree nine without constant term in t = 1 / (1 + 0.35 z), fitted over 0 <= z <= 15 for the least
// relative error (7e-8 with these coefficients; as evaluated here at most 12 * 2^-24).  With exp_half_square the tail keeps its relative accuracy, which
// 1 + erf(g / sqrt 2) loses, and the exponential is the one that the slope needs as well; with exp_f32 the tail is off by 1.2 g^2 2^-24 besides.
QMM_DEV float normal_cdf(float g, float e)                       // e = exp(-g^2 / 2)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(g), 0.35f, 1.0f));
    float q = -0.029163843020796776f;
    q = fmaf(q, t, 0.1440604031085968f);
    q = fmaf(q, t, -0.2559010684490204f);
    q = fmaf(q, t, 0.15939202904701233f);
    q = fmaf(q, t, -0.02326325699687004f);
    q = fmaf(q, t, 0.10557457059621811f);
    q = fmaf(q, t, 0.11981555074453354f);
    q = fmaf(q, t, 0.13986432552337646f);
    q = fmaf(q, t, 0.13962125778198242f);
    q = q * t * e;
    return g < 0.0f ? q : 1.0f - q;
}

// act(g)
template <int ACT> QMM_DEV float activate(float g)
{
    if constexpr (ACT == QMM_ACT_SILU) return g * logistic(g);
    else return g * normal_cdf(g, exp_f32(-0.5f * g * g));
}
// act(g) and act'(g); SQUARE: g is a bfloat16 value
template <int ACT, bool SQUARE> QMM_DEV void activate_slope(float g, float& value, float& slope)
{
    if constexpr (ACT == QMM_ACT_SILU) {
        float rest;
        const float s = logistic_exact(g, rest);
        value = g * s;
        slope = s * fmaf(g, rest, 1.0f);
    } else {
        const float e = exp_half_square<SQUARE>(g), p = normal_cdf(g, e);
        value = g * p;
        slope = fmaf(g * 0.3989422804f, e, p);                   // Phi + g phi, phi = e / sqrt(2 pi)
    }
}

}  // namespace qmm
