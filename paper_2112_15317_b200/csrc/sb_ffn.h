// Shared by the gated feed-forward block's files: the activations.
#pragma once

#include "../../include/splitbrain.h"
#include "sb_internal.h"

namespace sb {

// Device status word of the operators that have no model: an array of the library's image, so that a call needs no memory of its own for it.
// (a model's own word, while the calling thread has set one)
uint32_t* ops_status();
inline uint32_t*& ops_status_of_model() { static thread_local uint32_t* word = nullptr; return word; }

#ifdef __CUDACC__
// GELU's share Phi(g) = erfc(-g / sqrt 2) / 2 for results that bf16 rounds, given bell = exp(-g^2 / 2), which the derivative needs as well.  With
// t = 1 / (1 + 0.3 |g|), Phi(-|g|) = bell t P(t): P of degree seven fitted to erfcx(|g| / sqrt 2) / (2 t) over |g| <= 14 (weighted least squares, weights
// raised where the relative error was largest): 2^-22.7 at most.  In floats, relative, negative gates: 2^-20 to -3, 2^-18 to -9 (the bell's exponent).
// (1 + erf(g / sqrt 2) loses the negative tail: several per cent at -5, all of it from -5.5 on; erfcf takes 4 to 15 % of the block's time more.)
__device__ __forceinline__ float gelu_share(float g, float bell)
{
    const float t = __fdividef(1.0f, fmaf(0.3f, fabsf(g), 1.0f));
    float p = 0.035674773f;
    p = fmaf(p, t, -0.15720308f);
    p = fmaf(p, t, 0.2063535f);
    p = fmaf(p, t, -0.053683642f);
    p = fmaf(p, t, 0.12856163f);
    p = fmaf(p, t, 0.09991349f);
    p = fmaf(p, t, 0.12075396f);
    p = fmaf(p, t, 0.1196293f);
    const float low = bell * t * p;
    return g < 0.f ? low : 1.0f - low;
}
// a(g).  EXACT: library exp, erfc and division; otherwise approximations, relative errors of 2^-21 (GELU: see gelu_share), for results that bf16 rounds.
template <bool EXACT>
__device__ __forceinline__ float ffn_act(float g, int act)
{
    if (act == SB_ACT_SILU) return EXACT ? g / (1.0f + expf(-g)) : __fdividef(g, 1.0f + __expf(-g));
    if (act == SB_ACT_GELU) return EXACT ? 0.5f * g * erfcf(g * -0.70710678f) : g * gelu_share(g, __expf(-0.5f * g * g));
    return g > 0.f ? g : g == g ? 0.f : g;
}
// a(g), and its derivative in da
template <bool EXACT>
__device__ __forceinline__ float ffn_act_grad(float g, int act, float& da)
{
    if (act == SB_ACT_SILU) {
        const float s = EXACT ? 1.0f / (1.0f + expf(-g)) : __fdividef(1.0f, 1.0f + __expf(-g));
        da = s * (1.0f + g * (1.0f - s));
        return g * s;
    }
    if (act == SB_ACT_GELU) {
        const float bell = EXACT ? expf(-0.5f * g * g) : __expf(-0.5f * g * g), cdf = EXACT ? 0.5f * erfcf(g * -0.70710678f) : gelu_share(g, bell);
        da = cdf + g * 0.39894228f * bell;
        return g * cdf;
    }
    da = g > 0.f ? 1.f : 0.f;
    return g > 0.f ? g : g == g ? 0.f : g;
}
#endif

}  // namespace sb
