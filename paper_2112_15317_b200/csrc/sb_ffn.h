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
// a(g).  EXACT: library exp and division; otherwise their approximations (errors of 2^-21, for results that bf16 rounds).
template <bool EXACT>
__device__ __forceinline__ float ffn_act(float g, int act)
{
    if (act == SB_ACT_SILU) return EXACT ? g / (1.0f + expf(-g)) : __fdividef(g, 1.0f + __expf(-g));
    if (act == SB_ACT_GELU) return 0.5f * g * (EXACT ? erfcf(g * -0.70710678f) : 1.0f + erff(g * 0.70710678f));
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
        const float cdf = 0.5f * (EXACT ? erfcf(g * -0.70710678f) : 1.0f + erff(g * 0.70710678f));
        da = cdf + g * 0.39894228f * (EXACT ? expf(-0.5f * g * g) : __expf(-0.5f * g * g));
        return g * cdf;
    }
    da = g > 0.f ? 1.f : 0.f;
    return g > 0.f ? g : g == g ? 0.f : g;
}
#endif

}  // namespace sb
