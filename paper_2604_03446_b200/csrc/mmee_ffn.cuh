// Shared by the kernels of the gated feed-forward block.
#pragma once

#include "mmee_chain.h"
#include "mmee_sm100.cuh"

namespace mmee {

// Activation and its derivative.
__device__ __forceinline__ float act_value(uint32_t act, float g) {
    if (act == MMEE_ACT_RELU) return g < 0.f ? 0.f : g;
    if (act == MMEE_ACT_GELU) return 0.5f * g * (1.f + erff(g * 0.70710678118654752f));
    const float s = __fdividef(1.f, 1.f + __expf(-g));
    return act == MMEE_ACT_SIGMOID ? s : g * s;
}

__device__ __forceinline__ void act_both(uint32_t act, float g, float* a, float* da) {
    if (act == MMEE_ACT_RELU) {
        *a = g < 0.f ? 0.f : g;
        *da = g > 0.f ? 1.f : 0.f;
    } else if (act == MMEE_ACT_GELU) {
        const float cdf = 0.5f * (1.f + erff(g * 0.70710678118654752f));
        *a = g * cdf;
        *da = cdf + g * 0.39894228040143268f * __expf(-0.5f * g * g);
    } else {
        const float s = __fdividef(1.f, 1.f + __expf(-g));
        *a = act == MMEE_ACT_SIGMOID ? s : g * s;
        *da = act == MMEE_ACT_SIGMOID ? s * (1.f - s) : s * (1.f + g * (1.f - s));
    }
}

// The block for up to kFewTokens tokens (mmee_ffn_tokens.cu).
constexpr uint32_t kFewTokens = 32;
struct FfnTokens {
    uint32_t tokens, d_in, d_ff, d_out, act;
    const void *x, *w_gate, *w_up, *w_down;
    int64_t x_stride, w_gate_stride, w_up_stride, w_down_stride;
    void *hidden, *y;
    float* kept;                       // gate, then up; or null
};
int ffn_tokens(const FfnTokens& p, bool bf16, cudaStream_t stream);

}  // namespace mmee
