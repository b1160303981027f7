// Shared by the kernels of the gated feed-forward block.
#pragma once

#include "mmee_chain.h"
#include "mmee_sm100.cuh"

namespace mmee {

// Activation and its derivative.  The kind is a constant where many values go through it: with a choice at every value, none starts
// before the one before it is done (the gradient's kernel of 4096 tokens, 4096-16384-4096, took 575 us so).
template <uint32_t ACT>
__device__ __forceinline__ void act_both(float g, float* a, float* da) {
    if (ACT == MMEE_ACT_RELU) {
        *a = g < 0.f ? 0.f : g;
        *da = g > 0.f ? 1.f : 0.f;
    } else if (ACT == MMEE_ACT_GELU) {
        const float cdf = 0.5f * (1.f + erff(g * 0.70710678118654752f));
        *a = g * cdf;
        *da = cdf + g * 0.39894228040143268f * __expf(-0.5f * g * g);
    } else {
        const float s = __fdividef(1.f, 1.f + __expf(-g));
        *a = ACT == MMEE_ACT_SIGMOID ? s : g * s;
        *da = ACT == MMEE_ACT_SIGMOID ? s * (1.f - s) : s * (1.f + g * (1.f - s));
    }
}

template <uint32_t ACT>
__device__ __forceinline__ float act_value(float g) {
    float a, da;
    act_both<ACT>(g, &a, &da);
    return a;
}

template <uint32_t V>
struct Kind {
    static constexpr uint32_t value = V;
};

template <typename F>
__device__ __forceinline__ void with_act(uint32_t act, F f) {
    if (act == MMEE_ACT_SILU)
        f(Kind<MMEE_ACT_SILU>());
    else if (act == MMEE_ACT_GELU)
        f(Kind<MMEE_ACT_GELU>());
    else if (act == MMEE_ACT_RELU)
        f(Kind<MMEE_ACT_RELU>());
    else
        f(Kind<MMEE_ACT_SIGMOID>());
}

__device__ __forceinline__ float act_value(uint32_t act, float g) {
    float a;
    with_act(act, [&](auto kind) { a = act_value<decltype(kind)::value>(g); });
    return a;
}

// The block for few tokens, which the weights' way from memory bounds.  Up to kNarrow tokens: mmee_ffn_narrow.cu; up to kFew
// tokens and weights of less than kFewBytes: mmee_ffn_tokens.cu, which starts faster and, with many rows, reads a little slower.
// us of a captured call, weights from memory, one token / eight, few and narrow: 13 MB of weights 5.9 and 9.8 / 6.2 and 10.4; 67 MB 17.6 and
// 19.3 / 20.1 and 20.1; 126 MB 25.3 and 26.6 / 27.0 and 27.8; 201 MB 36.3 and 38.3 / 38.4 and 40.1; 252 MB 46.2 and 45.2 / 50.2 and 46.7; 302 MB
// 51.0 and 59.8 / 54.0 and 62.2; 403 MB 67.5 and 67.2 / 71.1 and 69.7 (two and four tokens in between): from 240 MB on it goes by how the rows
// divide.  128 tokens (narrow, tiles of 128 x 256): 25 MB 41 and 40, 67 MB 55 and 78, 403 MB 119 and 151.
constexpr uint32_t kFew = 8, kNarrow = 128;
constexpr uint64_t kFewBytes = 224ull << 20;
struct FfnTokens {
    uint32_t tokens, d_in, d_ff, d_out, act;
    const void *x, *w_gate, *w_up, *w_down;
    int64_t x_stride, w_gate_stride, w_up_stride, w_down_stride;
    void *hidden, *y;
    float* kept;                       // gate, then up; or null
};
int ffn_tokens(const FfnTokens& p, bool bf16, cudaStream_t stream);
int ffn_narrow(const FfnTokens& p, bool bf16, cudaStream_t stream);

}  // namespace mmee
