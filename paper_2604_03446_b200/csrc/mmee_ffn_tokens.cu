// The gated feed-forward block for up to eight tokens and weights of moderate size: every weight is read once, and that is what
// bounds it.  (Where the weights are large, or the tokens more, mmee_ffn_narrow.cu.)
//
// A CTA takes 16 rows of the weights, its warps take the reduction in turns of 128.  Weights go from memory straight into the
// registers of the matrix instructions as their 16 rows, tokens are the columns (mma.sync: the rate does not matter here, and a
// 128-row tcgen05 tile of tokens would be mostly empty).  Which positions of the reduction a lane holds is free as long as both
// operands agree, so that it reads sixteen consecutive bytes of a row.  The warps' sums are added in order through shared memory.
// The second kernel is launched before the first has ended and has its first weights under way when it waits for it.
#include "mmee_ffn.cuh"

namespace mmee {

namespace {

constexpr uint32_t kMostWarps = 8;

// Tokens' values: they come back to L1 for the next rows.
__device__ __forceinline__ uint4 read_token(const uint16_t* p) {
    uint4 v;
    asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

// GATE: hidden from x, w_gate and w_up; otherwise y from hidden and w_down.
// A warp has two turns of eight sixteen-byte reads a lane under way.  Measured at 4096-16384-4096, one token: two CTAs of eight
// warps a multiprocessor with the second turn 73.7 us; four CTAs without it 79; one turn of sixteen reads 85; three CTAs, whose
// registers do not hold two turns, 94.
template <bool GATE, bool BF16>
__global__ void __launch_bounds__(kMostWarps * 32, 2) ffn_tokens_kernel(const FfnTokens p) {
    constexpr int kW = GATE ? 2 : 1;   // weight matrices
    constexpr int kC = 4 / kW;         // steps of 32 in a turn
    constexpr uint32_t kTurn = 32 * kC;
    __shared__ float sums[kMostWarps][kW][16][9];
    const uint32_t warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, g = lane >> 2, c = lane & 3u;
    const uint32_t row0 = blockIdx.x * 16, rows = GATE ? p.d_ff : p.d_out, depth = GATE ? p.d_in : p.d_ff;
    const uint16_t *w0[kW], *w1[kW];   // this lane's two rows
    bool in[2] = {row0 + g < rows, row0 + g + 8 < rows};
#pragma unroll
    for (int m = 0; m < kW; ++m) {
        const uint16_t* const base = static_cast<const uint16_t*>(GATE ? m ? p.w_up : p.w_gate : p.w_down);
        const int64_t stride = GATE ? m ? p.w_up_stride : p.w_gate_stride : p.w_down_stride;
        w0[m] = base + (int64_t)(row0 + g) * stride + 8 * c;
        w1[m] = w0[m] + 8 * stride;
    }
    const uint16_t* const x = static_cast<const uint16_t*>(GATE ? p.x : p.hidden);
    const int64_t x_stride = GATE ? p.x_stride : (int64_t)p.d_ff;
    const uint16_t* const xr = x + (int64_t)g * x_stride + 8 * c;
    const bool token_in = g < p.tokens;
    float acc[kW][4];
#pragma unroll
    for (int i = 0; i < kW * 4; ++i) (&acc[0][0])[i] = 0.f;
    const uint4 none = make_uint4(0, 0, 0, 0);
    uint4 w[2][kC][kW][2];
    auto weights = [&](uint4 (&to)[kC][kW][2], uint32_t k) {
#pragma unroll
        for (int j = 0; j < kC; ++j)
#pragma unroll
            for (int m = 0; m < kW; ++m) {
                const bool deep = k + 32 * j + 8 * c < depth;
                to[j][m][0] = in[0] && deep ? read_once(w0[m] + k + 32 * j) : none;
                to[j][m][1] = in[1] && deep ? read_once(w1[m] + k + 32 * j) : none;
            }
    };
    auto multiply = [&](const uint4 (&v)[kC][kW][2], uint32_t k) {
#pragma unroll
        for (int j = 0; j < kC; ++j) {
            const bool deep = k + 32 * j + 8 * c < depth;
            const uint4 b = token_in && deep ? read_token(xr + k + 32 * j) : none;
#pragma unroll
            for (int m = 0; m < kW; ++m) {
                mma16<BF16>(acc[m], v[j][m][0].x, v[j][m][1].x, v[j][m][0].y, v[j][m][1].y, b.x, b.y);
                mma16<BF16>(acc[m], v[j][m][0].z, v[j][m][1].z, v[j][m][0].w, v[j][m][1].w, b.z, b.w);
            }
        }
    };
    const uint32_t step = warps * kTurn;
    uint32_t k = warp * kTurn;
    if (GATE) wait_for_stream();                       // (the weights of the second kernel do not come from the first)
    weights(w[0], k);
    weights(w[1], k + step);
    if (!GATE) wait_for_stream();
    release_stream();
    for (; k < depth; k += 2 * step) {
        multiply(w[0], k);
        weights(w[0], k + 2 * step);
        multiply(w[1], k + step);
        weights(w[1], k + 3 * step);
    }
#pragma unroll
    for (int m = 0; m < kW; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[warp][m][g + 8 * (i >> 1)][2 * c + (i & 1)] = acc[m][i];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < 16 * p.tokens; i += blockDim.x) {
        const uint32_t r = i % 16, token = i / 16;
        if (row0 + r >= rows) continue;
        float v[kW];
#pragma unroll
        for (int m = 0; m < kW; ++m) {
            v[m] = 0.f;
            for (uint32_t s = 0; s < warps; ++s) v[m] += sums[s][m][r][token];
        }
        const uint64_t at = (uint64_t)token * rows + row0 + r;
        if (GATE && p.kept) {
            p.kept[at] = v[0];
            p.kept[(uint64_t)p.tokens * rows + at] = v[kW - 1];
        }
        const float out = GATE ? act_value(p.act, v[0]) * v[kW - 1] : v[0];
        static_cast<uint16_t*>(GATE ? p.hidden : p.y)[at] = (uint16_t)pack2<BF16>(out, 0.f);
    }
}

template <bool BF16>
int launch_both(const FfnTokens& p, cudaStream_t stream) {
    // As many warps to a CTA as there are turns, eight at most.
    auto threads = [](uint32_t depth, uint32_t turn) {
        uint32_t n = 1;
        while (n < kMostWarps && n * 2 * turn <= depth) n *= 2;
        return 32 * n;
    };
    const LaunchAt gate{dim3((uint32_t)ceil_div(p.d_ff, 16)), threads(p.d_in, 64), 0, 1, true, stream};
    const LaunchAt down{dim3((uint32_t)ceil_div(p.d_out, 16)), threads(p.d_ff, 128), 0, 1, true, stream};
    const int rc = launch<ffn_tokens_kernel<true, BF16>>(gate, p);
    return rc ? rc : launch<ffn_tokens_kernel<false, BF16>>(down, p);
}

}  // namespace

int ffn_tokens(const FfnTokens& p, bool bf16, cudaStream_t stream) { return bf16 ? launch_both<true>(p, stream) : launch_both<false>(p, stream); }

}  // namespace mmee
