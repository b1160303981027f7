// Attention of few query rows (a token or a few, all heads that share a key head: up to 16 rows) over many keys: the keys and
// values are read once, and that is what bounds it.
//
// A warp takes 16 keys at a time straight from memory into the registers of the matrix instructions, without shared memory:
// which of the reduction's positions a lane holds is free as long as both operands agree, so that a lane reads sixteen
// consecutive bytes.  S^T = K Q^T has the keys along its rows and eight query rows along its columns (mma.sync: 128-row
// tcgen05 tiles would be filled to an eighth at most, and the rate does not matter here); O^T = V^T P^T takes V's columns as rows.
// Warps, the CTAs of a cluster (over distributed shared memory) and clusters (a join afterwards) each take a part of the keys.
#include <cooperative_groups.h>

#include "mmee_attention.cuh"

namespace mmee {

namespace {

namespace cg = cooperative_groups;

constexpr uint32_t kWarps = 4, kStep = 16;

struct TokenParams {
    AttentionParams a;
    const uint16_t *q, *k, *v;
    Strides qs, ks, vs;
    uint32_t cluster;                  // CTAs that join their parts themselves; a.splits counts clusters
};

__device__ __forceinline__ uint32_t transposed8x8(uint32_t v) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

template <int DK, int DV, int NT, bool BF16>
__global__ void __launch_bounds__(kWarps * 32, NT == 1 ? 3 : 2) attention_token_kernel(const TokenParams p) {
    constexpr uint32_t kRows = 8 * NT, kPitch = DV + 4;
    __shared__ __align__(16) float sums[kWarps][kRows][kPitch];
    __shared__ float tops[kWarps][kRows], totals[kWarps][kRows];
    wait_for_stream();
    release_stream();
    const AttentionParams& a = p.a;
    const uint32_t head = blockIdx.y, b = blockIdx.z, parts = gridDim.x, part = blockIdx.x;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, g = lane >> 2, c = lane & 3u;
    const uint32_t keys = valid_keys(a.kv_len, b, a.seq_kv), rows = a.group * a.seq_q;
    const uint32_t share = (keys + parts * kStep - 1) / (parts * kStep) * kStep;
    const uint32_t begin = min(keys, part * share), end = min(keys, begin + share);
    const uint16_t* const kp = p.k + (int64_t)b * p.ks.batch + (int64_t)head * p.ks.head;
    const uint16_t* const vp = p.v + (int64_t)b * p.vs.batch + (int64_t)head * p.vs.head;
    const uint4 none = make_uint4(0, 0, 0, 0);

    uint4 q[NT][DK / 32];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const uint32_t r = 8 * t + g, h = r / a.seq_q, token = r % a.seq_q;
        const uint16_t* const row = p.q + (int64_t)b * p.qs.batch + (int64_t)token * p.qs.token + (int64_t)(head * a.group + h) * p.qs.head;
#pragma unroll
        for (int j = 0; j < DK / 32; ++j) q[t][j] = r < rows && 32 * j + 8 * c < a.d_qk ? read_once(row + 32 * j + 8 * c) : none;
    }
    float acc[NT][DV / 64][4][4];
    float m[NT][2], l[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        m[t][0] = m[t][1] = -INFINITY;
        l[t][0] = l[t][1] = 0.f;
#pragma unroll
        for (int i = 0; i < DV / 64 * 16; ++i) (&acc[t][0][0][0])[i] = 0.f;
    }
    const float sl2 = a.scale * kLog2e;

    // The next step's keys are under way while this one's probabilities are made, its values while the next scores are.
    uint4 kf[2][DK / 32], vf[DV / 64][4];
    auto load_keys = [&](uint32_t key) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t at = key + g + 8 * i;
            const uint16_t* const row = kp + (int64_t)at * p.ks.token + 8 * c;
#pragma unroll
            for (int j = 0; j < DK / 32; ++j) kf[i][j] = at < end && 32 * j + 8 * c < a.d_qk ? read_once(row + 32 * j) : none;
        }
    };
    auto load_values = [&](uint32_t key) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t at = key + 2 * c + (i & 1) + 8 * (i >> 1);
            const uint16_t* const row = vp + (int64_t)at * p.vs.token + 8 * g;
#pragma unroll
            for (int j = 0; j < DV / 64; ++j) vf[j][i] = at < end && 64 * j + 8 * g < a.d_v ? read_once(row + 64 * j) : none;
        }
    };
    load_keys(begin + warp * kStep);
    load_values(begin + warp * kStep);
    for (uint32_t key = begin + warp * kStep; key < end; key += kWarps * kStep) {
        float s[NT][4];
        bool more = false;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) s[t][i] = 0.f;
#pragma unroll
            for (int j = 0; j < DK / 32; ++j) {
                mma16<BF16>(s[t], kf[0][j].x, kf[1][j].x, kf[0][j].y, kf[1][j].y, q[t][j].x, q[t][j].y);
                mma16<BF16>(s[t], kf[0][j].z, kf[1][j].z, kf[0][j].w, kf[1][j].w, q[t][j].z, q[t][j].w);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) s[t][i] = key + g + 8 * (i >> 1) < end ? s[t][i] * sl2 : -INFINITY;
            more |= fmaxf(s[t][0], s[t][2]) > m[t][0] + kSlack || fmaxf(s[t][1], s[t][3]) > m[t][1] + kSlack;
        }
        load_keys(key + kWarps * kStep);
        if (__any_sync(0xffffffffu, more)) {           // the reference moves, for the columns that need it
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float top = fmaxf(s[t][e], s[t][2 + e]);
                    for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                    const float to = top > m[t][e] + kSlack ? top : m[t][e], by = to == m[t][e] ? 1.f : exp2_fast(m[t][e] - to);
                    m[t][e] = to;
                    l[t][e] *= by;
#pragma unroll
                    for (int j = 0; j < DV / 64; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            acc[t][j][i][e] *= by;
                            acc[t][j][i][2 + e] *= by;
                        }
                }
            }
        }
        uint32_t pr[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = exp2_fast(s[t][i] - ((m[t][i & 1] == -INFINITY ? 0.f : m[t][i & 1]) - kBias<BF16>));
            l[t][0] += w[0] + w[2];
            l[t][1] += w[1] + w[3];
            pr[t][0] = transposed8x8(pack2<BF16>(w[0], w[1]));
            pr[t][1] = transposed8x8(pack2<BF16>(w[2], w[3]));
        }
#pragma unroll
        for (int j = 0; j < DV / 64; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t v0 = word(vf[j][0], i), v1 = word(vf[j][1], i), v2 = word(vf[j][2], i), v3 = word(vf[j][3], i);
                const uint32_t a0 = __byte_perm(v0, v1, 0x5410), a1 = __byte_perm(v0, v1, 0x7632);
                const uint32_t a2 = __byte_perm(v2, v3, 0x5410), a3 = __byte_perm(v2, v3, 0x7632);
#pragma unroll
                for (int t = 0; t < NT; ++t) mma16<BF16>(acc[t][j][i], a0, a1, a2, a3, pr[t][0], pr[t][1]);
            }
        load_values(key + kWarps * kStep);
    }

    // The warps' parts, each relative to its own reference.
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t r = 8 * t + 2 * c + e;
            float sum = l[t][e];
            for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            if (g == 0) {
                tops[warp][r] = m[t][e];
                totals[warp][r] = sum;
            }
#pragma unroll
            for (int j = 0; j < DV / 64; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<float2*>(&sums[warp][r][64 * j + 8 * g + 2 * i]) = make_float2(acc[t][j][i][e], acc[t][j][i][2 + e]);
        }
    cg::cluster_group cluster = cg::this_cluster();
    if (p.cluster > 1)
        cluster.sync();
    else
        __syncthreads();

    // Each CTA of the cluster joins a share of the rows' values, four at a time, in the order of the parts.
    const uint32_t rank = part % p.cluster, id = part / p.cluster, quads = a.d_v / 4;
    const uint64_t all = (uint64_t)a.batch * a.q_heads * a.seq_q;
    for (uint32_t i = rank * blockDim.x + threadIdx.x; i < rows * quads; i += p.cluster * blockDim.x) {
        const uint32_t r = i / quads, d = i % quads * 4;
        float top = -INFINITY;
        for (uint32_t n = 0; n < p.cluster; ++n) {
            const float* const remote = p.cluster > 1 ? cluster.map_shared_rank(&tops[0][0], n) : &tops[0][0];
            for (uint32_t w = 0; w < kWarps; ++w) top = fmaxf(top, remote[w * kRows + r]);
        }
        const float from = top == -INFINITY ? 0.f : top;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        float total = 0.f;
        for (uint32_t n = 0; n < p.cluster; ++n) {
            const float* const rt = p.cluster > 1 ? cluster.map_shared_rank(&tops[0][0], n) : &tops[0][0];
            const float* const rl = p.cluster > 1 ? cluster.map_shared_rank(&totals[0][0], n) : &totals[0][0];
            const float* const rs = p.cluster > 1 ? cluster.map_shared_rank(&sums[0][0][0], n) : &sums[0][0][0];
            for (uint32_t w = 0; w < kWarps; ++w) {
                const float by = exp2_fast(rt[w * kRows + r] - from), t = rl[w * kRows + r];
                const float4 x = *reinterpret_cast<const float4*>(rs + (w * kRows + r) * kPitch + d);
                total += by * t;
                o.x += by * x.x, o.y += by * x.y, o.z += by * x.z, o.w += by * x.w;
            }
        }
        const float inv = total == 0.f ? 0.f : 1.f / total;
        const uint32_t h = head * a.group + r / a.seq_q, token = r % a.seq_q;
        const uint64_t at = ((uint64_t)b * a.q_heads + h) * a.seq_q + token;
        const float log = total == 0.f ? -INFINITY : from - kBias<BF16> + log2f(total);
        if (a.splits > 1) {
            if (d == 0) a.part_lse[id * all + at] = log;
            if (total != 0.f) *reinterpret_cast<float4*>(a.part_o + (id * all + at) * a.d_v + d) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
        } else {
            if (d == 0 && a.lse) a.lse[at] = log * kLn2;
            uint16_t* const to = static_cast<uint16_t*>(a.o) + (int64_t)b * a.os.batch + (int64_t)token * a.os.token + (int64_t)h * a.os.head;
            o.x *= inv, o.y *= inv, o.z *= inv, o.w *= inv;
            const uint2 w = make_uint2(pack2<BF16>(o.x, o.y), pack2<BF16>(o.z, o.w));
            *reinterpret_cast<uint2*>(to + d) = w;
            if (a.rest)
                *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.rest) + rest_at(a, b, token, h) + d) =
                    make_uint2(rest2<BF16>(o.x, o.y, w.x), rest2<BF16>(o.z, o.w, w.y));
        }
    }
    if (p.cluster > 1) cluster.sync();                 // shared memory stays until the others have read it
}

template <int DK, int DV, int NT>
int launch_tokens(const TokenParams& p, bool bf16, cudaStream_t stream) {
    const LaunchAt at{dim3(p.cluster * p.a.splits, p.a.q_heads / p.a.group, p.a.batch), kWarps * 32, 0, p.cluster, true, stream};
    return bf16 ? launch<attention_token_kernel<DK, DV, NT, true>>(at, p) : launch<attention_token_kernel<DK, DV, NT, false>>(at, p);
}

template <int NT>
int tokens_sized(const TokenParams& p, bool bf16, cudaStream_t stream) {
    const bool k = p.a.d_qk > 64, v = p.a.d_v > 64;
    return k ? v ? launch_tokens<128, 128, NT>(p, bf16, stream) : launch_tokens<128, 64, NT>(p, bf16, stream)
             : v ? launch_tokens<64, 128, NT>(p, bf16, stream) : launch_tokens<64, 64, NT>(p, bf16, stream);
}

}  // namespace

int token_splits(const AttentionParams& a, uint32_t* cluster, uint32_t* clusters) {
    uint32_t sms;
    const int rc = sm_count(&sms);
    if (rc) return rc;
    // Three CTAs fit a multiprocessor.  Parts of 64 keys at least (a step of every warp).  Where they fill the multiprocessors, long ones are
    // halved once more, so that sequences of different lengths keep them all at work (32 sequences of up to 8192 keys: 126 us, 116 us
    // with four parts instead of two; with parts of 512 keys it does not pay).
    const uint64_t heads = (uint64_t)a.batch * (a.q_heads / a.group), room = 3ull * sms, most = ceil_div(a.seq_kv, kWarps * kStep);
    uint64_t parts = 1;
    while (parts < 8 && 2 * parts <= most && (parts * heads < room || (parts * heads < 2 * room && a.seq_kv >= 2048 * parts))) parts *= 2;
    *cluster = (uint32_t)parts;
    // Few heads with very many keys: more clusters, of at least 16 steps a CTA, which pay for the launch that joins them.
    uint64_t more = 1;
    while (more < 16 && more * parts * heads < room && 2 * more * parts * 16 <= most) more *= 2;
    *clusters = (uint32_t)more;
    return MMEE_OK;
}

int attention_tokens(const Problem& x, uint32_t cluster, cudaStream_t stream) {
    TokenParams p{};
    p.a = x.p;
    p.q = static_cast<const uint16_t*>(x.q.base);
    p.k = static_cast<const uint16_t*>(x.k.base);
    p.v = static_cast<const uint16_t*>(x.v.base);
    p.qs = x.q.s;
    p.ks = x.k.s;
    p.vs = x.v.s;
    p.cluster = cluster;
    return x.p.group * x.p.seq_q <= 8 ? tokens_sized<1>(p, x.bf16, stream) : tokens_sized<2>(p, x.bf16, stream);
}

}  // namespace mmee
