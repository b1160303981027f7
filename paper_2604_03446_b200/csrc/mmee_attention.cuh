// Shared by the forward and the backward pass of attention: sizes, checks of arguments, small device helpers.
#pragma once

#include <math.h>

#include "mmee_chain.h"
#include "mmee_sm100.cuh"

namespace mmee {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr uint32_t kTile = 128;                        // query rows and keys of a tile

// A row's sums refer to a maximum that is moved only when the scores pass it by more than this (in powers of two): the
// results are the same up to rounding, and moving it means going through the row's sums in tensor memory.
constexpr float kSlack = 8.f;
// fp16 has its smallest normal value at 2^-14: probabilities are kept 2^7 larger (at most 2^15 with the slack), which the
// division by their sum takes out again.
template <bool BF16>
__device__ constexpr float kBias = BF16 ? 0.f : 7.f;

struct Strides {
    int64_t batch, token, head;        // elements
};

struct AttentionParams {
    uint32_t batch, q_heads, group, seq_q, seq_kv, d_qk, d_v;
    // Query tiles (blocks of `tile_rows` rows of a head, `tiles_q` of them, `tiles` in all) from `whole` on have their keys cut into
    // `splits` parts of `tiles_per_split` tiles of keys, which are joined afterwards.
    uint32_t tile_rows, tiles_q, tiles, whole, splits, tiles_per_split;
    float scale;
    const int32_t* kv_len;
    void* o;
    Strides os;
    float* lse;                        // [batch][q_heads][seq_q], or null
    void* rest;                        // [batch][seq_q][q_heads][d_v]: what the rounding of o took off, or null
    float *part_o, *part_lse;          // [split][tiles - whole][tile_rows] rows of d_v; log2 of the sums
};

// (Not through the read-only path, see read_once.)
__device__ __forceinline__ uint32_t valid_keys(const int32_t* kv_len, uint32_t b, uint32_t seq_kv) {
    if (!kv_len) return seq_kv;
    int32_t n;
    asm volatile("ld.global.b32 %0, [%1];" : "=r"(n) : "l"(kv_len + b) : "memory");
    return n < 0 ? 0u : min((uint32_t)n, seq_kv);
}

// Zeroes rows [from, to) of a tile of `blocks` blocks of 64 columns, by a whole warp: keys behind a sequence's end may hold
// anything, and nothing times infinity would count.  (The swizzle moves sixteen-byte pieces within a row only.)
__device__ __forceinline__ void zero_rows(uint32_t tile, uint32_t blocks, uint32_t from, uint32_t to) {
    const uint32_t pieces = (to - from) * (kRowBytes / 16);
    for (uint32_t b = 0; b < blocks; ++b)
        for (uint32_t i = threadIdx.x & 31u; i < pieces; i += 32)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(tile + b * kTile * kRowBytes + from * kRowBytes + i * 16), "r"(0) : "memory");
    fence_async_shared();
    __syncwarp();
}

// Matrix instructions on whole tiles.  The full count of steps is unrolled: in a loop with a variable end each costs the one thread
// that issues them over a hundred cycles, more than the instruction takes (forward pass of 4096 queries, 8192 keys, d 128: 538 us
// so, 463 us unrolled).

// The product of two tiles in shared memory, both with the reduction along their rows.
template <int D>
__device__ __forceinline__ void tile_product(uint32_t to, uint32_t a, uint32_t b, uint32_t desc, uint32_t steps) {
    const uint64_t da = tile_desc(a, 16), db = tile_desc(b, 16);
    auto one = [&](uint32_t k) {
        const uint64_t at = (uint64_t)(k / 4) * (kTile * kRowBytes >> 4) + (k % 4) * kStepK;
        mma_ss(to, da + at, db + at, desc, k);
    };
    if (steps == D / 16) {
#pragma unroll
        for (uint32_t k = 0; k < D / 16; ++k) one(k);
    } else {
#pragma unroll 1
        for (uint32_t k = 0; k < steps; ++k) one(k);
    }
}

// Adds the product of an operand in tensor memory (four steps of packed values, eight columns each, to a stretch of STRIDE columns) and
// a tile whose rows are the reduction.
template <int STEPS, int STRIDE>
__device__ __forceinline__ void turned_product(uint32_t to, uint32_t a, uint32_t b, uint32_t desc, uint32_t steps, bool add) {
    const uint64_t db = tile_desc(b, kTile * kRowBytes);
    auto one = [&](uint32_t k) { mma_ts(to, a + (k / 4) * STRIDE + (k % 4) * 8, db + k * kStepMN, desc, add || k); };
    if (steps >= STEPS) {
#pragma unroll
        for (uint32_t k = 0; k < STEPS; ++k) one(k);
    } else {
#pragma unroll 1
        for (uint32_t k = 0; k < steps; ++k) one(k);
    }
}

// What a rounding to two 16-bit values took off, rounded to 16 bits itself.
template <bool BF16>
__device__ __forceinline__ uint32_t rest2(float lo, float hi, uint32_t rounded) {
    const float2 r = unpack2<BF16>(rounded);
    return pack2<BF16>(lo - r.x, hi - r.y);
}

// Writes 8 * n values of a row; REST: what that rounds off, instead.
template <bool BF16, bool REST = false>
__device__ __forceinline__ void write_row(void* to, int64_t at, const float* v, uint32_t from, uint32_t cols) {
    uint4* const p = reinterpret_cast<uint4*>(static_cast<uint16_t*>(to) + at + from);
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (from + 8 * j < cols) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float lo = v[8 * j + 2 * e], hi = v[8 * j + 2 * e + 1];
                w[e] = pack2<BF16>(lo, hi);
                if (REST) w[e] = rest2<BF16>(lo, hi, w[e]);
            }
            p[j] = make_uint4(w[0], w[1], w[2], w[3]);
        }
}

__device__ __forceinline__ int64_t rest_at(const AttentionParams& p, uint32_t b, uint32_t token, uint32_t head) {
    return (((int64_t)b * p.seq_q + token) * p.q_heads + head) * p.d_v;
}

// --- host -----------------------------------------------------------------------------------------------------------

struct View {
    const void* base;
    uint32_t seq, heads, d;
    Strides s;
};

inline int view_map(CUtensorMap* map, bool bf16, uint32_t batch, const View& v) {
    const uint64_t extent[4] = {v.d, v.seq, v.heads, batch};
    const int64_t stride[3] = {v.s.token, v.s.head, v.s.batch};
    return tile_map(map, bf16, v.base, 4, extent, stride, kTile);
}

inline Strides strides(const int64_t s[3]) { return {s[0], s[1], s[2]}; }

inline int check_view(const View& v, uint32_t batch) {
    if (!v.base || !aligned16(v.base)) return MMEE_ERR_ARG;
    const int64_t s[3] = {v.s.batch, v.s.token, v.s.head};
    const uint32_t n[3] = {batch, v.seq, v.heads};
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1 && (s[i] <= 0 || s[i] % 8 || s[i] >> 38)) return MMEE_ERR_ARG;
    return MMEE_OK;
}

struct Problem {
    AttentionParams p;
    View q, k, v, o;
    bool bf16;
};

inline int check(const mmee_workload_t* w, const mmee_attention_t* a, Problem* out) {
    if (!w || !a) return MMEE_ERR_ARG;
    if (!w->batch || !w->q_heads || !w->kv_heads || !w->seq_q || !w->seq_kv || !w->d_qk || !w->d_v) return MMEE_ERR_ARG;
    if (w->q_heads % w->kv_heads || w->word_bytes != 2 || (w->d_qk | w->d_v) % 8) return MMEE_ERR_ARG;
    if (w->d_qk > MMEE_ATTENTION_MAX_D || w->d_v > MMEE_ATTENTION_MAX_D) return MMEE_ERR_RANGE;
    if (w->batch > 4095 || w->q_heads > 65535 || (w->seq_q | w->seq_kv) >> 30) return MMEE_ERR_RANGE;
    if (a->dtype != MMEE_F16 && a->dtype != MMEE_BF16) return MMEE_ERR_ARG;
    // (times log2 e it has to stay a normal number: masked scores, -infinity, are multiplied by it)
    if (!(a->scale >= 0x1p-126f) || !(a->scale <= 0x1p127f)) return MMEE_ERR_ARG;
    if (((uintptr_t)a->lse | (uintptr_t)a->kv_len) % 4) return MMEE_ERR_ARG;
    out->q = {a->q, w->seq_q, w->q_heads, w->d_qk, strides(a->q_stride)};
    out->k = {a->k, w->seq_kv, w->kv_heads, w->d_qk, strides(a->k_stride)};
    out->v = {a->v, w->seq_kv, w->kv_heads, w->d_v, strides(a->v_stride)};
    out->o = {a->o, w->seq_q, w->q_heads, w->d_v, strides(a->o_stride)};
    for (const View* v : {&out->q, &out->k, &out->v, &out->o}) {
        const int rc = check_view(*v, w->batch);
        if (rc) return rc;
    }
    AttentionParams& p = out->p;
    p = AttentionParams{};
    p.batch = w->batch;
    p.q_heads = w->q_heads;
    p.group = w->q_heads / w->kv_heads;
    p.seq_q = w->seq_q;
    p.seq_kv = w->seq_kv;
    p.d_qk = w->d_qk;
    p.d_v = w->d_v;
    p.scale = a->scale;
    p.kv_len = a->kv_len;
    p.o = a->o;
    p.os = out->o.s;
    p.lse = a->lse;
    p.rest = a->o_rest;
    if (p.rest && !aligned16(p.rest)) return MMEE_ERR_ARG;
    out->bf16 = a->dtype == MMEE_BF16;
    return MMEE_OK;
}

// The kernel for up to 16 query rows to a key head (mmee_attention_token.cu): into how many parts it cuts the keys -- CTAs of a
// cluster, and clusters -- and its launch (splits: clusters).
int token_splits(const AttentionParams& a, uint32_t* cluster, uint32_t* clusters);
int attention_tokens(const Problem& x, uint32_t cluster, cudaStream_t stream);

}  // namespace mmee
