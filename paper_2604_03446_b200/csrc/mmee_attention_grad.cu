// The gradients of attention.  With P = exp(S - lse) and delta = rowsum(dO * O):
//   dV = P^T dO,  dS = P * (dO V^T - delta),  dK = scale dS^T Q,  dQ = scale dS K.
//
// Two kernels, so that every sum has one owner and one order: one holds a tile of keys and goes through the query tiles of all
// heads that share them (dK, dV), the other holds a tile of queries and goes through the keys (dQ).  Each makes P and dS anew;
// that is seven products instead of five, and no atomics.  P and dS go from tensor memory through registers and back, in place,
// and are operands of the next matrix instruction there.
//
// 2 x 32/8 heads, 2048 queries, 4096 keys, d 128, bf16: dK and dV 480 us (1140 TFLOP/s of its four products), dQ 357 us (1150 of its
// three).  The tensor cores are at work 60 to 67 % of active cycles; what bounds them is the chain of a turn (scores, P, its product,
// dP, dS, its product), of which half is the registers' and half the tensor cores', with one tile of each to a CTA: tensor memory is full.
//
// In fp16 P is kept 2^12 larger, and dS by a power of two for which the largest value that a sequence and key head allow,
// 2 d_v max|dO| max|V| over its rows and valid keys, still fits: gradients much smaller than one keep their bits, whatever other
// sequences and heads hold.  Both leave the results exactly.
#include "mmee_attention.cuh"

namespace mmee {

namespace {

struct GradParams {
    AttentionParams a;                 // (lse: in)
    const void* d_o;
    Strides dos;
    const void* v;
    Strides vs;
    uint32_t kv_heads;
    float* delta;                      // [batch][q_heads][seq_q]
    uint32_t* most;                    // fp16: [batch][kv_heads] bits of max|dO| and of max|V|
    void *dq, *dk, *dv;
    Strides dqs, dks, dvs;
};

template <bool BF16>
__device__ constexpr float kPShift = BF16 ? 0.f : 12.f;

// Power of two that dS of a key head is kept larger by.
template <bool BF16>
__device__ __forceinline__ int ds_shift(const GradParams& p, uint32_t b, uint32_t kv_head) {
    if (BF16) return 0;
    const uint32_t* const most = p.most + 2 * ((uint64_t)b * p.kv_heads + kv_head);
    return fp16_shift(2.f * (float)p.a.d_v * __uint_as_float(most[0]) * __uint_as_float(most[1]), 100);
}

// delta of every query row, half a warp to a row, from o and what its rounding took off (o alone would add four fifths of the error that
// a rounding of dQ and dK is: 384 queries, 512 keys, fp16); in fp16 also the largest sizes in dO and in V's valid rows, of each key head
// (their order does not matter).  A block takes 64 tokens of a head.
constexpr uint32_t kRowsOfBlock = 64;
template <bool BF16>
__global__ void __launch_bounds__(256) grad_rows_kernel(const GradParams p) {
    wait_for_stream();
    release_stream();
    const AttentionParams& a = p.a;
    const uint32_t lane = threadIdx.x & 15u, head = blockIdx.y, b = blockIdx.z, t0 = blockIdx.x * kRowsOfBlock + (threadIdx.x >> 4);
    const uint16_t* const d_o = static_cast<const uint16_t*>(p.d_o) + (int64_t)b * p.dos.batch + (int64_t)head * p.dos.head + 8 * lane;
    const uint16_t* const o = static_cast<const uint16_t*>(a.o) + (int64_t)b * a.os.batch + (int64_t)head * a.os.head + 8 * lane;
    const uint16_t* const rest = static_cast<const uint16_t*>(a.rest) + rest_at(a, b, 0, head) + 8 * lane;
    const uint16_t* const v = static_cast<const uint16_t*>(p.v) + (int64_t)b * p.vs.batch + (int64_t)head * p.vs.head + 8 * lane;
    uint32_t keys = 0;
    if constexpr (!BF16) keys = head < p.kv_heads ? valid_keys(a.kv_len, b, a.seq_kv) : 0;
    const bool in = 8 * lane < a.d_v;
    float most[2] = {0.f, 0.f};
    uint4 x[kRowsOfBlock / 16], y[kRowsOfBlock / 16], y2[kRowsOfBlock / 16], z[kRowsOfBlock / 16];
#pragma unroll
    for (uint32_t i = 0; i < kRowsOfBlock / 16; ++i) {
        const uint32_t token = t0 + 16 * i;
        const uint4 none = make_uint4(0, 0, 0, 0);
        x[i] = in && token < a.seq_q ? *reinterpret_cast<const uint4*>(d_o + (int64_t)token * p.dos.token) : none;
        y[i] = in && token < a.seq_q ? *reinterpret_cast<const uint4*>(o + (int64_t)token * a.os.token) : none;
        y2[i] = in && a.rest && token < a.seq_q ? *reinterpret_cast<const uint4*>(rest + (int64_t)token * a.q_heads * a.d_v) : none;
        if constexpr (!BF16) z[i] = in && token < keys ? *reinterpret_cast<const uint4*>(v + (int64_t)token * p.vs.token) : none;
    }
#pragma unroll
    for (uint32_t i = 0; i < kRowsOfBlock / 16; ++i) {
        const uint32_t token = t0 + 16 * i;
        const uint32_t xs[4] = {x[i].x, x[i].y, x[i].z, x[i].w}, ys[4] = {y[i].x, y[i].y, y[i].z, y[i].w};
        const uint32_t rs[4] = {y2[i].x, y2[i].y, y2[i].z, y2[i].w};
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 f = unpack2<BF16>(xs[j]), g = unpack2<BF16>(ys[j]), r = unpack2<BF16>(rs[j]);
            sum += f.x * (g.x + r.x) + f.y * (g.y + r.y);
            if (!BF16) most[0] = fmaxf(most[0], fmaxf(finite_size(f.x), finite_size(f.y)));
        }
        if (!BF16) {
            const uint32_t zs[4] = {z[i].x, z[i].y, z[i].z, z[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 f = unpack2<BF16>(zs[j]);
                most[1] = fmaxf(most[1], fmaxf(finite_size(f.x), finite_size(f.y)));
            }
        }
        for (int d = 8; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (lane == 0 && token < a.seq_q) p.delta[((uint64_t)b * a.q_heads + head) * a.seq_q + token] = sum;
    }
    if (!BF16) {                                       // (one atomic a block and value: their number is what they cost)
        __shared__ float largest[2][8];
        for (int i = 0; i < 2; ++i) {
            float m = most[i];
            for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
            if ((threadIdx.x & 31u) == 0) largest[i][threadIdx.x >> 5] = m;
        }
        __syncthreads();
        if (threadIdx.x < 2) {
            float m = 0.f;
            for (int w = 0; w < 8; ++w) m = fmaxf(m, largest[threadIdx.x][w]);
            // dO counts for the key head that this query head shares; V comes with the blocks of the first heads, its own head's.
            const uint32_t kv_head = threadIdx.x == 0 ? head / a.group : head;
            if (kv_head < p.kv_heads) atomicMax(p.most + 2 * ((uint64_t)b * p.kv_heads + kv_head) + threadIdx.x, __float_as_uint(m));
        }
    }
}

// A row's lse in powers of two, from which P follows; rows that count nothing get P = 0.
__device__ __forceinline__ float row_log(const GradParams& p, uint64_t at, bool in) {
    if (!in) return INFINITY;
    const float l = p.a.lse[at];
    return l == -INFINITY ? INFINITY : l * kLog2e;
}

template <int DK, int DV>
struct GradShape {
    // Tiles that stay, and rings of those that stream: the operand of d_qk values serves the first and the last product of a turn, so
    // that three are needed for its load to be hidden (with two, and one barrier for both operands, every turn waited for its loads:
    // dQ of 2 x 32 heads, 2048 queries, 4096 keys, d 128: 478 us).
    static constexpr uint32_t kQ = (DK / 64) * kTile * kRowBytes, kV = (DV / 64) * kTile * kRowBytes, kRingQ = 3, kRingV = 2;
    static constexpr uint32_t tiles = (1 + kRingQ) * kQ + (1 + kRingV) * kV, smem = tiles + 1024;
    // The kernel for keys has 2 KB beside: the largest tiles leave no whole KB for their alignment, but less is needed behind that.
    struct Beside {
        float row_stats[kRingV][2][kTile];             // with each query tile: log2 of the sums, delta; both negative
        uint64_t bars[2 * kRingQ + 2 * kRingV + 7];
        uint32_t tmem_base, gave_up;
    };
    static constexpr uint32_t kMost = 227 * 1024, smem_keys = smem + sizeof(Beside) < kMost ? smem : kMost - sizeof(Beside);
    static_assert(round_up(sizeof(Beside), 1024) + tiles <= kMost);
};

// --- dK and dV ------------------------------------------------------------------------------------------------------

template <int DK, int DV, bool BF16>
__global__ void __launch_bounds__(320, 1)
grad_keys_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                 const __grid_constant__ CUtensorMap mo, const GradParams p) {
    using Shape = GradShape<DK, DV>;
    constexpr uint32_t kRingQ = Shape::kRingQ, kRingV = Shape::kRingV;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(16) typename Shape::Beside beside;
    auto& row_stats = beside.row_stats;
    auto& gave_up = beside.gave_up;

    const AttentionParams& a = p.a;
    const uint32_t b = blockIdx.z, head = blockIdx.y, k0 = blockIdx.x * kTile;
    const uint32_t keys = valid_keys(a.kv_len, b, a.seq_kv);
    const uint32_t tiles_q = (a.seq_q + kTile - 1) / kTile, n = k0 < keys ? a.group * tiles_q : 0;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;

    const uint32_t base = (smem_addr(raw) + 1023u) & ~1023u;
    const uint32_t k_tile = base, v_tile = base + Shape::kQ;
    auto q_tile = [&](uint32_t i) { return base + Shape::kV + (1 + i % kRingQ) * Shape::kQ; };
    auto o_tile = [&](uint32_t i) { return base + (1 + kRingQ) * Shape::kQ + (1 + i % kRingV) * Shape::kV; };
    const uint32_t bar0 = smem_addr(beside.bars);
    auto q_full = [&](uint32_t i) { return bar0 + 8 * (i % kRingQ); };
    auto q_empty = [&](uint32_t i) { return bar0 + 8 * (kRingQ + i % kRingQ); };
    auto o_full = [&](uint32_t i) { return bar0 + 8 * (2 * kRingQ + i % kRingV); };
    auto o_empty = [&](uint32_t i) { return bar0 + 8 * (2 * kRingQ + kRingV + i % kRingV); };
    auto q_turn = [](uint32_t i) { return (i / kRingQ) & 1; };
    auto o_turn = [](uint32_t i) { return (i / kRingV) & 1; };
    const uint32_t kv_full = bar0 + 8 * (2 * kRingQ + 2 * kRingV), s_full = kv_full + 8, dp_full = kv_full + 16, p_full = kv_full + 24, ds_full = kv_full + 32,
                   sums_full = kv_full + 40, drained = kv_full + 48;
    if (threadIdx.x == 0) {
        gave_up = 0;
        for (uint32_t i = 0; i < 2 * kRingQ + 2 * kRingV; ++i) mbar_init(bar0 + 8 * i, 1);
        mbar_init(kv_full, 1);
        mbar_init(s_full, 1);
        mbar_init(dp_full, 1);
        mbar_init(p_full, 8);                          // (an arrival of every warp)
        mbar_init(ds_full, 8);
        mbar_init(sums_full, 1);
        mbar_init(drained, 1);
        mbar_init_visible();
    }
    if (warp == 9) tmem_alloc(&beside.tmem_base, 512);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = beside.tmem_base, s_col = tmem, dp_col = tmem + 128, dv_col = tmem + 256, dk_col = dv_col + DV;
    volatile uint32_t* const lost = &gave_up;
    // The rows' kernel is done from here on.  The kernel of dQ, which needs it too, may start where this one leaves room.
    wait_for_stream();
    release_stream();
    uint32_t q_sent = 0, o_sent = 0;                   // loads on their way or landed

    if (warp == 8) {
        const int32_t bb = (int32_t)b, hk = (int32_t)head;
        if (lane == 0 && n) {
            mbar_expect(kv_full, Shape::kQ + Shape::kV);
            for (int32_t j = 0; j < DK / 64; ++j) tma_load_4d(k_tile + j * kTile * kRowBytes, &mk, kv_full, 64 * j, (int32_t)k0, hk, bb);
            for (int32_t j = 0; j < DV / 64; ++j) tma_load_4d(v_tile + j * kTile * kRowBytes, &mv, kv_full, 64 * j, (int32_t)k0, hk, bb);
        }
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t s = i % kRingV, h = head * a.group + i / tiles_q, row = i % tiles_q * kTile;
            const uint64_t at = ((uint64_t)b * a.q_heads + h) * a.seq_q + row + 4 * lane;
            float logs[4], deltas[4];
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                const bool in = row + 4 * lane + j < a.seq_q;
                logs[j] = kPShift<BF16> - row_log(p, at + j, in);
                deltas[j] = in ? -p.delta[at + j] : 0.f;
            }
            if (!mbar_wait(q_empty(i), q_turn(i) ^ 1, lost)) break;
            if (lane == 0) {
                mbar_expect(q_full(i), Shape::kQ);
                for (int32_t j = 0; j < DK / 64; ++j) tma_load_4d(q_tile(i) + j * kTile * kRowBytes, &mq, q_full(i), 64 * j, (int32_t)row, (int32_t)h, bb);
            }
            ++q_sent;
            if (!mbar_wait(o_empty(i), o_turn(i) ^ 1, lost)) break;
            *reinterpret_cast<float4*>(&row_stats[s][0][4 * lane]) = make_float4(logs[0], logs[1], logs[2], logs[3]);
            *reinterpret_cast<float4*>(&row_stats[s][1][4 * lane]) = make_float4(deltas[0], deltas[1], deltas[2], deltas[3]);
            __syncwarp();
            if (lane == 0) {
                mbar_expect(o_full(i), Shape::kV);
                for (int32_t j = 0; j < DV / 64; ++j) tma_load_4d(o_tile(i) + j * kTile * kRowBytes, &mo, o_full(i), 64 * j, (int32_t)row, (int32_t)h, bb);
            }
            ++o_sent;
        }
        __syncwarp();
    } else if (warp == 9) {
        constexpr uint32_t desc = mma_desc(BF16, kTile, kTile, false, false);
        const uint32_t steps_k = (a.d_qk + 15) / 16, steps_v = (a.d_v + 15) / 16;
        const uint32_t desc_dv = mma_desc(BF16, kTile, 16 * steps_v, false, true), desc_dk = mma_desc(BF16, kTile, 16 * steps_k, false, true);
        bool sound = n > 0 && mbar_wait(kv_full, 0, lost) && mbar_wait(q_full(0), 0, lost) && mbar_wait(o_full(0), 0, lost);
        if (sound) {
            tcgen05_fence_after();
            if (elect_one()) {
                tile_product<DK>(s_col, k_tile, q_tile(0), desc, steps_k);
                mma_commit(s_full);
                tile_product<DV>(dp_col, v_tile, o_tile(0), desc, steps_v);
                mma_commit(dp_full);
            }
            __syncwarp();
        }
        for (uint32_t i = 0; i < n && sound; ++i) {
            const bool more = i + 1 < n;
            if (!(sound = mbar_wait(p_full, i & 1, lost))) break;
            tcgen05_fence_after();
            if (elect_one()) {
                turned_product<8, 64>(dv_col, s_col, o_tile(i), desc_dv, 8, i);
            }
            __syncwarp();
            if (more) {
                if (!(sound = mbar_wait(q_full(i + 1), q_turn(i + 1), lost))) break;
                tcgen05_fence_after();
                if (elect_one()) {
                    tile_product<DK>(s_col, k_tile, q_tile(i + 1), desc, steps_k);
                    mma_commit(s_full);
                }
                __syncwarp();
            }
            if (!(sound = mbar_wait(ds_full, i & 1, lost))) break;
            tcgen05_fence_after();
            if (elect_one()) {
                turned_product<8, 64>(dk_col, dp_col, q_tile(i), desc_dk, 8, i);
                mma_commit(q_empty(i));
                mma_commit(o_empty(i));                // (with the rows' numbers, which dS needs)
                if (!more) mma_commit(sums_full);
            }
            __syncwarp();
            if (more) {
                if (!(sound = mbar_wait(o_full(i + 1), o_turn(i + 1), lost))) break;
                tcgen05_fence_after();
                if (elect_one()) {
                    tile_product<DV>(dp_col, v_tile, o_tile(i + 1), desc, steps_v);
                    mma_commit(dp_full);
                }
                __syncwarp();
            }
        }
    } else {
        const uint32_t half = warp / 4, row = (warp % 4) * 32 + lane, lanes = ((warp % 4) * 32) << 16;
        const float sl2 = a.scale * kLog2e;
        const int shift = n ? ds_shift<BF16>(p, b, head) : 0;
        const float ds_scale = power_of_two(shift - (int)kPShift<BF16>);
        const bool valid = k0 + row < keys, whole = k0 + kTile <= keys;
        const uint64_t scale2 = pair(sl2, sl2), ds_scale2 = pair(ds_scale, ds_scale);
        const uint32_t s_at = s_col + lanes + 64 * half, dp_at = dp_col + lanes + 64 * half;
        auto hand_over = [&](uint32_t bar) {
            tmem_stored();
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
        };
        // (keys behind the end: their rows of P and dS are nothing, whatever K and V hold there)
        auto only_valid = [&](uint32_t* pk) {
            if (!whole && !valid) {
#pragma unroll
                for (int j = 0; j < 16; ++j) pk[j] = 0;
            }
        };
        bool sound = true;
#pragma unroll 1
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t s = i % kRingV;
            const float* const logs = &row_stats[s][0][64 * half];
            const float* const deltas = &row_stats[s][1][64 * half];
            uint32_t x[64], pk[16];
            uint64_t pr[32];
            if (!(sound = mbar_wait(o_full(i), o_turn(i), lost)) || !(sound = mbar_wait(s_full, i & 1, lost))) break;
            tcgen05_fence_after();
            tmem_load32(s_at, x);
            tmem_load32(s_at + 32, x + 32);
            tmem_loaded32(x);
            tmem_loaded32(x + 32);
#pragma unroll
            for (int c = 0; c < 64; c += 32) {         // P over scores that have been read
#pragma unroll
                for (int j = 0; j < 32; j += 4) {
                    const float4 l = *reinterpret_cast<const float4*>(logs + c + j);
                    const float2 a0 = unpair(fma_pair(pair(__uint_as_float(x[c + j]), __uint_as_float(x[c + j + 1])), scale2, pair(l.x, l.y)));
                    const float2 a1 = unpair(fma_pair(pair(__uint_as_float(x[c + j + 2]), __uint_as_float(x[c + j + 3])), scale2, pair(l.z, l.w)));
                    const float w[4] = {exp2_fast(a0.x), exp2_fast(a0.y), exp2_fast(a1.x), exp2_fast(a1.y)};
                    pr[(c + j) / 2] = pair(w[0], w[1]);
                    pr[(c + j) / 2 + 1] = pair(w[2], w[3]);
                    pk[j / 2] = pack2<BF16>(w[0], w[1]);
                    pk[j / 2 + 1] = pack2<BF16>(w[2], w[3]);
                }
                only_valid(pk);
                tmem_store16(s_at + c / 2, pk);
            }
            hand_over(p_full);
            if (!(sound = mbar_wait(dp_full, i & 1, lost))) break;
            tcgen05_fence_after();
            tmem_load32(dp_at, x);
            tmem_load32(dp_at + 32, x + 32);
            tmem_loaded32(x);
            tmem_loaded32(x + 32);
#pragma unroll
            for (int c = 0; c < 64; c += 32) {
#pragma unroll
                for (int j = 0; j < 32; j += 4) {
                    const float4 d = *reinterpret_cast<const float4*>(deltas + c + j);
                    uint64_t v0 = mul_pair(pr[(c + j) / 2], add_pair(pair(__uint_as_float(x[c + j]), __uint_as_float(x[c + j + 1])), pair(d.x, d.y)));
                    uint64_t v1 = mul_pair(pr[(c + j) / 2 + 1], add_pair(pair(__uint_as_float(x[c + j + 2]), __uint_as_float(x[c + j + 3])), pair(d.z, d.w)));
                    if (!BF16) v0 = mul_pair(v0, ds_scale2), v1 = mul_pair(v1, ds_scale2);
                    const float2 w0 = unpair(v0), w1 = unpair(v1);
                    pk[j / 2] = pack2<BF16>(w0.x, w0.y);
                    pk[j / 2 + 1] = pack2<BF16>(w1.x, w1.y);
                }
                only_valid(pk);
                tmem_store16(dp_at + c / 2, pk);
            }
            hand_over(ds_full);
        }
        if (n && sound) sound = mbar_wait(sums_full, 0, lost);
        tcgen05_fence_after();
        if (sound) {
            const uint32_t token = k0 + row;
            const float by_v = power_of_two(-(int)kPShift<BF16>), by_k = a.scale * power_of_two(-shift);
            auto write = [&](uint32_t col, uint32_t d, uint32_t width, void* to, const Strides& st, float by) {
                for (uint32_t c = half * d / 2; c < (half + 1) * d / 2; c += 32) {
                    uint32_t x[32];
                    if (n) {
                        tmem_load32(col + lanes + c, x);
                        tmem_loaded32(x);
                    }
                    if (token < a.seq_kv && c < width) {
                        float v[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = valid ? __uint_as_float(x[j]) * by : 0.f;
                        write_row<BF16>(to, (int64_t)b * st.batch + (int64_t)token * st.token + (int64_t)head * st.head, v, c, width);
                    }
                    __syncwarp();
                }
            };
            write(dv_col, DV, a.d_v, p.dv, p.dvs, by_v);
            write(dk_col, DK, a.d_qk, p.dk, p.dks, by_k);
        }
    }
    tcgen05_fence_before();
    __syncthreads();
    if (gave_up && warp == 8 && n) {                   // what is in flight lands before the CTA ends
        mbar_wait(kv_full, 0, nullptr);
        for (uint32_t s = 1; s <= kRingQ; ++s)
            if (q_sent >= s) mbar_wait(q_full(q_sent - s), q_turn(q_sent - s), nullptr);
        for (uint32_t s = 1; s <= kRingV; ++s)
            if (o_sent >= s) mbar_wait(o_full(o_sent - s), o_turn(o_sent - s), nullptr);
    }
    if (warp == 9) {
        if (gave_up) {                                 // matrix instructions in flight end before their memory is freed
            if (elect_one()) {
                g_gave_up = 1;
                mma_commit(drained);
                mbar_wait(drained, 0, nullptr);
            }
            __syncwarp();
        }
        tcgen05_fence_after();
        tmem_free(tmem, 512);
    }
}

// --- dQ -------------------------------------------------------------------------------------------------------------

template <int DK, int DV, bool BF16>
__global__ void __launch_bounds__(320, 1)
grad_queries_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                    const __grid_constant__ CUtensorMap mo, const GradParams p) {
    using Shape = GradShape<DK, DV>;
    constexpr uint32_t kRingK = Shape::kRingQ, kRingV = Shape::kRingV;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[2 * kRingK + 2 * kRingV + 7];
    __shared__ uint32_t tmem_base, gave_up;

    const AttentionParams& a = p.a;
    const uint32_t b = blockIdx.z, head = blockIdx.y, q0 = blockIdx.x * kTile;
    const uint32_t keys = valid_keys(a.kv_len, b, a.seq_kv), n = (keys + kTile - 1) / kTile;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;

    const uint32_t base = (smem_addr(raw) + 1023u) & ~1023u;
    const uint32_t q_tile = base, o_tile = base + Shape::kQ;
    auto k_tile = [&](uint32_t i) { return base + Shape::kV + (1 + i % kRingK) * Shape::kQ; };
    auto v_tile = [&](uint32_t i) { return base + (1 + kRingK) * Shape::kQ + (1 + i % kRingV) * Shape::kV; };
    const uint32_t bar0 = smem_addr(bars);
    auto k_full = [&](uint32_t i) { return bar0 + 8 * (i % kRingK); };
    auto k_empty = [&](uint32_t i) { return bar0 + 8 * (kRingK + i % kRingK); };
    auto v_full = [&](uint32_t i) { return bar0 + 8 * (2 * kRingK + i % kRingV); };
    auto v_empty = [&](uint32_t i) { return bar0 + 8 * (2 * kRingK + kRingV + i % kRingV); };
    auto k_turn = [](uint32_t i) { return (i / kRingK) & 1; };
    auto v_turn = [](uint32_t i) { return (i / kRingV) & 1; };
    const uint32_t q_full = bar0 + 8 * (2 * kRingK + 2 * kRingV), dp_full = q_full + 24, ds_full = q_full + 32, sums_full = q_full + 40, drained = q_full + 48;
    auto s_full = [&](uint32_t t) { return q_full + 8 + 8 * t; };
    if (threadIdx.x == 0) {
        gave_up = 0;
        for (uint32_t i = 0; i < 2 * kRingK + 2 * kRingV; ++i) mbar_init(bar0 + 8 * i, 1);
        mbar_init(q_full, 1);
        mbar_init(s_full(0), 1);
        mbar_init(s_full(1), 1);
        mbar_init(dp_full, 1);
        mbar_init(ds_full, 8);                         // (an arrival of every warp)
        mbar_init(sums_full, 1);
        mbar_init(drained, 1);
        mbar_init_visible();
    }
    if (warp == 9) tmem_alloc(&tmem_base, 512);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_base, dp_col = tmem + 256, dq_col = tmem + 384;
    auto s_col = [&](uint32_t t) { return tmem + 128 * t; };
    volatile uint32_t* const lost = &gave_up;
    // Without a wait: the kernel of dK and dV, beside which this one starts, has released the stream after the rows' kernel was done, and
    // writes nothing that is read here.
    release_stream();
    uint32_t k_sent = 0, v_sent = 0;                   // loads on their way or landed (of the thread that issues them)

    if (warp == 8) {
        if (elect_one() && n) {
            const int32_t bb = (int32_t)b, h = (int32_t)head, hk = (int32_t)(head / a.group);
            mbar_expect(q_full, Shape::kQ + Shape::kV);
            for (int32_t j = 0; j < DK / 64; ++j) tma_load_4d(q_tile + j * kTile * kRowBytes, &mq, q_full, 64 * j, (int32_t)q0, h, bb);
            for (int32_t j = 0; j < DV / 64; ++j) tma_load_4d(o_tile + j * kTile * kRowBytes, &mo, q_full, 64 * j, (int32_t)q0, h, bb);
            for (uint32_t i = 0; i < n; ++i) {
                if (!mbar_wait(k_empty(i), k_turn(i) ^ 1, lost)) break;
                mbar_expect(k_full(i), Shape::kQ);
                for (int32_t j = 0; j < DK / 64; ++j) tma_load_4d(k_tile(i) + j * kTile * kRowBytes, &mk, k_full(i), 64 * j, (int32_t)(i * kTile), hk, bb);
                ++k_sent;
                if (!mbar_wait(v_empty(i), v_turn(i) ^ 1, lost)) break;
                mbar_expect(v_full(i), Shape::kV);
                for (int32_t j = 0; j < DV / 64; ++j) tma_load_4d(v_tile(i) + j * kTile * kRowBytes, &mv, v_full(i), 64 * j, (int32_t)(i * kTile), hk, bb);
                ++v_sent;
            }
        }
        __syncwarp();
    } else if (warp == 9) {
        constexpr uint32_t desc = mma_desc(BF16, kTile, kTile, false, false);
        const uint32_t steps_k = (a.d_qk + 15) / 16, steps_v = (a.d_v + 15) / 16;
        const uint32_t desc_dq = mma_desc(BF16, kTile, 16 * steps_k, false, true);
        // Tile i of K has landed; keys behind the end become zeros (in dS K they meet zeros).
        auto landed = [&](uint32_t i) {
            if (!mbar_wait(k_full(i), k_turn(i), lost)) return false;
            const uint32_t left = keys - i * kTile;
            if (left < kTile && left % 16) zero_rows(k_tile(i), DK / 64, left, (left + 15) / 16 * 16);
            tcgen05_fence_after();
            return true;
        };
        auto gradient_of_p = [&](uint32_t i) {            // dP of tile i
            if (!mbar_wait(v_full(i), v_turn(i), lost)) return false;
            tcgen05_fence_after();
            if (elect_one()) {
                tile_product<DV>(dp_col, o_tile, v_tile(i), desc, steps_v);
                mma_commit(dp_full);
                mma_commit(v_empty(i));
            }
            __syncwarp();
            return true;
        };
        bool sound = n > 0 && mbar_wait(q_full, 0, lost) && landed(0);
        if (sound) {
            if (elect_one()) {
                tile_product<DK>(s_col(0), q_tile, k_tile(0), desc, steps_k);
                mma_commit(s_full(0));
            }
            __syncwarp();
            sound = gradient_of_p(0);
        }
        for (uint32_t i = 0; i < n && sound; ++i) {
            if (i + 1 < n) {
                if (!(sound = landed(i + 1))) break;
                if (elect_one()) {
                    tile_product<DK>(s_col((i + 1) & 1), q_tile, k_tile(i + 1), desc, steps_k);
                    mma_commit(s_full((i + 1) & 1));
                }
                __syncwarp();
            }
            if (!(sound = mbar_wait(ds_full, i & 1, lost))) break;
            tcgen05_fence_after();
            if (i + 1 < n && !(sound = gradient_of_p(i + 1))) break;
            if (elect_one()) {
                turned_product<8, 64>(dq_col, s_col(i & 1), k_tile(i), desc_dq, (min(kTile, keys - i * kTile) + 15) / 16, i);
                mma_commit(k_empty(i));
                if (i + 1 == n) mma_commit(sums_full);
            }
            __syncwarp();
        }
    } else {
        const uint32_t half = warp / 4, row = (warp % 4) * 32 + lane, lanes = ((warp % 4) * 32) << 16, token = q0 + row;
        const float sl2 = a.scale * kLog2e;
        const int shift = n ? ds_shift<BF16>(p, b, head / a.group) : 0;
        const uint64_t at = ((uint64_t)b * a.q_heads + head) * a.seq_q + token;
        const bool in = token < a.seq_q;
        // dS = 2^shift exp2(S sl2 - log) (dP - delta): the power goes into the exponent.  Rows that count nothing: exp2(-infinity).
        const float from = (float)shift - row_log(p, at, in), delta = in ? -p.delta[at] : 0.f;
        const uint64_t scale2 = pair(sl2, sl2), from2 = pair(from, from), delta2 = pair(delta, delta);
        bool sound = true;
#pragma unroll 1
        for (uint32_t i = 0; i < n; ++i) {
            const int valid = (int)(keys - i * kTile) - 64 * (int)half;        // columns of this half that count
            const uint32_t s = s_col(i & 1) + lanes + 64 * half;
            uint32_t x[64];
            uint64_t pr[32];
            if (!(sound = mbar_wait(s_full(i & 1), (i >> 1) & 1, lost))) break;
            tcgen05_fence_after();
            tmem_load32(s, x);
            tmem_load32(s + 32, x + 32);
            tmem_loaded32(x);
            tmem_loaded32(x + 32);
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                const float2 w = unpair(fma_pair(pair(__uint_as_float(x[2 * j]), __uint_as_float(x[2 * j + 1])), scale2, from2));
                pr[j] = pair(exp2_fast(w.x), exp2_fast(w.y));
            }
            if (!(sound = mbar_wait(dp_full, i & 1, lost))) break;
            tcgen05_fence_after();
            tmem_load32(dp_col + lanes + 64 * half, x);
            tmem_load32(dp_col + lanes + 64 * half + 32, x + 32);
            tmem_loaded32(x);
            tmem_loaded32(x + 32);
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                const float2 w = unpair(mul_pair(pr[j], add_pair(pair(__uint_as_float(x[2 * j]), __uint_as_float(x[2 * j + 1])), delta2)));
                x[j] = pack2<BF16>(w.x, w.y);
            }
            if (valid < 64) {                          // keys behind the end: nothing, whatever K and V hold there
#pragma unroll
                for (int j = 0; j < 32; ++j) x[j] = 2 * j >= valid ? 0u : 2 * j + 1 >= valid ? x[j] & 0xffffu : x[j];
            }
            tmem_store32(s, x);
            tmem_stored();
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(ds_full);
        }
        if (n && sound) sound = mbar_wait(sums_full, 0, lost);
        tcgen05_fence_after();
        if (sound) {
            const float by = a.scale * power_of_two(-shift);
            for (uint32_t c = half * DK / 2; c < (half + 1) * DK / 2; c += 32) {
                uint32_t x[32];
                if (n) {
                    tmem_load32(dq_col + lanes + c, x);
                    tmem_loaded32(x);
                }
                if (in && c < a.d_qk) {
                    float v[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = n ? __uint_as_float(x[j]) * by : 0.f;
                    write_row<BF16>(p.dq, (int64_t)b * p.dqs.batch + (int64_t)token * p.dqs.token + (int64_t)head * p.dqs.head, v, c, a.d_qk);
                }
                __syncwarp();
            }
        }
    }
    // (it was launched beside the kernel of dK and dV, and ends after it: what follows in the stream needs both)
    wait_for_stream();
    tcgen05_fence_before();
    __syncthreads();
    if (gave_up && warp == 8 && n) {                   // what is in flight lands before the CTA ends
        if (elect_one()) {
            mbar_wait(q_full, 0, nullptr);
            for (uint32_t s = 1; s <= kRingK; ++s)
                if (k_sent >= s) mbar_wait(k_full(k_sent - s), k_turn(k_sent - s), nullptr);
            for (uint32_t s = 1; s <= kRingV; ++s)
                if (v_sent >= s) mbar_wait(v_full(v_sent - s), v_turn(v_sent - s), nullptr);
        }
        __syncwarp();
    }
    if (warp == 9) {
        if (gave_up) {                                 // matrix instructions in flight end before their memory is freed
            if (elect_one()) {
                g_gave_up = 1;
                mma_commit(drained);
                mbar_wait(drained, 0, nullptr);
            }
            __syncwarp();
        }
        tcgen05_fence_after();
        tmem_free(tmem, 512);
    }
}

// --- host -----------------------------------------------------------------------------------------------------------

template <int DK, int DV, bool BF16>
int launch_grads(const Problem& x, const View& d_o, const GradParams& p, cudaStream_t stream) {
    const AttentionParams& a = p.a;
    CUtensorMap mq, mk, mv, mo;
    int rc = view_map(&mq, BF16, a.batch, x.q);
    if (!rc) rc = view_map(&mk, BF16, a.batch, x.k);
    if (!rc) rc = view_map(&mv, BF16, a.batch, x.v);
    if (!rc) rc = view_map(&mo, BF16, a.batch, d_o);
    if (rc) return rc;
    if (!BF16 && (rc = cuda_status(cudaMemsetAsync(p.most, 0, 8ull * a.batch * p.kv_heads, stream)))) return rc;
    const uint32_t longest = BF16 ? a.seq_q : max(a.seq_q, a.seq_kv);
    using Shape = GradShape<DK, DV>;
    const LaunchAt rows{dim3((uint32_t)ceil_div(longest, kRowsOfBlock), a.q_heads, a.batch), 256, 0, 1, BF16, stream};       // (fp16: after the memset)
    const LaunchAt keys{dim3((uint32_t)ceil_div(a.seq_kv, kTile), p.kv_heads, a.batch), 320, Shape::smem_keys, 1, true, stream};
    const LaunchAt queries{dim3((uint32_t)ceil_div(a.seq_q, kTile), a.q_heads, a.batch), 320, Shape::smem, 1, true, stream};
    rc = launch<grad_rows_kernel<BF16>>(rows, p);
    if (!rc) rc = launch<grad_keys_kernel<DK, DV, BF16>>(keys, mq, mk, mv, mo, p);
    return rc ? rc : launch<grad_queries_kernel<DK, DV, BF16>>(queries, mq, mk, mv, mo, p);
}

template <int DK, int DV>
int grads_typed(const Problem& x, const View& d_o, const GradParams& p, cudaStream_t stream) {
    return x.bf16 ? launch_grads<DK, DV, true>(x, d_o, p, stream) : launch_grads<DK, DV, false>(x, d_o, p, stream);
}

// The workspace: delta, then the largest sizes of each sequence and key head.
uint64_t rows_bytes(const mmee_workload_t& w) { return round_up((uint64_t)w.batch * w.q_heads * w.seq_q * 4, 16); }
uint64_t space_bytes(const mmee_workload_t& w) { return rows_bytes(w) + round_up((uint64_t)w.batch * w.kv_heads * 8, 16); }

}  // namespace

int attention_grad_waits(uint32_t* gave_up, const uint64_t* limit_ns) { return waits_of_file(gave_up, limit_ns); }

}  // namespace mmee

using namespace mmee;

extern "C" int mmee_attention_backward_workspace(const mmee_workload_t* w, uint64_t* bytes) {
    if (!w || !bytes) return MMEE_ERR_ARG;
    *bytes = space_bytes(*w);
    return MMEE_OK;
}

extern "C" int mmee_attention_backward(const mmee_workload_t* workload, const mmee_attention_t* attention, const mmee_attention_grad_t* g,
                                       void* cuda_stream) {
    Problem x;
    const int rc = check(workload, attention, &x);
    if (rc) return rc;
    if (!g || !attention->lse) return MMEE_ERR_ARG;
    const mmee_workload_t& w = *workload;
    const View d_o{g->d_o, w.seq_q, w.q_heads, w.d_v, strides(g->d_o_stride)};
    const View dq{g->d_q, w.seq_q, w.q_heads, w.d_qk, strides(g->d_q_stride)}, dk{g->d_k, w.seq_kv, w.kv_heads, w.d_qk, strides(g->d_k_stride)};
    const View dv{g->d_v, w.seq_kv, w.kv_heads, w.d_v, strides(g->d_v_stride)};
    for (const View* v : {&d_o, &dq, &dk, &dv})
        if (check_view(*v, w.batch)) return MMEE_ERR_ARG;
    if (!g->workspace || !aligned16(g->workspace) || g->workspace_bytes < space_bytes(w)) return MMEE_ERR_ARG;
    GradParams p{};
    p.a = x.p;
    p.d_o = g->d_o;
    p.dos = d_o.s;
    p.v = attention->v;
    p.vs = x.v.s;
    p.kv_heads = w.kv_heads;
    p.delta = static_cast<float*>(g->workspace);
    p.most = reinterpret_cast<uint32_t*>(static_cast<char*>(g->workspace) + rows_bytes(w));
    p.dq = g->d_q;
    p.dk = g->d_k;
    p.dv = g->d_v;
    p.dqs = dq.s;
    p.dks = dk.s;
    p.dvs = dv.s;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const bool bk = w.d_qk > 64, bv = w.d_v > 64;
    return bk ? bv ? grads_typed<128, 128>(x, d_o, p, stream) : grads_typed<128, 64>(x, d_o, p, stream)
              : bv ? grads_typed<64, 128>(x, d_o, p, stream) : grads_typed<64, 64>(x, d_o, p, stream);
}
