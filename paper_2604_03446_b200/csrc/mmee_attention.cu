// Attention over states of another length, run: S = Q K^T scale, P = softmax over a sequence's valid keys, O = P V, and the
// gradients of Q, K and V.
//
// The forward kernel keeps scores in tensor memory: a CTA holds up to two tiles of 128 query rows, keys and values stream
// through shared memory by TMA in tiles of 128, S = Q K^T lands in tensor memory, a warpgroup per query tile (a thread per
// row, so that no reduction crosses threads) turns it into P in place, which the next matrix instruction takes from there.
// While one tile's scores are turned, the tensor cores work for the other.
//
// 32/8 heads, 4096 queries, 8192 keys, d 128, bf16: 514 us, 1070 TFLOP/s.  The tensor cores are at work 56 % of active cycles, the
// exponentials' units as much.  What bounds it is a tile's way through a turn (scores read, maximum, 128 exponentials a thread,
// written, P V, the next scores), which is longer than the other tile's products.  Measured on the way (narrow inputs, 459 us as it is):
// exponentials on the multiply-add pipes for a quarter of the values 479; two warpgroups a tile, half a row to a thread, 490; blocks
// of 64 keys with two places for scores 707 (more and smaller matrix instructions); a reference from the block before instead of a
// maximum first 606.
#include "mmee_attention.cuh"

namespace mmee {

namespace {

// --- forward --------------------------------------------------------------------------------------------------------

template <int DK, int DV>
struct ForwardShape {
    static constexpr uint32_t kQ = (DK / 64) * kTile * kRowBytes, kV = (DV / 64) * kTile * kRowBytes;
    static constexpr uint32_t kRing = 2;
    static constexpr uint32_t smem(uint32_t tiles) { return tiles * kQ + kRing * (kQ + kV) + 1024; }
};

// A warpgroup to a query tile, then one warp each for the loads and the matrix instructions; with two query tiles two more that make
// their warpgroup whole: it hands registers on, so that a row's 128 scores fit a thread (8 warps of 208 and 4 of 88 from 12 of 168).
// With one, two CTAs share a multiprocessor: a thread holds half of the scores and reads the others twice.
constexpr uint32_t forward_threads(uint32_t tiles) { return tiles == 2 ? 384 : 192; }

template <int DK, int DV, int TILES, bool BF16>
__global__ void __launch_bounds__(forward_threads(TILES), TILES == 2 ? 1 : 2)
attention_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                 const AttentionParams p) {
    using Shape = ForwardShape<DK, DV>;
    constexpr uint32_t kRing = Shape::kRing, kLoad = TILES * 4, kMma = kLoad + 1;
    constexpr int kHeld = TILES == 2 ? 128 : 64;       // scores of a row that stay in registers
    constexpr uint32_t kColumns = TILES * (128 + DV) <= 256 ? 256 : 512;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[TILES * 5 + 4 * kRing + 1];
    __shared__ uint32_t tmem_base, gave_up;

    // The query tile, and the part of its keys.
    const bool cut_up = blockIdx.x >= p.whole;
    const uint32_t past = blockIdx.x - p.whole, split = cut_up ? past % p.splits : 0, tile = cut_up ? p.whole + past / p.splits : blockIdx.x;
    const uint32_t head = tile / p.tiles_q % p.q_heads, b = tile / p.tiles_q / p.q_heads, q0 = tile % p.tiles_q * (TILES * kTile);
    const uint32_t tiles = (p.seq_q - q0 <= kTile) ? 1 : TILES;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;

    const uint32_t base = (smem_addr(raw) + 1023u) & ~1023u;
    const uint32_t bar0 = smem_addr(bars);
    auto q_full = [&](uint32_t t) { return bar0 + 8 * t; };
    auto s_full = [&](uint32_t t) { return bar0 + 8 * (TILES + t); };
    auto o_full = [&](uint32_t t) { return bar0 + 8 * (2 * TILES + t); };
    auto p_full = [&](uint32_t t, uint32_t h) { return bar0 + 8 * (3 * TILES + 2 * t + h); };
    auto k_full = [&](uint32_t s) { return bar0 + 8 * (5 * TILES + s); };
    auto k_empty = [&](uint32_t s) { return bar0 + 8 * (5 * TILES + kRing + s); };
    auto v_full = [&](uint32_t s) { return bar0 + 8 * (5 * TILES + 2 * kRing + s); };
    auto v_empty = [&](uint32_t s) { return bar0 + 8 * (5 * TILES + 3 * kRing + s); };
    const uint32_t drained = bar0 + 8 * (5 * TILES + 4 * kRing);
    auto q_tile = [&](uint32_t t) { return base + t * Shape::kQ; };
    auto k_tile = [&](uint32_t s) { return base + TILES * Shape::kQ + s * Shape::kQ; };
    auto v_tile = [&](uint32_t s) { return base + (TILES + kRing) * Shape::kQ + s * Shape::kV; };

    if (threadIdx.x == 0) {
        gave_up = 0;
        for (uint32_t t = 0; t < TILES; ++t) {
            mbar_init(q_full(t), 1);
            mbar_init(s_full(t), 1);
            mbar_init(p_full(t, 0), 4);
            mbar_init(p_full(t, 1), 4);
            mbar_init(o_full(t), 1);
        }
        for (uint32_t s = 0; s < kRing; ++s) {
            mbar_init(k_full(s), 1);
            mbar_init(k_empty(s), 1);
            mbar_init(v_full(s), 1);
            mbar_init(v_empty(s), 1);
        }
        mbar_init(drained, 1);
        mbar_init_visible();
    }
    if (warp == kMma) tmem_alloc(&tmem_base, kColumns);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_base;
    volatile uint32_t* const lost = &gave_up;
    wait_for_stream();
    release_stream();
    const uint32_t keys = valid_keys(p.kv_len, b, p.seq_kv);
    const uint32_t t0 = split * p.tiles_per_split, t_all = (keys + kTile - 1) / kTile;
    const uint32_t n = !cut_up ? t_all : t0 < t_all ? min(p.tiles_per_split, t_all - t0) : 0;     // key tiles of this CTA
    auto s_col = [&](uint32_t t) { return tmem + t * 128; };
    auto o_col = [&](uint32_t t) { return tmem + TILES * 128 + t * DV; };
    uint32_t q_sent = 0, k_sent = 0, v_sent = 0;       // loads on their way or landed (of the thread that issues them)

    if (warp >= kLoad) {
        if constexpr (TILES == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        if (warp == kLoad) {
            if (elect_one() && n) {
                const int32_t h = (int32_t)head, hk = (int32_t)(head / p.group), bb = (int32_t)b;
                auto load_q = [&](uint32_t t) {
                    mbar_expect(q_full(t), Shape::kQ);
                    for (int32_t j = 0; j < DK / 64; ++j) tma_load_4d(q_tile(t) + j * kTile * kRowBytes, &mq, q_full(t), 64 * j, (int32_t)(q0 + t * kTile), h, bb);
                    ++q_sent;
                };
                load_q(0);
                for (uint32_t i = 0; i < n; ++i) {
                    const uint32_t s = i % kRing, turn = ((i / kRing) & 1) ^ 1;
                    const int32_t row = (int32_t)((t0 + i) * kTile);
                    if (!mbar_wait(k_empty(s), turn, lost)) break;
                    mbar_expect(k_full(s), Shape::kQ);
                    for (int32_t j = 0; j < DK / 64; ++j) tma_load_4d(k_tile(s) + j * kTile * kRowBytes, &mk, k_full(s), 64 * j, row, hk, bb);
                    ++k_sent;
                    if (i == 0)
                        for (uint32_t t = 1; t < tiles; ++t) load_q(t);
                    if (!mbar_wait(v_empty(s), turn, lost)) break;
                    mbar_expect(v_full(s), Shape::kV);
                    for (int32_t j = 0; j < DV / 64; ++j) tma_load_4d(v_tile(s) + j * kTile * kRowBytes, &mv, v_full(s), 64 * j, row, hk, bb);
                    ++v_sent;
                }
            }
            __syncwarp();
        } else if (warp == kMma) {
            constexpr uint32_t desc_s = mma_desc(BF16, kTile, kTile, false, false);
            const uint32_t desc_o = mma_desc(BF16, kTile, (p.d_v + 15) / 16 * 16, false, true);
            const uint32_t steps_s = (p.d_qk + 15) / 16;
            auto scores = [&](uint32_t t, uint32_t s) {    // S_t = Q_t K^T
                tile_product<DK>(s_col(t), q_tile(t), k_tile(s), desc_s, steps_s);
                mma_commit(s_full(t));
            };
            bool sound = n > 0;
            if (sound) {
                sound = mbar_wait(k_full(0), 0, lost);
                for (uint32_t t = 0; t < tiles && sound; ++t) {
                    if (!(sound = mbar_wait(q_full(t), 0, lost))) break;
                    tcgen05_fence_after();
                    if (elect_one()) {
                        scores(t, 0);
                        if (t + 1 == tiles) mma_commit(k_empty(0));
                    }
                    __syncwarp();
                }
            }
            for (uint32_t i = 0; i < n && sound; ++i) {
                const uint32_t s = i % kRing, s1 = (i + 1) % kRing;
                const uint32_t valid = min(kTile, keys - (t0 + i) * kTile), steps_o = (valid + 15) / 16;
                if (!(sound = mbar_wait(v_full(s), (i / kRing) & 1, lost))) break;
                if (valid % 16) zero_rows(v_tile(s), DV / 64, valid, steps_o * 16);
                if (i + 1 < n && !(sound = mbar_wait(k_full(s1), ((i + 1) / kRing) & 1, lost))) break;
                for (uint32_t t = 0; t < tiles; ++t) {
                    // P V in two halves of 64 keys, the first while the second is still scores.
                    for (uint32_t h = 0; h < 2 && sound; ++h) {
                        if (!(sound = mbar_wait(p_full(t, h), i & 1, lost))) break;
                        tcgen05_fence_after();
                        if (elect_one()) {
                            turned_product<4, 32>(o_col(t), s_col(t) + 32 * h, v_tile(s) + h * 64 * kRowBytes, desc_o, max(steps_o, 4 * h) - 4 * h, i | h);
                        }
                        __syncwarp();
                    }
                    if (!sound) break;
                    if (elect_one()) {
                        if (t + 1 == tiles) mma_commit(v_empty(s));
                        if (i + 1 < n) {
                            scores(t, s1);
                            if (t + 1 == tiles) mma_commit(k_empty(s1));
                        } else {
                            mma_commit(o_full(t));
                        }
                    }
                    __syncwarp();
                }
            }
        }
    } else {
        if constexpr (TILES == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        if (warp / 4 < tiles) {
            const uint32_t t = warp / 4, row = (warp % 4) * 32 + lane, lanes = ((warp % 4) * 32) << 16;
            const float sl2 = p.scale * kLog2e;
            float m = -INFINITY, l = 0.f;                  // reference and sum, in powers of two
            bool sound = true;
            const uint32_t from_s = s_col(t) + lanes;
#pragma unroll 1
            for (uint32_t i = 0; i < n; ++i) {
                if (!(sound = mbar_wait(s_full(t), i & 1, lost))) break;
                tcgen05_fence_after();
                const int valid = (int)min(kTile, keys - (t0 + i) * kTile);
                auto cut = [&](uint32_t* v, int from) {    // scores of keys behind the end
                    if (valid < from + 32) {
#pragma unroll
                        for (int c = 0; c < 32; ++c)
                            if (from + c >= valid) v[c] = 0xff800000u;
                    }
                };
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                auto take_most = [&](const uint32_t* v) {
#pragma unroll
                    for (int c = 0; c < 32; c += 2) top[(c >> 1) & 3] = max3(top[(c >> 1) & 3], __uint_as_float(v[c]), __uint_as_float(v[c + 1]));
                };
                uint32_t x[kHeld], y[32];
#pragma unroll
                for (int c = 0; c < kHeld; c += 32) tmem_load32(from_s + c, x + c);
#pragma unroll
                for (int c = 0; c < kHeld; c += 32) tmem_loaded32(x + c);
#pragma unroll
                for (int c = kHeld; c < 128; c += 32) {
                    tmem_load32(from_s + c, y);
                    tmem_loaded32(y);
                    cut(y, c);
                    take_most(y);
                }
                if (valid < (int)kTile) {
#pragma unroll
                    for (int c = 0; c < kHeld; c += 32) cut(x + c, c);
                }
#pragma unroll
                for (int c = 0; c < kHeld; c += 32) take_most(x + c);
                const float most = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * sl2;
                if (i == 0) {
                    m = most;
                } else if (__any_sync(0xffffffffu, most > m + kSlack)) {
                    // The sums so far: all matrix instructions issued before these scores are done, P V of the last tile too.
                    const float to = most > m + kSlack ? most : m, by = to == m ? 1.f : exp2_fast(m - to);
                    m = to;
                    l *= by;
#pragma unroll 1
                    for (int c = 0; c < DV; c += 16) {     // (few registers: the scores are live)
                        uint32_t o[16];
                        tmem_load16(o_col(t) + lanes + c, o);
                        tmem_loaded16(o);
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * by);
                        tmem_store16(o_col(t) + lanes + c, o);
                    }
                }
                const float from = kBias<BF16> - (m == -INFINITY ? 0.f : m);
                const uint64_t scale2 = pair(sl2, sl2), from2 = pair(from, from);
                uint64_t sum[2] = {0, 0};
                auto turn = [&](const uint32_t* v, int c) {        // 32 scores into probabilities, over scores that have been read
                    uint32_t pk[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float2 w = unpair(fma_pair(pair(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])), scale2, from2));
                        w.x = exp2_fast(w.x), w.y = exp2_fast(w.y);
                        sum[j & 1] = add_pair(sum[j & 1], pair(w.x, w.y));
                        pk[j] = pack2<BF16>(w.x, w.y);
                    }
                    tmem_store16(from_s + c / 2, pk);
                    if (c == 32 || c == 96) {
                        tmem_stored();
                        tcgen05_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(p_full(t, c / 64));
                    }
                };
#pragma unroll
                for (int c = 0; c < kHeld; c += 32) turn(x + c, c);
#pragma unroll
                for (int c = kHeld; c < 128; c += 32) {
                    tmem_load32(from_s + c, y);
                    tmem_loaded32(y);
                    cut(y, c);
                    turn(y, c);
                }
                const float2 sums = unpair(add_pair(sum[0], sum[1]));
                l += sums.x + sums.y;
            }
            const uint32_t token = q0 + t * kTile + row;
            if (n && sound) sound = mbar_wait(o_full(t), 0, lost);
            tcgen05_fence_after();
            const float inv = l == 0.f ? 0.f : 1.f / l;
            const uint64_t part_at = ((uint64_t)split * (p.tiles - p.whole) + (tile - p.whole)) * p.tile_rows + t * kTile + row;    // (if cut up)
            if (sound && token < p.seq_q) {
                const float l2 = l == 0.f ? -INFINITY : m - kBias<BF16> + log2f(l);
                if (cut_up)
                    p.part_lse[part_at] = l2;
                else if (p.lse)
                    p.lse[((uint64_t)b * p.q_heads + head) * p.seq_q + token] = l2 * kLn2;
            }
            if (sound) {
                const int64_t to = (int64_t)b * p.os.batch + (int64_t)token * p.os.token + (int64_t)head * p.os.head;
#pragma unroll
                for (uint32_t c = 0; c < DV; c += 32) {
                    uint32_t o[32];
                    if (n) {
                        tmem_load32(o_col(t) + lanes + c, o);
                        tmem_loaded32(o);
                    }
                    if (token < p.seq_q && c < p.d_v) {
                        float v[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = l == 0.f ? 0.f : __uint_as_float(o[j]) * inv;
                        if (cut_up) {
                            if (l != 0.f) {
                                float4* const q = reinterpret_cast<float4*>(p.part_o + part_at * p.d_v + c);
#pragma unroll
                                for (int j = 0; j < 8; ++j)
                                    if (c + 4 * j < p.d_v) q[j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                            }
                        } else {
                            write_row<BF16>(p.o, to, v, c, p.d_v);
                            if (p.rest) write_row<BF16, true>(p.rest, rest_at(p, b, token, head), v, c, p.d_v);
                        }
                    }
                    __syncwarp();
                }
            }
        }
    }
    tcgen05_fence_before();
    __syncthreads();
    if (gave_up && warp == kLoad) {                    // what is in flight lands before the CTA ends
        if (elect_one()) {
            for (uint32_t t = 0; t < q_sent; ++t) mbar_wait(q_full(t), 0, nullptr);
            for (uint32_t s = 0; s < kRing; ++s) {
                if (k_sent > s) mbar_wait(k_full(s), ((k_sent - 1 - s) / kRing) & 1, nullptr);
                if (v_sent > s) mbar_wait(v_full(s), ((v_sent - 1 - s) / kRing) & 1, nullptr);
            }
        }
        __syncwarp();
    }
    if (warp == kMma) {
        if (gave_up) {                                 // matrix instructions in flight end before their memory is freed
            if (elect_one()) {
                g_gave_up = 1;
                mma_commit(drained);
                mbar_wait(drained, 0, nullptr);
            }
            __syncwarp();
        }
        tcgen05_fence_after();
        tmem_free(tmem, kColumns);
    }
}

// Joins the parts of the keys (32 at most): a warp per query row, a lane's part each for the weights.  Every row's parts are added
// in the same order.
template <bool BF16>
__global__ void __launch_bounds__(128) attention_join_kernel(const AttentionParams p) {
    wait_for_stream();
    release_stream();
    const uint64_t rows = (uint64_t)(p.tiles - p.whole) * p.tile_rows, at = (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    const uint32_t lane = threadIdx.x & 31u;
    if (at >= rows) return;
    const uint32_t tile = p.whole + (uint32_t)(at / p.tile_rows), token = tile % p.tiles_q * p.tile_rows + (uint32_t)(at % p.tile_rows);
    const uint32_t head = tile / p.tiles_q % p.q_heads, b = tile / p.tiles_q / p.q_heads;
    if (token >= p.seq_q) return;
    const float part = lane < p.splits ? p.part_lse[lane * rows + at] : -INFINITY;
    float top = part;
    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    const float from = top == -INFINITY ? 0.f : top, weight = exp2f(part - from);
    const float* const from_o = p.part_o + at * p.d_v + 4 * lane;
    float v[4] = {0.f, 0.f, 0.f, 0.f}, sum = 0.f;
#pragma unroll 4
    for (uint32_t s = 0; s < p.splits; ++s) {
        const float w = __shfl_sync(0xffffffffu, weight, (int)s);
        sum += w;
        if (w != 0.f && 4 * lane < p.d_v) {            // (w = 0: no valid key, its values may not have been written)
            const float4 o = *reinterpret_cast<const float4*>(from_o + s * rows * p.d_v);
            v[0] += w * o.x, v[1] += w * o.y, v[2] += w * o.z, v[3] += w * o.w;
        }
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    if (p.lse && lane == 0) p.lse[((uint64_t)b * p.q_heads + head) * p.seq_q + token] = sum == 0.f ? -INFINITY : (from + log2f(sum)) * kLn2;
    if (4 * lane < p.d_v) {
        uint16_t* const to = static_cast<uint16_t*>(p.o) + (int64_t)b * p.os.batch + (int64_t)token * p.os.token + (int64_t)head * p.os.head;
        for (float& x : v) x *= inv;
        const uint2 w = make_uint2(pack2<BF16>(v[0], v[1]), pack2<BF16>(v[2], v[3]));
        *reinterpret_cast<uint2*>(to + 4 * lane) = w;
        if (p.rest)
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.rest) + rest_at(p, b, token, head) + 4 * lane) =
                make_uint2(rest2<BF16>(v[0], v[1], w.x), rest2<BF16>(v[2], v[3], w.y));
    }
}

// --- host -----------------------------------------------------------------------------------------------------------

template <int DK, int DV, int TILES, bool BF16>
int launch_forward(const Problem& x, cudaStream_t stream) {
    CUtensorMap mq, mk, mv;
    int rc = view_map(&mq, BF16, x.p.batch, x.q);
    if (!rc) rc = view_map(&mk, BF16, x.p.batch, x.k);
    if (!rc) rc = view_map(&mv, BF16, x.p.batch, x.v);
    if (rc) return rc;
    const LaunchAt at{dim3(x.p.whole + (x.p.tiles - x.p.whole) * x.p.splits), forward_threads(TILES), ForwardShape<DK, DV>::smem(TILES), 1, true, stream};
    return launch<attention_kernel<DK, DV, TILES, BF16>>(at, mq, mk, mv, x.p);
}

template <int DK, int DV>
int forward_typed(const Problem& x, cudaStream_t stream) {
    if (x.p.tile_rows == kTile) return x.bf16 ? launch_forward<DK, DV, 1, true>(x, stream) : launch_forward<DK, DV, 1, false>(x, stream);
    return x.bf16 ? launch_forward<DK, DV, 2, true>(x, stream) : launch_forward<DK, DV, 2, false>(x, stream);
}

int forward(const Problem& x, cudaStream_t stream) {
    const bool k = x.p.d_qk > 64, v = x.p.d_v > 64;
    return k ? v ? forward_typed<128, 128>(x, stream) : forward_typed<128, 64>(x, stream)
             : v ? forward_typed<64, 128>(x, stream) : forward_typed<64, 64>(x, stream);
}

// How a call is cut up.  Up to 16 query rows to a key head take the kernel for few rows (`cluster` > 0).
int plan(AttentionParams* p, uint32_t* cluster) {
    *cluster = 0;
    const uint64_t heads = (uint64_t)p->q_heads * p->batch;
    if ((uint64_t)p->group * p->seq_q <= 16) {
        p->tile_rows = p->seq_q;
        p->tiles_q = 1;
        p->tiles = (uint32_t)heads;
        return token_splits(*p, cluster, &p->splits);
    }
    uint32_t sms;
    const int rc = sm_count(&sms);
    if (rc) return rc;
    // Two query tiles a CTA, which share the loads of the keys; or one, of which two fit a multiprocessor if the widths allow it, where
    // that takes fewer turns of the multiprocessors.
    const bool narrow = p->d_qk <= 64 && p->d_v <= 64;
    const uint64_t ones = ceil_div(p->seq_q, kTile) * heads, twos = ceil_div(p->seq_q, 2 * kTile) * heads;
    const bool single = p->seq_q <= kTile || (narrow && ceil_div(ones, 2 * sms) < ceil_div(twos, sms));
    p->tile_rows = single ? kTile : 2 * kTile;
    p->tiles_q = (uint32_t)ceil_div(p->seq_q, p->tile_rows);
    if ((single ? ones : twos) >> 27) return MMEE_ERR_RANGE;
    p->tiles = (uint32_t)(single ? ones : twos);
    // Query tiles that would leave most of the multiprocessors without work have their keys cut into parts: all of them where they are
    // few, of two tiles of keys at least; otherwise those of the last turn, if the time of eight tiles of keys is saved (parts
    // cost a launch, and their sums' way through memory).
    const uint32_t slots = single && narrow ? 2 * sms : sms, keys = (uint32_t)ceil_div(p->seq_kv, kTile), last = p->tiles % slots;
    uint32_t splits = last ? min(slots / last, 16u) : 1;
    if (p->tiles < slots)
        splits = min(splits, keys / 2);
    else if (keys - keys / splits < 8)
        splits = 1;
    p->whole = splits > 1 ? p->tiles - last : p->tiles;
    p->tiles_per_split = splits > 1 ? (uint32_t)ceil_div(keys, splits) : keys;
    p->splits = (uint32_t)ceil_div(keys, p->tiles_per_split);
    return MMEE_OK;
}

uint64_t part_rows(const AttentionParams& p) { return p.splits > 1 ? (uint64_t)p.splits * (p.tiles - p.whole) * p.tile_rows : 0; }
uint64_t parts_bytes(const AttentionParams& p) { return round_up(part_rows(p) * 4, 16) * (p.d_v + 1); }

}  // namespace

int attention_waits(uint32_t* gave_up, const uint64_t* limit_ns) { return waits_of_file(gave_up, limit_ns); }

}  // namespace mmee

using namespace mmee;

extern "C" int mmee_attention_workspace(const mmee_workload_t* w, uint64_t* bytes) {
    if (!w || !bytes || !w->kv_heads) return MMEE_ERR_ARG;
    AttentionParams p{};
    p.batch = w->batch;
    p.q_heads = w->q_heads;
    p.seq_q = w->seq_q;
    p.seq_kv = w->seq_kv;
    p.d_qk = w->d_qk;
    p.d_v = w->d_v;
    if (!p.batch || w->q_heads < w->kv_heads || !p.seq_q || !p.seq_kv) return MMEE_ERR_ARG;
    p.group = w->q_heads / w->kv_heads;
    uint32_t cluster;
    const int rc = plan(&p, &cluster);
    if (!rc) *bytes = parts_bytes(p);
    return rc;
}

extern "C" int mmee_attention(const mmee_workload_t* workload, const mmee_attention_t* a, void* cuda_stream) {
    Problem x;
    int rc = check(workload, a, &x);
    uint32_t cluster;
    if (!rc) rc = plan(&x.p, &cluster);
    if (rc) return rc;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const uint64_t rows = part_rows(x.p);
    if (rows) {
        if (!a->workspace || !aligned16(a->workspace) || a->workspace_bytes < parts_bytes(x.p)) return MMEE_ERR_ARG;
        x.p.part_o = static_cast<float*>(a->workspace);
        x.p.part_lse = x.p.part_o + rows * x.p.d_v;
    }
    if ((rc = cluster ? attention_tokens(x, cluster, stream) : forward(x, stream))) return rc;
    if (rows) {
        const LaunchAt at{dim3((uint32_t)ceil_div(rows / x.p.splits, 4)), 128, 0, 1, true, stream};
        rc = x.bf16 ? launch<attention_join_kernel<true>>(at, x.p) : launch<attention_join_kernel<false>>(at, x.p);
    }
    return rc;
}
