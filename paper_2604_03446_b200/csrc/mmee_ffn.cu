// The gated feed-forward block, run: h = act(x Wg^T) * (x Wu^T), y = h Wd^T, and its gradients.
//
// Every product is one kernel template: pairs of CTAs go through tiles of 256 x 256 results (single ones through smaller
// tiles where those would be too few), operands stream through shared memory by TMA, one thread issues the matrix
// instructions into one of two accumulators in tensor memory, four warps a CTA empty the other.  Operands lie with the
// reduction along their rows (K-major) or along their columns (MN-major), so that no product needs a transposed copy.  The
// gate kernel puts rows of Wg and the same rows of Wu into one operand tile: both projections of a value of h end in one
// thread, which applies activation and product.
//
// Roundings: sums, gate, up and the gradient of h in 32 bits; h, dg and du are rounded once each to the type of the
// operands, which the tensor cores need; results once.  In fp16 dg and du are kept larger by a power of two for which a bound on
// them fits (grad_bound_kernel), which leaves the results exactly: gradients far below one keep their bits, large ones do not
// overflow on the way.
#include "mmee_ffn.cuh"

namespace mmee {

namespace {

enum Epilogue { kPlain, kGate, kGrad };

// One product of a launch.
struct Product {
    uint32_t m, n;                     // results: rows, columns (kGate: columns of h)
    uint32_t chunks0, chunks1;         // steps of 64 along the reduction, first and second pair of operands
    uint32_t tiles_m, tiles_n, end;    // `end`: tiles of the launch up to here
    uint32_t splits, part_chunks;      // kPlain: parts of the reduction, steps of each; parts are added up afterwards
    uint32_t a_mn, b_mn;               // the operand lies with the reduction along its columns
    uint32_t act;
    void *out, *out2;                  // kPlain: the product; kGate: h; kGrad: dg, du
    int64_t out_stride;                // elements from row to row of out and out2
    float* parts;                      // splits > 1: [splits][m][n]
    float *gate, *up;                  // kGate: where to keep them, or null; kGrad: what was kept.  Rows of n
    uint32_t scaled;                   // fp16: dg and du leave it (kGrad) or go into it a power of two larger
};

constexpr uint32_t kMostProducts = 4;
struct Products {
    CUtensorMap a0[kMostProducts], b0[kMostProducts], a1[kMostProducts], b1[kMostProducts];
    CUtensorMap out[kMostProducts];    // the result, or its parts
    CUtensorMap out2, gate, up;        // kGate, kGrad: of the only product
    Product of[kMostProducts];
    uint32_t count;
    // fp16: bounds by grad_bound_kernel, of the tokens' parts, then of the weights'; multiples of four
    const float* bounds;
    uint32_t token_bounds, weight_bounds;
};

// A tile: 128 rows to a CTA, PAIR: of two CTAs that share the columns' operand.
// Results leave through shared memory: each warp lays 32 rows of 128 bytes down and has the TMA store them, so that memory sees
// whole lines (a thread has a row, its sixteen-byte stores would each be a line of their own, in the way of the operands as well:
// of the training step of 4096 tokens, 4096-16384-4096, the gradient's kernel, which reads what was kept the same way, took 771 us).
constexpr uint32_t kPart = 32 * kRowBytes;             // a warp's rows
template <int EPI, bool PAIR, int TN>
struct TileShape {
    static constexpr uint32_t kM = PAIR ? 256 : 128, kRowsB = PAIR ? TN / 2 : TN;      // rows of a tile; of B in a CTA
    static constexpr uint32_t kA = 128 * kRowBytes, kB = kRowsB * kRowBytes;
    // A warp's places: two of results (kGate: gate and up, then h, or h by turns; kGrad: dg and du), for kGrad two of gate and up each.
    static constexpr uint32_t kParts = EPI == kGrad ? 6 : 2, kStages = (226 * 1024 - 4 * kParts * kPart) / (kA + kB);
    static constexpr uint32_t smem = kStages * (kA + kB) + 4 * kParts * kPart + 1024;
};

constexpr uint32_t kGroupRows = 2048;  // result rows that are gone through together, so that their operands stay in L2

template <uint32_t TM>
__device__ __forceinline__ void tile_of(const Product& p, uint32_t i, uint32_t* tm, uint32_t* tn, uint32_t* split) {
    constexpr uint32_t kGroup = kGroupRows / TM;
    *split = i / (p.tiles_m * p.tiles_n);
    i -= *split * (p.tiles_m * p.tiles_n);
    const uint32_t per = kGroup * p.tiles_n, g = i / per, first = g * kGroup;
    const uint32_t rows = min(kGroup, p.tiles_m - first), r = i - g * per;
    *tm = first + r % rows;
    *tn = r / rows;
}

// Power of two that dg and du are kept larger by in fp16, by a whole warp.  (Not above 2^60: dh, which meets it first, stays finite
// in 32 bits.)
__device__ __forceinline__ int grad_shift(const Products& ps) {
    const uint32_t lane = threadIdx.x & 31u;
    auto largest = [&](const float* from, uint32_t n) {
        float most = 0.f;
#pragma unroll 8
        for (uint32_t i = 4 * lane; i < n; i += 128) {
            const float4 v = __ldcg(reinterpret_cast<const float4*>(from + i));
            most = fmaxf(fmaxf(most, fmaxf(v.x, v.y)), fmaxf(v.z, v.w));
        }
        for (int d = 16; d; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
        return most;
    };
    return fp16_shift(largest(ps.bounds, ps.token_bounds) * largest(ps.bounds + ps.token_bounds, ps.weight_bounds), 60);
}

template <int EPI, bool PAIR, int TN, bool BF16>
__global__ void __launch_bounds__(192, 1) product_kernel(const __grid_constant__ Products ps) {
    using Shape = TileShape<EPI, PAIR, TN>;
    constexpr uint32_t kStages = Shape::kStages, kStage = Shape::kA + Shape::kB;
    constexpr uint32_t kCols = EPI == kGate ? TN / 2 : TN;             // columns of the result in a tile
    constexpr uint32_t kRowsX = EPI == kGate && !PAIR ? TN / 2 : Shape::kRowsB;    // rows of B from one matrix in a CTA
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[2 * kStages + 5 + 8];
    __shared__ uint32_t tmem_base, gave_up, others_sent;       // others_sent: loads of the pair's other CTA, told to the leader
    const uint32_t tiles = (smem_addr(raw) + 1023u) & ~1023u;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    const uint32_t rank = PAIR ? cluster_rank() : 0, workers = PAIR ? gridDim.x / 2 : gridDim.x, worker = PAIR ? blockIdx.x / 2 : blockIdx.x;
    const uint32_t bar0 = smem_addr(bars);
    auto full = [&](uint32_t s) { return bar0 + 8 * s; };
    auto empty = [&](uint32_t s) { return bar0 + 8 * (kStages + s); };
    auto acc_full = [&](uint32_t b) { return bar0 + 8 * (2 * kStages + b); };
    auto acc_empty = [&](uint32_t b) { return bar0 + 8 * (2 * kStages + 2 + b); };
    const uint32_t drained = bar0 + 8 * (2 * kStages + 4);
    auto kept_full = [&](uint32_t w, uint32_t b) { return drained + 8 * (1 + 2 * w + b); };
    if (threadIdx.x == 0) {
        gave_up = 0;
        for (uint32_t s = 0; s < kStages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (uint32_t b = 0; b < 2; ++b) {
            mbar_init(acc_full(b), 1);
            mbar_init(acc_empty(b), PAIR ? 8 : 4);     // an arrival of every warp that empties it
        }
        mbar_init(drained, 1);
        for (uint32_t w = 0; w < 4; ++w)
            for (uint32_t b = 0; b < 2; ++b) mbar_init(kept_full(w, b), 1);
        mbar_init_visible();
    }
    if (warp == 5) {
        if constexpr (PAIR)
            tmem_alloc_pair(&tmem_base, 2 * TN);
        else
            tmem_alloc(&tmem_base, 2 * TN);
    }
    tcgen05_fence_before();
    if constexpr (PAIR)
        cluster_barrier();
    else
        __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_base;
    volatile uint32_t* const lost = &gave_up;
    // fp16 gradients: the kernel before this one finds their bounds, which the results alone need; operands come from before that
    // kernel, which has waited for them.
    constexpr bool kBounds = EPI == kGrad && !BF16;
    if constexpr (!kBounds) {
        wait_for_stream();
        release_stream();
    }
    const uint32_t n_tiles = ps.of[ps.count - 1].end;
    // The product that tile i is part of, and the tile's number there.
    auto product_of = [&](uint32_t i, uint32_t* at) {
        uint32_t k = 0;
        while (i >= ps.of[k].end) ++k;
        *at = i - (k ? ps.of[k - 1].end : 0);
        return k;
    };

    auto commit = [](uint32_t bar) {
        if constexpr (PAIR)
            mma_commit_pair(bar);
        else
            mma_commit(bar);
    };

    uint32_t sent = 0;                                 // steps whose loads are on their way or landed (of the thread that issues them)
    if (warp == 4) {                                   // operands
        if (elect_one()) {
            uint32_t& it = sent;
            bool sound = true;
            for (uint32_t i = worker; i < n_tiles && sound; i += workers) {
                uint32_t at, tm, tn, split;
                const uint32_t k = product_of(i, &at);
                const Product& p = ps.of[k];
                tile_of<Shape::kM>(p, at, &tm, &tn, &split);
                const int32_t m0 = (int32_t)(tm * Shape::kM + rank * 128), n0 = (int32_t)(tn * kCols + (EPI == kGate ? 0 : rank * Shape::kRowsB));
                const uint32_t end = min((split + 1) * p.part_chunks, p.chunks0 + p.chunks1);
                for (uint32_t c = split * p.part_chunks; c < end; ++c, ++it) {
                    const uint32_t s = it % kStages;
                    if (!mbar_wait(empty(s), ((it / kStages) & 1) ^ 1, lost)) {
                        sound = false;
                        break;
                    }
                    const bool one = c < p.chunks0;
                    const CUtensorMap *ma = one ? &ps.a0[k] : &ps.a1[k], *mb = one ? &ps.b0[k] : &ps.b1[k];
                    if (EPI == kGate) mb = PAIR && rank ? &ps.b1[k] : &ps.b0[k];
                    const int32_t d = (int32_t)((one ? c : c - p.chunks0) * 64);
                    const uint32_t sa = tiles + s * kStage, sb = sa + Shape::kA;
                    // The leader's barrier counts both CTAs' bytes (the other's may come before it is told how many).
                    const uint32_t f = PAIR ? pair_leader(full(s)) : full(s);
                    if (rank == 0) mbar_expect(full(s), (PAIR ? 2 : 1) * kStage);
                    auto load = [&](uint32_t to, const CUtensorMap* map, int32_t x, int32_t y) {
                        if constexpr (PAIR)
                            tma_load_2d_pair(to, map, f, x, y);
                        else
                            tma_load_2d(to, map, f, x, y);
                    };
                    if (p.a_mn) {
                        for (int32_t j = 0; j < 2; ++j) load(sa + j * 64 * kRowBytes, ma, m0 + 64 * j, d);
                    } else {
                        load(sa, ma, d, m0);
                    }
                    if (p.b_mn) {
                        for (int32_t j = 0; j < (int32_t)Shape::kRowsB / 64; ++j) load(sb + j * 64 * kRowBytes, mb, n0 + 64 * j, d);
                    } else {
                        // (boxes of 128 rows, of 64 where a CTA holds no more)
                        constexpr int32_t kBox = kRowsX < 128 ? kRowsX : 128;
                        for (int32_t j = 0; j < (int32_t)kRowsX / kBox; ++j) load(sb + j * kBox * kRowBytes, mb, d, n0 + kBox * j);
                        if (EPI == kGate && !PAIR) load(sb + kRowsX * kRowBytes, &ps.b1[k], d, n0);
                    }
                }
            }
            if (PAIR && rank) store_cluster(pair_leader(smem_addr(&others_sent)), sent);
        }
        __syncwarp();
    } else if (warp == 5) {                            // matrix instructions, of a pair the leader's
        uint32_t it = 0, n = 0;
        bool sound = rank == 0;
        for (uint32_t i = worker; i < n_tiles && sound; i += workers, ++n) {
            const uint32_t b = n & 1;
            uint32_t at;
            const Product& p = ps.of[product_of(i, &at)];
            const uint32_t split = at / (p.tiles_m * p.tiles_n), chunks = min(p.part_chunks, p.chunks0 + p.chunks1 - split * p.part_chunks);
            const uint32_t desc = mma_desc(BF16, Shape::kM, TN, p.a_mn, p.b_mn);
            const uint64_t step_a = p.a_mn ? kStepMN : kStepK, step_b = p.b_mn ? kStepMN : kStepK;
            if (!mbar_wait(acc_empty(b), ((n >> 1) & 1) ^ 1, lost)) break;
            tcgen05_fence_after();
            for (uint32_t c = 0; c < chunks; ++c, ++it) {
                const uint32_t s = it % kStages;
                if (!mbar_wait(full(s), (it / kStages) & 1, lost)) {
                    sound = false;
                    break;
                }
                tcgen05_fence_after();
                const uint32_t sa = tiles + s * kStage, sb = sa + Shape::kA;
                const uint64_t da = tile_desc(sa, p.a_mn ? 64 * kRowBytes : 16), db = tile_desc(sb, p.b_mn ? 64 * kRowBytes : 16);
                if (elect_one()) {
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k) {
                        if constexpr (PAIR)
                            mma_ss_pair(tmem + b * TN, da + k * step_a, db + k * step_b, desc, c | k);
                        else
                            mma_ss(tmem + b * TN, da + k * step_a, db + k * step_b, desc, c | k);
                    }
                    commit(empty(s));
                    if (c + 1 == chunks) commit(acc_full(b));
                }
                __syncwarp();
            }
        }
    } else {                                           // results
        uint32_t n = 0, stores = 0, kept = 0, asked = 0;       // tiles, groups of stores, pieces of gate and up: used, asked for
        bool sound = true;
        const uint32_t mine = tiles + kStages * kStage + warp * Shape::kParts * kPart;
        if constexpr (kBounds) {
            wait_for_stream();
            release_stream();
        }
        float larger = 1.f;                            // fp16: the power of two in dh; out of it again in the products of dg and du
        if constexpr (!BF16 && EPI != kGate)
            if (ps.of[0].scaled) larger = power_of_two(EPI == kGrad ? grad_shift(ps) : -grad_shift(ps));
        auto part = [&](uint32_t i) { return mine + i * kPart; };
        // Lays a row of 64 results down, two to a word.
        auto lay = [&](uint32_t to, const uint32_t* v) {
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) store_shared16(swizzled(to, lane, j), v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        };
        auto ready = [] {
            fence_async_shared();
            __syncwarp();
        };
        for (uint32_t i = worker; i < n_tiles && sound; i += workers, ++n) {
            const uint32_t b = n & 1;
            uint32_t at, tm, tn, split;
            const uint32_t k = product_of(i, &at);
            const Product& p = ps.of[k];
            tile_of<Shape::kM>(p, at, &tm, &tn, &split);
            const uint32_t row0 = tm * Shape::kM + rank * 128 + warp * 32, col0 = tn * kCols;
            const uint32_t cols = row0 < p.m ? min(kCols, p.n - col0) : 0;     // of this warp's rows, inside
            auto ask_kept = [&](uint32_t c) {          // gate and up of 32 columns
                if (c >= cols) return;
                if (lane == 0) {
                    const uint32_t q = asked & 1, bar = kept_full(warp, q);
                    mbar_expect(bar, 2 * kPart);
                    tma_load_2d(part(2 + 2 * q), &ps.gate, bar, (int32_t)(col0 + c), (int32_t)row0);
                    tma_load_2d(part(3 + 2 * q), &ps.up, bar, (int32_t)(col0 + c), (int32_t)row0);
                }
                ++asked;
            };
            if (EPI == kGrad) {
                ask_kept(0);
                ask_kept(32);
            }
            if (!mbar_wait(acc_full(b), (n >> 1) & 1, lost)) break;
            tcgen05_fence_after();
            const uint32_t acc = tmem + b * TN + ((warp * 32) << 16);
#pragma unroll 1
            for (uint32_t c = 0; c < kCols && sound; c += 64) {
                uint32_t o[32], o2[32];
#pragma unroll
                for (uint32_t half = 0; half < 2; ++half) {
                    uint32_t x[32], y[32];
                    const uint32_t d = c + 32 * half;
                    tmem_load32(acc + d, x);
                    if (EPI == kGate) tmem_load32(acc + TN / 2 + d, y);
                    tmem_loaded32(x);
                    if (EPI == kGate) tmem_loaded32(y);
                    if constexpr (!BF16 && EPI != kGate) {
                        if (p.scaled) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) x[j] = __float_as_uint(__uint_as_float(x[j]) * larger);
                        }
                    }
                    if (EPI == kPlain && p.splits > 1) {
                        if (d < cols) {                // a part, in 32 bits
                            const uint32_t to = part(stores & 1);
                            if (lane == 0) tma_store_read<1>();
                            __syncwarp();
#pragma unroll
                            for (uint32_t j = 0; j < 8; ++j) store_shared16(swizzled(to, lane, j), x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
                            ready();
                            if (lane == 0) {
                                tma_store_3d(&ps.out[k], to, (int32_t)(col0 + d), (int32_t)row0, (int32_t)split);
                                tma_store_commit();
                            }
                            ++stores;
                        }
                    } else if (EPI == kPlain) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[16 * half + j] = pack2<BF16>(__uint_as_float(x[2 * j]), __uint_as_float(x[2 * j + 1]));
                    } else if (EPI == kGate) {
                        if (p.gate && d < cols) {
                            if (lane == 0) tma_store_read<0>();
                            __syncwarp();
#pragma unroll
                            for (uint32_t j = 0; j < 8; ++j) {
                                store_shared16(swizzled(part(0), lane, j), x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
                                store_shared16(swizzled(part(1), lane, j), y[4 * j], y[4 * j + 1], y[4 * j + 2], y[4 * j + 3]);
                            }
                            ready();
                            if (lane == 0) {
                                tma_store_2d(&ps.gate, part(0), (int32_t)(col0 + d), (int32_t)row0);
                                tma_store_2d(&ps.up, part(1), (int32_t)(col0 + d), (int32_t)row0);
                                tma_store_commit();
                            }
                        }
                        with_act(p.act, [&](auto kind) {
                            constexpr uint32_t kAct = decltype(kind)::value;
#pragma unroll
                            for (int j = 0; j < 16; ++j)
                                o[16 * half + j] = pack2<BF16>(act_value<kAct>(__uint_as_float(x[2 * j])) * __uint_as_float(y[2 * j]),
                                                               act_value<kAct>(__uint_as_float(x[2 * j + 1])) * __uint_as_float(y[2 * j + 1]));
                        });
                    } else if (d < cols && sound) {
                        const uint32_t q = kept & 1;
                        if (!(sound = mbar_wait(kept_full(warp, q), (kept >> 1) & 1, lost))) continue;
                        with_act(p.act, [&](auto kind) {
#pragma unroll
                            for (uint32_t j = 0; j < 8; ++j) {
                                const float4 gv = load_shared16(swizzled(part(2 + 2 * q), lane, j)), uv = load_shared16(swizzled(part(3 + 2 * q), lane, j));
                                const float gg[4] = {gv.x, gv.y, gv.z, gv.w}, uu[4] = {uv.x, uv.y, uv.z, uv.w};
                                float dg[4], du[4];
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    float a, da;
                                    act_both<decltype(kind)::value>(gg[e], &a, &da);
                                    const float dh = __uint_as_float(x[4 * j + e]);
                                    dg[e] = dh * uu[e] * da;
                                    du[e] = dh * a;
                                }
                                o[16 * half + 2 * j] = pack2<BF16>(dg[0], dg[1]);
                                o[16 * half + 2 * j + 1] = pack2<BF16>(dg[2], dg[3]);
                                o2[16 * half + 2 * j] = pack2<BF16>(du[0], du[1]);
                                o2[16 * half + 2 * j + 1] = pack2<BF16>(du[2], du[3]);
                            }
                        });
                        __syncwarp();                  // all have read these places: the next but one goes there
                        ask_kept(d + 64);
                        ++kept;
                    }
                }
                if (c >= cols || !sound || (EPI == kPlain && p.splits > 1)) continue;      // (the same for the whole warp)
                const uint32_t to = EPI == kGrad ? part(0) : part(stores & 1);
                if (lane == 0) {
                    if (EPI == kGrad || (EPI == kGate && p.gate))
                        tma_store_read<0>();
                    else
                        tma_store_read<1>();
                }
                __syncwarp();
                lay(to, o);
                if (EPI == kGrad) lay(part(1), o2);
                ready();
                if (lane == 0) {
                    tma_store_2d(&ps.out[k], to, (int32_t)(col0 + c), (int32_t)row0);
                    if (EPI == kGrad) tma_store_2d(&ps.out2, part(1), (int32_t)(col0 + c), (int32_t)row0);
                    tma_store_commit();
                }
                ++stores;
            }
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0 && sound) {
                if constexpr (PAIR)
                    mbar_arrive_cluster(pair_leader(acc_empty(b)));
                else
                    mbar_arrive(acc_empty(b));
            }
        }
        // Shared memory stays until it has been read; after a wait that ran out, until what was asked for is there.
        if (lane == 0) tma_store_read<0>();
        for (; EPI == kGrad && kept < asked; ++kept) mbar_wait(kept_full(warp, kept & 1), (kept >> 1) & 1, nullptr);
    }
    __syncwarp();
    tcgen05_fence_before();
    // (of a pair: neither's shared or tensor memory goes away while the other uses it)
    if constexpr (PAIR) {
        if (gave_up && lane == 0) store_cluster(cluster_addr(smem_addr(&gave_up), rank ^ 1), 1);       // both know before either ends
        __syncwarp();
        cluster_barrier();
    } else {
        __syncthreads();
    }
    if (gave_up) {                                     // what is in flight lands, matrix instructions end
        if (warp == 4 && rank == 0) {
            if (elect_one()) {
                // Steps that only one CTA of a pair has issued: the barrier is told of the bytes that come, or that do not.
                const uint32_t others = PAIR ? others_sent : sent, all = max(sent, others);
                for (uint32_t i = min(sent, others); i < all; ++i) {
                    if (sent > others)
                        mbar_count_landed(full(i % kStages), kStage);
                    else
                        mbar_expect(full(i % kStages), kStage);
                }
                for (uint32_t s = 0; s < kStages; ++s)
                    if (all > s) mbar_wait(full(s), ((all - 1 - s) / kStages) & 1, nullptr);
            }
            __syncwarp();
        } else if (warp == 5) {
            if (elect_one()) {
                g_gave_up = 1;
                if (rank == 0) commit(drained);
                mbar_wait(drained, 0, nullptr);
            }
            __syncwarp();
        }
        if constexpr (PAIR) cluster_barrier();
    }
    if (warp == 5) {
        tcgen05_fence_after();
        if constexpr (PAIR)
            tmem_free_pair(tmem, 2 * TN);
        else
            tmem_free(tmem, 2 * TN);
    }
}

struct Operand {
    const void* base;
    uint64_t rows, cols;               // as it lies in memory: `cols` values side by side
    int64_t stride;
    bool mn;                           // the reduction is along its rows
};

// Adds a product to a launch.  a1, b1: the second pair of operands (kGate: b1 is the second projection; kPlain: added), or null.
void add_product(Products* ps, Operand* (&ops)[kMostProducts][4], Product p, Operand* a0, Operand* b0, Operand* a1, Operand* b1) {
    p.a_mn = a0->mn;
    p.b_mn = b0->mn;
    p.chunks0 = (uint32_t)ceil_div(a0->mn ? a0->rows : a0->cols, 64);
    p.chunks1 = a1 ? (uint32_t)ceil_div(a1->mn ? a1->rows : a1->cols, 64) : 0;
    Operand* const all[4] = {a0, b0, a1, b1};
    for (int i = 0; i < 4; ++i) ops[ps->count][i] = all[i];
    ps->of[ps->count++] = p;
}

// What dg and du are at most, as the product of two maxima over its blocks: of |w_down|, and over the tokens of sqrt(J) |d_y| times
// the largest of what dh meets -- |dh| is at most the 2-norm of the token's d_y times that of a column of w_down.  Typical values lie
// some 2^12 below the bound, 16 bits above fp16's smallest normal value then.
// Bound by memory, as gate, up and w_down are read once more; a token to a block at a time, so that few tokens have many loads under
// way.  The gradient's kernel, which needs the bounds for its results alone, starts beside it.  us of forward and gradients without and
// with all this: 777 tokens, 1000-2728-712, 112 and 116; 512 tokens, 1024-4096-1024, 85 and 87; 64 tokens, 2048-5464-2048, 96 and 103; eight
// tokens, 4096-16384-4096, 304 and 333 (25 of them w_down's 134 MB); 4096 tokens of that 4577 and 4750.
constexpr uint32_t kTokenBounds = 1024, kWeightBounds = 592;
struct BoundParams {
    const uint16_t *d_y, *w_down;
    int64_t d_y_stride, w_down_stride;
    const float *gate, *up;
    uint32_t tokens, d_ff, d_out, act;
    float* bounds;
    uint32_t token_bounds;
};

__global__ void __launch_bounds__(256) grad_bound_kernel(const BoundParams p) {
    __shared__ float found[2][8];
    wait_for_stream();
    release_stream();
    const uint32_t warp = threadIdx.x >> 5;
    auto over_block = [&](float v, uint32_t at, bool sum) {
        for (int d = 16; d; d >>= 1) {
            const float x = __shfl_xor_sync(0xffffffffu, v, d);
            v = sum ? v + x : fmaxf(v, x);
        }
        if ((threadIdx.x & 31u) == 0) found[at][warp] = v;
        __syncthreads();
        v = found[at][0];
        for (int w = 1; w < 8; ++w) v = sum ? v + found[at][w] : fmaxf(v, found[at][w]);
        return v;
    };
    float most = 0.f;
    if (blockIdx.x >= p.token_bounds) {
        for (uint32_t row = blockIdx.x - p.token_bounds; row < p.d_out; row += gridDim.x - p.token_bounds) {
            const uint16_t* const from = p.w_down + (int64_t)row * p.w_down_stride;
#pragma unroll 4
            for (uint32_t i = threadIdx.x * 8; i < p.d_ff; i += 256 * 8) {
                const uint4 v = *reinterpret_cast<const uint4*>(from + i);
                for (const uint32_t w : {v.x, v.y, v.z, v.w}) {
                    const float2 f = unpack2<false>(w);
                    most = fmaxf(most, fmaxf(finite_size(f.x), finite_size(f.y)));
                }
            }
        }
        most = over_block(most, 0, false);
    } else {
        for (uint32_t token = blockIdx.x; token < p.tokens; token += p.token_bounds) {
            // dh meets up times the activation's slope (1.13 at most, gelu's) and the activation: one at most for sigmoid, |gate| for the others.
            float meets = 0.f, squares = 0.f;
            const uint64_t at = (uint64_t)token * p.d_ff;
            const bool by_gate = p.act != MMEE_ACT_SIGMOID;
#pragma unroll 4
            for (uint32_t i = threadIdx.x * 4; i < p.d_ff; i += 256 * 4) {
                const float4 g = by_gate ? __ldcs(reinterpret_cast<const float4*>(p.gate + at + i)) : make_float4(1.f, 1.f, 1.f, 1.f);
                const float4 u = __ldcs(reinterpret_cast<const float4*>(p.up + at + i));
                for (const float v : {g.x, g.y, g.z, g.w, 1.13f * u.x, 1.13f * u.y, 1.13f * u.z, 1.13f * u.w}) meets = fmaxf(meets, finite_size(v));
            }
            const uint16_t* const d_y = p.d_y + (int64_t)token * p.d_y_stride;
            for (uint32_t i = threadIdx.x * 8; i < p.d_out; i += 256 * 8) {
                const uint4 v = *reinterpret_cast<const uint4*>(d_y + i);
                for (const uint32_t w : {v.x, v.y, v.z, v.w}) {
                    const float2 f = unpack2<false>(w);
                    const float a = finite_size(f.x), b = finite_size(f.y);
                    squares += a * a + b * b;
                }
            }
            meets = over_block(meets, 0, false);
            squares = over_block(squares, 1, true);
            most = fmaxf(most, sqrtf(squares * (float)p.d_out) * meets);
            __syncthreads();                           // (before the next token's are written)
        }
    }
    if (threadIdx.x == 0) p.bounds[blockIdx.x] = most;
}

// Adds the parts of a product up, in order: eight values of a row to a thread.
template <bool BF16>
__global__ void __launch_bounds__(256) join_parts_kernel(const float* parts, uint32_t splits, uint32_t m, uint32_t n, void* out, int64_t out_stride) {
    wait_for_stream();
    release_stream();
    const uint64_t size = (uint64_t)m * n, at = ((uint64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (at >= size) return;
    float4 sum[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll 4
    for (uint32_t s = 0; s < splits; ++s) {
        const float4* const from = reinterpret_cast<const float4*>(parts + s * size + at);
        const float4 x = __ldcg(from), y = __ldcg(from + 1);
        sum[0].x += x.x, sum[0].y += x.y, sum[0].z += x.z, sum[0].w += x.w;
        sum[1].x += y.x, sum[1].y += y.y, sum[1].z += y.z, sum[1].w += y.w;
    }
    uint16_t* const to = static_cast<uint16_t*>(out) + (int64_t)(at / n) * out_stride + at % n;
    *reinterpret_cast<uint4*>(to) = make_uint4(pack2<BF16>(sum[0].x, sum[0].y), pack2<BF16>(sum[0].z, sum[0].w), pack2<BF16>(sum[1].x, sum[1].y),
                                               pack2<BF16>(sum[1].z, sum[1].w));
}

// Cuts the reductions of products of few tiles into parts, so that no pair of CTAs has much more to do than its share of the launch; parts
// of eight steps at least.  Returns the values of all parts.
// 512 tokens, 1024-4096-1024: the down product is 8 tiles of 64 steps each, and took 24 us on 8 of 74 pairs.
uint64_t cut_up(Products* ps, uint32_t sms) {
    const uint32_t pairs = sms / 2;
    uint64_t all = 0, values = 0;
    for (uint32_t i = 0; i < ps->count; ++i) {
        const Product& p = ps->of[i];
        all += ceil_div(p.m, 256) * ceil_div(p.n, 256) * (p.chunks0 + p.chunks1);
    }
    const uint32_t share = (uint32_t)max(ceil_div(all, pairs), (uint64_t)8);
    for (uint32_t i = 0; i < ps->count; ++i) {
        Product& p = ps->of[i];
        const uint32_t chunks = p.chunks0 + p.chunks1, splits = min((uint32_t)ceil_div(chunks, share), 8u);
        p.part_chunks = (uint32_t)ceil_div(chunks, splits);
        p.splits = (uint32_t)ceil_div(chunks, p.part_chunks);
        if (p.splits > 1) values += (uint64_t)p.splits * p.m * p.n;
    }
    return values;
}

template <int EPI, bool PAIR, int TN, bool BF16>
int launch_products(Products& ps, Operand* (&ops)[kMostProducts][4], uint32_t sms, float* parts, cudaStream_t stream) {
    using Shape = TileShape<EPI, PAIR, TN>;
    constexpr uint32_t kRowsX = EPI == kGate && !PAIR ? TN / 2 : Shape::kRowsB;
    uint32_t end = 0;
    int rc = MMEE_OK;
    for (uint32_t i = 0; i < ps.count && !rc; ++i) {
        Product& p = ps.of[i];
        p.tiles_m = (uint32_t)ceil_div(p.m, Shape::kM);
        p.tiles_n = (uint32_t)ceil_div(p.n, EPI == kGate ? TN / 2 : TN);
        p.end = end += p.tiles_m * p.tiles_n * p.splits;
        CUtensorMap* const maps[4] = {&ps.a0[i], &ps.b0[i], &ps.a1[i], &ps.b1[i]};
        for (int k = 0; k < 4 && !rc; ++k) {
            const Operand* const o = ops[i][k];
            if (!o) continue;
            const uint64_t extent[2] = {o->cols, o->rows};
            rc = tile_map(maps[k], BF16, o->base, 2, extent, &o->stride, o->mn ? 64 : k % 2 ? min(128u, kRowsX) : 128);
        }
        const uint64_t result[3] = {p.n, p.m, p.splits};
        const int64_t packed[2] = {p.n, (int64_t)p.m * p.n};
        if (p.splits > 1) {
            p.parts = parts;
            parts += (uint64_t)p.splits * p.m * p.n;
        }
        if (!rc) rc = p.splits > 1 ? tile_map(&ps.out[i], Values::f32, p.parts, 3, result, packed, 32) : tile_map(&ps.out[i], BF16, p.out, 2, result, &p.out_stride, 32);
        if (!rc && EPI == kGrad) rc = tile_map(&ps.out2, BF16, p.out2, 2, result, &p.out_stride, 32);
        if (!rc && p.gate) rc = tile_map(&ps.gate, Values::f32, p.gate, 2, result, packed, 32);
        if (!rc && p.gate) rc = tile_map(&ps.up, Values::f32, p.up, 2, result, packed, 32);
    }
    if (rc) return rc;
    const LaunchAt at{dim3(PAIR ? 2 * min(sms / 2, end) : min(sms, end)), 192, Shape::smem, PAIR ? 2u : 1u, true, stream};
    rc = launch<product_kernel<EPI, PAIR, TN, BF16>>(at, ps);
    for (uint32_t i = 0; i < ps.count && !rc; ++i) {
        const Product& p = ps.of[i];
        if (p.splits == 1) continue;
        const LaunchAt join{dim3((uint32_t)ceil_div((uint64_t)p.m * p.n, 8 * 256)), 256, 0, 1, true, stream};
        rc = launch<join_parts_kernel<BF16>>(join, (const float*)p.parts, p.splits, p.m, p.n, p.out, p.out_stride);
    }
    return rc;
}

// Tiles of 256 x 256 by pairs of CTAs.  The kernels with work at the end of a tile take tiles of 128 x 128 by single CTAs where the large ones
// would leave multiprocessors idle (us, large and small: gate of 512 x 4096 x 1024, 64 large tiles, 15 and 18; gradient, 32 tiles, 22 and 17;
// gradient of 2048 x 4096 x 1024, 128 tiles, 39 and 43).  parts: room for what cut_up says.
template <int EPI>
int products(bool bf16, Products& ps, Operand* (&ops)[kMostProducts][4], float* parts, cudaStream_t stream) {
    uint32_t sms;
    const int rc = sm_count(&sms);
    if (rc) return rc;
    if constexpr (EPI == kPlain) {
        cut_up(&ps, sms);
    } else {
        Product& p = ps.of[0];
        p.splits = 1;
        p.part_chunks = p.chunks0 + p.chunks1;
        const uint64_t large = ceil_div(p.m, 256) * ceil_div(p.n, EPI == kGate ? 128 : 256);
        if (large < (EPI == kGate ? sms / 4 : sms / 2))
            return bf16 ? launch_products<EPI, false, 128, true>(ps, ops, sms, parts, stream) : launch_products<EPI, false, 128, false>(ps, ops, sms, parts, stream);
    }
    return bf16 ? launch_products<EPI, true, 256, true>(ps, ops, sms, parts, stream) : launch_products<EPI, true, 256, false>(ps, ops, sms, parts, stream);
}

Product plain(uint32_t m, uint32_t n, void* out, bool scaled = false) {
    Product p{};
    p.m = m;
    p.n = n;
    p.out = out;
    p.out_stride = n;
    p.scaled = scaled;
    return p;
}

// The block's sizes out of a two-GEMM workload: I tokens, K in, L inside, J out.
struct Sizes {
    uint32_t tokens, d_in, d_ff, d_out;
};

int check(const mmee_workload_t* w, const mmee_gated_ffn_t* f, Sizes* s) {
    if (!w || !f) return MMEE_ERR_ARG;
    if (w->batch != 1 || w->q_heads != 1 || w->kv_heads != 1 || w->word_bytes != 2) return MMEE_ERR_ARG;
    *s = {w->seq_q, w->d_qk, w->seq_kv, w->d_v};
    if (!s->tokens || !s->d_in || !s->d_ff || !s->d_out || (s->d_in | s->d_ff | s->d_out) % 8) return MMEE_ERR_ARG;
    if ((s->tokens | s->d_in | s->d_ff | s->d_out) >> 28) return MMEE_ERR_RANGE;
    if (f->dtype != MMEE_F16 && f->dtype != MMEE_BF16) return MMEE_ERR_ARG;
    if (f->activation > MMEE_ACT_SIGMOID) return MMEE_ERR_ARG;
    const void* in[4] = {f->x, f->w_gate, f->w_up, f->w_down};
    const int64_t stride[4] = {f->x_stride, f->w_gate_stride, f->w_up_stride, f->w_down_stride};
    const uint32_t rows[4] = {s->tokens, s->d_ff, s->d_ff, s->d_out}, cols[4] = {s->d_in, s->d_in, s->d_in, s->d_ff};
    for (int i = 0; i < 4; ++i) {
        if (!in[i] || !aligned16(in[i])) return MMEE_ERR_ARG;
        if (rows[i] > 1 && (stride[i] < (int64_t)cols[i] || stride[i] % 8 || stride[i] >> 38)) return MMEE_ERR_ARG;
    }
    if (!f->hidden || !aligned16(f->hidden)) return MMEE_ERR_ARG;
    return MMEE_OK;
}

// The products of one launch with their operands.
struct Plan {
    Products ps;
    Operand* ops[kMostProducts][4];
    Operand held[10];
};

void plan_forward(const Sizes& s, const mmee_gated_ffn_t& f, Plan* gate, Plan* down) {
    Operand* const g = gate->held;
    g[0] = {f.x, s.tokens, s.d_in, f.x_stride, false};
    g[1] = {f.w_gate, s.d_ff, s.d_in, f.w_gate_stride, false};
    g[2] = {f.w_up, s.d_ff, s.d_in, f.w_up_stride, false};
    Product p = plain(s.tokens, s.d_ff, f.hidden);
    p.act = f.activation;
    p.gate = f.kept;
    p.up = f.kept ? f.kept + (uint64_t)s.tokens * s.d_ff : nullptr;
    gate->ps.count = 0;
    add_product(&gate->ps, gate->ops, p, &g[0], &g[1], nullptr, &g[2]);
    Operand* const d = down->held;
    d[0] = {f.hidden, s.tokens, s.d_ff, s.d_ff, false};
    d[1] = {f.w_down, s.d_out, s.d_ff, f.w_down_stride, false};
    down->ps.count = 0;
    add_product(&down->ps, down->ops, plain(s.tokens, s.d_out, f.y), &d[0], &d[1], nullptr, nullptr);
}

// The backward workspace: dg and du, the bounds, parts.
uint64_t pair_bytes(const Sizes& s) { return 4 * (uint64_t)s.tokens * s.d_ff; }
uint32_t token_bounds(const Sizes& s) { return (uint32_t)round_up(min(s.tokens, kTokenBounds), 4); }
uint32_t weight_bounds(const Sizes& s) { return (uint32_t)round_up(min(s.d_out, kWeightBounds), 4); }
uint64_t fixed_bytes(const Sizes& s) { return pair_bytes(s) + 4 * (token_bounds(s) + weight_bounds(s)); }

void plan_backward(const Sizes& s, const mmee_gated_ffn_t& f, const mmee_gated_ffn_grad_t& g, Plan* grad, Plan* rest) {
    const uint64_t inner = (uint64_t)s.tokens * s.d_ff;            // (a multiple of eight)
    const bool scaled = f.dtype == MMEE_F16;
    for (Plan* const plan : {grad, rest}) {
        plan->ps.bounds = reinterpret_cast<const float*>(static_cast<char*>(f.workspace) + pair_bytes(s));
        plan->ps.token_bounds = token_bounds(s);
        plan->ps.weight_bounds = weight_bounds(s);
    }
    uint16_t* const dg = static_cast<uint16_t*>(f.workspace);
    uint16_t* const du = dg ? dg + inner : nullptr;
    Operand* const o = grad->held;
    o[0] = {g.d_y, s.tokens, s.d_out, g.d_y_stride, false};
    o[1] = {f.w_down, s.d_out, s.d_ff, f.w_down_stride, true};
    Product p = plain(s.tokens, s.d_ff, dg);
    p.out2 = du;
    p.act = f.activation;
    p.gate = f.kept;
    p.up = f.kept ? f.kept + inner : nullptr;
    p.scaled = scaled;
    grad->ps.count = 0;
    add_product(&grad->ps, grad->ops, p, &o[0], &o[1], nullptr, nullptr);
    // The other four products depend on nothing but these, and are one launch: the one with the longest reduction first.
    Operand* const r = rest->held;
    r[0] = {dg, s.tokens, s.d_ff, s.d_ff, false};
    r[1] = {du, s.tokens, s.d_ff, s.d_ff, false};
    r[2] = {f.w_gate, s.d_ff, s.d_in, f.w_gate_stride, true};
    r[3] = {f.w_up, s.d_ff, s.d_in, f.w_up_stride, true};
    r[4] = {dg, s.tokens, s.d_ff, s.d_ff, true};
    r[5] = {du, s.tokens, s.d_ff, s.d_ff, true};
    r[6] = {f.x, s.tokens, s.d_in, f.x_stride, true};
    r[7] = {f.hidden, s.tokens, s.d_ff, s.d_ff, true};
    r[8] = {g.d_y, s.tokens, s.d_out, g.d_y_stride, true};
    rest->ps.count = 0;
    add_product(&rest->ps, rest->ops, plain(s.tokens, s.d_in, g.d_x, scaled), &r[0], &r[2], &r[1], &r[3]);
    add_product(&rest->ps, rest->ops, plain(s.d_ff, s.d_in, g.d_w_gate, scaled), &r[4], &r[6], nullptr, nullptr);
    add_product(&rest->ps, rest->ops, plain(s.d_ff, s.d_in, g.d_w_up, scaled), &r[5], &r[6], nullptr, nullptr);
    add_product(&rest->ps, rest->ops, plain(s.d_out, s.d_ff, g.d_w_down), &r[8], &r[7], nullptr, nullptr);
}

int grad_bound(const Sizes& s, const mmee_gated_ffn_t& f, const mmee_gated_ffn_grad_t& g, cudaStream_t stream) {
    const BoundParams p{static_cast<const uint16_t*>(g.d_y), static_cast<const uint16_t*>(f.w_down), g.d_y_stride, f.w_down_stride, f.kept,
                        f.kept + (uint64_t)s.tokens * s.d_ff, s.tokens, s.d_ff, s.d_out, f.activation,
                        reinterpret_cast<float*>(static_cast<char*>(f.workspace) + pair_bytes(s)), token_bounds(s)};
    return launch<grad_bound_kernel>(LaunchAt{dim3(token_bounds(s) + weight_bounds(s)), 256, 0, 1, true, stream}, p);
}

// Workspace of a call: `fixed` bytes and the parts of the plan's products.
int space_of(Plan* plan, uint64_t fixed, uint64_t* bytes) {
    uint32_t sms;
    const int rc = sm_count(&sms);
    if (!rc) *bytes = fixed + 4 * cut_up(&plan->ps, sms);
    return rc;
}

int check_space(const void* space, uint64_t bytes, Plan* plan, uint64_t fixed) {
    uint64_t need = 0;
    const int rc = space_of(plan, fixed, &need);
    return rc ? rc : need && (!space || !aligned16(space) || bytes < need) ? MMEE_ERR_ARG : MMEE_OK;
}

}  // namespace

int ffn_waits(uint32_t* gave_up, const uint64_t* limit_ns) { return waits_of_file(gave_up, limit_ns); }

}  // namespace mmee

using namespace mmee;

extern "C" int mmee_gated_ffn(const mmee_workload_t* workload, const mmee_gated_ffn_t* f, void* cuda_stream) {
    Sizes s;
    int rc = check(workload, f, &s);
    if (rc) return rc;
    if (!f->y || !aligned16(f->y) || (f->kept && !aligned16(f->kept))) return MMEE_ERR_ARG;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const bool bf16 = f->dtype == MMEE_BF16;
    if (s.tokens <= kNarrow) {
        const FfnTokens few{s.tokens, s.d_in, s.d_ff, s.d_out, f->activation, f->x, f->w_gate, f->w_up, f->w_down,
                            f->x_stride, f->w_gate_stride, f->w_up_stride, f->w_down_stride, f->hidden, f->y, f->kept};
        const uint64_t bytes = 2ull * s.d_ff * (2ull * s.d_in + s.d_out);
        return s.tokens <= kFew && bytes < kFewBytes ? ffn_tokens(few, bf16, stream) : ffn_narrow(few, bf16, stream);
    }
    Plan gate, down;
    plan_forward(s, *f, &gate, &down);
    if ((rc = check_space(f->workspace, f->workspace_bytes, &down, 0))) return rc;
    if ((rc = products<kGate>(bf16, gate.ps, gate.ops, nullptr, stream))) return rc;
    return products<kPlain>(bf16, down.ps, down.ops, static_cast<float*>(f->workspace), stream);
}

extern "C" int mmee_gated_ffn_backward(const mmee_workload_t* workload, const mmee_gated_ffn_t* f, const mmee_gated_ffn_grad_t* g,
                                       void* cuda_stream) {
    Sizes s;
    int rc = check(workload, f, &s);
    if (rc) return rc;
    if (!g || !f->kept || !aligned16(f->kept) || !g->d_y || !aligned16(g->d_y)) return MMEE_ERR_ARG;
    if (s.tokens > 1 && (g->d_y_stride < (int64_t)s.d_out || g->d_y_stride % 8 || g->d_y_stride >> 38)) return MMEE_ERR_ARG;
    void* outs[4] = {g->d_x, g->d_w_gate, g->d_w_up, g->d_w_down};
    for (void* o : outs)
        if (!o || !aligned16(o)) return MMEE_ERR_ARG;
    Plan grad, rest;
    plan_backward(s, *f, *g, &grad, &rest);
    if ((rc = check_space(f->workspace, f->workspace_bytes, &rest, fixed_bytes(s)))) return rc;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const bool bf16 = f->dtype == MMEE_BF16;
    if (!bf16 && (rc = grad_bound(s, *f, *g, stream))) return rc;
    if ((rc = products<kGrad>(bf16, grad.ps, grad.ops, nullptr, stream))) return rc;
    return products<kPlain>(bf16, rest.ps, rest.ops, reinterpret_cast<float*>(static_cast<char*>(f->workspace) + fixed_bytes(s)), stream);
}

extern "C" int mmee_gated_ffn_workspace(const mmee_workload_t* w, uint32_t backward, uint64_t* bytes) {
    if (!w || !bytes || backward > 1) return MMEE_ERR_ARG;
    const Sizes s{w->seq_q, w->d_qk, w->seq_kv, w->d_v};
    if (!s.tokens || !s.d_in || !s.d_ff || !s.d_out) return MMEE_ERR_ARG;
    *bytes = 0;
    if (!backward && s.tokens <= kNarrow) return MMEE_OK;
    Plan first, rest;
    if (backward)
        plan_backward(s, mmee_gated_ffn_t{}, mmee_gated_ffn_grad_t{}, &first, &rest);
    else
        plan_forward(s, mmee_gated_ffn_t{}, &first, &rest);
    return space_of(&rest, backward ? fixed_bytes(s) : 0, bytes);
}
