// The gated feed-forward block for up to 128 tokens: every weight is read once, and that is what bounds it.
//
// Weights are the 128 rows of a matrix instruction, tokens its columns.  A cluster of CTAs takes 128 rows of the weights (of the
// gate kernel: of both projections, so that both of a value of `hidden` end in one thread), its CTAs a part of the reduction each;
// two CTAs fit a multiprocessor and together keep about 200 KB of weights on their way from memory.  The parts are added in order
// over distributed shared memory.  The second kernel is launched before the first has ended: its first weights are under way
// when it waits for `hidden`.
#include <cooperative_groups.h>

#include "mmee_ffn.cuh"

namespace mmee {

namespace {

namespace cg = cooperative_groups;

constexpr uint32_t kRowsW = 128, kTileW = kRowsW * kRowBytes;
constexpr uint32_t kNarrowSmem = 112 * 1024;           // a CTA's share of a multiprocessor
constexpr uint32_t kSlice = 32;                        // columns that are joined at a time

struct NarrowShape {
    uint32_t cols;                     // tokens rounded up to 16
    uint32_t stages, stage_bytes;
    uint32_t columns;                  // of tensor memory
};

template <bool GATE, bool BF16>
__global__ void __launch_bounds__(192) ffn_narrow_kernel(const __grid_constant__ CUtensorMap mw0, const __grid_constant__ CUtensorMap mw1,
                                                         const __grid_constant__ CUtensorMap mx, const FfnTokens p, const NarrowShape z) {
    constexpr uint32_t kW = GATE ? 2 : 1, kMostStages = 6;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[2 * kMostStages + 2];
    __shared__ uint32_t tmem_base, gave_up;
    const uint32_t base = (smem_addr(raw) + 1023u) & ~1023u;
    float* const slice = reinterpret_cast<float*>(raw + (base - smem_addr(raw)));      // [kW][kSlice][128], after the stages are done with
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t parts = cluster.num_blocks(), part = cluster.block_rank(), row0 = blockIdx.x / parts * kRowsW;
    const uint32_t depth = GATE ? p.d_in : p.d_ff, rows = GATE ? p.d_ff : p.d_out, all = (depth + 63) / 64;
    const uint32_t first = (uint32_t)((uint64_t)all * part / parts), n = (uint32_t)((uint64_t)all * (part + 1) / parts) - first;
    const uint32_t bar0 = smem_addr(bars);
    auto full = [&](uint32_t s) { return bar0 + 8 * s; };
    auto empty = [&](uint32_t s) { return bar0 + 8 * (kMostStages + s); };
    const uint32_t sums_full = bar0 + 8 * 2 * kMostStages, drained = sums_full + 8;
    if (threadIdx.x == 0) {
        gave_up = 0;
        for (uint32_t s = 0; s < z.stages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        mbar_init(sums_full, 1);
        mbar_init(drained, 1);
        mbar_init_visible();
    }
    if (warp == 4 && lane == 0) {
        tma_prefetch(&mw0);
        if (GATE) tma_prefetch(&mw1);
        tma_prefetch(&mx);
    }
    if (warp == 5) tmem_alloc(&tmem_base, z.columns);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_base;
    volatile uint32_t* const lost = &gave_up;
    if (GATE) {
        wait_for_stream();
        release_stream();
    }

    uint32_t sent = 0;                                 // steps whose loads are on their way or landed (of the thread that issues them)
    if (warp == 4) {
        if (elect_one()) {
            auto load_w = [&](uint32_t i) {
                const uint32_t s = i % z.stages, to = base + s * z.stage_bytes;
                const int32_t k = (int32_t)((first + i) * 64);
                mbar_expect(full(s), kW * kTileW + z.cols * kRowBytes);
                tma_load_2d(to, &mw0, full(s), k, (int32_t)row0);
                if (GATE) tma_load_2d(to + kTileW, &mw1, full(s), k, (int32_t)row0);
            };
            auto load_x = [&](uint32_t i) {
                const uint32_t s = i % z.stages;
                tma_load_2d(base + s * z.stage_bytes + kW * kTileW, &mx, full(s), (int32_t)((first + i) * 64), 0);
            };
            const uint32_t ahead = min(n, z.stages);
            for (uint32_t i = 0; i < ahead; ++i) load_w(i);
            if (!GATE) {                               // (the weights do not come from the gate kernel)
                wait_for_stream();
                release_stream();
            }
            for (uint32_t i = 0; i < ahead; ++i) load_x(i);
            sent = ahead;
            for (uint32_t i = ahead; i < n; ++i) {
                if (!mbar_wait(empty(i % z.stages), ((i / z.stages) & 1) ^ 1, lost)) break;
                load_w(i);
                load_x(i);
                ++sent;
            }
        }
        __syncwarp();
    } else if (warp == 5) {
        const uint32_t desc = mma_desc(BF16, kRowsW, z.cols, false, false);
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t s = i % z.stages;
            if (!mbar_wait(full(s), (i / z.stages) & 1, lost)) break;
            tcgen05_fence_after();
            if (elect_one()) {
                const uint32_t at = base + s * z.stage_bytes;
                const uint64_t dx = tile_desc(at + kW * kTileW, 16);
#pragma unroll
                for (uint32_t m = 0; m < kW; ++m) {
                    const uint64_t dw = tile_desc(at + m * kTileW, 16);
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k) mma_ss(tmem + m * z.cols, dw + k * kStepK, dx + k * kStepK, desc, i | k);
                }
                mma_commit(empty(s));
                if (i + 1 == n) mma_commit(sums_full);
            }
            __syncwarp();
        }
    }
    bool sound = true;
    if (warp < 4 && n) {
        sound = mbar_wait(sums_full, 0, lost);
        tcgen05_fence_after();
    }
    // A slice of columns at a time: every CTA lays its sums down (the stages are done with), each adds up its share of the rows, in
    // the order of the parts.
    const uint32_t share = (kRowsW + parts - 1) / parts, mine = min(share, kRowsW - min(kRowsW, part * share));
    for (uint32_t c0 = 0; c0 < p.tokens; c0 += kSlice) {
        if (warp < 4) {
#pragma unroll
            for (uint32_t m = 0; m < kW; ++m) {
#pragma unroll
                for (uint32_t h = 0; h < kSlice; h += 16) {
                    if (c0 + h >= z.cols) break;
                    uint32_t v[16];
                    if (n && sound) {
                        tmem_load16(tmem + m * z.cols + c0 + h + ((warp * 32) << 16), v);
                        tmem_loaded16(v);
                    }
#pragma unroll
                    for (uint32_t j = 0; j < 16; ++j) slice[(m * kSlice + h + j) * kRowsW + threadIdx.x] = n ? __uint_as_float(v[j]) : 0.f;
                }
            }
        }
        if (parts > 1)
            cluster.sync();
        else
            __syncthreads();
        for (uint32_t i = threadIdx.x; i < mine * min(kSlice, p.tokens - c0); i += blockDim.x) {
            const uint32_t col = i / mine, row_in = part * share + i % mine, row = row0 + row_in, token = c0 + col;
            if (row >= rows) continue;
            float sum[kW];
#pragma unroll
            for (uint32_t m = 0; m < kW; ++m) {
                float v[8];
#pragma unroll
                for (uint32_t r = 0; r < 8; ++r)
                    v[r] = r < parts ? (parts > 1 ? cluster.map_shared_rank(slice, r) : slice)[(m * kSlice + col) * kRowsW + row_in] : 0.f;
                sum[m] = v[0];
#pragma unroll
                for (uint32_t r = 1; r < 8; ++r) sum[m] += v[r];
            }
            const uint64_t at = (uint64_t)token * rows + row;
            if (GATE && p.kept) {
                p.kept[at] = sum[0];
                p.kept[(uint64_t)p.tokens * rows + at] = sum[kW - 1];
            }
            const float out = GATE ? act_value(p.act, sum[0]) * sum[kW - 1] : sum[0];
            static_cast<uint16_t*>(GATE ? p.hidden : p.y)[at] = (uint16_t)pack2<BF16>(out, 0.f);
        }
        if (parts > 1)                                 // nobody's slice changes while others read it
            cluster.sync();
        else
            __syncthreads();
    }
    tcgen05_fence_before();
    __syncthreads();
    if (gave_up && warp == 4) {                        // what is in flight lands before the CTA ends
        if (elect_one())
            for (uint32_t s = 0; s < z.stages; ++s)
                if (sent > s) mbar_wait(full(s), ((sent - 1 - s) / z.stages) & 1, nullptr);
        __syncwarp();
    }
    if (warp == 5) {
        if (gave_up) {                                 // matrix instructions in flight end before their memory is freed
            if (elect_one()) {
                g_gave_up = 1;
                mma_commit(drained);
                mbar_wait(drained, 0, nullptr);
            }
            __syncwarp();
        }
        tcgen05_fence_after();
        tmem_free(tmem, z.columns);
    }
}

int matrix_map(CUtensorMap* map, bool bf16, const void* base, uint64_t rows, uint64_t cols, int64_t stride, uint32_t box_rows) {
    const uint64_t extent[2] = {cols, rows};
    return tile_map(map, bf16, base, 2, extent, &stride, box_rows);
}

template <bool GATE, bool BF16>
int launch_narrow(const FfnTokens& p, cudaStream_t stream) {
    const uint32_t rows = GATE ? p.d_ff : p.d_out, depth = GATE ? p.d_in : p.d_ff, matrices = GATE ? 2 : 1;
    NarrowShape z;
    z.cols = (uint32_t)round_up(p.tokens, 16);
    z.stage_bytes = matrices * kTileW + z.cols * kRowBytes;
    z.stages = min(6u, (kNarrowSmem - 1024) / z.stage_bytes);
    z.columns = 32;
    while (z.columns < matrices * z.cols) z.columns *= 2;
    CUtensorMap w0, w1, x;
    int rc = GATE ? matrix_map(&w0, BF16, p.w_gate, rows, depth, p.w_gate_stride, kRowsW) : matrix_map(&w0, BF16, p.w_down, rows, depth, p.w_down_stride, kRowsW);
    if (!rc && GATE) rc = matrix_map(&w1, BF16, p.w_up, rows, depth, p.w_up_stride, kRowsW);
    if (!rc) rc = GATE ? matrix_map(&x, BF16, p.x, p.tokens, depth, p.x_stride, z.cols) : matrix_map(&x, BF16, p.hidden, p.tokens, depth, depth, z.cols);
    uint32_t sms;
    if (!rc) rc = sm_count(&sms);
    if (rc) return rc;
    // Parts of the reduction: as many as fill the multiprocessors twice, of two steps at least.
    const uint32_t tiles = (uint32_t)ceil_div(rows, kRowsW), most = (uint32_t)ceil_div(depth, 128);
    const uint32_t parts = max(1u, min(min(8u, 2 * sms / tiles), most));
    const LaunchAt at{dim3(tiles * parts), 192, kNarrowSmem, parts, true, stream};
    return launch<ffn_narrow_kernel<GATE, BF16>>(at, w0, GATE ? w1 : w0, x, p, z);
}

}  // namespace

int ffn_narrow(const FfnTokens& p, bool bf16, cudaStream_t stream) {
    const int rc = bf16 ? launch_narrow<true, true>(p, stream) : launch_narrow<true, false>(p, stream);
    return rc ? rc : bf16 ? launch_narrow<false, true>(p, stream) : launch_narrow<false, false>(p, stream);
}

int ffn_narrow_waits(uint32_t* gave_up, const uint64_t* limit_ns) { return waits_of_file(gave_up, limit_ns); }

}  // namespace mmee
