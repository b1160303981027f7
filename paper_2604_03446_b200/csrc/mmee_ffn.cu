// The gated feed-forward block, run: h = act(x Wg^T) * (x Wu^T), y = h Wd^T, and its gradients.
//
// Every product is one kernel template: a CTA per SM goes through tiles of 128 x 256 results, operands stream through
// shared memory by TMA, one thread issues the matrix instructions into one of two accumulators in tensor memory, four
// warps empty the other.  Operands lie with the reduction along their rows (K-major) or along their columns (MN-major), so
// that no product needs a transposed copy.  The gate kernel puts 128 rows of Wg and the same 128 rows of Wu into one
// operand tile: both projections of a value of h end in one thread, which applies activation and product.
//
// Roundings: sums, gate, up and the gradient of h in 32 bits; h, dg and du are rounded once each to the type of the
// operands, which the tensor cores need; results once.
#include "mmee_ffn.cuh"

namespace mmee {

namespace {

__device__ uint32_t g_gave_up;

enum Epilogue { kPlain, kGate, kGrad };

struct ProductParams {
    uint32_t m, n;                     // results: rows, columns (kGate: columns of h)
    uint32_t chunks0, chunks1;         // steps of 64 along the reduction, first and second pair of operands
    uint32_t tiles_m, tiles_n;
    uint32_t act;
    void *out, *out2;                  // kPlain: the product; kGate: h; kGrad: dg, du
    int64_t out_stride;                // elements from row to row of out and out2
    float *gate, *up;                  // kGate: where to keep them, or null; kGrad: what was kept.  Rows of n
};

constexpr uint32_t kTileM = 128, kTileN = 256, kStages = 4;
constexpr uint32_t kTileABytes = kTileM * kRowBytes, kTileBBytes = kTileN * kRowBytes;
constexpr uint32_t kProductSmem = kStages * (kTileABytes + kTileBBytes) + 1024;
constexpr uint32_t kGroupM = 16;       // tile rows that are gone through together, so that their operands stay in L2

__device__ __forceinline__ void tile_of(const ProductParams& p, uint32_t i, uint32_t* tm, uint32_t* tn) {
    const uint32_t per = kGroupM * p.tiles_n, g = i / per, first = g * kGroupM;
    const uint32_t rows = min(kGroupM, p.tiles_m - first), r = i - g * per;
    *tm = first + r % rows;
    *tn = r / rows;
}

template <int EPI, bool A_MN, bool B_MN, bool BF16>
__global__ void __launch_bounds__(192, 1)
product_kernel(const __grid_constant__ CUtensorMap a0, const __grid_constant__ CUtensorMap b0,
               const __grid_constant__ CUtensorMap a1, const __grid_constant__ CUtensorMap b1, const ProductParams p) {
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[2 * kStages + 5];
    __shared__ uint32_t tmem_base, gave_up;
    const uint32_t tiles = (smem_addr(raw) + 1023u) & ~1023u;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    const uint32_t bar0 = smem_addr(bars);
    auto full = [&](uint32_t s) { return bar0 + 8 * s; };
    auto empty = [&](uint32_t s) { return bar0 + 8 * (kStages + s); };
    auto acc_full = [&](uint32_t b) { return bar0 + 8 * (2 * kStages + b); };
    auto acc_empty = [&](uint32_t b) { return bar0 + 8 * (2 * kStages + 2 + b); };
    const uint32_t drained = bar0 + 8 * (2 * kStages + 4);
    if (threadIdx.x == 0) {
        gave_up = 0;
        for (uint32_t s = 0; s < kStages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (uint32_t b = 0; b < 2; ++b) {
            mbar_init(acc_full(b), 1);
            mbar_init(acc_empty(b), 128);
        }
        mbar_init(drained, 1);
        mbar_init_visible();
    }
    if (warp == 5) tmem_alloc(&tmem_base, 512);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_base;
    volatile uint32_t* const lost = &gave_up;
    const uint32_t n_tiles = p.tiles_m * p.tiles_n, chunks = p.chunks0 + p.chunks1;
    constexpr uint32_t kCols = EPI == kGate ? kTileN / 2 : kTileN;      // columns of the result in a tile

    if (warp == 4) {                                   // operands
        if (elect_one()) {
            uint32_t it = 0;
            bool sound = true;
            for (uint32_t i = blockIdx.x; i < n_tiles && sound; i += gridDim.x) {
                uint32_t tm, tn;
                tile_of(p, i, &tm, &tn);
                const int32_t m0 = (int32_t)(tm * kTileM), n0 = (int32_t)(tn * kCols);
                for (uint32_t c = 0; c < chunks; ++c, ++it) {
                    const uint32_t s = it % kStages;
                    if (!mbar_wait(empty(s), ((it / kStages) & 1) ^ 1, lost)) {
                        sound = false;
                        break;
                    }
                    const CUtensorMap *ma = c < p.chunks0 ? &a0 : &a1, *mb = c < p.chunks0 || EPI == kGate ? &b0 : &b1;
                    const int32_t k = (int32_t)((c < p.chunks0 ? c : c - p.chunks0) * 64);
                    const uint32_t sa = tiles + s * (kTileABytes + kTileBBytes), sb = sa + kTileABytes, f = full(s);
                    mbar_expect(f, kTileABytes + kTileBBytes);
                    if (A_MN) {
                        for (int32_t j = 0; j < 2; ++j) tma_load_2d(sa + j * 64 * kRowBytes, ma, f, m0 + 64 * j, k);
                    } else {
                        tma_load_2d(sa, ma, f, k, m0);
                    }
                    if (EPI == kGate) {
                        tma_load_2d(sb, &b0, f, k, n0);
                        tma_load_2d(sb + 128 * kRowBytes, &b1, f, k, n0);
                    } else if (B_MN) {
                        for (int32_t j = 0; j < 4; ++j) tma_load_2d(sb + j * 64 * kRowBytes, mb, f, n0 + 64 * j, k);
                    } else {
                        for (int32_t j = 0; j < 2; ++j) tma_load_2d(sb + j * 128 * kRowBytes, mb, f, k, n0 + 128 * j);
                    }
                }
            }
            if (!sound)                                // what is in flight lands before the CTA ends
                for (uint32_t s = 0; s < kStages; ++s)
                    if (it > s) mbar_wait(full(s), ((it - 1 - s) / kStages) & 1, nullptr);
        }
        __syncwarp();
    } else if (warp == 5) {                            // matrix instructions
        constexpr uint32_t desc = mma_desc(BF16, kTileM, kTileN, A_MN, B_MN);
        uint32_t it = 0, n = 0;
        bool sound = true;
        for (uint32_t i = blockIdx.x; i < n_tiles && sound; i += gridDim.x, ++n) {
            const uint32_t b = n & 1;
            if (!mbar_wait(acc_empty(b), ((n >> 1) & 1) ^ 1, lost)) break;
            tcgen05_fence_after();
            for (uint32_t c = 0; c < chunks; ++c, ++it) {
                const uint32_t s = it % kStages;
                if (!mbar_wait(full(s), (it / kStages) & 1, lost)) {
                    sound = false;
                    break;
                }
                tcgen05_fence_after();
                const uint32_t sa = tiles + s * (kTileABytes + kTileBBytes), sb = sa + kTileABytes;
                const uint64_t da = tile_desc(sa, A_MN ? 64 * kRowBytes : 16), db = tile_desc(sb, B_MN ? 64 * kRowBytes : 16);
                if (elect_one()) {
                    for (uint32_t k = 0; k < 4; ++k)
                        mma_ss(tmem + b * kTileN, da + k * (A_MN ? kStepMN : kStepK), db + k * (B_MN ? kStepMN : kStepK), desc, c | k);
                    mma_commit(empty(s));
                    if (c + 1 == chunks) mma_commit(acc_full(b));
                }
                __syncwarp();
            }
        }
    } else {                                           // results
        uint32_t n = 0;
        const uint32_t row_in = warp * 32 + lane;
        for (uint32_t i = blockIdx.x; i < n_tiles; i += gridDim.x, ++n) {
            const uint32_t b = n & 1;
            uint32_t tm, tn;
            tile_of(p, i, &tm, &tn);
            if (!mbar_wait(acc_full(b), (n >> 1) & 1, lost)) break;
            tcgen05_fence_after();
            const uint32_t acc = tmem + b * kTileN + ((warp * 32) << 16);
            const uint32_t row = tm * kTileM + row_in;
            const bool in = row < p.m;
            for (uint32_t c = 0; c < kCols; c += 32) {
                const uint32_t col = tn * kCols + c;
                uint32_t x[32], y[32];
                tmem_load32(acc + c, x);
                if (EPI == kGate) tmem_load32(acc + kTileN / 2 + c, y);
                tmem_loaded32(x);
                if (EPI == kGate) tmem_loaded32(y);
                if (in && col < p.n) {
                    uint32_t o[16], o2[16];
                    if (EPI == kPlain) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[j] = pack2<BF16>(__uint_as_float(x[2 * j]), __uint_as_float(x[2 * j + 1]));
                    } else if (EPI == kGate) {
                        if (p.gate) {
                            float4* const g = reinterpret_cast<float4*>(p.gate + (uint64_t)row * p.n + col);
                            float4* const u = reinterpret_cast<float4*>(p.up + (uint64_t)row * p.n + col);
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                if (col + 4 * j < p.n) {
                                    g[j] = make_float4(__uint_as_float(x[4 * j]), __uint_as_float(x[4 * j + 1]), __uint_as_float(x[4 * j + 2]), __uint_as_float(x[4 * j + 3]));
                                    u[j] = make_float4(__uint_as_float(y[4 * j]), __uint_as_float(y[4 * j + 1]), __uint_as_float(y[4 * j + 2]), __uint_as_float(y[4 * j + 3]));
                                }
                        }
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            o[j] = pack2<BF16>(act_value(p.act, __uint_as_float(x[2 * j])) * __uint_as_float(y[2 * j]),
                                               act_value(p.act, __uint_as_float(x[2 * j + 1])) * __uint_as_float(y[2 * j + 1]));
                    } else {
                        const float4* const g = reinterpret_cast<const float4*>(p.gate + (uint64_t)row * p.n + col);
                        const float4* const u = reinterpret_cast<const float4*>(p.up + (uint64_t)row * p.n + col);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            if (col + 4 * j >= p.n) break;
                            const float4 gv = g[j], uv = u[j];
                            const float gg[4] = {gv.x, gv.y, gv.z, gv.w}, uu[4] = {uv.x, uv.y, uv.z, uv.w};
                            float dg[4], du[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                float a, da;
                                act_both(p.act, gg[e], &a, &da);
                                const float dh = __uint_as_float(x[4 * j + e]);
                                dg[e] = dh * uu[e] * da;
                                du[e] = dh * a;
                            }
                            o[2 * j] = pack2<BF16>(dg[0], dg[1]);
                            o[2 * j + 1] = pack2<BF16>(dg[2], dg[3]);
                            o2[2 * j] = pack2<BF16>(du[0], du[1]);
                            o2[2 * j + 1] = pack2<BF16>(du[2], du[3]);
                        }
                    }
                    // (rows are multiples of eight values long, so that sixteen bytes are inside or outside as one)
                    uint4* const to = reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + (int64_t)row * p.out_stride + col);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (col + 8 * j < p.n) to[j] = make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
                    if (EPI == kGrad) {
                        uint4* const to2 = reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out2) + (int64_t)row * p.out_stride + col);
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (col + 8 * j < p.n) to2[j] = make_uint4(o2[4 * j], o2[4 * j + 1], o2[4 * j + 2], o2[4 * j + 3]);
                    }
                }
                __syncwarp();
            }
            tcgen05_fence_before();
            mbar_arrive(acc_empty(b));
        }
    }
    __syncthreads();
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
        tmem_free(tmem, 512);
    }
}

struct Operand {
    const void* base;
    uint64_t rows, cols;               // as it lies in memory: `cols` values side by side
    int64_t stride;
};

int operand_map(CUtensorMap* map, bool bf16, const Operand& o, uint32_t box_rows) {
    const uint64_t extent[2] = {o.cols, o.rows};
    return tile_map(map, bf16, o.base, 2, extent, &o.stride, box_rows);
}

// One product.  a1, b1: the second pair of operands (kGate: b1 is the second projection; kPlain: added), or null.
template <int EPI, bool A_MN, bool B_MN>
int product(bool bf16, const Operand& a0, const Operand& b0, const Operand* a1, const Operand* b1, ProductParams p, cudaStream_t stream) {
    CUtensorMap ma0, mb0, ma1, mb1;
    const uint32_t rows_a = A_MN ? 64 : 128, rows_b = B_MN ? 64 : 128;
    int rc = operand_map(&ma0, bf16, a0, rows_a);
    if (!rc) rc = operand_map(&mb0, bf16, b0, rows_b);
    if (!rc) rc = operand_map(&ma1, bf16, a1 ? *a1 : a0, rows_a);
    if (!rc) rc = operand_map(&mb1, bf16, b1 ? *b1 : b0, rows_b);
    if (rc) return rc;
    p.chunks0 = (uint32_t)ceil_div(A_MN ? a0.rows : a0.cols, 64);
    p.chunks1 = a1 ? (uint32_t)ceil_div(A_MN ? a1->rows : a1->cols, 64) : 0;
    p.tiles_m = (uint32_t)ceil_div(p.m, kTileM);
    p.tiles_n = (uint32_t)ceil_div(p.n, EPI == kGate ? kTileN / 2 : kTileN);
    uint32_t sms;
    if ((rc = sm_count(&sms))) return rc;
    const void* kernel = bf16 ? (const void*)product_kernel<EPI, A_MN, B_MN, true> : (const void*)product_kernel<EPI, A_MN, B_MN, false>;
    if ((rc = allow_smem(kernel, kProductSmem))) return rc;
    const uint32_t grid = min(sms, p.tiles_m * p.tiles_n);
    if (bf16)
        product_kernel<EPI, A_MN, B_MN, true><<<grid, 192, kProductSmem, stream>>>(ma0, mb0, ma1, mb1, p);
    else
        product_kernel<EPI, A_MN, B_MN, false><<<grid, 192, kProductSmem, stream>>>(ma0, mb0, ma1, mb1, p);
    return cuda_status(cudaGetLastError());
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

}  // namespace

int ffn_gave_up(uint32_t* word) {
    const uint32_t zero = 0;
    int rc = cuda_status(cudaMemcpyFromSymbol(word, g_gave_up, sizeof *word));
    if (!rc && *word) rc = cuda_status(cudaMemcpyToSymbol(g_gave_up, &zero, sizeof zero));
    return rc;
}

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
    const Operand x{f->x, s.tokens, s.d_in, f->x_stride}, wg{f->w_gate, s.d_ff, s.d_in, f->w_gate_stride};
    const Operand wu{f->w_up, s.d_ff, s.d_in, f->w_up_stride}, wd{f->w_down, s.d_out, s.d_ff, f->w_down_stride};
    const Operand h{f->hidden, s.tokens, s.d_ff, s.d_ff};
    ProductParams p{};
    p.m = s.tokens;
    p.n = s.d_ff;
    p.act = f->activation;
    p.out = f->hidden;
    p.out_stride = s.d_ff;
    p.gate = f->kept;
    p.up = f->kept ? f->kept + (uint64_t)s.tokens * s.d_ff : nullptr;
    if ((rc = product<kGate, false, false>(bf16, x, wg, nullptr, &wu, p, stream))) return rc;
    ProductParams q{};
    q.m = s.tokens;
    q.n = s.d_out;
    q.out = f->y;
    q.out_stride = s.d_out;
    return product<kPlain, false, false>(bf16, h, wd, nullptr, nullptr, q, stream);
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
    const uint64_t inner = (uint64_t)s.tokens * s.d_ff;
    if (!g->workspace || !aligned16(g->workspace) || g->workspace_bytes < 4 * inner) return MMEE_ERR_ARG;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const bool bf16 = f->dtype == MMEE_BF16;
    uint16_t* const dg = static_cast<uint16_t*>(g->workspace);
    uint16_t* const du = dg + inner;                   // (inner is a multiple of eight)
    const Operand x{f->x, s.tokens, s.d_in, f->x_stride}, wg{f->w_gate, s.d_ff, s.d_in, f->w_gate_stride};
    const Operand wu{f->w_up, s.d_ff, s.d_in, f->w_up_stride}, wd{f->w_down, s.d_out, s.d_ff, f->w_down_stride};
    const Operand h{f->hidden, s.tokens, s.d_ff, s.d_ff}, dy{g->d_y, s.tokens, s.d_out, g->d_y_stride};
    const Operand odg{dg, s.tokens, s.d_ff, s.d_ff}, odu{du, s.tokens, s.d_ff, s.d_ff};
    ProductParams p{};
    p.m = s.tokens;
    p.n = s.d_ff;
    p.act = f->activation;
    p.out = dg;
    p.out2 = du;
    p.out_stride = s.d_ff;
    p.gate = f->kept;
    p.up = f->kept + inner;
    if ((rc = product<kGrad, false, true>(bf16, dy, wd, nullptr, nullptr, p, stream))) return rc;
    auto plain = [](uint32_t m, uint32_t n, void* out) {
        ProductParams q{};
        q.m = m;
        q.n = n;
        q.out = out;
        q.out_stride = n;
        return q;
    };
    if ((rc = product<kPlain, false, true>(bf16, odg, wg, &odu, &wu, plain(s.tokens, s.d_in, g->d_x), stream))) return rc;
    if ((rc = product<kPlain, true, true>(bf16, odg, x, nullptr, nullptr, plain(s.d_ff, s.d_in, g->d_w_gate), stream))) return rc;
    if ((rc = product<kPlain, true, true>(bf16, odu, x, nullptr, nullptr, plain(s.d_ff, s.d_in, g->d_w_up), stream))) return rc;
    return product<kPlain, true, true>(bf16, dy, h, nullptr, nullptr, plain(s.d_out, s.d_ff, g->d_w_down), stream);
}

extern "C" int mmee_gated_ffn_workspace(const mmee_workload_t* w, uint64_t* bytes) {
    if (!w || !bytes) return MMEE_ERR_ARG;
    *bytes = 4 * (uint64_t)w->seq_q * w->seq_kv;
    return MMEE_OK;
}
