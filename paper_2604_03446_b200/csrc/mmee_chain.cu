// Host side shared by the calls that run a chain: tensor maps, device limits, the status of past launches.
#include "mmee_chain.h"

#include <initializer_list>

namespace mmee {

namespace {

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
    static const EncodeTiled f = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return f;
}

}  // namespace

int tile_map(CUtensorMap* map, Values type, const void* base, uint32_t rank, const uint64_t* extent, const int64_t* stride, uint32_t rows) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return cuda_status(cudaErrorNotSupported);
    const uint32_t size = type == Values::f32 ? 4 : 2;
    cuuint64_t dims[5], bytes[5];
    cuuint32_t box[5], step[5];
    for (uint32_t i = 0; i < rank; ++i) {
        dims[i] = extent[i];
        box[i] = i == 0 ? 128 / size : i == 1 ? rows : 1;
        step[i] = 1;
    }
    // (a dimension of one entry may carry any stride: a legal one stands in)
    for (uint32_t i = 0; i + 1 < rank; ++i) bytes[i] = extent[i + 1] == 1 ? 16 : (cuuint64_t)stride[i] * size;
    const CUresult r = encode(map, type == Values::f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : type == Values::bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                              rank, const_cast<void*>(base), dims, bytes, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? MMEE_OK : MMEE_ERR_ARG;
}

int sm_count(uint32_t* out) {
    static std::atomic<uint32_t> known[64];            // (asking takes longer than a launch's other preparations)
    int device = 0, n = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return cuda_status(e);
    if (device < 64 && (*out = known[device].load(std::memory_order_relaxed))) return MMEE_OK;
    e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device);
    if (e != cudaSuccess) return cuda_status(e);
    *out = (uint32_t)n;
    if (device < 64) known[device].store(*out, std::memory_order_relaxed);
    return MMEE_OK;
}

}  // namespace mmee

static int all_waits(uint32_t* any, const uint64_t* limit_ns) {
    const int done = mmee::cuda_status(cudaDeviceSynchronize());     // (streams that do not wait for the default one, too)
    if (done) return done;
    for (const auto waits : {mmee::attention_waits, mmee::attention_grad_waits, mmee::ffn_waits, mmee::ffn_narrow_waits}) {
        uint32_t w = 0;
        const int rc = waits(any ? &w : nullptr, limit_ns);
        if (rc) return rc;
        if (any) *any |= w;
    }
    return MMEE_OK;
}

extern "C" int mmee_chain_status(void) {
    uint32_t any = 0;
    const int rc = all_waits(&any, nullptr);
    return rc ? rc : any ? MMEE_ERR_TIMEOUT : MMEE_OK;
}

extern "C" int mmee_chain_wait_limit(uint64_t nanoseconds) {
    if (nanoseconds >> 62) return MMEE_ERR_ARG;        // (it is added to the clock)
    return all_waits(nullptr, &nanoseconds);
}
