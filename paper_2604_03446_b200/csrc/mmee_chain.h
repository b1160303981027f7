// Host side shared by the calls that run a chain (attention, gated feed-forward).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/mmee.h"

namespace mmee {

int cuda_status(cudaError_t e);                // mmee_api.cu

// Tensor map of a tensor, innermost dimension contiguous, with 128-byte swizzle and boxes of 128 bytes by `rows` (by one in
// further dimensions).  extent: rank entries, innermost first; stride: rank - 1 entries in elements.
enum class Values { f16, bf16, f32 };
int tile_map(CUtensorMap* map, Values type, const void* base, uint32_t rank, const uint64_t* extent, const int64_t* stride, uint32_t rows);
inline int tile_map(CUtensorMap* map, bool bf16, const void* base, uint32_t rank, const uint64_t* extent, const int64_t* stride, uint32_t rows) {
    return tile_map(map, bf16 ? Values::bf16 : Values::f16, base, rank, extent, stride, rows);
}

// Streaming multiprocessors of the current device.
int sm_count(uint32_t* out);

// A launch of KERNEL with up to 227 KB of dynamic shared memory; `cluster` CTAs to a cluster; `early`: it may start before the kernel
// before it in the stream has ended, and waits for it itself.
struct LaunchAt {
    dim3 grid;
    uint32_t block, smem, cluster;
    bool early;
    cudaStream_t stream;
};

template <auto KERNEL, typename... Args>
int launch(const LaunchAt& at, const Args&... args) {
    // Devices on which the kernel may use its shared memory: asked for once, and again where the device has been reset since.
    static std::atomic<uint64_t> allowed{0};
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return cuda_status(e);
    const uint64_t bit = device < 64 ? 1ull << device : 0;
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t c{};
    c.gridDim = at.grid;
    c.blockDim = dim3(at.block);
    c.dynamicSmemBytes = at.smem;
    c.stream = at.stream;
    c.attrs = attr;
    if (at.cluster > 1) {
        attr[c.numAttrs].id = cudaLaunchAttributeClusterDimension;
        attr[c.numAttrs].val.clusterDim.x = at.cluster;
        attr[c.numAttrs].val.clusterDim.y = attr[c.numAttrs].val.clusterDim.z = 1;
        ++c.numAttrs;
    }
    if (at.early) {
        attr[c.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[c.numAttrs].val.programmaticStreamSerializationAllowed = 1;
        ++c.numAttrs;
    }
    for (bool ask = at.smem > 48 * 1024 && !(allowed.load(std::memory_order_relaxed) & bit);; ask = true) {
        if (ask) {
            e = cudaFuncSetAttribute((const void*)KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)at.smem);
            if (e != cudaSuccess) return cuda_status(e);
            allowed.fetch_or(bit, std::memory_order_relaxed);
        }
        e = cudaLaunchKernelEx(&c, KERNEL, args...);
        if (e != cudaErrorInvalidValue || ask || at.smem <= 48 * 1024) return cuda_status(e);
        cudaGetLastError();
    }
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
constexpr uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }
constexpr uint64_t round_up(uint64_t a, uint64_t b) { return ceil_div(a, b) * b; }

// For each file with kernels that wait: reads and clears the word that they set when a wait ran out, sets the limit of their waits
// (either may be null).
int attention_waits(uint32_t* gave_up, const uint64_t* limit_ns);
int attention_grad_waits(uint32_t* gave_up, const uint64_t* limit_ns);
int ffn_waits(uint32_t* gave_up, const uint64_t* limit_ns);
int ffn_narrow_waits(uint32_t* gave_up, const uint64_t* limit_ns);

}  // namespace mmee
