// Host side shared by the calls that run a chain (attention, gated feed-forward).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

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

// Lets a kernel use that much dynamic shared memory on the current device.
int allow_smem(const void* kernel, uint32_t bytes);

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
constexpr uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }
constexpr uint64_t round_up(uint64_t a, uint64_t b) { return ceil_div(a, b) * b; }

// The words that kernels set when a wait ran out, read and cleared (one for each file with such kernels).
int attention_gave_up(uint32_t* word);
int attention_grad_gave_up(uint32_t* word);
int ffn_gave_up(uint32_t* word);
int ffn_narrow_gave_up(uint32_t* word);

}  // namespace mmee
