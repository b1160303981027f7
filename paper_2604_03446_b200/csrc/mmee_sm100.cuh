// The sm_100a instructions that the chain kernels are built from: mbarriers with limited waits, TMA loads, tensor memory
// and the fifth-generation matrix instructions, with the descriptors of 128-byte-swizzled tiles.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

namespace mmee {

int cuda_status(cudaError_t e);        // mmee_api.cu

constexpr uint32_t kRowBytes = 128;            // one row of a swizzled tile: 64 values of 16 bits
constexpr uint32_t kGroupBytes = 8 * kRowBytes;    // eight rows: the unit of the swizzle pattern

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ bool elect_one() {
    uint32_t is;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.b32 %0, 1, 0, p;\n}" : "=r"(is));
    return is != 0;
}

// --- mbarriers ------------------------------------------------------------------------------------------------------

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}

__device__ __forceinline__ void mbar_init_visible() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }

__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.b32 %0, 1, 0, p;\n}"
                 : "=r"(done)
                 : "r"(bar), "r"(parity)
                 : "memory");
    return done != 0;
}

__device__ __forceinline__ uint64_t global_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}

constexpr uint64_t kWaitNs = 4000000000ull;    // no wait of a sound launch comes near this
// One of each for every file with waits: what holds as the limit, and a word that a kernel sets when a wait ran out.
static __device__ uint64_t g_wait_ns = kWaitNs;
static __device__ uint32_t g_gave_up;

// Host side of the two: reads and clears the word, sets the limit (either may be null).
inline int waits_of_file(uint32_t* gave_up, const uint64_t* limit_ns) {
    const uint32_t zero = 0;
    cudaError_t e = cudaSuccess;
    if (gave_up) e = cudaMemcpyFromSymbol(gave_up, g_gave_up, sizeof *gave_up);
    if (e == cudaSuccess && gave_up && *gave_up) e = cudaMemcpyToSymbol(g_gave_up, &zero, sizeof zero);
    if (e == cudaSuccess && limit_ns) e = cudaMemcpyToSymbol(g_wait_ns, limit_ns, sizeof *limit_ns);
    return cuda_status(e);
}

// Waits until the barrier's phase of this parity is over.  False: the wait ran out, here or in another role of the CTA
// (`gave_up`, one word of shared memory); the role then leaves its loop.  With gave_up = nullptr: for what is in flight when a
// kernel gives up, with a limit of its own.
// (Lanes of a warp wait in step: each try, and each look at the clock and the word, is one instruction for them all, so that they
// leave together.  A vote after every wait would cost attention 3 to 4 %.)
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile uint32_t* gave_up) {
    uint64_t end = 0;
    for (uint32_t tries = 1; !mbar_try(bar, parity); ++tries) {
        if (tries % 256) continue;                     // (a look at the clock would delay what waits)
        const uint64_t now = global_ns();
        if (!end) end = now + (gave_up ? g_wait_ns : kWaitNs);
        if ((gave_up && *gave_up) || now >= end) {
            if (gave_up) *gave_up = 1;
            return false;
        }
    }
    return true;
}

// --- the order of kernels in a stream -------------------------------------------------------------------------------

// A kernel that was launched early (LaunchAt::early) may run beside the one before it until it waits here; then that one is done, and
// so is all before it: every kernel here waits before it ends.  Before the wait it touches no memory but what nothing that may still
// run writes.  What that is goes by the call: its first kernel may stand behind anything (a search, which releases at its start, with
// others still running before it) and touches nothing before; a later one may read what no kernel of the call writes, if the
// one before it releases after its own wait.
__device__ __forceinline__ void wait_for_stream() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// From here on (in every block) the next kernel may be launched early.  After the wait, so that the next one knows all but the
// kernel before it to be done.  One exception: the kernel of dQ, which releases at once, beside that of dK and dV; what comes next is
// a call's first kernel.
__device__ __forceinline__ void release_stream() { asm volatile("griddepcontrol.launch_dependents;"); }

// Sixteen bytes that are read once.  Not through the read-only path, which is for what nothing writes as long as a kernel runs: an
// earlier kernel of the stream may still be writing them when one that was launched early starts.
__device__ __forceinline__ uint4 read_once(const uint16_t* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

// --- TMA ------------------------------------------------------------------------------------------------------------

__device__ __forceinline__ void tma_prefetch(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

__device__ __forceinline__ void tma_load_2d(uint32_t to, const CUtensorMap* map, uint32_t bar, int32_t x, int32_t y) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(to),
                 "l"(map), "r"(bar), "r"(x), "r"(y)
                 : "memory");
}

__device__ __forceinline__ void tma_load_4d(uint32_t to, const CUtensorMap* map, uint32_t bar, int32_t x, int32_t y, int32_t z, int32_t w) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(to),
                 "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w)
                 : "memory");
}

// From shared memory; the thread's stores so far are a group after tma_store_commit.
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, uint32_t from, int32_t x, int32_t y) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(from), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, uint32_t from, int32_t x, int32_t y, int32_t z) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(from), "r"(x), "r"(y), "r"(z)
                 : "memory");
}
__device__ __forceinline__ void tma_store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// Waits until all of the thread's groups but the last `LEFT` have been read from shared memory.
template <int LEFT>
__device__ __forceinline__ void tma_store_read() {
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(LEFT) : "memory");
}

// By a CTA of a pair that works on one tile: the bytes are counted at `bar`, which may be the other CTA's (pair_leader).
__device__ __forceinline__ void tma_load_2d_pair(uint32_t to, const CUtensorMap* map, uint32_t bar, int32_t x, int32_t y) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(to),
                 "l"(map), "r"(bar), "r"(x), "r"(y)
                 : "memory");
}

// --- clusters -------------------------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// The same place in the shared memory of the cluster's CTA `rank`.
__device__ __forceinline__ uint32_t cluster_addr(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ uint32_t pair_leader(uint32_t addr) { return cluster_addr(addr, 0); }

__device__ __forceinline__ void store_cluster(uint32_t at, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory");
}

// Counts bytes at a barrier as landed that will not come.
__device__ __forceinline__ void mbar_count_landed(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.complete_tx.relaxed.cluster.shared::cluster.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// What threads wrote to shared memory, seen by the tensor cores.
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// --- tensor memory --------------------------------------------------------------------------------------------------

__device__ __forceinline__ void tmem_alloc(uint32_t* to_smem, uint32_t columns) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(to_smem)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
}

__device__ __forceinline__ void tmem_alloc_pair(uint32_t* to_smem, uint32_t columns) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(to_smem)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void tmem_free_pair(uint32_t base, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
}

__device__ __forceinline__ void tcgen05_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tcgen05_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

#define MMEE_R8(r, i) "=r"((r)[(i)]), "=r"((r)[(i) + 1]), "=r"((r)[(i) + 2]), "=r"((r)[(i) + 3]), "=r"((r)[(i) + 4]), "=r"((r)[(i) + 5]), "=r"((r)[(i) + 6]), "=r"((r)[(i) + 7])
#define MMEE_RW8(r, i) "+r"((r)[(i)]), "+r"((r)[(i) + 1]), "+r"((r)[(i) + 2]), "+r"((r)[(i) + 3]), "+r"((r)[(i) + 4]), "+r"((r)[(i) + 5]), "+r"((r)[(i) + 6]), "+r"((r)[(i) + 7])
#define MMEE_IN8(r, i) "r"((r)[(i)]), "r"((r)[(i) + 1]), "r"((r)[(i) + 2]), "r"((r)[(i) + 3]), "r"((r)[(i) + 4]), "r"((r)[(i) + 5]), "r"((r)[(i) + 6]), "r"((r)[(i) + 7])

// 32 columns of the warp's 32 lanes; the values are there after tmem_loaded of the same registers.
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
        "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : MMEE_R8(r, 0), MMEE_R8(r, 8), MMEE_R8(r, 16), MMEE_R8(r, 24)
        : "r"(addr));
}

__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t* r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : MMEE_R8(r, 0), MMEE_R8(r, 8)
                 : "r"(addr));
}

// The registers are operands, so that no use of them moves before the wait.
__device__ __forceinline__ void tmem_loaded32(uint32_t* r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" : MMEE_RW8(r, 0), MMEE_RW8(r, 8), MMEE_RW8(r, 16), MMEE_RW8(r, 24)::"memory");
}

__device__ __forceinline__ void tmem_loaded16(uint32_t* r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" : MMEE_RW8(r, 0), MMEE_RW8(r, 8)::"memory");
}

__device__ __forceinline__ void tmem_store32(uint32_t addr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
        "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(addr),
        MMEE_IN8(r, 0), MMEE_IN8(r, 8), MMEE_IN8(r, 16), MMEE_IN8(r, 24)
        : "memory");
}

__device__ __forceinline__ void tmem_store16(uint32_t addr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr),
                 MMEE_IN8(r, 0), MMEE_IN8(r, 8)
                 : "memory");
}

__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Sixteen bytes of a swizzled row: the row's piece j lies at j xor (row mod 8).
__device__ __forceinline__ uint32_t swizzled(uint32_t tile, uint32_t row, uint32_t piece) { return tile + row * kRowBytes + ((piece ^ (row & 7u)) << 4); }

__device__ __forceinline__ void store_shared16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

__device__ __forceinline__ float4 load_shared16(uint32_t at) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}

// --- matrix instructions --------------------------------------------------------------------------------------------

// Shared-memory descriptor of a tile with 128-byte swizzle.  Reduction along the row (K-major): rows in groups of eight,
// `lbo` unused.  Reduction along the rows (MN-major): `lbo` is the distance between blocks of 64 columns.  A step of 16
// along the reduction adds 32 bytes (K-major, within a block of 64) or two groups of rows (MN-major).
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr, uint32_t lbo) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | ((uint64_t)(lbo >> 4) << 16) | ((uint64_t)(kGroupBytes >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
constexpr uint64_t kStepK = 32 >> 4, kStepMN = (2 * kGroupBytes) >> 4;

// Instruction descriptor: 16-bit operands of one type, 32-bit sums.
__host__ __device__ constexpr uint32_t mma_desc(bool bf16, uint32_t m, uint32_t n, bool a_mn, bool b_mn) {
    return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) | ((n >> 3) << 17) | ((m >> 4) << 24);
}

__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, bool add) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b),
                 "r"(desc), "r"((uint32_t)add)
                 : "memory");
}

// A from tensor memory (two values of 16 bits to a column).
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t desc, bool add) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a), "l"(b),
                 "r"(desc), "r"((uint32_t)add)
                 : "memory");
}

// On a tile of a pair of CTAs: each holds half of A's rows, half of B's columns and its rows of the sums, at the same places.
__device__ __forceinline__ void mma_ss_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, bool add) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b),
                 "r"(desc), "r"((uint32_t)add)
                 : "memory");
}

// As mma_commit, at the same place in both CTAs.
__device__ __forceinline__ void mma_commit_pair(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3)
                 : "memory");
}

// The barrier gets an arrival when all matrix instructions that this thread has issued are done.
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// The instruction of a warp, operands in registers: for few rows, which fill no 128-row tile.
template <bool BF16>
__device__ __forceinline__ void mma16(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (BF16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// --- values ---------------------------------------------------------------------------------------------------------

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Two 32-bit values in one register pair.
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 unpair(uint64_t v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.ftz.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.ftz.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul_pair(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.ftz.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// An entry's size for a bound that a power of two is chosen by.  Infinities and NaN make their own row or column no number under
// any power, and are not to take the others' bits.
__device__ __forceinline__ float finite_size(float x) {
    const float a = fabsf(x);
    return a < INFINITY ? a : 0.f;
}

// The power of two (-100 to `most`) that values up to `bound` are kept larger by in fp16: they then end at 2^15.
__device__ __forceinline__ int fp16_shift(float bound, int most) {
    return bound > 0.f ? max(-100, min(most, 14 - ilogbf(bound))) : 0;
}

// 2^n for n from -126 to 127, exactly.
__device__ __forceinline__ float power_of_two(int n) { return __uint_as_float((uint32_t)(127 + n) << 23); }

template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    if (BF16)
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

template <bool BF16>
__device__ __forceinline__ float2 unpack2(uint32_t v) {
    if (BF16) return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2*>(&v));
}

}  // namespace mmee
