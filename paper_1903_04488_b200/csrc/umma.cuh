// umma.cuh -- what the matrix products need of the fifth-generation tensor cores: mbarriers with bounded waits, bulk copies
// into shared memory, tensor memory, tcgen05.mma on fp16 operands with fp32 accumulators, and the descriptors of operands that
// lie in shared memory as blocks.
//
// A block is 64 x 64 fp16 numbers, 8 KB: 64 rows of 128 bytes, the 16-byte pieces of row r permuted by xor with r mod 8 (the
// 128-byte swizzle of the tensor cores' operands).  Blocks lie in global memory as they lie in shared memory, so a bulk copy without
// a tensor map moves them, and one block serves as an operand in both directions: its columns along the contraction (K-major) or
// its rows (MN-major).
#pragma once
#include <cuda.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace ssgd {
namespace umma {

constexpr int BLOCK = 64;
constexpr int BLOCK_BYTES = BLOCK * BLOCK * 2;

// Byte offset of the 16-byte piece that holds columns [8 piece, 8 piece + 8) of a block's row
__device__ __forceinline__ uint32_t piece_at(int row, int piece) { return (uint32_t)(row * 128 + ((piece ^ (row & 7)) << 4)); }

__device__ __forceinline__ uint32_t shared_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// ---- mbarriers ---------------------------------------------------------------------------------------

__device__ __forceinline__ void bar_init(uint64_t* bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(shared_addr(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_init_fence() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void bar_expect(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(shared_addr(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(shared_addr(bar)), "r"(parity) : "memory");
    return ok != 0;
}
// Arrives at the barrier in the same place of the pair's first CTA.  Relaxed: what it hands over is tensor memory, ordered by the fence
// before it (fence_before), and a release would wait for all results that are on their way to global memory.
__device__ __forceinline__ void bar_arrive_first(uint64_t* bar) {
    uint32_t remote;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(remote) : "r"(shared_addr(bar)));
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(remote) : "memory");
}
__device__ __forceinline__ void pair_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Only that both have come here: nothing written before is handed over (a release would wait for all of it, some 2 us)
__device__ __forceinline__ void pair_meet() {
    asm volatile("barrier.cluster.arrive.relaxed.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t pair_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ void bar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(shared_addr(bar)) : "memory");
}
// False after two seconds (`limit`), or when another thread of the CTA has given up.  Nothing here takes a thousandth of that.
constexpr uint64_t WAIT_NS = 2000000000ull;
__device__ __forceinline__ bool bar_wait_long(uint64_t* bar, uint32_t parity, volatile int* gave_up, uint64_t limit) {
    const uint64_t t0 = now_ns();
    for (uint32_t i = 1;; ++i) {
        if (bar_try(bar, parity)) return true;
        if ((i & 63u) == 0 && (*gave_up || now_ns() - t0 > limit)) {
            *gave_up = 1;
            return false;
        }
    }
}
__device__ __forceinline__ bool bar_wait(uint64_t* bar, uint32_t parity, volatile int* gave_up, uint64_t limit = WAIT_NS) {
    return bar_try(bar, parity) || bar_wait_long(bar, parity, gave_up, limit);
}
// By a whole warp, with one answer for all of it: its lanes wait each for itself, and where some give up just before the barrier completes for
// the others, what follows (instructions of the whole warp) would be done by a part of it.
__device__ __forceinline__ bool bar_wait_warp(uint64_t* bar, uint32_t parity, volatile int* gave_up, uint64_t limit = WAIT_NS) {
    return __all_sync(0xffffffffu, bar_wait(bar, parity, gave_up, limit));
}

// ---- copies ------------------------------------------------------------------------------------------

// A block into the CTA's own shared memory; what has arrived is counted at the barrier in this place of the pair's first CTA.  The
// tensor map (blocks_map) reads the blocks' memory as rows of 128 bytes, as they are: it is there because a copy without one cannot
// count at another CTA's barrier.  Forwarding by a thread of the second CTA took 1000 cycles per stage, twice the products' time.
__device__ __forceinline__ void block_load(void* shared, const CUtensorMap* map, int32_t block, uint64_t* bar) {
    asm volatile(
        "{\n\t.reg .b32 first;\n\tmapa.shared::cluster.u32 first, %4, 0;\n\t"
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [first];\n\t}"
        ::"r"(shared_addr(shared)), "l"(map), "r"(0), "r"(block * BLOCK), "r"(shared_addr(bar)) : "memory");
}

// ---- tensor memory -----------------------------------------------------------------------------------

// PAIR: for products of two CTAs, where one warp of each calls.  columns: a power of two of at least 32.  The address goes to shared memory.
template <bool PAIR>
__device__ __forceinline__ void tmem_alloc(uint32_t* where, uint32_t columns) {
    if (PAIR) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_addr(where)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_addr(where)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
}
template <bool PAIR>
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t columns) {
    if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns));
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns));
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 columns of the thread's lane (warp w of four has lanes 32 w ..); wait before use
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]),
          "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]),
          "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_load16(uint32_t addr, float (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
          "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_store16(uint32_t addr, const float (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
        ::"r"(addr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]),
          "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]) : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// ---- products ----------------------------------------------------------------------------------------

// Operands are stacks of blocks.  K-major (rows along M or N, 64 columns of the contraction): groups of 8 rows are 1024 bytes apart.
// MN-major (columns along M or N, 64 rows of the contraction): 8 rows of the contraction are 1024 bytes apart, and the next 64
// columns are the next block, or `blocks` blocks further.
__device__ __forceinline__ uint64_t operand(uint32_t addr, bool mn_major, int blocks = 1) {
    const uint64_t leading = mn_major ? (uint64_t)(blocks * (BLOCK_BYTES / 16)) : 1, stride = 1024 / 16;
    return (uint64_t)((addr & 0x3ffff) >> 4) | leading << 16 | stride << 32 | 1ull << 46 | 2ull << 61;
}
// What 16 steps of the contraction add to a descriptor: 32 bytes of a row, or 16 rows
__device__ __forceinline__ uint64_t operand_step(bool mn_major) { return mn_major ? 2048 / 16 : 32 / 16; }

// fp16 x fp16 -> fp32
__device__ __forceinline__ uint32_t instruction(int m, int n, bool a_mn, bool b_mn) {
    return 1u << 4 | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}
// One thread; PAIR: of the first CTA, for both: each holds half of the rows of A and of the result, and half of the columns of B.
template <bool PAIR>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t instr, bool accumulate) {
    if (PAIR)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
            ::"r"(d), "l"(a), "l"(b), "r"(instr), "r"(accumulate ? 1u : 0u) : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
            ::"r"(d), "l"(a), "l"(b), "r"(instr), "r"(accumulate ? 1u : 0u) : "memory");
}
// The barrier (PAIR: of both CTAs) is arrived at when everything this thread has issued is done.
template <bool PAIR>
__device__ __forceinline__ void commit(uint64_t* bar) {
    if (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(shared_addr(bar)),
                     "h"((uint16_t)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(shared_addr(bar)) : "memory");
}

// ---- host side ---------------------------------------------------------------------------------------

// Map of `blocks` blocks from `base` on
inline bool blocks_map(CUtensorMap* map, void* base, int64_t blocks) {
    using Encode = decltype(&cuTensorMapEncodeTiled);
    static const Encode encode = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<Encode>(f);
    }();
    const cuuint64_t dims[2] = {BLOCK, (cuuint64_t)blocks * BLOCK}, strides[1] = {BLOCK * 2};
    const cuuint32_t box[2] = {BLOCK, BLOCK}, each[2] = {1, 1};
    return encode && encode(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, base, dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace umma
}  // namespace ssgd
