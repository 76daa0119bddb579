// sm_100a building blocks of the attention kernels: mbarriers with bounded waits, asynchronous copies, tensor memory, and the
// fifth-generation matrix instructions with their descriptors.
#pragma once
#include <stdint.h>
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace tiga {

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// ---- mbarriers
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
// one arrival, and `bytes` that bulk copies will bring
__device__ __forceinline__ void mbar_arrive_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok;
}
// Waits for the phase of this parity, about two seconds at most: then the block's abort word is set, every other wait of the block
// ends as well, and the block leaves through its usual end (rows that it did not finish are NaN).
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile uint32_t* abort_word) {
    if (mbar_try(bar, parity)) return true;
    const long long t0 = clock64();
    for (uint32_t n = 0;; ++n) {
        if (mbar_try(bar, parity)) return true;
        if ((n & 15) == 15) {
            if (*abort_word) return false;
            if (clock64() - t0 > (1LL << 32)) { *abort_word = 1; return false; }
        }
    }
}
// Without the abort word: waits for other warps of the block, whose own waits all end (a minute), or for what is still on its way.
constexpr long long A_MINUTE = 1LL << 37, HALF_A_SECOND = 1LL << 30;
__device__ __forceinline__ bool mbar_wait_for(uint32_t bar, uint32_t parity, long long cycles) {
    const long long t0 = clock64();
    while (!mbar_try(bar, parity))
        if (clock64() - t0 > cycles) return false;
    return true;
}

// ---- asynchronous copies (generic proxy) and the fence in front of their use by the matrix instructions
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
// arrives on the barrier (as one of its expected arrivals) once all earlier copies of this thread have landed
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// a box of a tensor map (four dimensions) to shared memory; arrives on the barrier with its bytes
__device__ __forceinline__ void box_copy(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2, int c3) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}

// ---- tensor memory
__device__ __forceinline__ void tmem_alloc(uint32_t slot, uint32_t columns) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns));
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

#define TIGA_R8(r, o) "=r"(r[o]), "=r"(r[o + 1]), "=r"(r[o + 2]), "=r"(r[o + 3]), "=r"(r[o + 4]), "=r"(r[o + 5]), "=r"(r[o + 6]), "=r"(r[o + 7])
#define TIGA_W8(r, o) "r"(r[o]), "r"(r[o + 1]), "r"(r[o + 2]), "r"(r[o + 3]), "r"(r[o + 4]), "r"(r[o + 5]), "r"(r[o + 6]), "r"(r[o + 7])

// Waits for this thread's loads.  The arrays that they fill are named, so that no use of them is moved in front of the wait, and no other
// value takes their registers before it (both happened: the load's results are outputs of the load as far as the compiler can see).
#define TIGA_RW8(r, o) "+r"(r[o]), "+r"(r[o + 1]), "+r"(r[o + 2]), "+r"(r[o + 3]), "+r"(r[o + 4]), "+r"(r[o + 5]), "+r"(r[o + 6]), "+r"(r[o + 7])
__device__ __forceinline__ void tmem_wait_ld(uint32_t (&r)[8]) { asm volatile("tcgen05.wait::ld.sync.aligned;" : TIGA_RW8(r, 0) :: "memory"); }
__device__ __forceinline__ void tmem_wait_ld(uint32_t (&r)[16]) { asm volatile("tcgen05.wait::ld.sync.aligned;" : TIGA_RW8(r, 0), TIGA_RW8(r, 8) :: "memory"); }
__device__ __forceinline__ void tmem_wait_ld(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" : TIGA_RW8(r, 0), TIGA_RW8(r, 8), TIGA_RW8(r, 16), TIGA_RW8(r, 24) :: "memory");
}

// 32 columns of this thread's lane
__device__ __forceinline__ void tmem_ld32(uint32_t at, uint32_t (&r)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : TIGA_R8(r, 0), TIGA_R8(r, 8), TIGA_R8(r, 16), TIGA_R8(r, 24) : "r"(at));
}
__device__ __forceinline__ void tmem_ld16(uint32_t at, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : TIGA_R8(r, 0), TIGA_R8(r, 8) : "r"(at));
}
__device__ __forceinline__ void tmem_ld8(uint32_t at, uint32_t (&r)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];" : TIGA_R8(r, 0) : "r"(at));
}
__device__ __forceinline__ void tmem_st8(uint32_t at, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(at), TIGA_W8(r, 0) : "memory");
}
template <int N>
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t (&r)[N]) {          // the first 16
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(at), TIGA_W8(r, 0), TIGA_W8(r, 8) : "memory");
}

// ---- matrix instructions (fp16 / bf16 operands of one type, fp32 accumulators; M = 128)
// Shared-memory operands are rows of 128 bytes (64 elements) in groups of eight, swizzled: the 16-byte piece c of row r lies at
// place c ^ (r & 7).  The same tile serves as a K-major operand (its rows are M or N, its features K) and as an MN-major one (its
// features are N, its rows K): then `next_block` is the distance to the next 64 features.
// A descriptor's low word: address and next_block; tiles differ in the address alone, which is added to it (in units of 16 bytes).  The
// high word is the same for all: 1024 bytes from one group of eight rows to the next, the swizzle of 128 bytes.
__device__ __forceinline__ uint32_t smem_desc(uint32_t addr, uint32_t next_block) { return (addr >> 4) | (next_block >> 4) << 16; }
#define TIGA_DESC_HIGH "0x40004040"
template <typename T> __device__ constexpr uint32_t operand_type();
template <> __device__ constexpr uint32_t operand_type<__half>() { return 0; }
template <> __device__ constexpr uint32_t operand_type<__nv_bfloat16>() { return 1; }
template <typename T>
__device__ __forceinline__ constexpr uint32_t mma_shape(int N, bool b_mn_major) {
    return (1u << 4) | (operand_type<T>() << 7) | (operand_type<T>() << 10) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(N / 8) << 17) | (8u << 24);
}
constexpr uint32_t MMA_NEGATE_A = 1u << 13;

// One thread of a converged warp.  (Where the compiler sees this election, the operands of the instructions below stay in the warp's
// uniform registers; behind a comparison of thread numbers each instruction paid about 80 cycles for their transfer.)
__device__ __forceinline__ bool elected() {
    uint32_t yes;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
    return yes;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t shape, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.u32 p, %4, 0;\n\tmov.b64 da, {%1, " TIGA_DESC_HIGH "};\n\tmov.b64 db, {%2, " TIGA_DESC_HIGH "};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(shape), "r"((uint32_t)add) : "memory");
}
// A from tensor memory: two consecutive K elements per 32-bit column
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t shape, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 db;\n\tsetp.ne.u32 p, %4, 0;\n\tmov.b64 db, {%2, " TIGA_DESC_HIGH "};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(shape), "r"((uint32_t)add) : "memory");
}
// arrives on the barrier once all matrix instructions that this thread issued so far are done
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// ---- arithmetic
__device__ __forceinline__ float ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float max3(float a, float b, float c) { float r; asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }
template <typename T> __device__ __forceinline__ uint32_t pack_half(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack_half<__half>(float lo, float hi) { uint32_t r; asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo)); return r; }
template <> __device__ __forceinline__ uint32_t pack_half<__nv_bfloat16>(float lo, float hi) { uint32_t r; asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo)); return r; }

}  // namespace tiga
