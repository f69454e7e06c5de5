// pf_tcgen.cuh -- the fifth generation's matrix instruction, its operands' descriptors, tensor memory, and barriers with bounded waits.
#pragma once

#include "pf_ops.cuh"

namespace pf {

// ------------------------------------------------------------------ barriers in shared memory
__device__ __forceinline__ void bar_init(uint32_t b, unsigned count) { asm volatile("mbarrier.init.shared.b64 [%0], %1;" ::"r"(b), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t b) { asm volatile("mbarrier.arrive.shared.b64 _, [%0];" ::"r"(b) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t b, uint32_t bytes)      // an arrival, and so many bytes to come
{
    asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"(b), "r"(bytes) : "memory");
}
// a bulk copy into shared memory: addresses and size are multiples of 16
__device__ __forceinline__ void bulk_in(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// Waits for the phase of that parity; false where `limit` polls of some 2 us each did not see it, or where another wait of the block gave up
// (`gave_up`, the address of a word of shared memory, which this one then sets too).  Written out, so that each of the many places is a dozen instructions: what the
// warps of a block go through has to fit the instruction cache.
__device__ __forceinline__ bool bar_wait(uint32_t b, unsigned parity, unsigned limit, uint32_t gave_up)
{
    uint32_t done;
    asm volatile("{\n.reg .pred p;\n.reg .u32 i, w;\n"
                 "mov.u32 i, %3;\n"
                 "AGAIN:\n"
                 "mbarrier.try_wait.parity.shared.b64 p, [%1], %2, 2000;\n"
                 "mov.u32 %0, 1;\n"
                 "@p bra END;\n"
                 "mov.u32 %0, 0;\n"
                 "ld.shared.u32 w, [%4];\n"
                 "setp.ne.u32 p, w, 0;\n"
                 "@p bra END;\n"
                 "sub.u32 i, i, 1;\n"
                 "setp.gt.s32 p, i, 0;\n"
                 "@p bra AGAIN;\n"
                 "st.shared.u32 [%4], 1;\n"
                 "END:\n}"
                 : "=&r"(done) : "r"(b), "r"(parity), "r"(limit), "r"(gave_up) : "memory");
    return done;
}
// what threads wrote to shared memory becomes visible to the matrix instruction
__device__ __forceinline__ void publish_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ------------------------------------------------------------------ tensor memory: 128 lanes of 512 32-bit columns
__device__ __forceinline__ void tmem_alloc(uint32_t where, uint32_t columns)       // by one warp; the address goes to shared memory
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t columns) { asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns)); }
__device__ __forceinline__ void tmem_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// r is named, so that nothing that reads it moves in front of a wait
template <int N>
__device__ __forceinline__ void tmem_named(uint32_t (&r)[N])
{
#pragma unroll
    for (int i = 0; i < N; i++) asm volatile("" : "+r"(r[i]));
}
// all loads are done, those into r among them
template <int N>
__device__ __forceinline__ void tmem_wait_ld(uint32_t (&r)[N])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
    tmem_named(r);
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// 16 columns of a warp's 32 lanes, a lane a thread
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                   "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr), "r"(r[0]), "r"(r[1]),
                 "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}

// ------------------------------------------------------------------ the matrix instruction: D[128 x N] (+)= A[128 x 16] B[16 x N], fp16 operands, fp32 sums in tensor memory
// Operands in shared memory are rows of 128 bytes, eight of them 1024, whose 16-byte chunks are permuted by the row's number (chunk ^ (row & 7)), at
// addresses that are multiples of 1024.  Either the summed index runs along a row (64 elements; a step of 16 is 32 bytes on), or the
// rows are the summed index (`across`: 64 columns of B a row; a step of 16 is 2048 bytes on; the next 64 columns are `apart` bytes on).
// A descriptor's lower word holds the address and `apart`, in 16 bytes; its upper word is the same for all.
__device__ __forceinline__ uint32_t operand_along(uint32_t addr) { return ((addr & 0x3FFFF) >> 4) | 1u << 16; }
__device__ __forceinline__ uint32_t operand_across(uint32_t addr, uint32_t apart) { return ((addr & 0x3FFFF) >> 4) | (apart >> 4) << 16; }
constexpr uint32_t kOperandHigh = (1024u >> 4) | 1u << 14 | 2u << 29;      // eight rows on: 1024 bytes; version 1; chunks permuted within 128 bytes
__host__ __device__ constexpr uint32_t mma_shape(int n, bool b_across) { return 1u << 4 | (b_across ? 1u << 16 : 0u) | (uint32_t)(n / 8) << 17 | (uint32_t)(128 / 16) << 24; }
// by one thread; `add`: 0 sets D
__device__ __forceinline__ void mma_shared(uint32_t d, uint32_t a, uint32_t b, uint32_t shape, uint32_t add)
{
    asm volatile("{\n.reg .pred p;\n.reg .b64 a, b;\nsetp.ne.b32 p, %4, 0;\nmov.b64 a, {%1, %5};\nmov.b64 b, {%2, %5};\n"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}" ::"r"(d), "r"(a), "r"(b), "r"(shape), "r"(add), "r"(kOperandHigh) : "memory");
}
// A from tensor memory: a lane a row, 16 elements in 8 columns
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint32_t b, uint32_t shape, uint32_t add)
{
    asm volatile("{\n.reg .pred p;\n.reg .b64 b;\nsetp.ne.b32 p, %4, 0;\nmov.b64 b, {%2, %5};\n"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}" ::"r"(d), "r"(a), "r"(b), "r"(shape), "r"(add), "r"(kOperandHigh) : "memory");
}
// one lane of a whole warp, the same one each time
__device__ __forceinline__ bool elected()
{
    uint32_t yes;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xFFFFFFFF;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(yes));
    return yes;
}
// the barrier gets an arrival when all of this thread's matrix instructions so far are done
__device__ __forceinline__ void mma_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

}  // namespace pf
