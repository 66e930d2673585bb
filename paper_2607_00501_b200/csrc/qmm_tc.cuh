// qmm_tc.cuh -- thin wrappers over the Blackwell tensor-core machinery used by
// the prefill and mixture-of-experts kernels: mbarriers with bounded waits,
// TMA tile loads, tensor-memory allocation / loads / stores and tcgen05.mma
// with the A operand in tensor memory.
#pragma once

#include <cuda.h>
#include <stdint.h>

namespace qmm {
namespace tc {

__device__ __forceinline__ uint32_t smem_u32(const void* p)
{
    return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

// One lane of a converged warp (the same lane every time).
__device__ __forceinline__ bool elect_one()
{
    uint32_t pred;
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "elect.sync _|p, 0xFFFFFFFF;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t"
        "}\n"
        : "=r"(pred));
    return pred != 0;
}

// ------------------------------------------------------------ mbarrier

__device__ __forceinline__ void mbar_init(uint64_t* bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory");
}

__device__ __forceinline__ void mbar_arrive(uint64_t* bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}

__device__ __forceinline__ void mbar_arrive_expect_tx(uint64_t* bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}

__device__ __forceinline__ bool mbar_try_wait(uint64_t* bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t"
        "}\n"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}

// Bounded wait: gives up after ~2^31 clock cycles (about a second), or at once
// when another role of the block has already given up (*abort != 0).  Returns
// false on give-up; the caller then raises the abort flag and unwinds.  No wait
// in these kernels can spin forever.
constexpr long long kWaitLimitCycles = 1LL << 31;

__device__ __forceinline__ bool mbar_wait(uint64_t* bar, uint32_t parity, volatile int* abort,
                                          long long limit_cycles = kWaitLimitCycles)
{
    if (mbar_try_wait(bar, parity)) return true;
    const long long t0 = clock64();
    while (true) {
        if (mbar_try_wait(bar, parity)) return true;
        if (*abort) return false;
        if (clock64() - t0 > limit_cycles) return false;
    }
}

__device__ __forceinline__ void fence_barrier_init()
{
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}

// ------------------------------------------------------------------ TMA

// 2-D tiled load global -> shared, completion counted on an mbarrier.  No
// multicast: every block fetches its own tile.
__device__ __forceinline__ void tma_load_2d(void* smem_dst, const CUtensorMap* map, int x, int y, uint64_t* bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
        ::"r"(smem_u32(smem_dst)), "l"(map), "r"(x), "r"(y), "r"(smem_u32(bar))
        : "memory");
}

__device__ __forceinline__ void st_shared_b32(uint32_t addr, uint32_t v)
{
    asm volatile("st.shared.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

__device__ __forceinline__ uint4 ld_shared_v4(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}

// Ask L2 for `bytes` (multiple of 16) of global memory starting at a 16-byte aligned address.
__device__ __forceinline__ void l2_prefetch(const void* gptr, uint32_t bytes)
{
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(gptr), "r"(bytes) : "memory");
}

__device__ __forceinline__ void prefetch_tensormap(const CUtensorMap* map)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// -------------------------------------------------------- tensor memory

// Allocate `cols` (power of two >= 32) columns; the base address is written to
// *slot in shared memory.  Whole warp, converged.
__device__ __forceinline__ void tmem_alloc(uint32_t* slot, uint32_t cols)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(cols)
                 : "memory");
}
__device__ __forceinline__ void tmem_relinquish()
{
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc(uint32_t base, uint32_t cols)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols) : "memory");
}

__device__ __forceinline__ void tc_fence_before_sync()
{
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tc_fence_after_sync()
{
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tmem_wait_st()
{
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_wait_ld()
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// 32 lanes x 32 columns: thread i of the warp writes lane (base lane + i),
// register j goes to column (base column + j).  Whole warp, converged.
__device__ __forceinline__ void tmem_st_32x32b_x32(uint32_t taddr, const uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}

__device__ __forceinline__ void tmem_ld_32x32b_x32(uint32_t taddr, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}

// ------------------------------------------------------------------ MMA

// Shared-memory matrix descriptor for a K-major tile whose rows are 128 bytes
// (64 fp16) in the 128-byte swizzle: 8-row groups are 1024 bytes apart.
__device__ __forceinline__ uint64_t smem_desc_k_sw128(uint32_t smem_addr)
{
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr >> 4) & 0x3FFFu);        // start address, 16-byte units
    d |= (uint64_t)1 << 16;                             // leading byte offset (unused with swizzle)
    d |= (uint64_t)(1024 >> 4) << 32;                   // stride byte offset: 8 rows
    d |= (uint64_t)1 << 46;                             // descriptor version (Blackwell)
    d |= (uint64_t)2 << 61;                             // layout: 128-byte swizzle
    return d;
}

// Instruction descriptor, kind::f16: fp16 A and B (both K-major), fp32 D, M = 128.
__host__ __device__ constexpr uint32_t idesc_f16_m128(int n)
{
    return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}

// D[tmem] (+)= A[tmem] * B[smem]^T.  The MMAs and commits of the issuing warp are executed by the
// whole converged warp with only the lane `sel != 0` acting (predicated instructions instead of a
// divergent branch).
//
// All MMAs of one 64-k stage for one weight tile set (four K = 16 steps) in one block of
// instructions: the predicates are set up once, the operands of the four steps are the first
// step's plus constants (8 tensor-memory columns, 2 descriptor units per step).  `first_acc` =
// accumulate flag of the first step (false at the start of a piece of work); the others accumulate.
__device__ __forceinline__ void mma_ts_f16_stage(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, bool first_acc,
                                                 uint32_t sel)
{
    asm volatile(
        "{\n\t"
        ".reg .pred q, p0, pt;\n\t"
        ".reg .b32 a1, a2, a3;\n\t"
        ".reg .b64 b1, b2, b3;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "setp.ne.b32 p0, %4, 0;\n\t"
        "setp.eq.b32 pt, %5, %5;\n\t"
        "add.u32 a1, %1, 8;\n\t"
        "add.u32 a2, %1, 16;\n\t"
        "add.u32 a3, %1, 24;\n\t"
        "add.u64 b1, %2, 2;\n\t"
        "add.u64 b2, %2, 4;\n\t"
        "add.u64 b3, %2, 6;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [a1], b1, %3, pt;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [a2], b2, %3, pt;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [a3], b3, %3, pt;\n\t"
        "}\n"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"((uint32_t)first_acc), "r"(sel)
        : "memory");
}
// Arrive on an mbarrier once every MMA issued so far by the acting lane has finished.
__device__ __forceinline__ void mma_commit_sel(uint64_t* bar, uint32_t sel)
{
    asm volatile(
        "{\n\t"
        ".reg .pred q;\n\t"
        "setp.ne.b32 q, %1, 0;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t"
        "}\n"
        ::"r"(smem_u32(bar)), "r"(sel)
        : "memory");
}

// ------------------------------------------- bulk copies, block-scaled MMA

// Contiguous global -> shared copy of `bytes` (a multiple of 16; both addresses 16-byte aligned), completion counted
// on an mbarrier; from a converged warp, the lane with sel != 0 acting.  The operands are then warp-uniform values; a single
// lane in a divergent branch needs ~190 cycles per copy to set them up, which bounded the loading warp.
__device__ __forceinline__ void bulk_load_sel(uint32_t smem_dst, const void* src, uint32_t bytes, uint32_t bar, uint32_t sel)
{
    asm volatile(
        "{\n\t"
        ".reg .pred q;\n\t"
        "setp.ne.b32 q, %4, 0;\n\t"
        "@q cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n\t"
        "}\n"
        ::"r"(smem_dst), "l"(src), "r"(bytes), "r"(bar), "r"(sel)
        : "memory");
}
__device__ __forceinline__ void mbar_arrive_expect_tx_sel(uint32_t bar, uint32_t bytes, uint32_t sel)
{
    asm volatile(
        "{\n\t"
        ".reg .pred q;\n\t"
        "setp.ne.b32 q, %2, 0;\n\t"
        "@q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t"
        "}\n"
        ::"r"(bar), "r"(bytes), "r"(sel)
        : "memory");
}

// Shared-memory descriptor of a 512-byte scale group (32 rows of 16 bytes, not swizzled: 8-row groups 128 bytes apart).
__device__ __forceinline__ uint64_t smem_desc_scales(uint32_t smem_addr)
{
    return (uint64_t)((smem_addr >> 4) & 0x3FFFu) | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}

// Instruction descriptor of the block-scaled 4-bit MMA: e2m1 A and B (K-major), fp32 D, M = 128 (or 256 over a pair of
// SMs); scales e8m0 (one per 32 k) or e4m3 (one per 16).  Bits 4 and 29 up (the byte of the scale words that a step starts at) are 0
// here and 2 in the second step of an e8m0 group.
__host__ __device__ constexpr uint32_t idesc_fp4(bool e8m0, int m, int n)
{
    return (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((e8m0 ? 1u : 0u) << 23) | ((uint32_t)(m >> 4) << 24);
}

// The scale groups of one operand of a stage (GROUPS of 512 bytes) -> 4 columns of tensor memory each, `pitch` columns apart,
// repeated in the four lane quarters.  CG = 2: of both blocks of the pair, each from its own shared memory.  One block of instructions
// (as the MMAs below): the predicate is set up once, the operands are the first ones plus constants.
template <int CG, int GROUPS>
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint64_t desc, uint32_t pitch, uint32_t sel)
{
    static_assert(GROUPS == 2 || GROUPS == 4, "two (32 k per scale) or four (16 k per scale) groups per stage");
    if constexpr (CG == 1 && GROUPS == 2)
        asm volatile(
            "{\n\t"
            ".reg .pred q;\n\t"
            ".reg .b32 t1;\n\t"
            ".reg .b64 s1;\n\t"
            "setp.ne.b32 q, %3, 0;\n\t"
            "add.u32 t1, %0, %2;\n\t"
            "add.u64 s1, %1, 32;\n\t"
            "@q tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t"
            "@q tcgen05.cp.cta_group::1.32x128b.warpx4 [t1], s1;\n\t"
            "}\n"
            ::"r"(taddr), "l"(desc), "r"(pitch), "r"(sel)
            : "memory");
    else if constexpr (CG == 1 && GROUPS == 4)
        asm volatile(
            "{\n\t"
            ".reg .pred q;\n\t"
            ".reg .b32 t1, t2, t3;\n\t"
            ".reg .b64 s1, s2, s3;\n\t"
            "setp.ne.b32 q, %3, 0;\n\t"
            "add.u32 t1, %0, %2;\n\t"
            "add.u64 s1, %1, 32;\n\t"
            "add.u32 t2, t1, %2;\n\t"
            "add.u64 s2, %1, 64;\n\t"
            "add.u32 t3, t2, %2;\n\t"
            "add.u64 s3, %1, 96;\n\t"
            "@q tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t"
            "@q tcgen05.cp.cta_group::1.32x128b.warpx4 [t1], s1;\n\t"
            "@q tcgen05.cp.cta_group::1.32x128b.warpx4 [t2], s2;\n\t"
            "@q tcgen05.cp.cta_group::1.32x128b.warpx4 [t3], s3;\n\t"
            "}\n"
            ::"r"(taddr), "l"(desc), "r"(pitch), "r"(sel)
            : "memory");
    else if constexpr (CG == 2 && GROUPS == 2)
        asm volatile(
            "{\n\t"
            ".reg .pred q;\n\t"
            ".reg .b32 t1;\n\t"
            ".reg .b64 s1;\n\t"
            "setp.ne.b32 q, %3, 0;\n\t"
            "add.u32 t1, %0, %2;\n\t"
            "add.u64 s1, %1, 32;\n\t"
            "@q tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;\n\t"
            "@q tcgen05.cp.cta_group::2.32x128b.warpx4 [t1], s1;\n\t"
            "}\n"
            ::"r"(taddr), "l"(desc), "r"(pitch), "r"(sel)
            : "memory");
    else if constexpr (CG == 2 && GROUPS == 4)
        asm volatile(
            "{\n\t"
            ".reg .pred q;\n\t"
            ".reg .b32 t1, t2, t3;\n\t"
            ".reg .b64 s1, s2, s3;\n\t"
            "setp.ne.b32 q, %3, 0;\n\t"
            "add.u32 t1, %0, %2;\n\t"
            "add.u64 s1, %1, 32;\n\t"
            "add.u32 t2, t1, %2;\n\t"
            "add.u64 s2, %1, 64;\n\t"
            "add.u32 t3, t2, %2;\n\t"
            "add.u64 s3, %1, 96;\n\t"
            "@q tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;\n\t"
            "@q tcgen05.cp.cta_group::2.32x128b.warpx4 [t1], s1;\n\t"
            "@q tcgen05.cp.cta_group::2.32x128b.warpx4 [t2], s2;\n\t"
            "@q tcgen05.cp.cta_group::2.32x128b.warpx4 [t3], s3;\n\t"
            "}\n"
            ::"r"(taddr), "l"(desc), "r"(pitch), "r"(sel)
            : "memory");
}

// The four K = 64 steps of one stage: D[tmem] (+)= (A[smem] sa) (B[smem] sb)^T.  sa / sb: scale columns of the first group, the next
// groups' 4 / sb_pitch columns further.  Scales e8m0 (E8M0: a group serves two steps, the second starts at byte 2 of its words)
// or e4m3 (a group per step).  CG = 2: rows from both blocks of a pair.
template <int CG, bool E8M0>
__device__ __forceinline__ void mma_fp4_stage(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t sb_pitch,
                                              uint32_t acc, uint32_t sel)
{
    if constexpr (CG == 1 && E8M0)
        asm volatile(
            "{\n\t"
            ".reg .pred q, p0, pt;\n\t"
            ".reg .b32 u1, v1, i1;\n\t"
            ".reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
            "setp.ne.b32 q, %8, 0;\n\t"
            "setp.ne.b32 p0, %7, 0;\n\t"
            "setp.eq.b32 pt, %8, %8;\n\t"
            "add.u64 a1, %1, 2;\n\t"
            "add.u64 b1, %2, 2;\n\t"
            "add.u64 a2, %1, 4;\n\t"
            "add.u64 b2, %2, 4;\n\t"
            "add.u64 a3, %1, 6;\n\t"
            "add.u64 b3, %2, 6;\n\t"
            "or.b32 i1, %3, 0x40000020;\n\t"
            "add.u32 u1, %4, 4;\n\t"
            "add.u32 v1, %5, %6;\n\t"
            "@q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p0;\n\t"
            "@q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], a1, b1, i1, [%4], [%5], pt;\n\t"
            "@q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], a2, b2, %3, [u1], [v1], pt;\n\t"
            "@q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], a3, b3, i1, [u1], [v1], pt;\n\t"
            "}\n"
            ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sa), "r"(sb), "r"(sb_pitch), "r"(acc), "r"(sel)
            : "memory");
    else if constexpr (CG == 1 && !E8M0)
        asm volatile(
            "{\n\t"
            ".reg .pred q, p0, pt;\n\t"
            ".reg .b32 u1, u2, u3, v1, v2, v3;\n\t"
            ".reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
            "setp.ne.b32 q, %8, 0;\n\t"
            "setp.ne.b32 p0, %7, 0;\n\t"
            "setp.eq.b32 pt, %8, %8;\n\t"
            "add.u64 a1, %1, 2;\n\t"
            "add.u64 b1, %2, 2;\n\t"
            "add.u64 a2, %1, 4;\n\t"
            "add.u64 b2, %2, 4;\n\t"
            "add.u64 a3, %1, 6;\n\t"
            "add.u64 b3, %2, 6;\n\t"
            "add.u32 u1, %4, 4;\n\t"
            "add.u32 u2, %4, 8;\n\t"
            "add.u32 u3, %4, 12;\n\t"
            "add.u32 v1, %5, %6;\n\t"
            "add.u32 v2, v1, %6;\n\t"
            "add.u32 v3, v2, %6;\n\t"
            "@q tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p0;\n\t"
            "@q tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], a1, b1, %3, [u1], [v1], pt;\n\t"
            "@q tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], a2, b2, %3, [u2], [v2], pt;\n\t"
            "@q tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], a3, b3, %3, [u3], [v3], pt;\n\t"
            "}\n"
            ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sa), "r"(sb), "r"(sb_pitch), "r"(acc), "r"(sel)
            : "memory");
    else if constexpr (CG == 2 && E8M0)
        asm volatile(
            "{\n\t"
            ".reg .pred q, p0, pt;\n\t"
            ".reg .b32 u1, v1, i1;\n\t"
            ".reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
            "setp.ne.b32 q, %8, 0;\n\t"
            "setp.ne.b32 p0, %7, 0;\n\t"
            "setp.eq.b32 pt, %8, %8;\n\t"
            "add.u64 a1, %1, 2;\n\t"
            "add.u64 b1, %2, 2;\n\t"
            "add.u64 a2, %1, 4;\n\t"
            "add.u64 b2, %2, 4;\n\t"
            "add.u64 a3, %1, 6;\n\t"
            "add.u64 b3, %2, 6;\n\t"
            "or.b32 i1, %3, 0x40000020;\n\t"
            "add.u32 u1, %4, 4;\n\t"
            "add.u32 v1, %5, %6;\n\t"
            "@q tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p0;\n\t"
            "@q tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], a1, b1, i1, [%4], [%5], pt;\n\t"
            "@q tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], a2, b2, %3, [u1], [v1], pt;\n\t"
            "@q tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], a3, b3, i1, [u1], [v1], pt;\n\t"
            "}\n"
            ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sa), "r"(sb), "r"(sb_pitch), "r"(acc), "r"(sel)
            : "memory");
    else if constexpr (CG == 2 && !E8M0)
        asm volatile(
            "{\n\t"
            ".reg .pred q, p0, pt;\n\t"
            ".reg .b32 u1, u2, u3, v1, v2, v3;\n\t"
            ".reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
            "setp.ne.b32 q, %8, 0;\n\t"
            "setp.ne.b32 p0, %7, 0;\n\t"
            "setp.eq.b32 pt, %8, %8;\n\t"
            "add.u64 a1, %1, 2;\n\t"
            "add.u64 b1, %2, 2;\n\t"
            "add.u64 a2, %1, 4;\n\t"
            "add.u64 b2, %2, 4;\n\t"
            "add.u64 a3, %1, 6;\n\t"
            "add.u64 b3, %2, 6;\n\t"
            "add.u32 u1, %4, 4;\n\t"
            "add.u32 u2, %4, 8;\n\t"
            "add.u32 u3, %4, 12;\n\t"
            "add.u32 v1, %5, %6;\n\t"
            "add.u32 v2, v1, %6;\n\t"
            "add.u32 v3, v2, %6;\n\t"
            "@q tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p0;\n\t"
            "@q tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], a1, b1, %3, [u1], [v1], pt;\n\t"
            "@q tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], a2, b2, %3, [u2], [v2], pt;\n\t"
            "@q tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], a3, b3, %3, [u3], [v3], pt;\n\t"
            "}\n"
            ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sa), "r"(sb), "r"(sb_pitch), "r"(acc), "r"(sel)
            : "memory");
}

// ------------------------------------------- pairs of SMs (cta_group::2)

// 2-D tiled load into this block's shared memory whose completion may be counted on a barrier of either block of the pair
// (bar: a shared::cluster address).  No multicast: every block fetches its own tile.
__device__ __forceinline__ void tma_load_2d_pair(uint32_t smem_dst, const CUtensorMap* map, int x, int y, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
        ::"r"(smem_dst), "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}

// shared::cluster address of the variable at this place in block `rank`.
__device__ __forceinline__ uint32_t cluster_addr(const void* p, uint32_t rank)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    return a;
}

// Arrive on the barrier at the same place in block `rank` of the cluster.  It orders the arriving thread's tensor-memory reads
// (after tcgen05.wait::ld and the fence before a thread sync), not its global stores: a release at cluster scope
// would wait for all of those, which was measured at 2 000 cycles in an epilogue.
__device__ __forceinline__ void mbar_arrive_remote(uint64_t* bar, uint32_t rank)
{
    asm volatile(
        "{\n\t"
        ".reg .b32 a;\n\t"
        "mapa.shared::cluster.u32 a, %0, %1;\n\t"
        "mbarrier.arrive.shared::cluster.b64 _, [a];\n\t"
        "}\n"
        ::"r"(smem_u32(bar)), "r"(rank)
        : "memory");
}

__device__ __forceinline__ void tmem_alloc_pair(uint32_t* slot, uint32_t cols)
{
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc_pair(uint32_t base, uint32_t cols)
{
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols) : "memory");
}

// Arrive on the barrier at this place in both blocks once everything the acting lane has issued so far has finished.
__device__ __forceinline__ void mma_commit_pair(uint64_t* bar, uint32_t sel)
{
    asm volatile(
        "{\n\t"
        ".reg .pred q;\n\t"
        ".reg .b16 m;\n\t"
        "setp.ne.b32 q, %1, 0;\n\t"
        "mov.b16 m, 3;\n\t"
        "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], m;\n\t"
        "}\n"
        ::"r"(smem_u32(bar)), "r"(sel)
        : "memory");
}

}  // namespace tc
}  // namespace qmm
