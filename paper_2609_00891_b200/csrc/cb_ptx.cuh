// Thin wrappers over the sm_100a PTX used by the tensor-core kernels: mbarriers with bounded waits, TMA tile
// loads, tcgen05 (TMEM allocation, MMA, commit, loads) and the UMMA descriptors.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace cb {
namespace ptx {

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

// True in one lane of a converged warp, always the same one.  The compiler keeps the operands of what follows under it in
// uniform registers when they are warp-uniform; under `lane == 0` it moves them there one by one for every instruction,
// which, beside busy warps, made a tcgen05.mma take 80 cycles to issue instead of the 48 to 64 it runs for (measured).
__device__ __forceinline__ bool elect_one()
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok));
    return ok != 0;
}

// ---- mbarrier ----------------------------------------------------------------------------------------
__device__ __forceinline__ void mbar_init(uint64_t *bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_fence_init()
{
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t *bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void mbar_arrive_expect_tx(uint64_t *bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint64_t *bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t"
        "}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}

// Bounded wait.  Returns false if the limit ran out or another thread of the block already gave up
// (abort_flag[0] != 0); the caller then leaves its loop and the block tears down.  abort_flag points at two ints in
// shared memory: [0] the block's abort flag, [1] the poll limit of this launch (kPollLimitDefault unless the host set
// a shorter one), read only once the fast polls are used up.  After `fast_polls` failed polls the thread sleeps
// `sleep_ns` between polls: every poll is a shared-memory transaction, and a block full of spinning threads slows
// down the shared-memory pipe for the threads that do the work.
constexpr uint32_t kPollLimitDefault = 1u << 22;
__device__ __forceinline__ bool mbar_wait(uint64_t *bar, uint32_t parity, volatile int *abort_flag,
                                          uint32_t fast_polls = 1u << 14, uint32_t sleep_ns = 64)
{
    for (uint32_t i = 0; i < fast_polls; ++i)
        if (mbar_try_wait(bar, parity)) return true;
    const uint32_t limit = (uint32_t)abort_flag[1];
    for (uint32_t i = fast_polls; i < limit; ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((i & 63) == 0 && abort_flag[0]) return false;
        __nanosleep(sleep_ns);
    }
    abort_flag[0] = 1;
    return false;
}

// Warp-wide wait with a warp-uniform outcome.  `one_lane`: only lane 0 polls (for long, uncritical waits: fewer
// shared-memory transactions); otherwise every lane polls, which reacts fastest.  All 32 lanes must call it.
__device__ __forceinline__ bool mbar_wait_warp(uint64_t *bar, uint32_t parity, volatile int *abort_flag, int lane,
                                               bool one_lane = false, uint32_t fast_polls = 1u << 14, uint32_t sleep_ns = 64)
{
    if (one_lane) {
        int ok = 1;
        if (lane == 0) ok = mbar_wait(bar, parity, abort_flag, fast_polls, sleep_ns) ? 1 : 0;
        return __shfl_sync(0xffffffffu, ok, 0) != 0;
    }
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, fast_polls, sleep_ns)) != 0;
}

// The same bounded wait for kernels whose waiting warps share a scheduler with warps that compute: the thread is suspended
// in the barrier unit, for 4 us a poll as measured (whatever longer time the hint names), instead of polling (a spinning
// warp takes issue slots: measured, the exponentials of an attention tile took 1,300 cycles beside a spinning warp and 600
// without one).  abort_flag as above; the limit counts in units of four polls: 2^20 of them, four seconds.
__device__ __forceinline__ bool mbar_poll_suspended(uint64_t *bar, uint32_t parity, volatile int *abort_flag)
{
    const uint32_t limit = 1u + ((uint32_t)abort_flag[1] >> 2);
    for (uint32_t i = 0; i < limit; ++i) {
        uint32_t ok;
        asm volatile(
            "{\n\t"
            ".reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t"
            "}"
            : "=r"(ok)
            : "r"(smem_u32(bar)), "r"(parity), "r"(1000000u)
            : "memory");
        if (ok) return true;
        if (abort_flag[0]) return false;
    }
    return false;
}
__device__ __forceinline__ bool mbar_wait_suspended(uint64_t *bar, uint32_t parity, volatile int *abort_flag)
{
    if (mbar_try_wait(bar, parity) || mbar_poll_suspended(bar, parity, abort_flag)) return true;
    abort_flag[0] = 1;
    return false;
}
// For a wait that lasts as long as others' work on many tiles: it runs out only when `moves`, which a warp of the block
// counts up with that work, has stood still for as long as the limit.
__device__ __forceinline__ bool mbar_wait_while_moving(uint64_t *bar, uint32_t parity, volatile int *abort_flag, volatile int *moves)
{
    if (mbar_try_wait(bar, parity)) return true;
    int seen, now = *moves;
    do {
        seen = now;
        if (mbar_poll_suspended(bar, parity, abort_flag)) return true;
        now = *moves;
    } while (now != seen && abort_flag[0] == 0);
    abort_flag[0] = 1;
    return false;
}
__device__ __forceinline__ bool mbar_wait_while_moving_warp(uint64_t *bar, uint32_t parity, volatile int *abort_flag, volatile int *moves)
{
    return __all_sync(0xffffffffu, mbar_wait_while_moving(bar, parity, abort_flag, moves)) != 0;
}
// Warp-wide, with a warp-uniform outcome; all 32 lanes must call it.
__device__ __forceinline__ bool mbar_wait_suspended_warp(uint64_t *bar, uint32_t parity, volatile int *abort_flag)
{
    return __all_sync(0xffffffffu, mbar_wait_suspended(bar, parity, abort_flag)) != 0;
}

// For a warp that issues copies, before it fills a stage again: the same wait, and false as well once any warp of the block
// has given up.  A warp that gave up releases stages whose copy it has not seen land; it sets the flag before that arrival,
// so the flag is seen here and no copy goes to such a stage.
__device__ __forceinline__ bool mbar_wait_to_issue_warp(uint64_t *bar, uint32_t parity, volatile int *abort_flag)
{
    return __all_sync(0xffffffffu, mbar_wait_suspended(bar, parity, abort_flag) && abort_flag[0] == 0) != 0;
}
// After a time-out: waits for a copy or a product in flight whatever the abort flag says (2^20 polls, a quarter of a second
// or more; those take microseconds).
__device__ __forceinline__ void mbar_drain(uint64_t *bar, uint32_t parity)
{
    for (uint32_t i = 0; i < (1u << 20) && !mbar_try_wait(bar, parity); ++i) __nanosleep(256);
}

// Make this thread's generic-proxy writes to shared memory visible to the async proxy (TMA, tensor cores).
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- TMA ---------------------------------------------------------------------------------------------
__device__ __forceinline__ void tma_load_4d(void *dst, const CUtensorMap *map, uint64_t *bar, int c0, int c1, int c2, int c3)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(smem_u32(dst)), "l"(map), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
        : "memory");
}
// One copy brings [c_hi][tokens][64 channels] (dims: c_lo, token, c_hi, head, layer).
__device__ __forceinline__ void tma_load_5d(void *dst, const CUtensorMap *map, uint64_t *bar, int c0, int c1, int c2, int c3, int c4)
{
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
        ::"r"(smem_u32(dst)), "l"(map), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4)
        : "memory");
}
// Plain bulk copy global -> shared (both 16-byte aligned, size a multiple of 16) that completes on an mbarrier.
__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes, uint64_t *bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}
// Store a shared-memory tile [c_hi][tokens][64 channels] to global memory (rows past the tensor's end are clipped).
__device__ __forceinline__ void tma_store_5d(const CUtensorMap *map, const void *src, int c0, int c1, int c2, int c3, int c4)
{
    asm volatile("cp.async.bulk.tensor.5d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4, %5, %6}], [%1];"
                 ::"l"(map), "r"(smem_u32(src)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4) : "memory");
}
__device__ __forceinline__ void tma_store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// All of this thread's committed stores have finished READING shared memory (the buffer may be rewritten).
__device__ __forceinline__ void tma_store_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
// All but the N most recent committed store groups have finished reading shared memory.
template <int N>
__device__ __forceinline__ void tma_store_wait_read_keep() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }
// All of this thread's committed stores are complete.
__device__ __forceinline__ void tma_store_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void tma_prefetch_desc(const CUtensorMap *map)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// ---- asynchronous 4-byte copies (any alignment, zero fill when src_bytes == 0) --------------------------
__device__ __forceinline__ void cp_async_4(void *dst_smem, const void *src, uint32_t src_bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(dst_smem)), "l"(src), "r"(src_bytes) : "memory");
}
// The barrier receives one arrival from this thread once all its earlier asynchronous copies have landed; the
// arrival must be part of the barrier's expected count.
__device__ __forceinline__ void cp_async_arrive_noinc(uint64_t *bar)
{
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// ---- tcgen05 -----------------------------------------------------------------------------------------
__device__ __forceinline__ void tmem_alloc(uint32_t *dst_smem, uint32_t ncols)   // whole warp
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(dst_smem)), "r"(ncols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc(uint32_t taddr, uint32_t ncols)     // whole warp
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// D[tmem] (+)= A[smem] * B[smem], bf16 inputs, fp32 accumulation; one thread issues.
__device__ __forceinline__ void umma_bf16_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t"
        "}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem]: the first operand is read from tensor memory (lane = row of A, two bf16 of
// consecutive K per 32-bit column: K = 16 takes 8 columns), K-major by construction.
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t"
        "}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Arrive on an mbarrier once all tcgen05 operations issued so far by this thread have completed.
__device__ __forceinline__ void umma_commit(uint64_t *bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// 32 lanes x 32 consecutive columns of 32-bit data: thread i of the warp gets lane (base lane + i).
__device__ __forceinline__ void tmem_ld_32x32(uint32_t taddr, uint32_t (&r)[32])
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
__device__ __forceinline__ void tmem_ld_32x16(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Store 16 lanes x 16 columns: thread i holds, for n = 0..3, register 2n = (lane i/4, column 4n + i%4) and register
// 2n+1 = (lane i/4 + 8, column 4n + i%4): the register layout that ldmatrix (8x8, 16-bit, transposed) produces.
__device__ __forceinline__ void tmem_st_16x128_x4(uint32_t taddr, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
// 32 lanes x 16 consecutive columns of 32-bit data from registers (thread i writes lane base + i).
__device__ __forceinline__ void tmem_st_32x16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr),
          "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Four 8x8 matrices of 16-bit elements, transposed: thread i supplies the address of row i%8 of matrix i/8 and
// receives in register j the elements (row 2(i%4), column i/4) [low half] and (row 2(i%4)+1, column i/4) of matrix j.
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t smem_addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(smem_addr) : "memory");
}

// Four fp32 added to 16-byte aligned global memory, no value returned.
__device__ __forceinline__ void red_add_f32x4(float *dst, float a, float b, float c, float d)
{
    asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(dst), "f"(a), "f"(b), "f"(c), "f"(d) : "memory");
}

// ---- descriptors -------------------------------------------------------------------------------------
// Shared-memory operand descriptor, 128-byte swizzle.  For an MN-major operand (the contraction index is the
// row of the tile in shared memory, 64 channels = 128 bytes per row): `lbo_bytes` is the distance between
// consecutive 64-channel blocks, `sbo_bytes` the distance between consecutive groups of 8 rows.
// For a K-major operand `sbo_bytes` is the distance between groups of 8 rows of M/N and lbo is unused.
__device__ __forceinline__ uint64_t umma_smem_desc_sw128(uint32_t smem_addr, uint32_t lbo_bytes, uint32_t sbo_bytes)
{
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr & 0x3FFFFu) >> 4);
    d |= (uint64_t)((lbo_bytes >> 4) & 0x3FFFu) << 16;
    d |= (uint64_t)((sbo_bytes >> 4) & 0x3FFFu) << 32;
    d |= (uint64_t)1 << 46;   // descriptor version for sm_100
    d |= (uint64_t)2 << 61;   // 128-byte swizzle
    return d;
}

// Instruction descriptor for kind::f16 with bf16 operands and fp32 accumulation.
__host__ __device__ constexpr uint32_t umma_idesc_bf16(int M, int N, bool a_mn_major, bool b_mn_major)
{
    return (1u << 4)                         // accumulator format: fp32
           | (1u << 7)                       // A: bf16
           | (1u << 10)                      // B: bf16
           | ((a_mn_major ? 1u : 0u) << 15)  // A major
           | ((b_mn_major ? 1u : 0u) << 16)  // B major
           | ((uint32_t)(N >> 3) << 17)
           | ((uint32_t)(M >> 4) << 24);
}

// The same with fp16 operands (format code 0 for A and B).
__host__ __device__ constexpr uint32_t umma_idesc_f16(int M, int N, bool a_mn_major, bool b_mn_major)
{
    return (1u << 4)                         // accumulator format: fp32
           | ((a_mn_major ? 1u : 0u) << 15)  // A major
           | ((b_mn_major ? 1u : 0u) << 16)  // B major
           | ((uint32_t)(N >> 3) << 17)
           | ((uint32_t)(M >> 4) << 24);
}

}  // namespace ptx
}  // namespace cb
