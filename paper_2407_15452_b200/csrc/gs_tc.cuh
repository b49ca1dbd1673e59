// The Blackwell instructions that the tensor-core attention kernels use, one thin wrapper each:
// mbarriers with bounded waits, TMA tile loads, tensor memory and tcgen05.mma.
//
// Waits are bounded.  A kernel whose wait runs out (which no finite input should cause) sets a flag in
// shared memory that ends every other wait of its block, drains what it has in flight, frees its
// tensor memory and adds one to the count that the next call finds and gs_stalled_kernels reads.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gs_common.cuh"

namespace gs {
namespace tc {

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

// ---- mbarriers ----------------------------------------------------------------------
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}

// In units of 2^32 cycles, about two seconds each: the upper half of the clock is all that a wait looks at, since the code
// of the waits is a good part of these kernels' and shows where items are short.  About twenty seconds: a warp that does
// rows again (gs_attn_again.cuh) keeps the others of its block waiting, and 32 keys of 8 query heads of 240000 positions
// take that long, one after the other.
static constexpr uint32_t WAIT_LIMIT = 9;
__device__ __forceinline__ uint32_t clock_upper()
{
    uint32_t t;
    asm volatile("mov.u32 %0, %%clock_hi;" : "=r"(t));
    return t;
}

// true once the barrier's phase has completed; false if the wait ran out here or elsewhere in the block
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *stalled, uint32_t limit = WAIT_LIMIT)
{
    if (bar_try(bar, parity)) return true;
    const uint32_t t0 = clock_upper();
    while (!bar_try(bar, parity)) {
        if (clock_upper() - t0 > limit) *stalled = 1;
        if (*stalled) return false;
    }
    return true;
}

__device__ __forceinline__ void fence_barrier_init() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
// orders this thread's shared-memory writes before later reads by TMA and tcgen05
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- TMA ------------------------------------------------------------------------------
__device__ __forceinline__ void tma_prefetch(const CUtensorMap *map)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
// one box of a [batch][head][position][dim] view; x must be a multiple of 8 (16 bytes)
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int pos, int head, int b)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
                 " [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(pos), "r"(head), "r"(b) : "memory");
}

// a box from shared memory; what lies outside the tensor is not written
__device__ __forceinline__ void tma_store(const CUtensorMap *map, uint32_t src, int x, int pos, int head, int b)
{
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4, %5}], [%1];"
                 ::"l"(map), "r"(src), "r"(x), "r"(pos), "r"(head), "r"(b) : "memory");
}
__device__ __forceinline__ void tma_store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// this thread's stores have read their shared memory
__device__ __forceinline__ void tma_stores_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
// ... and have been written
__device__ __forceinline__ void tma_stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// ---- work of blocks that have not started -----------------------------------------------------
// asks for the cancellation of one block's launch; the 16-byte answer arrives at `answer` and counts 16 bytes on `bar`
__device__ __forceinline__ void cancel_block(uint32_t answer, uint32_t bar)
{
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];"
                 ::"r"(answer), "r"(bar) : "memory");
}
// index of the block that an answer gives, UINT32_MAX if none is left
__device__ __forceinline__ uint32_t canceled_block(uint32_t answer)
{
    uint32_t x;
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b128 h;\n\t.reg .b32 c;\n\t"
                 "ld.shared.b128 h, [%1];\n\t"
                 "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n\t"
                 "mov.b32 %0, 0xffffffff;\n\t"
                 "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 c, h;\n\t"
                 "@p mov.b32 %0, c;\n\t}"
                 : "=r"(x) : "r"(answer) : "memory");
    return x;
}

// ---- tensor memory ----------------------------------------------------------------------
__device__ __forceinline__ void tmem_alloc(uint32_t where, uint32_t columns)       // whole warp
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t columns)          // the same warp
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

#define GS_R8(a, o) "=r"(a[o]), "=r"(a[o + 1]), "=r"(a[o + 2]), "=r"(a[o + 3]), "=r"(a[o + 4]), "=r"(a[o + 5]), "=r"(a[o + 6]), "=r"(a[o + 7])
#define GS_I8(a, o) "r"(a[o]), "r"(a[o + 1]), "r"(a[o + 2]), "r"(a[o + 3]), "r"(a[o + 4]), "r"(a[o + 5]), "r"(a[o + 6]), "r"(a[o + 7])

// 32 consecutive columns of this thread's lane (warp w of four reads lanes 32w..32w+31)
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t *r)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : GS_R8(r, 0), GS_R8(r, 8), GS_R8(r, 16), GS_R8(r, 24) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t *r)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : GS_R8(r, 0), GS_R8(r, 8) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
                 ::GS_I8(r, 0), GS_I8(r, 8), GS_I8(r, 16), GS_I8(r, 24), "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
                 ::GS_I8(r, 0), GS_I8(r, 8), "r"(addr) : "memory");
}

// one lane of the warp, the same each time.  The warp that issues products runs its loop whole and lets this lane
// issue: everything that an instruction is given is then known to be the same in all lanes and stays in uniform
// registers.  With one lane alone in the loop each tcgen05.mma cost about 120 cycles to set up, twice what it runs.
__device__ __forceinline__ bool elect_one()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}

// ---- tcgen05.mma, 16-bit operands, fp32 accumulators, one CTA, M = 128 -------------------------
// Operand tiles sit in shared memory as the 128-byte-swizzled boxes that TMA writes: [rows][64 values],
// rows 128 bytes apart, groups of eight rows 1024 bytes apart.
//  along the rows' values (row . row products): a step of 16 values is 32 bytes further
//  along the rows (the product sums over rows, values are the other extent): a step of 16 rows is 2048
//  bytes further, the next 64 values sit `half` bytes further
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t leading, uint32_t stride)
{
    return (uint64_t)((addr >> 4) & 0x3FFF) | ((uint64_t)((leading >> 4) & 0x3FFF) << 16) |
           ((uint64_t)((stride >> 4) & 0x3FFF) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ uint64_t desc_values(uint32_t addr) { return smem_desc(addr, 16, 1024); }
__device__ __forceinline__ uint64_t desc_rows(uint32_t addr, uint32_t half) { return smem_desc(addr, half, 1024); }
// the same, `bytes` further (tiles lie below 256 KB, so the address field does not carry)
__device__ __forceinline__ constexpr uint64_t desc_step(uint32_t bytes) { return bytes >> 4; }

// instruction descriptor: fp32 result, both operands bf16 or both f16; b_rows: B sums over its rows
__host__ __device__ constexpr uint32_t mma_desc(bool bf16, int m, int n, bool b_rows)
{
    return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((b_rows ? 1u : 0u) << 16) |
           ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
// A from tensor memory: row = lane, two 16-bit values per column
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
// the barrier completes once every mma issued by this thread so far has finished
__device__ __forceinline__ void mma_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// ---- packed fp32 arithmetic and conversions ---------------------------------------------------------
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(*reinterpret_cast<uint64_t *>(&d))
        : "l"(*reinterpret_cast<uint64_t *>(&a)), "l"(*reinterpret_cast<uint64_t *>(&b)), "l"(*reinterpret_cast<uint64_t *>(&c)));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("add.rn.f32x2 %0, %1, %2;"
        : "=l"(*reinterpret_cast<uint64_t *>(&d))
        : "l"(*reinterpret_cast<uint64_t *>(&a)), "l"(*reinterpret_cast<uint64_t *>(&b)));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 d;
    asm("mul.rn.f32x2 %0, %1, %2;"
        : "=l"(*reinterpret_cast<uint64_t *>(&d))
        : "l"(*reinterpret_cast<uint64_t *>(&a)), "l"(*reinterpret_cast<uint64_t *>(&b)));
    return d;
}
// The unit's own approximations of 2^x, log2 x and 1 / x, one instruction each, with relative errors of about 2^-22, 2^-22
// (absolute, near 1) and 2^-23: as much as the products in front of them are off by, where a correctly rounded exponential
// would be a third of these kernels' instructions.
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float log2_fast(float x)
{
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp_fast(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// fp32 on the tensor cores: x = hi + lo, hi rounded to the 11 significant bits that tf32 keeps and lo what is left (exact;
// its own last bits beyond 11 are dropped), and x y = hi hi + hi lo + lo hi with a relative error below 2^-21.  Chosen
// for speed: multiply-adds in fp32 on the CUDA cores are half as fast at length (16 heads of 4096 x 64 forward 2111 us
// against 1381), and a sum over 64 columns is off by about as much in either; the error of the results is 1 to 3
// times theirs (root mean square, of the results' own; tensor cores | everything in fp32): 512 x 2 heads of 10 x 32 output 2.3e-7 |
// 1.5e-7, 200 heads of 128 x 64 6.5e-7 | 3.9e-7 and dq 8.8e-7 | 4.0e-7, 16 heads of 2048 x 64 8.2e-7 | 9.4e-7 and 1.1e-6 | 9.6e-7.
__device__ __forceinline__ void split(float x, uint32_t &hi, uint32_t &lo)
{
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(hi) : "f"(x));
    lo = __float_as_uint(x - __uint_as_float(hi));
}
// over the four lanes that share a row of an mma.sync accumulator
__device__ __forceinline__ float quad_max(float v)
{
    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
    return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
}
__device__ __forceinline__ float quad_sum(float v)
{
    v += __shfl_xor_sync(0xffffffffu, v, 1);
    return v + __shfl_xor_sync(0xffffffffu, v, 2);
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    uint32_t u;
    if constexpr (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(hi), "f"(lo));
    return u;
}

}  // namespace tc
}  // namespace gs
