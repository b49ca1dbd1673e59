// What the forward and backward tensor-core attention kernels share.
#pragma once

#include "gs_attn.cuh"
#include "gs_tc.cuh"

namespace gs {

// host side: whether TMA can address a tensor, and its map with boxes of `rows` positions x `values` values (32, 64 or
// 128 bytes), swizzled over their width
bool attn_tma_ok(const AttnTensor &t, int32_t dtype, int64_t batch, int64_t len, int64_t heads);
gs_status attn_tensor_map(CUtensorMap *m, const AttnTensor &t, int32_t dtype, int64_t batch, int64_t len, int64_t heads,
                          int dim, int values, int rows);

static constexpr int HALF_TILE = 128 * 128;          // bytes of one box: 128 rows of 64 16-bit values

// Work items, sorted from the longest to the shortest as far as their indexes tell.  Two ways to hand them out:
//  fixed : as many blocks as SMs; block b takes every gridDim.x-th item, in rounds of alternating direction, which evens
//          out what a block gets.  For sequences of one length, whose items' lengths follow from their indexes.
//  asked : for ragged batches.  The grid has one block per item.  A block that runs takes the item of its own index
//          and then, as long as there are any, those of blocks that have not started yet: it cancels their
//          launch (clusterlaunchcontrol) and does their work where its memory and barriers are set up already.
//          The warp that loads asks, when it has nothing left to load: an item taken earlier is one that another SM
//          could have begun (asking two items ahead took 278 instead of 128 us where 256 items meet 148 SMs).
// Measured: three sequences of up to 5003 x 64, 12 heads, forward 272 us fixed and 254 us asked; 16 heads of 8192 x 128
// 465 and 481 us; the last answer, which ends a block, costs small grids 2 to 4 us, so they are fixed.
// Every warp that works on items goes through the same sequence.
struct ItemQueue {
    uint32_t count;                                             // items; 0: asked
    uint32_t answers, full, empty;                              // shared memory: two 16-byte slots, two barriers each
    volatile int *stalled;
    __device__ __forceinline__ void init(uint32_t listeners) const          // one thread; warps other than the asking one
    {
        for (int i = 0; i < 2; ++i) {
            tc::bar_init(full + 8 * i, 1);
            tc::bar_init(empty + 8 * i, listeners);
        }
    }
    // item of answer k, or UINT32_MAX when there are no more
    __device__ __forceinline__ uint32_t answer(uint32_t k) const
    {
        if (!__all_sync(0xffffffffu, tc::bar_wait(full + 8 * (k & 1), (k >> 1) & 1, stalled))) return 0xffffffffu;
        return tc::canceled_block(answers + 16 * (k & 1));
    }
};
template <bool ASKS>
struct Items {
    const ItemQueue &q;
    uint32_t at, k;
    __device__ __forceinline__ explicit Items(const ItemQueue &queue) : q(queue), at(blockIdx.x), k(0) {}
    __device__ __forceinline__ bool more() const { return at != 0xffffffffu; }
    __device__ __forceinline__ void next()                      // a whole warp; not again after the end
    {
        if (q.count) {                                          // rounds: 0, 1, .. and .., 1, 0 in turn
            at += k & 1 ? 2 * blockIdx.x + 1 : 2 * (gridDim.x - blockIdx.x) - 1;
            if (at >= q.count) at = 0xffffffffu;
            ++k;
            return;
        }
        const bool one = (threadIdx.x & 31) == 0;
        if (ASKS) {
            const bool ok = k < 2 || __all_sync(0xffffffffu, tc::bar_wait(q.empty + 8 * (k & 1), (k / 2 - 1) & 1, q.stalled));
            if (ok && one) {
                tc::bar_expect(q.full + 8 * (k & 1), 16);
                tc::cancel_block(q.answers + 16 * (k & 1), q.full + 8 * (k & 1));
            }
            __syncwarp();
            at = ok ? q.answer(k) : 0xffffffffu;
        } else {
            at = q.answer(k);
            tc::fence_async_shared();                           // this read before the next answer is written
            __syncwarp();
            if (one) tc::bar_arrive(q.empty + 8 * (k & 1));
        }
        ++k;
    }
};
// host side: whether a launch's items are asked for
static inline bool items_asked(const AttnArgs &a, int64_t items)
{
    return (a.q_lens != nullptr || a.k_lens != nullptr) && items > sm_count();
}

// One 128-row tile of DP values into shared memory at `dst` (DP / 64 boxes)
template <int DP>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap *map, uint32_t bar, int pos, int head, int b)
{
#pragma unroll
    for (int x = 0; x < DP / 64; ++x) tc::tma_load(dst + x * HALF_TILE, map, bar, x * 64, pos, head, b);
}

// 32 columns of one row, times mul (0: zeros whatever o holds)
template <bool BF16>
__device__ __forceinline__ void store32(uint16_t *row, int c, int dim, bool vec, const float (&o)[32], float mul)
{
    uint32_t u[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) u[i] = mul != 0.f ? tc::pack2<BF16>(o[2 * i] * mul, o[2 * i + 1] * mul) : 0u;
    if (vec) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + 8 * i < dim)
                *reinterpret_cast<uint4 *>(row + c + 8 * i) = make_uint4(u[4 * i], u[4 * i + 1], u[4 * i + 2], u[4 * i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (c + i < dim) row[c + i] = (uint16_t)(i & 1 ? u[i / 2] >> 16 : u[i / 2]);
    }
}

template <bool BF16> struct Tensor16 { using T = __half; };
template <> struct Tensor16<true> { using T = __nv_bfloat16; };

// sums whose only use is that they are NaN if one of the values is
struct NanSums {
    float2 t[4] = {};
    __device__ __forceinline__ void add(const float (&o)[32])
    {
#pragma unroll
        for (int i = 0; i < 32; i += 2) t[i / 2 % 4] = tc::add2(t[i / 2 % 4], make_float2(o[i], o[i + 1]));
    }
    __device__ __forceinline__ bool found() const
    {
        const float2 s = tc::add2(tc::add2(t[0], t[1]), tc::add2(t[2], t[3]));
        return s.x + s.y != s.x + s.y;
    }
};

// rows that 16-byte stores may write
__device__ __forceinline__ bool rows16(const AttnTensor &t, int dim)
{
    return dim % 8 == 0 && (((uintptr_t)t.p | (uintptr_t)(2 * t.sb) | (uintptr_t)(2 * t.sl) | (uintptr_t)(2 * t.sh)) & 15) == 0;
}

// Rows [from, 128) of a tile that TMA has just written (bar `done`, first phase `parity`) become zeros,
// then `full` is announced in TMA's stead.  Whole warp.  For operands whose rows are summed over: what lies
// past a sequence's end must not meet a zero factor (0 * NaN).
template <int DP>
__device__ __forceinline__ bool patch_tile(uint32_t tile, int from, uint32_t done, uint32_t parity, uint32_t full,
                                           volatile int *stalled)
{
    const bool ok = __all_sync(0xffffffffu, tc::bar_wait(done, parity, stalled));
    const int lane = threadIdx.x & 31;
    for (int e = from * 8 + lane; e < 128 * 8; e += 32)
#pragma unroll
        for (int x = 0; x < DP / 64; ++x)
            asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(tile + x * HALF_TILE + e * 16), "r"(0) : "memory");
    tc::fence_async_shared();
    __syncwarp();
    if (lane == 0) tc::bar_arrive(full);
    return ok;
}

// end of a block one of whose waits ran out: loads and products in flight get a bounded time to end
// before the block's memory goes
__device__ __forceinline__ void drain_stalled(unsigned long long *stalls)
{
    if (threadIdx.x == 0) {
        for (int i = 0; i < 64; ++i) __nanosleep(100000);
        if (stalls) atomicAdd_system(stalls, 1ull);
    }
    __syncthreads();
}

}  // namespace gs
