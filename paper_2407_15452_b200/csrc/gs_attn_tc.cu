// Forward attention of 16-bit tensors on the fifth-generation tensor cores.
//
// One block owns 256 query rows of a head as two tiles of 128 and walks the key tiles (128 keys)
// that any of them sees.  Roles:
//   warps 0-3, 4-7  softmax of tile 0 and tile 1: thread = row.  Scores come from tensor memory,
//                   probabilities go back there as 16-bit values over the scores they came from
//   warp 8          one thread issues the tcgen05.mma: S_t = Q_t K^T (both from shared memory) and
//                   O_t += P_t V (P from tensor memory)
//   warp 9          TMA loads of Q and of the ring of K and V tiles
// While one tile's warps exponentiate, the tensor core works on the other tile.  Tensor memory: S_0,
// S_1, O_0, O_1 of 128 columns.  The order of one thread's tcgen05.mma is kept, so S_t of the next
// keys, issued behind P_t V, may overwrite P_t without another barrier; and the barrier that
// announces it also says that O_t is at rest, which is when its owner may rescale it.
//
// The running maximum moves only when the new one is above it by more than 8 (a factor 256 in p):
// most tiles then leave O and the sum alone, exact in any case because the quotient O / sum uses one base.
// p is rounded to the tensors' type for the product with V; the sum takes it in fp32.
#include "gs_attn_tc.cuh"

namespace gs {

using namespace tc;

static constexpr int ROWS = 256, KEYS = 128;

template <int DP>
struct FwdSmem {
    static constexpr int TILE = 128 * DP * 2;                   // bytes of one 128-row tile
    static constexpr int SLOTS = DP == 128 ? 4 : 8;
    static constexpr int Q = 0, RING = 2 * TILE, BARS = RING + SLOTS * TILE;
    static constexpr int BYTES = BARS + 256 + 1024;             // 1024: alignment of the tiles
};

struct TcMaps {
    CUtensorMap q, k, v;
};

template <bool BF16, int DP>
__global__ void __launch_bounds__(384, 1)
attn_tc_forward_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ TcMaps maps, unsigned long long *stalls)
{
    using L = FwdSmem<DP>;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    __shared__ volatile int stalled;
    __shared__ uint32_t tmem_base;
    const uint32_t bars = base + L::BARS;
    const uint32_t q_full = bars, fix = bars + 8, s_full = bars + 16, p_full = bars + 32, o_full = bars + 48,
                   kv_full = bars + 64, kv_empty = bars + 64 + 8 * L::SLOTS;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    const int64_t heads = a.batch * a.q_heads;
    const int tiles = (a.q_len + ROWS - 1) / ROWS;
    const int tile = tiles - 1 - (int)(blockIdx.x / heads);
    const int64_t bh = blockIdx.x % heads, b = bh / a.q_heads;
    const int h = (int)(bh % a.q_heads), g = h / a.group;
    const AttnSeq s = attn_seq(a, b);
    const int r0 = tile * ROWS;

    // key tiles [first[t], last[t]) of the two row tiles
    int first[2], last[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int rt = r0 + 128 * t, re = min(rt + 128, s.nq);
        first[t] = last[t] = 0;
        if (rt < re) {
            const int lo = attn_lo(a, s, rt), hi = attn_hi(a, s, re - 1);
            if (lo < hi) {
                first[t] = lo / KEYS;
                last[t] = (hi + KEYS - 1) / KEYS;
            }
        }
    }
    const bool any0 = first[0] < last[0], any1 = first[1] < last[1];
    const int it0 = any0 ? (any1 ? min(first[0], first[1]) : first[0]) : first[1];
    const int it1 = any0 ? (any1 ? max(last[0], last[1]) : last[0]) : last[1];

    if (threadIdx.x == 0) {
        stalled = 0;
        bar_init(q_full, 1);
        bar_init(fix, 1);
        for (int t = 0; t < 2; ++t) {
            bar_init(s_full + 8 * t, 1);
            bar_init(p_full + 8 * t, 128);
            bar_init(o_full + 8 * t, 1);
        }
        for (int i = 0; i < L::SLOTS; ++i) {
            bar_init(kv_full + 8 * i, 1);
            bar_init(kv_empty + 8 * i, 1);
        }
        fence_barrier_init();
    }
    if (warp == 8) tmem_alloc(smem_u32(&tmem_base), 512);
    if (warp == 9 && lane == 0) {
        tma_prefetch(&maps.q);
        tma_prefetch(&maps.k);
        tma_prefetch(&maps.v);
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = tmem_base;

    // 384 threads start with 168 registers each; the softmax warps hold a row of scores:
    // 256 x 224 + 128 x 56 = 384 x 168
    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == 9) {
            // ---- loads: Q, then K and V of every key tile through the ring
            if (it0 < it1) {
                if (lane == 0) {
                    bar_expect(q_full, 2 * L::TILE);
                    load_tile<DP>(base + L::Q, &maps.q, q_full, r0, h, (int)b);
                    load_tile<DP>(base + L::Q + L::TILE, &maps.q, q_full, r0 + 128, h, (int)b);
                }
                int n = 0;
                bool ok = true;
                for (int it = it0; it < it1 && ok; ++it) {
                    for (int kv = 0; kv < 2 && ok; ++kv, ++n) {
                        const int slot = n % L::SLOTS, round = n / L::SLOTS;
                        if (round > 0) ok = __all_sync(0xffffffffu, bar_wait(kv_empty + 8 * slot, (round - 1) & 1, &stalled));
                        if (!ok) break;
                        const uint32_t dst = base + L::RING + slot * L::TILE, full = kv_full + 8 * slot;
                        // values past the sequence's end (not past the tensor's, which TMA fills with zeros)
                        // must not meet a zero probability: 0 * NaN.  They are overwritten with zeros.
                        const bool patch = kv == 1 && s.nk < a.k_len && (it + 1) * KEYS > s.nk;
                        if (lane == 0) {
                            bar_expect(patch ? fix : full, L::TILE);
                            load_tile<DP>(dst, kv ? &maps.v : &maps.k, patch ? fix : full, it * KEYS, g, (int)b);
                        }
                            // only ever the last tile: `fix` is used once
                        if (patch) ok = patch_tile<DP>(dst, s.nk - it * KEYS, fix, 0, full, &stalled);
                    }
                }
            }
        } else if (warp == 8) {
            // ---- products
            if (lane == 0 && it0 < it1) {
                constexpr uint32_t DESC_S = mma_desc(BF16, 128, KEYS, false), DESC_O = mma_desc(BF16, 128, DP, true);
                bool ok = bar_wait(q_full, 0, &stalled);
                int n = 0;                                        // ring position of K of step it; V of it - 1 is n - 1
                uint32_t p_phase[2] = {0, 0};
                for (int it = it0; it <= it1 && ok; ++it, n += 2) {
                    const int ks = n % L::SLOTS, vs = (n + L::SLOTS - 1) % L::SLOTS;
                    const bool have_k = it < it1, have_v = it > it0;
                    if (have_v) ok = ok && bar_wait(kv_full + 8 * vs, ((n - 1) / L::SLOTS) & 1, &stalled);
                    if (have_k) ok = ok && bar_wait(kv_full + 8 * ks, (n / L::SLOTS) & 1, &stalled);
                    if (!ok) break;
                    fence_after();
                    const uint32_t kt = base + L::RING + ks * L::TILE, vt = base + L::RING + vs * L::TILE;
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        if (it - 1 >= first[t] && it - 1 < last[t]) {
                            ok = ok && bar_wait(p_full + 8 * t, p_phase[t], &stalled);
                            if (!ok) break;
                            p_phase[t] ^= 1;
                            fence_after();
#pragma unroll
                            for (int k = 0; k < KEYS / 16; ++k)
                                mma_ts(tmem + 256 + 128 * t, tmem + 128 * t + 8 * k, desc_rows(vt + 2048 * k, HALF_TILE), DESC_O,
                                       it - 1 > first[t] || k > 0);
                            if (it == last[t]) mma_commit(o_full + 8 * t);
                        }
                        if (it >= first[t] && it < last[t]) {
#pragma unroll
                            for (int k = 0; k < DP / 16; ++k) {
                                const uint32_t at = (k / 4) * HALF_TILE + (k % 4) * 32;
                                mma_ss(tmem + 128 * t, desc_values(base + L::Q + t * L::TILE + at), desc_values(kt + at), DESC_S, k > 0);
                            }
                            mma_commit(s_full + 8 * t);
                        }
                    }
                    if (!ok) break;
                    if (have_v) mma_commit(kv_empty + 8 * vs);
                    if (have_k) mma_commit(kv_empty + 8 * ks);
                }
            }
            __syncwarp();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        // ---- softmax of one row
        const int t = warp >> 2;
        const int r = r0 + 128 * t + (threadIdx.x & 127);
        const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
        const uint32_t ts = tmem + lanes + 128 * t, to = tmem + lanes + 256 + 128 * t;
        const float mul = a.scale * LOG2E;                      // exponents are taken in base 2
        const bool row = r < s.nq;
        const int lo = row ? attn_lo(a, s, r) : 0, hi = row ? attn_hi(a, s, r) : s.nk;
        // tiles that every row of this tile sees whole need no mask
        const int whole_lo = attn_lo(a, s, min(r0 + 128 * t + 127, max(s.nq - 1, 0))), whole_hi = attn_hi(a, s, r0 + 128 * t);
        float top = -INFINITY, sum = 0.f;                         // top: base of the exponents, in units of log2
        bool ok = true;
        uint32_t phase = 0;
        const int it_first = t == 0 ? first[0] : first[1], it_last = t == 0 ? last[0] : last[1];
        for (int it = it_first; it < it_last; ++it) {
            ok = __all_sync(0xffffffffu, bar_wait(s_full + 8 * t, phase, &stalled));
            if (!ok) break;
            phase ^= 1;
            fence_after();
            float x[KEYS];
#pragma unroll
            for (int c = 0; c < KEYS; c += 32) tmem_ld32(ts + c, reinterpret_cast<uint32_t *>(x) + c);
            wait_ld();
            if (it * KEYS < whole_lo || (it + 1) * KEYS > whole_hi) {
                const int c0 = lo - it * KEYS, c1 = hi - it * KEYS;
#pragma unroll
                for (int c = 0; c < KEYS; ++c) x[c] = c >= c0 && c < c1 ? x[c] : -INFINITY;
            }
            float m4[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
            for (int c = 4; c < KEYS; c += 4)
#pragma unroll
                for (int i = 0; i < 4; ++i) m4[i] = fmaxf(m4[i], x[c + i]);
            const float m = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * mul;
            const bool move = m > top + 8.f;                      // also from -inf
            if (__any_sync(0xffffffffu, move)) {
                const float to_top = move ? m : top;
                const float keep = move ? exp2_fast(top - to_top) : 1.f;
                top = to_top;
                sum *= keep;
                if (it > it_first) {
#pragma unroll
                    for (int c = 0; c < DP; c += 16) {
                        float o[16];
                        tmem_ld16(to + c, reinterpret_cast<uint32_t *>(o));
                        wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] *= keep;
                        tmem_st16(to + c, reinterpret_cast<uint32_t *>(o));
                    }
                }
            }
            const float2 mul2v = make_float2(mul, mul);
            const float sub = top == -INFINITY ? 0.f : -top;      // nothing visible yet: every p is exp2(-inf) = 0
            const float2 sub2 = make_float2(sub, sub);
            float2 acc[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
            for (int c = 0; c < KEYS; c += 32) {
                uint32_t p[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float2 e = fma2(make_float2(x[c + 2 * i], x[c + 2 * i + 1]), mul2v, sub2);
                    e.x = exp2_fast(e.x);
                    e.y = exp2_fast(e.y);
                    acc[i & 1] = add2(acc[i & 1], e);
                    p[i] = pack2<BF16>(e.x, e.y);
                }
                tmem_st16(ts + c / 2, p);
            }
            wait_st();
            fence_before();
            bar_arrive(p_full + 8 * t);
            const float2 part = add2(acc[0], acc[1]);
            sum += part.x + part.y;
        }
        const bool some = it_first < it_last;
        if (ok && some) ok = __all_sync(0xffffffffu, bar_wait(o_full + 8 * t, 0, &stalled));
        fence_after();
        const float inv = row && some && sum != 0.f ? 1.f / sum : 0.f;
        if (r < a.q_len) a.lse[bh * a.q_len + r] = inv != 0.f ? (top + log2f(sum)) * LN2 : -INFINITY;
        uint16_t *out = reinterpret_cast<uint16_t *>(a.out.p) + b * a.out.sb + (int64_t)r * a.out.sl + h * a.out.sh;
        const bool vec = rows16(a.out, a.dim);
#pragma unroll
        for (int c = 0; c < DP; c += 32) {
            float o[32];
            __syncwarp();
            if (some && ok) {
                tmem_ld32(to + c, reinterpret_cast<uint32_t *>(o));
                wait_ld();
            }
            if (r < a.q_len) store32<BF16>(out, c, a.dim, vec, o, inv);
        }
    }

    fence_before();
    __syncthreads();
    fence_after();
    if (stalled) drain_stalled(stalls);
    if (warp == 8) tmem_free(tmem, 512);
}

// ---- tensor maps -----------------------------------------------------------------------------------
typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeTiled encoder()
{
    static EncodeTiled fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            p = nullptr;
        return (EncodeTiled)p;
    }();
    return fn;
}

bool attn_tma_ok(const AttnTensor &t, int64_t batch, int64_t len, int64_t heads)
{
    auto stride_ok = [](int64_t extent, int64_t s) {
        return extent <= 1 || (s > 0 && s % 8 == 0 && s < ((int64_t)1 << 38));
    };
    return (uintptr_t)t.p % 16 == 0 && stride_ok(batch, t.sb) && stride_ok(len, t.sl) && stride_ok(heads, t.sh);
}

gs_status attn_tensor_map(CUtensorMap *m, const AttnTensor &t, bool bf16, int64_t batch, int64_t len, int64_t heads,
                          int dim, int values, int rows)
{
    EncodeTiled fn = encoder();
    if (!fn) {
        set_error("cuTensorMapEncodeTiled is not available from this driver");
        return GS_ERR_CUDA;
    }
    const cuuint64_t extent[4] = {(cuuint64_t)dim, (cuuint64_t)len, (cuuint64_t)heads, (cuuint64_t)batch};
    const cuuint64_t stride[3] = {(cuuint64_t)(len > 1 ? 2 * t.sl : 256), (cuuint64_t)(heads > 1 ? 2 * t.sh : 256),
                                  (cuuint64_t)(batch > 1 ? 2 * t.sb : 256)};
    const cuuint32_t box[4] = {(cuuint32_t)values, (cuuint32_t)rows, 1, 1}, step[4] = {1, 1, 1, 1};
    const CUresult r = fn(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, t.p, extent, stride,
                          box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          values == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : values == 32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        set_error("cuTensorMapEncodeTiled failed with %d", (int)r);
        return GS_ERR_CUDA;
    }
    return GS_OK;
}

template <bool BF16, int DP>
static gs_status forward_t(const AttnArgs &a, const TcMaps &maps, cudaStream_t st)
{
    const int64_t blocks = a.batch * a.q_heads * ((a.q_len + ROWS - 1) / ROWS);
    if (blocks > 0x7FFFFFFF) {
        set_error("attention of %lld row tiles exceeds one launch", (long long)blocks);
        return GS_ERR_UNSUPPORTED;
    }
    auto kernel = attn_tc_forward_kernel<BF16, DP>;
    static SharedRecord record;
    gs_status s = allow_shared(kernel, FwdSmem<DP>::BYTES, record);
    if (s != GS_OK) return s;
    kernel<<<(unsigned)blocks, 384, FwdSmem<DP>::BYTES, st>>>(a, maps, stall_counter());
    GS_CUDA_TRY(cudaGetLastError());
    return GS_OK;
}

bool attn_tc_forward_ok(const AttnArgs &a)
{
    return a.dtype != GS_TABLE_F32 && a.batch < ((int64_t)1 << 31) && attn_tma_ok(a.q, a.batch, a.q_len, a.q_heads) &&
           attn_tma_ok(a.k, a.batch, a.k_len, a.kv_heads) && attn_tma_ok(a.v, a.batch, a.k_len, a.kv_heads);
}

gs_status attn_tc_forward(const AttnArgs &a, cudaStream_t st)
{
    const bool bf16 = a.dtype == GS_TABLE_BF16;
    TcMaps m;
    gs_status s;
    if ((s = attn_tensor_map(&m.q, a.q, bf16, a.batch, a.q_len, a.q_heads, a.dim, 64, 128)) != GS_OK) return s;
    if ((s = attn_tensor_map(&m.k, a.k, bf16, a.batch, a.k_len, a.kv_heads, a.dim, 64, 128)) != GS_OK) return s;
    if ((s = attn_tensor_map(&m.v, a.v, bf16, a.batch, a.k_len, a.kv_heads, a.dim, 64, 128)) != GS_OK) return s;
    if (a.dim <= 64) return bf16 ? forward_t<true, 64>(a, m, st) : forward_t<false, 64>(a, m, st);
    return bf16 ? forward_t<true, 128>(a, m, st) : forward_t<false, 128>(a, m, st);
}

}  // namespace gs
