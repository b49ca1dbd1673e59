// Forward attention of 16-bit tensors on the fifth-generation tensor cores.
//
// A work item is 256 query rows of a head, as two tiles of 128, and the key tiles (128 keys) that any of them
// sees.  One block per SM goes through its items; loads and products of the next item run while the last
// one's rows are divided and stored.  Roles:
//   warps 0-3, 4-7  softmax of tile 0 and tile 1: thread = row.  Scores come from tensor memory,
//                   probabilities go back there as 16-bit values over the scores they came from
//   warp 8          one thread issues the tcgen05.mma: S_t = Q_t K^T (both from shared memory) and
//                   O_t += P_t V (P from tensor memory)
//   warp 9          TMA loads of Q and of the ring of K and V tiles; asks for the next item
// While one tile's warps exponentiate, the tensor core works on the other tile.  Tensor memory: S_0,
// S_1, O_0, O_1 of 128 columns.  The order of one thread's tcgen05.mma is kept, so S_t of the next
// keys, issued behind P_t V, may overwrite P_t without another barrier; and the barrier that
// announces it also says that O_t is at rest, which is when its owner may rescale it.
//
// The running maximum moves only when the new one is above it by more than 8 (a factor 256 in p):
// most tiles then leave O and the sum alone, exact in any case because the quotient O / sum uses one base.
// p is rounded to the tensors' type for the product with V; the sum takes it in fp32.
#include "gs_attn_again.cuh"
#include "gs_attn_tc.cuh"

namespace gs {

using namespace tc;

static constexpr int ROWS = 256, KEYS = 128;

template <int DP>
struct FwdSmem {
    static constexpr int TILE = 128 * DP * 2;                   // bytes of one 128-row tile
    static constexpr int SLOTS = DP == 128 ? 4 : 8;
    static constexpr int Q = 0, RING = 2 * TILE, BARS = RING + SLOTS * TILE;
    static constexpr int QUEUE = (BARS + 8 * (13 + 2 * SLOTS) + 15) / 16 * 16;      // answers and barriers of the items
    static constexpr int WORDS = QUEUE + 64;                    // stalled, address of the tensor memory
    static constexpr int BYTES = WORDS + 16;
};

struct FwdItem {
    AttnSeq s;
    int b, h, g, r0;
    int first[2], last[2];                                      // key tiles of the two row tiles
    int it0, it1;                                               // of either
    __device__ __forceinline__ FwdItem(const AttnArgs &a, uint32_t i)
    {
        const uint32_t heads = (uint32_t)a.batch * a.q_heads, tile = i / heads, bh = i - tile * heads;
        h = (int)(bh / (uint32_t)a.batch);                    // neighbours in the list are other sequences: lengths mix
        b = (int)(bh - (uint32_t)h * (uint32_t)a.batch);
        g = h / a.group;
        s = attn_seq(a, b);
        r0 = ((a.q_len + ROWS - 1) / ROWS - 1 - (int)tile) * ROWS;      // the last rows of a causal bound are the longest
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
        it0 = any0 ? (any1 ? min(first[0], first[1]) : first[0]) : first[1];
        it1 = any0 ? (any1 ? max(last[0], last[1]) : last[0]) : last[1];
    }
};

struct TcMaps {
    CUtensorMap q, k, v;
};

template <bool BF16, int DP>
__global__ void __launch_bounds__(384, 1)
attn_tc_forward_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ TcMaps maps, uint32_t count,
                       unsigned long long *stalls)
{
    using L = FwdSmem<DP>;
    extern __shared__ __align__(1024) uint8_t smem[];           // no static shared memory: this starts at its beginning
    const uint32_t base = smem_u32(smem);
    volatile int &stalled = *reinterpret_cast<volatile int *>(smem + L::WORDS);
    uint32_t &tmem_base = *reinterpret_cast<uint32_t *>(smem + L::WORDS + 4);
    const uint32_t bars = base + L::BARS;
    const uint32_t q_full = bars, q_empty = bars + 8, fix = bars + 16, s_full = bars + 24, p_full = bars + 40, o_full = bars + 56,
                   o_empty = bars + 72, p_half = bars + 88, kv_full = bars + 104, kv_empty = kv_full + 8 * L::SLOTS;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const ItemQueue queue{count, base + L::QUEUE, base + L::QUEUE + 32, base + L::QUEUE + 48, &stalled};

    if (threadIdx.x == 0) {
        stalled = 0;
        queue.init(9);                                          // warps 0-8
        bar_init(q_full, 1);
        bar_init(q_empty, 1);
        bar_init(fix, 1);
        for (int t = 0; t < 2; ++t) {
            bar_init(s_full + 8 * t, 1);
            bar_init(p_half + 8 * t, 128);
            bar_init(p_full + 8 * t, 128);
            bar_init(o_full + 8 * t, 1);
            bar_init(o_empty + 8 * t, 128);
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
            // ---- loads: Q of each item, K and V of its key tiles through the ring
            int n = 0, items = 0;                                 // tiles loaded, items begun
            uint32_t patched = 0;
            bool ok = true;
            for (Items<true> i(queue); i.more() && ok; i.next()) {
                const FwdItem w(a, i.at);
                if (w.it0 >= w.it1) continue;
                if (items > 0) ok = __all_sync(0xffffffffu, bar_wait(q_empty, (items - 1) & 1, &stalled));
                ++items;
                if (ok && lane == 0) {
                    bar_expect(q_full, 2 * L::TILE);
                    load_tile<DP>(base + L::Q, &maps.q, q_full, w.r0, w.h, w.b);
                    load_tile<DP>(base + L::Q + L::TILE, &maps.q, q_full, w.r0 + 128, w.h, w.b);
                }
                for (int it = w.it0; it < w.it1 && ok; ++it) {
                    for (int kv = 0; kv < 2 && ok; ++kv, ++n) {
                        const int slot = n % L::SLOTS, round = n / L::SLOTS;
                        if (round > 0) ok = __all_sync(0xffffffffu, bar_wait(kv_empty + 8 * slot, (round - 1) & 1, &stalled));
                        if (!ok) break;
                        const uint32_t dst = base + L::RING + slot * L::TILE, full = kv_full + 8 * slot;
                        // values past the sequence's end (not past the tensor's, which TMA fills with zeros)
                        // must not meet a zero probability: 0 * NaN.  They are overwritten with zeros.
                        const bool patch = kv == 1 && w.s.nk < a.k_len && (it + 1) * KEYS > w.s.nk;
                        if (lane == 0) {
                            bar_expect(patch ? fix : full, L::TILE);
                            load_tile<DP>(dst, kv ? &maps.v : &maps.k, patch ? fix : full, it * KEYS, w.g, w.b);
                        }
                        if (patch) {
                            ok = patch_tile<DP>(dst, w.s.nk - it * KEYS, fix, patched, full, &stalled);
                            patched ^= 1;
                        }
                    }
                }
            }
        } else if (warp == 8) {
            // ---- products
            {
                const bool one = elect_one();
                constexpr uint32_t DESC_S = mma_desc(BF16, 128, KEYS, false), DESC_O = mma_desc(BF16, 128, DP, true);
                int n = 0, items = 0;                             // ring position of K of step it; V of it - 1 is n - 1
                uint32_t p_phase[2] = {0, 0}, o_used[2] = {0, 0};
                bool ok = true;
                for (Items<false> i(queue); i.more() && ok; i.next()) {
                    const FwdItem w(a, i.at);
                    if (w.it0 >= w.it1) continue;
                    ok = __all_sync(0xffffffffu, bar_wait(q_full, items & 1, &stalled));
                    ++items;
                    for (int it = w.it0; it <= w.it1 && ok; ++it) {
                        const bool have_k = it < w.it1, have_v = it > w.it0;
                        const int ks = n % L::SLOTS, vs = (n + L::SLOTS - 1) % L::SLOTS;
                        if (have_v) ok = bar_wait(kv_full + 8 * vs, ((n - 1) / L::SLOTS) & 1, &stalled);
                        if (have_k) ok = bar_wait(kv_full + 8 * ks, (n / L::SLOTS) & 1, &stalled) && ok;
                        ok = __all_sync(0xffffffffu, ok);
                        if (!ok) break;
                        fence_after();
                        const uint32_t kt = base + L::RING + ks * L::TILE, vt = base + L::RING + vs * L::TILE;
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            if (it - 1 >= w.first[t] && it - 1 < w.last[t]) {
                                ok = bar_wait(p_half + 8 * t, p_phase[t], &stalled);
                                if (ok && it - 1 == w.first[t] && o_used[t]++ > 0)      // the last item's rows have been read
                                    ok = bar_wait(o_empty + 8 * t, o_used[t] & 1, &stalled);
                                ok = __all_sync(0xffffffffu, ok);
                                if (!ok) break;
                                const uint64_t v0 = desc_rows(vt, HALF_TILE);
#pragma unroll
                                for (int part = 0; part < 2; ++part) {
                                    if (part == 1) ok = __all_sync(0xffffffffu, bar_wait(p_full + 8 * t, p_phase[t], &stalled));
                                    if (!ok) break;
                                    fence_after();
                                    if (one) {
#pragma unroll
                                        for (int k = part * KEYS / 32; k < (part + 1) * KEYS / 32; ++k)
                                            mma_ts(tmem + 256 + 128 * t, tmem + 128 * t + 8 * k, v0 + desc_step(2048 * k), DESC_O,
                                                   it - 1 > w.first[t] || k > 0);
                                        if (part == 1 && it == w.last[t]) mma_commit(o_full + 8 * t);
                                    }
                                }
                                if (!ok) break;
                                p_phase[t] ^= 1;
                            }
                            if (it >= w.first[t] && it < w.last[t]) {
                                if (one) {
const uint64_t q0 = desc_values(base + L::Q + t * L::TILE), k0 = desc_values(kt);
#pragma unroll
                                for (int k = 0; k < DP / 16; ++k) {
                                    const uint64_t at = desc_step((k / 4) * HALF_TILE + (k % 4) * 32);
                                    mma_ss(tmem + 128 * t, q0 + at, k0 + at, DESC_S, k > 0);
                                }
                                mma_commit(s_full + 8 * t);
                                }
                            }
                        }
                        if (!ok) break;
                        if (one) {
                            if (have_v) mma_commit(kv_empty + 8 * vs);
                            if (have_k) mma_commit(kv_empty + 8 * ks);
                            if (it + 1 == w.it1) mma_commit(q_empty);
                        }
                        if (have_k) n += 2;
                    }
                }
            }
            __syncwarp();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        // ---- softmax of one row
        const int t = warp >> 2;
        const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
        const uint32_t ts = tmem + lanes + 128 * t, to = tmem + lanes + 256 + 128 * t;
        const float mul = a.scale * LOG2E;                        // exponents are taken in base 2
        const bool vec = rows16(a.out, a.dim);
        bool ok = true;
        uint32_t phase = 0, o_phase = 0;
        for (Items<false> i(queue); i.more() && ok; i.next()) {
        const FwdItem w(a, i.at);
        const AttnSeq &s = w.s;
        const int r = w.r0 + 128 * t + (threadIdx.x & 127);
        const bool row = r < s.nq;
        const int lo = row ? attn_lo(a, s, r) : 0, hi = row ? attn_hi(a, s, r) : s.nk;
        // tiles that every row of this tile sees whole need no mask
        const int whole_lo = attn_lo(a, s, min(w.r0 + 128 * t + 127, max(s.nq - 1, 0))), whole_hi = attn_hi(a, s, w.r0 + 128 * t);
        float top = -INFINITY, sum = 0.f;                         // top: base of the exponents, in units of log2
        const int it_first = t == 0 ? w.first[0] : w.first[1], it_last = t == 0 ? w.last[0] : w.last[1];
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
                for (int k = 0; k < 16; ++k) {
                    float2 e = fma2(make_float2(x[c + 2 * k], x[c + 2 * k + 1]), mul2v, sub2);
                    e = make_float2(exp2_fast(e.x), exp2_fast(e.y));
                    acc[k & 1] = add2(acc[k & 1], e);
                    p[k] = pack2<BF16>(e.x, e.y);
                }
                tmem_st16(ts + c / 2, p);
                if (c == KEYS / 2 - 32 || c == KEYS - 32) {       // the product with V starts on the first half
                    wait_st();
                    fence_before();
                    bar_arrive((c == KEYS - 32 ? p_full : p_half) + 8 * t);
                }
            }
            const float2 part = add2(acc[0], acc[1]);
            sum += part.x + part.y;
        }
        const bool some = it_first < it_last;
        if (ok && some) {
            ok = __all_sync(0xffffffffu, bar_wait(o_full + 8 * t, o_phase, &stalled));
            o_phase ^= 1;
        }
        fence_after();
        const float inv = row && some ? again::row_factor(top, 1.f / sum) : 0.f;
        if (r < a.q_len) a.lse[((int64_t)w.b * a.q_heads + w.h) * a.q_len + r] = again::row_lse(top, inv, log2f(sum));
        uint16_t *out = reinterpret_cast<uint16_t *>(a.out.p) + w.b * a.out.sb + (int64_t)r * a.out.sl + w.h * a.out.sh;
        NanSums total;                     // whether one of the row's values is NaN
#pragma unroll
        for (int c = 0; c < DP; c += 32) {
            float o[32];
            __syncwarp();
            if (some && ok) {
                tmem_ld32(to + c, reinterpret_cast<uint32_t *>(o));
                wait_ld();
                if (c + 32 == DP) {
                    fence_before();
                    bar_arrive(o_empty + 8 * t);
                }
                total.add(o);
            }
            if (r < a.q_len) store32<BF16>(out, c, a.dim, vec, o, inv);
        }
        if (__any_sync(0xffffffffu, row && (total.found() || again::is_nan(inv)))) {
            const int r32 = w.r0 + 128 * t + 32 * (warp & 3);
            again::outputs<typename Tensor16<BF16>::T>(a, w.b, w.h, r32, r32 + 32);
        }
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

bool attn_tma_ok(const AttnTensor &t, int32_t dtype, int64_t batch, int64_t len, int64_t heads)
{
    const int n = dtype == GS_TABLE_F32 ? 4 : 8;                // strides of whole 16 bytes, below 2^40
    auto stride_ok = [&](int64_t extent, int64_t s) {
        return extent <= 1 || (s > 0 && s % n == 0 && s < ((int64_t)1 << 37));
    };
    return (uintptr_t)t.p % 16 == 0 && stride_ok(batch, t.sb) && stride_ok(len, t.sl) && stride_ok(heads, t.sh);
}

gs_status attn_tensor_map(CUtensorMap *m, const AttnTensor &t, int32_t dtype, int64_t batch, int64_t len, int64_t heads,
                          int dim, int values, int rows)
{
    EncodeTiled fn = encoder();
    if (!fn) {
        set_error("cuTensorMapEncodeTiled is not available from this driver");
        return GS_ERR_CUDA;
    }
    const cuuint64_t extent[4] = {(cuuint64_t)dim, (cuuint64_t)len, (cuuint64_t)heads, (cuuint64_t)batch};
    const int es = dtype == GS_TABLE_F32 ? 4 : 2;
    const cuuint64_t stride[3] = {(cuuint64_t)(len > 1 ? es * t.sl : 512), (cuuint64_t)(heads > 1 ? es * t.sh : 512),
                                  (cuuint64_t)(batch > 1 ? es * t.sb : 512)};
    const cuuint32_t box[4] = {(cuuint32_t)values, (cuuint32_t)rows, 1, 1}, step[4] = {1, 1, 1, 1};
    auto encode = [&] {
        return fn(m, dtype == GS_TABLE_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                  : dtype == GS_TABLE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, t.p, extent, stride,
                              box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              values * es == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : values * es == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    };
    CUresult r = encode();
    if (r == CUDA_ERROR_INVALID_CONTEXT) {          // a thread that has not used the device yet, such as autograd's
        int dev = 0;
        GS_CUDA_TRY(cudaGetDevice(&dev));
        GS_CUDA_TRY(cudaSetDevice(dev));
        r = encode();
    }
    if (r != CUDA_SUCCESS) {
        set_error("cuTensorMapEncodeTiled failed with %d", (int)r);
        return GS_ERR_CUDA;
    }
    return GS_OK;
}

template <bool BF16, int DP>
static gs_status forward_t(const AttnArgs &a, const TcMaps &maps, cudaStream_t st)
{
    const int64_t items = a.batch * a.q_heads * ((a.q_len + ROWS - 1) / ROWS);
    if (items > 0x7FFFFFFF) {
        set_error("attention of %lld row tiles exceeds one launch", (long long)items);
        return GS_ERR_UNSUPPORTED;
    }
    auto kernel = attn_tc_forward_kernel<BF16, DP>;
    static SharedRecord record;
    gs_status s = allow_shared(kernel, FwdSmem<DP>::BYTES, record);
    if (s != GS_OK) return s;
    const int64_t sms = sm_count();
    const bool asked = items_asked(a, items);
    kernel<<<(unsigned)(asked || items < sms ? items : sms), 384, FwdSmem<DP>::BYTES, st>>>(a, maps, asked ? 0u : (uint32_t)items, stall_counter());
    GS_CUDA_TRY(cudaGetLastError());
    return GS_OK;
}

bool attn_tc_forward_ok(const AttnArgs &a)
{
    return a.dtype != GS_TABLE_F32 && a.batch < ((int64_t)1 << 31) && attn_tma_ok(a.q, a.dtype, a.batch, a.q_len, a.q_heads) &&
           attn_tma_ok(a.k, a.dtype, a.batch, a.k_len, a.kv_heads) && attn_tma_ok(a.v, a.dtype, a.batch, a.k_len, a.kv_heads);
}

gs_status attn_tc_forward(const AttnArgs &a, cudaStream_t st)
{
    const bool bf16 = a.dtype == GS_TABLE_BF16;
    TcMaps m;
    gs_status s;
    if ((s = attn_tensor_map(&m.q, a.q, a.dtype, a.batch, a.q_len, a.q_heads, a.dim, 64, 128)) != GS_OK) return s;
    if ((s = attn_tensor_map(&m.k, a.k, a.dtype, a.batch, a.k_len, a.kv_heads, a.dim, 64, 128)) != GS_OK) return s;
    if ((s = attn_tensor_map(&m.v, a.v, a.dtype, a.batch, a.k_len, a.kv_heads, a.dim, 64, 128)) != GS_OK) return s;
    if (a.dim <= 64) return bf16 ? forward_t<true, 64>(a, m, st) : forward_t<false, 64>(a, m, st);
    return bf16 ? forward_t<true, 128>(a, m, st) : forward_t<false, 128>(a, m, st);
}

// One block whose wait nothing ends; it gives up within about two seconds and is counted like any other
__global__ void attn_stall_drill_kernel(unsigned long long *stalls)
{
    __shared__ __align__(8) uint64_t never;
    __shared__ volatile int stalled;
    const uint32_t bar = smem_u32(&never);
    if (threadIdx.x == 0) {
        stalled = 0;
        bar_init(bar, 1);
        fence_barrier_init();
    }
    __syncthreads();
    bar_wait(bar, 0, &stalled, 0);
    __syncthreads();
    if (stalled) drain_stalled(stalls);
}

gs_status attn_stall_drill(cudaStream_t st)
{
    unsigned long long *stalls = stall_counter();
    if (!stalls) {
        set_error("no page-locked host memory for the count");
        return GS_ERR_OOM;
    }
    attn_stall_drill_kernel<<<1, 32, 0, st>>>(stalls);
    GS_CUDA_TRY(cudaGetLastError());
    return GS_OK;
}

}  // namespace gs
