// Backward attention of 16-bit tensors on the fifth-generation tensor cores: two kernels that both
// compute the scores again, so that every gradient has one owner and no value is summed with atomics
// (seven products of 128 x 128 tiles where a single kernel with atomics on dq needs five).
//
//  dq     : one block per 128 query rows.  S = Q K^T, dP = dO V^T, dS = P (dP - delta), dQ += dS K.
//           Thread = query row; S of the next keys is computed while this one's dS is formed, dP's columns are
//           free for the next product as soon as they are in registers.  Leaves delta = dO.O for the other kernel.
//  dk, dv : one block per 128 keys, looping over the query heads of their group and their query tiles.
//           Everything transposed: S^T = K Q^T, dP^T = V dO^T, so that P^T and dS^T come out with one key per
//           lane and feed dV += P^T dO, dK += dS^T Q from tensor memory without passing through shared memory.
//           Tensor memory is full (S^T, dP^T, dV, dK: 128 columns each); the order dV(i), S^T(i+1) while dS(i)
//           is formed, then dK(i), dP^T(i+1) while P(i+1) is formed, keeps both sides busy.
// In both, eight warps do the elementwise part, four per 64 columns of a tile; a warp overwrites only
// columns that it has read itself.  Warp 8 issues the products, warp 9 the loads, warp 10 brings the
// row statistics of dk/dv's query tiles.
//
// P and dS are rounded to the tensors' type for their products.  binary16 has no range for that as it
// stands: P is scaled by 2^15 (P <= 1), dS by the power of two that brings its bound
// |dS| <= 2 max|do| max|v| (row norms) near 2^15; the bound needs a pass over dO and V, for binary16 only.
#include "gs_attn_tc.cuh"

namespace gs {

using namespace tc;

static constexpr int T = 128;                     // rows of every tile

struct BwdMaps {
    CUtensorMap q, k, v, dout;
};

struct BwdNorms {                                 // binary16: largest row norm of each 128-row tile
    float *dout, *v;                              // [batch * q_heads][q tiles], [batch * kv_heads][k tiles]
};

template <int DP>
struct BwdSmem {
    static constexpr int TILE = T * DP * 2;
    // Two resident tiles, then two rings of tiles: X for the operand that a step needs first and last (K for dq, Q for
    // dk/dv), Y for the other.  Three X tiles, because one is free only when its step's last product is done.
    static constexpr int XS = DP == 128 ? 3 : 4, YS = DP == 128 ? 2 : 4, SS = 2;
    static constexpr int A = 0, B = TILE, X = 2 * TILE, Y = X + XS * TILE;
    static constexpr int STATS = Y + YS * TILE;                 // dk/dv: lse and delta of a query tile, SS of them
    static constexpr int BARS = STATS + SS * 2 * T * 4;
    static constexpr int WORDS = BARS + 8 * (10 + 2 * XS + 2 * YS + 2 * SS);    // stalled, address of the tensor memory
    static constexpr int BYTES = WORDS + 16;
    static_assert(BYTES <= 227 * 1024, "shared memory of one block");
};

// D[128 x 128] = A B^T over the head dimension, both tiles [rows][values]
template <int DP>
__device__ __forceinline__ void mul_values(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc)
{
    const uint64_t a0 = desc_values(a), b0 = desc_values(b);
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
        const uint64_t at = desc_step((k / 4) * HALF_TILE + (k % 4) * 32);
        mma_ss(d, a0 + at, b0 + at, idesc, k > 0);
    }
}

// D[128 x DP] += A B, A 128 x 128 in tensor memory (two halves of 32 columns, 64 apart), B [rows][values]
__device__ __forceinline__ void mul_rows(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add)
{
    const uint64_t b0 = desc_rows(b, HALF_TILE);
#pragma unroll
    for (int k = 0; k < T / 16; ++k)
        mma_ts(d, a + (k / 4) * 64 + (k % 4) * 8, b0 + desc_step(2048 * k), idesc, add || k > 0);
}

__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// power of two that brings 2 max|do| max|v| to [2^14, 2^15); heads [h0, h1) of one key/value head
__device__ __forceinline__ float ds_scale(const AttnArgs &a, const BwdNorms &nm, int64_t b, int h0, int h1, int g)
{
    const int qt = (a.q_len + T - 1) / T, kt = (a.k_len + T - 1) / T, lane = threadIdx.x & 31;
    float x = 0.f, y = 0.f;
    const float *p = nm.dout + (b * a.q_heads + h0) * qt;
    for (int i = lane; i < (h1 - h0) * qt; i += 32) x = fmaxf(x, p[i]);
    const float *w = nm.v + (b * a.kv_heads + g) * kt;
    for (int i = lane; i < kt; i += 32) y = fmaxf(y, w[i]);
    const float top = 2.f * warp_max(x) * warp_max(y);
    if (!(top > 0.f) || !isfinite(top)) return 1.f;
    int e;
    frexpf(top, &e);                              // top in [2^(e-1), 2^e)
    return ldexpf(1.f, min(max(15 - e, -100), 100));
}

// largest row norm of each 128-row tile of dO and V.  Block: one tile; a warp takes every fourth row.
__global__ void __launch_bounds__(128) attn_tc_norms_kernel(const __grid_constant__ AttnArgs a, BwdNorms nm)
{
    const int qt = (a.q_len + T - 1) / T, kt = (a.k_len + T - 1) / T;
    int64_t i = blockIdx.x;
    const int64_t nq = a.batch * a.q_heads * qt;
    const bool on_q = i < nq;
    if (!on_q) i -= nq;
    const int tiles = on_q ? qt : kt, nh = on_q ? a.q_heads : a.kv_heads;
    const int tile = (int)(i % tiles);
    const int64_t bh = i / tiles, b = bh / nh;
    const int h = (int)(bh % nh);
    const AttnTensor &t = on_q ? a.dout : a.v;
    const AttnSeq s = attn_seq(a, b);
    const int end = min((tile + 1) * T, on_q ? s.nq : s.nk), lane = threadIdx.x & 31;
    const __half *base = reinterpret_cast<const __half *>(t.p) + b * t.sb + h * t.sh;
    float top = 0.f;
    for (int r = tile * T + (threadIdx.x >> 5); r < end; r += 4) {
        float x = 0.f;
        for (int c = lane; c < a.dim; c += 32) {
            const float v = __half2float(base[(int64_t)r * t.sl + c]);
            x = fmaf(v, v, x);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        top = fmaxf(top, x);
    }
    __shared__ float sh[4];
    if (lane == 0) sh[threadIdx.x >> 5] = top;
    __syncthreads();
    if (threadIdx.x == 0)
        (on_q ? nm.dout : nm.v)[i] = sqrtf(fmaxf(fmaxf(sh[0], sh[1]), fmaxf(sh[2], sh[3])));
}

template <bool BF16>
__device__ __forceinline__ float2 unpack2(uint32_t u)
{
    if constexpr (BF16) return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
    else return __half22float2(*reinterpret_cast<__half2 *>(&u));
}

// dot product of two rows of 16-bit values in global memory; 128 bytes of each are on their way at a time
template <bool BF16, int DP>
__device__ __forceinline__ float dot16(const uint16_t *x, const uint16_t *y, int dim, bool vec)
{
    float d = 0.f;
    if (vec) {
#pragma unroll
        for (int c0 = 0; c0 < DP; c0 += 64) {
            uint4 u[8], w[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const bool in = c0 + 8 * k < dim;
                u[k] = in ? __ldg(reinterpret_cast<const uint4 *>(x + c0 + 8 * k)) : make_uint4(0, 0, 0, 0);
                w[k] = in ? __ldg(reinterpret_cast<const uint4 *>(y + c0 + 8 * k)) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t p[4] = {u[k].x, u[k].y, u[k].z, u[k].w}, q[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = unpack2<BF16>(p[i]), g = unpack2<BF16>(q[i]);
                    d = fmaf(f.x, g.x, d);
                    d = fmaf(f.y, g.y, d);
                }
            }
        }
    } else {
        for (int c = 0; c < dim; ++c) d = fmaf(unpack2<BF16>(x[c]).x, unpack2<BF16>(y[c]).x, d);
    }
    return d;
}

template <bool BF16, int DP>
__global__ void __launch_bounds__(384, 1)
attn_tc_dq_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ BwdMaps maps, const BwdNorms norms,
                  unsigned long long *stalls)
{
    using L = BwdSmem<DP>;
    extern __shared__ __align__(1024) uint8_t smem[];           // no static shared memory: this starts at its beginning
    const uint32_t base = smem_u32(smem);
    volatile int &stalled = *reinterpret_cast<volatile int *>(smem + L::WORDS);
    uint32_t &tmem_base = *reinterpret_cast<uint32_t *>(smem + L::WORDS + 4);
    const uint32_t bars = base + L::BARS;
    const uint32_t q_full = bars, fix = bars + 8, s_full = bars + 16, dp_full = bars + 32, dp_free = bars + 40,
                   ds_full = bars + 48, done = bars + 56, k_full = bars + 80, k_empty = k_full + 8 * L::XS,
                   v_full = k_empty + 8 * L::XS, v_empty = v_full + 8 * L::YS;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    const int64_t heads = a.batch * a.q_heads;
    const int tiles = (a.q_len + T - 1) / T;
    const int r0 = (tiles - 1 - (int)(blockIdx.x / heads)) * T;     // the longest rows of a causal bound go first
    const int64_t bh = blockIdx.x % heads, b = bh / a.q_heads;
    const int h = (int)(bh % a.q_heads), g = h / a.group;
    const AttnSeq s = attn_seq(a, b);
    int first = 0, n = 0;
    if (r0 < s.nq) {
        const int lo = attn_lo(a, s, r0), hi = attn_hi(a, s, min(r0 + T, s.nq) - 1);
        if (lo < hi) {
            first = lo / T;
            n = (hi + T - 1) / T - first;
        }
    }

    if (threadIdx.x == 0) {
        stalled = 0;
        bar_init(q_full, 1);
        bar_init(fix, 1);
        bar_init(s_full, 1);
        bar_init(s_full + 8, 1);
        bar_init(dp_full, 1);
        bar_init(dp_free, 256);
        bar_init(ds_full, 256);
        bar_init(done, 1);
        for (int i = 0; i < 2 * (L::XS + L::YS); ++i) bar_init(k_full + 8 * i, 1);
        fence_barrier_init();
    }
    if (warp == 8) tmem_alloc(smem_u32(&tmem_base), 512);
    if (warp == 9 && lane == 0) {
        tma_prefetch(&maps.q);
        tma_prefetch(&maps.k);
        tma_prefetch(&maps.v);
        tma_prefetch(&maps.dout);
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = tmem_base;                  // S of even and odd steps, dP, dQ

    if (warp == 9) {
        if (n > 0) {
            if (lane == 0) {
                bar_expect(q_full, 2 * L::TILE);
                load_tile<DP>(base + L::A, &maps.q, q_full, r0, h, (int)b);
                load_tile<DP>(base + L::B, &maps.dout, q_full, r0, h, (int)b);
            }
            bool ok = true;
            for (int i = 0; i < n && ok; ++i) {
                const int kst = i % L::XS, vst = i % L::YS, j0 = (first + i) * T;
                const uint32_t kt = base + L::X + kst * L::TILE, vt = base + L::Y + vst * L::TILE;
                const bool patch = s.nk < a.k_len && j0 + T > s.nk;        // K is summed over its rows in dS K
                if (i >= L::XS) ok = __all_sync(0xffffffffu, bar_wait(k_empty + 8 * kst, (i / L::XS - 1) & 1, &stalled));
                if (!ok) break;
                if (lane == 0) {
                    const uint32_t bar = patch ? fix : k_full + 8 * kst;
                    bar_expect(bar, L::TILE);
                    load_tile<DP>(kt, &maps.k, bar, j0, g, (int)b);
                }
                if (i >= L::YS) ok = __all_sync(0xffffffffu, bar_wait(v_empty + 8 * vst, (i / L::YS - 1) & 1, &stalled));
                if (!ok) break;
                if (lane == 0) {
                    bar_expect(v_full + 8 * vst, L::TILE);
                    load_tile<DP>(vt, &maps.v, v_full + 8 * vst, j0, g, (int)b);
                }
                if (patch) ok = patch_tile<DP>(kt, s.nk - j0, fix, 0, k_full + 8 * kst, &stalled);
            }
        }
    } else if (warp == 8) {
        if (n > 0) {
            const bool one = elect_one();
            constexpr uint32_t DESC_S = mma_desc(BF16, T, T, false), DESC_Q = mma_desc(BF16, T, DP, true);
            auto kt = [&](int i) { return base + L::X + (i % L::XS) * L::TILE; };
            auto vt = [&](int i) { return base + L::Y + (i % L::YS) * L::TILE; };
            auto k_here = [&](int i) { return bar_wait(k_full + 8 * (i % L::XS), (i / L::XS) & 1, &stalled); };
            auto v_here = [&](int i) { return bar_wait(v_full + 8 * (i % L::YS), (i / L::YS) & 1, &stalled); };
            bool ok = __all_sync(0xffffffffu, bar_wait(q_full, 0, &stalled) && k_here(0));
            if (ok) {
                fence_after();
                if (one) {
                    mul_values<DP>(tmem, base + L::A, kt(0), DESC_S);
                    mma_commit(s_full);
                }
                ok = __all_sync(0xffffffffu, v_here(0));
            }
            if (ok) {
                fence_after();
                if (one) {
                    mul_values<DP>(tmem + 256, base + L::B, vt(0), DESC_S);
                    mma_commit(dp_full);
                    mma_commit(v_empty);
                }
            }
            for (int i = 0; i < n && ok; ++i) {
                if (i + 1 < n) {                      // the other S: its dS went into dQ(i - 1), issued before
                    ok = __all_sync(0xffffffffu, k_here(i + 1));
                    if (!ok) break;
                    fence_after();
                    if (one) {
                        mul_values<DP>(tmem + 128 * ((i + 1) & 1), base + L::A, kt(i + 1), DESC_S);
                        mma_commit(s_full + 8 * ((i + 1) & 1));
                    }
                    ok = __all_sync(0xffffffffu, v_here(i + 1) && bar_wait(dp_free, i & 1, &stalled));
                    if (!ok) break;
                    fence_after();
                    if (one) {
                        mul_values<DP>(tmem + 256, base + L::B, vt(i + 1), DESC_S);
                        mma_commit(dp_full);
                        mma_commit(v_empty + 8 * ((i + 1) % L::YS));
                    }
                }
                ok = __all_sync(0xffffffffu, bar_wait(ds_full, i & 1, &stalled));
                if (!ok) break;
                fence_after();
                if (one) {
                    mul_rows(tmem + 384, tmem + 128 * (i & 1), kt(i), DESC_Q, i > 0);
                    mma_commit(k_empty + 8 * (i % L::XS));
                }
            }
            if (ok && one) mma_commit(done);
        }
        __syncwarp();
    } else if (warp < 8) {
        const int half = warp >> 2;                   // columns [64 half, 64 half + 64)
        const int r = r0 + (threadIdx.x & 127);
        const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
        const bool row = r < s.nq;
        const int lo = row ? attn_lo(a, s, r) : 0, hi = row ? attn_hi(a, s, r) : 0;
        const int whole_lo = attn_lo(a, s, min(r0 + T, s.nq) - 1), whole_hi = attn_hi(a, s, r0);
        const bool whole = r0 + T <= s.nq;
        float delta = 0.f, lse2 = 0.f;
        if (row) {
            const bool vec = rows16(a.out, a.dim) && rows16(a.dout, a.dim);
            delta = dot16<BF16, DP>(reinterpret_cast<const uint16_t *>(a.out.p) + b * a.out.sb + (int64_t)r * a.out.sl + h * a.out.sh,
                                reinterpret_cast<const uint16_t *>(a.dout.p) + b * a.dout.sb + (int64_t)r * a.dout.sl + h * a.dout.sh,
                                a.dim, vec);
            lse2 = a.lse[bh * a.q_len + r] * LOG2E;
        }
        if (half == 0 && r < a.q_len) a.delta[bh * a.q_len + r] = delta;
        const float mul = a.scale * LOG2E;
        float up = 1.f;
        if constexpr (!BF16) up = ds_scale(a, norms, b, h, h + 1, g);
        bool ok = true;
        for (int i = 0; i < n; ++i) {
            ok = __all_sync(0xffffffffu, bar_wait(s_full + 8 * (i & 1), (i >> 1) & 1, &stalled) &&
                                             bar_wait(dp_full, i & 1, &stalled));
            if (!ok) break;
            fence_after();
            float x[64], dp[64];
            const uint32_t ts = tmem + lanes + 128 * (i & 1) + 64 * half, td = tmem + lanes + 256 + 64 * half;
            tmem_ld32(td, reinterpret_cast<uint32_t *>(dp));
            tmem_ld32(td + 32, reinterpret_cast<uint32_t *>(dp) + 32);
            tmem_ld32(ts, reinterpret_cast<uint32_t *>(x));
            tmem_ld32(ts + 32, reinterpret_cast<uint32_t *>(x) + 32);
            wait_ld();
            fence_before();
            bar_arrive(dp_free);
            const int j0 = (first + i) * T;
#pragma unroll
            for (int c = 0; c < 64; c += 2) {
                const float2 e = fma2(make_float2(x[c], x[c + 1]), make_float2(mul, mul), make_float2(-lse2, -lse2));
                float2 p = make_float2(exp2_fast(e.x), exp2_fast(e.y));
                if constexpr (!BF16) p = mul2(p, make_float2(up, up));
                const float2 d = mul2(p, add2(make_float2(dp[c], dp[c + 1]), make_float2(-delta, -delta)));
                x[c] = d.x;
                x[c + 1] = d.y;
            }
            if (!whole || j0 < whole_lo || j0 + T > whole_hi) {
                const int c0 = lo - j0 - 64 * half, c1 = hi - j0 - 64 * half;
#pragma unroll
                for (int c = 0; c < 64; ++c) x[c] = c >= c0 && c < c1 ? x[c] : 0.f;
            }
            uint32_t u[32];
#pragma unroll
            for (int c = 0; c < 32; ++c) u[c] = pack2<BF16>(x[2 * c], x[2 * c + 1]);
            tmem_st32(ts, u);
            wait_st();
            fence_before();
            bar_arrive(ds_full);
        }
        if (ok && n > 0) ok = __all_sync(0xffffffffu, bar_wait(done, 0, &stalled));
        fence_after();
        const float factor = row && n > 0 ? a.scale / up : 0.f;
        uint16_t *out = reinterpret_cast<uint16_t *>(a.dq.p) + b * a.dq.sb + (int64_t)r * a.dq.sl + h * a.dq.sh;
        const bool vec = rows16(a.dq, a.dim);
#pragma unroll
        for (int c = 0; c < DP / 2; c += 32) {        // each half of the warps stores half of the columns
            const int col = half * (DP / 2) + c;
            float o[32];
            __syncwarp();
            if (n > 0 && ok) {
                tmem_ld32(tmem + lanes + 384 + col, reinterpret_cast<uint32_t *>(o));
                wait_ld();
            }
            if (r < a.q_len) store32<BF16>(out, col, a.dim, vec, o, factor);
        }
    }

    fence_before();
    __syncthreads();
    fence_after();
    if (stalled) drain_stalled(stalls);
    if (warp == 8) tmem_free(tmem, 512);
}

template <bool BF16, int DP>
__global__ void __launch_bounds__(384, 1)
attn_tc_dkdv_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ BwdMaps maps, const BwdNorms norms,
                    unsigned long long *stalls)
{
    using L = BwdSmem<DP>;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    float *stats = reinterpret_cast<float *>(smem + L::STATS);            // [slot][lse, delta][128]
    volatile int &stalled = *reinterpret_cast<volatile int *>(smem + L::WORDS);
    uint32_t &tmem_base = *reinterpret_cast<uint32_t *>(smem + L::WORDS + 4);
    const uint32_t bars = base + L::BARS;
    const uint32_t kv_full = bars, fix = bars + 8, s_full = bars + 24, dp_full = bars + 32, p_full = bars + 40,
                   ds_full = bars + 48, done = bars + 56, q_full = bars + 80, q_empty = q_full + 8 * L::XS,
                   do_full = q_empty + 8 * L::XS, do_empty = do_full + 8 * L::YS,
                   st_full = do_empty + 8 * L::YS, st_empty = st_full + 8 * L::SS;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    const int64_t heads = a.batch * a.kv_heads;
    const int j0 = (int)(blockIdx.x / heads) * T;                   // the first keys of a causal bound have most queries
    const int64_t bg = blockIdx.x % heads, b = bg / a.kv_heads;
    const int g = (int)(bg % a.kv_heads);
    const AttnSeq s = attn_seq(a, b);
    int first = 0, per_head = 0;
    if (j0 < s.nk) {
        const int lo = attn_q_first(a, s, j0), hi = attn_q_last(a, s, min(j0 + T, s.nk));
        if (lo < hi) {
            first = lo / T;
            per_head = (hi + T - 1) / T - first;
        }
    }
    const int n = per_head * a.group;                               // steps: query heads of the group x their tiles

    if (threadIdx.x == 0) {
        stalled = 0;
        bar_init(kv_full, 1);
        bar_init(fix, 1);
        bar_init(fix + 8, 1);
        bar_init(s_full, 1);
        bar_init(dp_full, 1);
        bar_init(p_full, 256);
        bar_init(ds_full, 256);
        bar_init(done, 1);
        for (int i = 0; i < 2 * (L::XS + L::YS); ++i) bar_init(q_full + 8 * i, 1);
        for (int i = 0; i < L::SS; ++i) {
            bar_init(st_full + 8 * i, 32);
            bar_init(st_empty + 8 * i, 256);
        }
        fence_barrier_init();
    }
    if (warp == 8) tmem_alloc(smem_u32(&tmem_base), 512);
    if (warp == 9 && lane == 0) {
        tma_prefetch(&maps.q);
        tma_prefetch(&maps.k);
        tma_prefetch(&maps.v);
        tma_prefetch(&maps.dout);
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = tmem_base;                                // S^T, dP^T, dV, dK

    if (warp == 9) {
        if (n > 0) {
            if (lane == 0) {
                bar_expect(kv_full, 2 * L::TILE);
                load_tile<DP>(base + L::A, &maps.k, kv_full, j0, g, (int)b);
                load_tile<DP>(base + L::B, &maps.v, kv_full, j0, g, (int)b);
            }
            bool ok = true;
            uint32_t patched = 0;
            for (int i = 0; i < n && ok; ++i) {
                const int qst = i % L::XS, ost = i % L::YS;
                const int r0 = (first + i % per_head) * T, h = g * a.group + i / per_head;
                const uint32_t qt = base + L::X + qst * L::TILE, dt = base + L::Y + ost * L::TILE;
                const bool patch = s.nq < a.q_len && r0 + T > s.nq;        // both are summed over their rows
                if (i >= L::XS) ok = __all_sync(0xffffffffu, bar_wait(q_empty + 8 * qst, (i / L::XS - 1) & 1, &stalled));
                if (!ok) break;
                if (lane == 0) {
                    const uint32_t bar = patch ? fix : q_full + 8 * qst;
                    bar_expect(bar, L::TILE);
                    load_tile<DP>(qt, &maps.q, bar, r0, h, (int)b);
                }
                if (i >= L::YS) ok = __all_sync(0xffffffffu, bar_wait(do_empty + 8 * ost, (i / L::YS - 1) & 1, &stalled));
                if (!ok) break;
                if (lane == 0) {
                    const uint32_t bar = patch ? fix + 8 : do_full + 8 * ost;
                    bar_expect(bar, L::TILE);
                    load_tile<DP>(dt, &maps.dout, bar, r0, h, (int)b);
                }
                if (patch) {
                    ok = patch_tile<DP>(qt, s.nq - r0, fix, patched, q_full + 8 * qst, &stalled) &&
                         patch_tile<DP>(dt, s.nq - r0, fix + 8, patched, do_full + 8 * ost, &stalled);
                    patched ^= 1;
                }
            }
        }
    } else if (warp == 8) {
        if (n > 0) {
            const bool one = elect_one();
            constexpr uint32_t DESC_S = mma_desc(BF16, T, T, false), DESC_G = mma_desc(BF16, T, DP, true);
            auto qt = [&](int i) { return base + L::X + (i % L::XS) * L::TILE; };
            auto dt = [&](int i) { return base + L::Y + (i % L::YS) * L::TILE; };
            auto q_here = [&](int i) { return bar_wait(q_full + 8 * (i % L::XS), (i / L::XS) & 1, &stalled); };
            auto do_here = [&](int i) { return bar_wait(do_full + 8 * (i % L::YS), (i / L::YS) & 1, &stalled); };
            bool ok = __all_sync(0xffffffffu, bar_wait(kv_full, 0, &stalled) && q_here(0));
            if (ok) {
                fence_after();
                if (one) {
                    mul_values<DP>(tmem, base + L::A, qt(0), DESC_S);
                    mma_commit(s_full);
                }
                ok = __all_sync(0xffffffffu, do_here(0));
            }
            if (ok) {
                fence_after();
                if (one) {
                    mul_values<DP>(tmem + 128, base + L::B, dt(0), DESC_S);
                    mma_commit(dp_full);
                }
            }
            for (int i = 0; i < n && ok; ++i) {
                ok = __all_sync(0xffffffffu, bar_wait(p_full, i & 1, &stalled));
                if (!ok) break;
                fence_after();
                if (one) {
                    mul_rows(tmem + 256, tmem, dt(i), DESC_G, i > 0);
                    mma_commit(do_empty + 8 * (i % L::YS));
                }
                if (i + 1 < n) {
                    ok = __all_sync(0xffffffffu, q_here(i + 1));
                    if (!ok) break;
                    fence_after();
                    if (one) {
                        mul_values<DP>(tmem, base + L::A, qt(i + 1), DESC_S);
                        mma_commit(s_full);
                    }
                }
                ok = __all_sync(0xffffffffu, bar_wait(ds_full, i & 1, &stalled));
                if (!ok) break;
                fence_after();
                if (one) {
                    mul_rows(tmem + 384, tmem + 128, qt(i), DESC_G, i > 0);
                    mma_commit(q_empty + 8 * (i % L::XS));
                }
                if (i + 1 < n) {
                    ok = __all_sync(0xffffffffu, do_here(i + 1));
                    if (!ok) break;
                    fence_after();
                    if (one) {
                        mul_values<DP>(tmem + 128, base + L::B, dt(i + 1), DESC_S);
                        mma_commit(dp_full);
                    }
                }
            }
            if (ok && one) mma_commit(done);
        }
        __syncwarp();
    } else if (warp == 10) {
        // lse (in units of log2; +inf where p is to be 0) and delta of each step's 128 queries
        bool ok = true;
        for (int i = 0; i < n && ok; ++i) {
            const int st = i % L::SS;
            const int r0 = (first + i % per_head) * T, h = g * a.group + i / per_head;
            const int64_t at = (b * a.q_heads + h) * a.q_len;
            float l[4], d[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int r = r0 + lane + 32 * x;
                l[x] = r < s.nq ? a.lse[at + r] * LOG2E : INFINITY;
                d[x] = r < s.nq ? a.delta[at + r] : 0.f;
                if (l[x] == -INFINITY) l[x] = INFINITY;              // a row that sees nothing
            }
            if (i >= L::SS) ok = __all_sync(0xffffffffu, bar_wait(st_empty + 8 * st, (i / L::SS - 1) & 1, &stalled));
            if (!ok) break;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                stats[st * 256 + lane + 32 * x] = -l[x];
                stats[st * 256 + 128 + lane + 32 * x] = -d[x];
            }
            bar_arrive(st_full + 8 * st);
        }
    } else if (warp < 8) {
        const int half = warp >> 2;                                 // queries [64 half, 64 half + 64) of a tile
        const int j = j0 + (threadIdx.x & 127);
        const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
        const bool row = j < s.nk;
        const int lo = row ? attn_q_first(a, s, j) : 0, hi = row ? attn_q_last(a, s, j + 1) : 0;
        // query tiles inside [whole_lo, whole_hi) are seen whole by every key of this block
        const int whole_lo = attn_q_first(a, s, min(j0 + T, s.nk) - 1), whole_hi = attn_q_last(a, s, j0 + 1);
        const float mul = a.scale * LOG2E;
        float up = 1.f;
        if constexpr (!BF16) up = ds_scale(a, norms, b, g * a.group, (g + 1) * a.group, g);
        const uint32_t ts = tmem + lanes + 64 * half, td = ts + 128;
        bool ok = true;
        for (int i = 0; i < n; ++i) {
            const int st = i % L::SS, r0 = (first + i % per_head) * T;
            const float *neg_lse = stats + st * 256 + 64 * half, *neg_delta = neg_lse + 128;
            ok = __all_sync(0xffffffffu, bar_wait(st_full + 8 * st, (i / L::SS) & 1, &stalled) &&
                                             bar_wait(s_full, i & 1, &stalled));
            if (!ok) break;
            fence_after();
            float x[64];
            tmem_ld32(ts, reinterpret_cast<uint32_t *>(x));
            tmem_ld32(ts + 32, reinterpret_cast<uint32_t *>(x) + 32);
            wait_ld();
#pragma unroll
            for (int c = 0; c < 64; c += 4) {
                const float4 l = *reinterpret_cast<const float4 *>(neg_lse + c);
                const float2 e = fma2(make_float2(x[c], x[c + 1]), make_float2(mul, mul), make_float2(l.x, l.y));
                const float2 f = fma2(make_float2(x[c + 2], x[c + 3]), make_float2(mul, mul), make_float2(l.z, l.w));
                x[c] = exp2_fast(e.x);
                x[c + 1] = exp2_fast(e.y);
                x[c + 2] = exp2_fast(f.x);
                x[c + 3] = exp2_fast(f.y);
            }
            if (r0 < whole_lo || r0 + T > whole_hi) {
                const int c0 = lo - r0 - 64 * half, c1 = hi - r0 - 64 * half;
#pragma unroll
                for (int c = 0; c < 64; ++c) x[c] = c >= c0 && c < c1 ? x[c] : 0.f;
            }
            {
                uint32_t u[32];
#pragma unroll
                for (int c = 0; c < 32; ++c)
                    u[c] = BF16 ? pack2<BF16>(x[2 * c], x[2 * c + 1]) : pack2<BF16>(x[2 * c] * 32768.f, x[2 * c + 1] * 32768.f);
                tmem_st32(ts, u);
            }
            wait_st();
            fence_before();
            bar_arrive(p_full);
            ok = __all_sync(0xffffffffu, bar_wait(dp_full, i & 1, &stalled));
            if (!ok) break;
            fence_after();
            uint32_t u[32];
#pragma unroll
            for (int c0 = 0; c0 < 64; c0 += 32) {
                float dp[32];
                tmem_ld32(td + c0, reinterpret_cast<uint32_t *>(dp));
                wait_ld();
#pragma unroll
                for (int c = 0; c < 32; c += 4) {
                    const float4 dl = *reinterpret_cast<const float4 *>(neg_delta + c0 + c);
                    float2 p = make_float2(x[c0 + c], x[c0 + c + 1]), q = make_float2(x[c0 + c + 2], x[c0 + c + 3]);
                    if constexpr (!BF16) {
                        p = mul2(p, make_float2(up, up));
                        q = mul2(q, make_float2(up, up));
                    }
                    p = mul2(p, add2(make_float2(dp[c], dp[c + 1]), make_float2(dl.x, dl.y)));
                    q = mul2(q, add2(make_float2(dp[c + 2], dp[c + 3]), make_float2(dl.z, dl.w)));
                    u[(c0 + c) / 2] = pack2<BF16>(p.x, p.y);
                    u[(c0 + c) / 2 + 1] = pack2<BF16>(q.x, q.y);
                }
            }
            tmem_st32(td, u);
            wait_st();
            fence_before();
            bar_arrive(ds_full);
            bar_arrive(st_empty + 8 * st);
        }
        if (ok && n > 0) ok = __all_sync(0xffffffffu, bar_wait(done, 0, &stalled));
        fence_after();
        // the first four warps store dV, the others dK
        const AttnTensor &to = half == 0 ? a.dv : a.dk;
        float factor = half == 0 ? (BF16 ? 1.f : 1.f / 32768.f) : a.scale / up;
        if (!row || n == 0) factor = 0.f;
        uint16_t *out = reinterpret_cast<uint16_t *>(to.p) + b * to.sb + (int64_t)j * to.sl + g * to.sh;
        const bool vec = rows16(to, a.dim);
#pragma unroll
        for (int c = 0; c < DP; c += 32) {
            float o[32];
            __syncwarp();
            if (n > 0 && ok) {
                tmem_ld32(tmem + lanes + 256 + 128 * half + c, reinterpret_cast<uint32_t *>(o));
                wait_ld();
            }
            if (j < a.k_len) store32<BF16>(out, c, a.dim, vec, o, factor);
        }
    }

    fence_before();
    __syncthreads();
    fence_after();
    if (stalled) drain_stalled(stalls);
    if (warp == 8) tmem_free(tmem, 512);
}

static int64_t tiles_of(int64_t n) { return (n + T - 1) / T; }

int64_t attn_tc_backward_work(int64_t batch, int32_t q_len, int32_t k_len, int32_t q_heads, int32_t kv_heads)
{
    return batch * q_heads * tiles_of(q_len) + batch * kv_heads * tiles_of(k_len);
}

bool attn_tc_backward_ok(const AttnArgs &a)
{
    return a.dtype != GS_TABLE_F32 && a.batch < ((int64_t)1 << 31) && attn_tma_ok(a.q, a.batch, a.q_len, a.q_heads) &&
           attn_tma_ok(a.dout, a.batch, a.q_len, a.q_heads) && attn_tma_ok(a.k, a.batch, a.k_len, a.kv_heads) &&
           attn_tma_ok(a.v, a.batch, a.k_len, a.kv_heads);
}

template <bool BF16, int DP>
static gs_status backward_t(const AttnArgs &a, const BwdMaps &maps, const BwdNorms &norms, cudaStream_t st)
{
    const int64_t q_blocks = a.batch * a.q_heads * tiles_of(a.q_len), k_blocks = a.batch * a.kv_heads * tiles_of(a.k_len);
    if (q_blocks + k_blocks > 0x7FFFFFFF) {
        set_error("attention of %lld row tiles exceeds one launch", (long long)(q_blocks + k_blocks));
        return GS_ERR_UNSUPPORTED;
    }
    unsigned long long *stalls = stall_counter();
    if (!BF16) {
        attn_tc_norms_kernel<<<(unsigned)(q_blocks + k_blocks), 128, 0, st>>>(a, norms);
        GS_CUDA_TRY(cudaGetLastError());
    }
    constexpr int smem = BwdSmem<DP>::BYTES;
    static SharedRecord record[2];
    gs_status s;
    if ((s = allow_shared(attn_tc_dq_kernel<BF16, DP>, smem, record[0])) != GS_OK ||
        (s = allow_shared(attn_tc_dkdv_kernel<BF16, DP>, smem, record[1])) != GS_OK)
        return s;
    attn_tc_dq_kernel<BF16, DP><<<(unsigned)q_blocks, 384, smem, st>>>(a, maps, norms, stalls);
    GS_CUDA_TRY(cudaGetLastError());
    attn_tc_dkdv_kernel<BF16, DP><<<(unsigned)k_blocks, 384, smem, st>>>(a, maps, norms, stalls);
    GS_CUDA_TRY(cudaGetLastError());
    return GS_OK;
}

gs_status attn_tc_backward(const AttnArgs &a, cudaStream_t st)
{
    const bool bf16 = a.dtype == GS_TABLE_BF16;
    BwdMaps m;
    gs_status s;
    if ((s = attn_tensor_map(&m.q, a.q, bf16, a.batch, a.q_len, a.q_heads, a.dim, 64, 128)) != GS_OK) return s;
    if ((s = attn_tensor_map(&m.dout, a.dout, bf16, a.batch, a.q_len, a.q_heads, a.dim, 64, 128)) != GS_OK) return s;
    if ((s = attn_tensor_map(&m.k, a.k, bf16, a.batch, a.k_len, a.kv_heads, a.dim, 64, 128)) != GS_OK) return s;
    if ((s = attn_tensor_map(&m.v, a.v, bf16, a.batch, a.k_len, a.kv_heads, a.dim, 64, 128)) != GS_OK) return s;
    BwdNorms nm;
    nm.dout = a.delta + a.batch * a.q_heads * (int64_t)a.q_len;
    nm.v = nm.dout + a.batch * a.q_heads * tiles_of(a.q_len);
    if (a.dim <= 64) return bf16 ? backward_t<true, 64>(a, m, nm, st) : backward_t<false, 64>(a, m, nm, st);
    return bf16 ? backward_t<true, 128>(a, m, nm, st) : backward_t<false, 128>(a, m, nm, st);
}

}  // namespace gs
