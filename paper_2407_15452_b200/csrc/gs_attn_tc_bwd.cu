// Backward attention of 16-bit tensors on the fifth-generation tensor cores: two kernels that both
// compute the scores again, so that every gradient has one owner and no value is summed with atomics
// (seven products of 128 x 128 tiles where a single kernel with atomics on dq needs five).
//
//  dq     : an item is 128 query rows.  S = Q K^T, dP = dO V^T, dS = P (dP - delta), dQ += dS K.
//           Thread = query row; S of the next keys is computed while this one's dS is formed, dP's columns are
//           free for the next product as soon as they are in registers.
//  dk, dv : an item is 128 keys, with the query heads of their group and their query tiles.
//           Everything transposed: S^T = K Q^T, dP^T = V dO^T, so that P^T and dS^T come out with one key per
//           lane and feed dV += P^T dO, dK += dS^T Q from tensor memory without passing through shared memory.
//           Tensor memory is full (S^T, dP^T, dV, dK: 128 columns each); the order dV(i), S^T(i+1) while dS(i)
//           is formed, then dK(i), dP^T(i+1) while P(i+1) is formed, keeps both sides busy.
// One block per SM goes through items; loads and products of the next item run while
// the last one's results are stored.  Eight warps do the elementwise part, four per 64 columns of a tile; a
// warp overwrites only columns that it has read itself.  Warp 8 issues the products, warp 9 loads and
// asks for the next item, warp 10 brings the row statistics.  A first kernel works out delta = dO.O.
//
// P and dS are rounded to the tensors' type for their products.  binary16 has no range for that as it
// stands: P is scaled by 2^15 (P <= 1), dS by the power of two that brings its bound
// |dS| <= 2 max|do| max|v| (row norms) near 2^15; the first kernel finds the norms too then.
#include "gs_attn_again.cuh"
#include "gs_attn_tc.cuh"

namespace gs {

using namespace tc;

static constexpr int T = 128;                     // rows of every tile
static constexpr int THREADS = 384;

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
    static constexpr int STATS = Y + YS * TILE;                 // SS of: -lse (log2) and -delta of a query tile, scale of dS
    static constexpr int STAT = 2 * T + 4;                      // floats of one
    static constexpr int BARS = STATS + SS * STAT * 4;
    static constexpr int QUEUE = (BARS + 8 * (12 + 2 * XS + 2 * YS + 2 * SS) + 15) / 16 * 16;      // answers and barriers of the items
    static constexpr int WORDS = QUEUE + 64;                    // stalled, address of the tensor memory
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

template <bool BF16>
__device__ __forceinline__ float2 unpack2(uint32_t u)
{
    if constexpr (BF16) return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
    else return __half22float2(*reinterpret_cast<__half2 *>(&u));
}

// dot product of the first min(8, n) values at two addresses, 16-byte aligned
template <bool BF16>
__device__ __forceinline__ float dot8(const uint16_t *x, const uint16_t *y, int n)
{
    float d = 0.f;
    if (n >= 8) {
        const uint4 u = __ldg(reinterpret_cast<const uint4 *>(x)), w = __ldg(reinterpret_cast<const uint4 *>(y));
        const uint32_t p[4] = {u.x, u.y, u.z, u.w}, q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = unpack2<BF16>(p[i]), g = unpack2<BF16>(q[i]);
            d = fmaf(f.x, g.x, d);
            d = fmaf(f.y, g.y, d);
        }
    } else {
        for (int i = 0; i < n; ++i) d = fmaf(unpack2<BF16>(x[i]).x, unpack2<BF16>(y[i]).x, d);
    }
    return d;
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v)
{
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Before the products: delta = dO.O of every query row and, for binary16, the largest row norm of each 128-row tile
// of dO and V.  One block per tile, DP / 8 lanes per row, all of a thread's loads on their way at once.
template <bool BF16, int DP>
__global__ void __launch_bounds__(256) attn_tc_prepare_kernel(const __grid_constant__ AttnArgs a, BwdNorms nm)
{
    constexpr int LANES = DP / 8, STEP = 256 / LANES, ROUNDS = T / STEP;
    cudaTriggerProgrammaticLaunchCompletion();                  // the dq kernel may set itself up meanwhile
    const int qt = (a.q_len + T - 1) / T, kt = (a.k_len + T - 1) / T;
    int64_t i = blockIdx.x;
    const int64_t nq = a.batch * a.q_heads * qt;
    const bool on_q = i < nq;
    if (!on_q) i -= nq;                                         // only binary16 has these blocks
    const int tiles = on_q ? qt : kt, nh = on_q ? a.q_heads : a.kv_heads;
    const int tile = (int)(i % tiles);
    const int64_t bh = i / tiles, b = bh / nh;
    const int h = (int)(bh % nh);
    const AttnSeq s = attn_seq(a, b);
    const int end = on_q ? s.nq : s.nk, col = ((int)threadIdx.x % LANES) * 8, n = a.dim - col;
    const AttnTensor &t = on_q ? a.dout : a.v;                  // both can be read by TMA: rows are aligned to 16 bytes
    const uint16_t *x = reinterpret_cast<const uint16_t *>(t.p) + b * t.sb + h * t.sh + col;
    const uint16_t *o = reinterpret_cast<const uint16_t *>(a.out.p) + b * a.out.sb + h * a.out.sh + col;
    const bool vec = rows16(a.out, a.dim);
    float top = 0.f, delta[ROUNDS], norm[ROUNDS];
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) {
        const int r = tile * T + (int)threadIdx.x / LANES + k * STEP;
        delta[k] = norm[k] = 0.f;
        if (r < end) {
            const uint16_t *y = x + (int64_t)r * t.sl, *z = o + (int64_t)r * a.out.sl;
            if (!BF16) norm[k] = dot8<BF16>(y, y, n);
            if (on_q && vec) delta[k] = dot8<BF16>(y, z, n);
            else if (on_q)
                for (int e = 0; e < min(8, n); ++e) delta[k] = fmaf(unpack2<BF16>(y[e]).x, unpack2<BF16>(z[e]).x, delta[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) {
        const int r = tile * T + (int)threadIdx.x / LANES + k * STEP;
        if (!BF16) {                              // a row that is not finite must not cost the others their scale
            const float n2 = lanes_sum<LANES>(norm[k]);
            top = fmaxf(top, n2 < INFINITY ? n2 : 0.f);
        }
        const float d = lanes_sum<LANES>(delta[k]);
        if (on_q && threadIdx.x % LANES == 0 && r < a.q_len) a.delta[bh * a.q_len + r] = d;
    }
    if constexpr (!BF16) {
        __shared__ float sh[8];
        top = warp_max(top);
        if (threadIdx.x % 32 == 0) sh[threadIdx.x >> 5] = top;
        __syncthreads();
        if (threadIdx.x == 0) {
#pragma unroll
            for (int w = 0; w < 8; ++w) top = fmaxf(top, sh[w]);
            (on_q ? nm.dout : nm.v)[i] = sqrtf(top);
        }
    }
}

struct DqItem {
    AttnSeq s;
    int b, h, g, r0;
    int first, n;                                               // key tiles
    __device__ __forceinline__ DqItem(const AttnArgs &a, uint32_t i)
    {
        const uint32_t heads = (uint32_t)a.batch * a.q_heads, tile = i / heads, bh = i - tile * heads;
        h = (int)(bh / (uint32_t)a.batch);                    // neighbours in the list are other sequences: lengths mix
        b = (int)(bh - (uint32_t)h * (uint32_t)a.batch);
        g = h / a.group;
        s = attn_seq(a, b);
        r0 = ((a.q_len + T - 1) / T - 1 - (int)tile) * T;       // the last rows of a causal bound are the longest
        first = n = 0;
        if (r0 < s.nq) {
            const int lo = attn_lo(a, s, r0), hi = attn_hi(a, s, min(r0 + T, s.nq) - 1);
            if (lo < hi) {
                first = lo / T;
                n = (hi + T - 1) / T - first;
            }
        }
    }
};

template <bool BF16, int DP>
__global__ void __launch_bounds__(THREADS, 1)
attn_tc_dq_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ BwdMaps maps, const BwdNorms norms,
                  uint32_t count, unsigned long long *stalls)
{
    using L = BwdSmem<DP>;
    extern __shared__ __align__(1024) uint8_t smem[];           // no static shared memory: this starts at its beginning
    const uint32_t base = smem_u32(smem);
    float *stats = reinterpret_cast<float *>(smem + L::STATS);
    volatile int &stalled = *reinterpret_cast<volatile int *>(smem + L::WORDS);
    uint32_t &tmem_base = *reinterpret_cast<uint32_t *>(smem + L::WORDS + 4);
    const uint32_t bars = base + L::BARS;
    const uint32_t q_full = bars, q_empty = bars + 8, fix = bars + 16, s_full = bars + 24, dp_full = bars + 40, dp_free = bars + 48,
                   ds_full = bars + 56, done = bars + 64, dq_empty = bars + 72, k_full = bars + 96, k_empty = k_full + 8 * L::XS,
                   v_full = k_empty + 8 * L::XS, v_empty = v_full + 8 * L::YS, st_full = v_empty + 8 * L::YS,
                   st_empty = st_full + 8 * L::SS;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const ItemQueue queue{count, base + L::QUEUE, base + L::QUEUE + 32, base + L::QUEUE + 48, &stalled};

    if (threadIdx.x == 0) {
        stalled = 0;
        queue.init(10);                               // warps 0-8 and 10
        bar_init(q_full, 1);
        bar_init(q_empty, 1);
        bar_init(fix, 1);
        bar_init(s_full, 1);
        bar_init(s_full + 8, 1);
        bar_init(dp_full, 1);
        bar_init(dp_free, 256);
        bar_init(ds_full, 256);
        bar_init(done, 1);
        bar_init(dq_empty, 256);
        for (int i = 0; i < 2 * (L::XS + L::YS); ++i) bar_init(k_full + 8 * i, 1);
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
    const uint32_t tmem = tmem_base;                  // S of even and odd steps, dP, dQ

    // c counts a block's steps (key tiles) over all its items, t the items that have any
    bool ok = true;
    int c = 0, t = 0;
    if (warp == 9) {
        uint32_t patched = 0;
        for (Items<true> it(queue); it.more() && ok; it.next()) {
            const DqItem w(a, it.at);
            if (w.n == 0) continue;
            if (t > 0) ok = __all_sync(0xffffffffu, bar_wait(q_empty, (t - 1) & 1, &stalled));
            ++t;
            if (ok && lane == 0) {
                bar_expect(q_full, 2 * L::TILE);
                load_tile<DP>(base + L::A, &maps.q, q_full, w.r0, w.h, w.b);
                load_tile<DP>(base + L::B, &maps.dout, q_full, w.r0, w.h, w.b);
            }
            for (int i = 0; i < w.n && ok; ++i, ++c) {
                const int kst = c % L::XS, vst = c % L::YS, j0 = (w.first + i) * T;
                const uint32_t kt = base + L::X + kst * L::TILE, vt = base + L::Y + vst * L::TILE;
                const bool patch = w.s.nk < a.k_len && j0 + T > w.s.nk;        // K is summed over its rows in dS K
                if (c >= L::XS) ok = __all_sync(0xffffffffu, bar_wait(k_empty + 8 * kst, (c / L::XS - 1) & 1, &stalled));
                if (!ok) break;
                if (lane == 0) {
                    const uint32_t bar = patch ? fix : k_full + 8 * kst;
                    bar_expect(bar, L::TILE);
                    load_tile<DP>(kt, &maps.k, bar, j0, w.g, w.b);
                }
                if (c >= L::YS) ok = __all_sync(0xffffffffu, bar_wait(v_empty + 8 * vst, (c / L::YS - 1) & 1, &stalled));
                if (!ok) break;
                if (lane == 0) {
                    bar_expect(v_full + 8 * vst, L::TILE);
                    load_tile<DP>(vt, &maps.v, v_full + 8 * vst, j0, w.g, w.b);
                }
                if (patch) {
                    ok = patch_tile<DP>(kt, w.s.nk - j0, fix, patched, k_full + 8 * kst, &stalled);
                    patched ^= 1;
                }
            }
        }
    } else if (warp == 8) {
        const bool one = elect_one();
        constexpr uint32_t DESC_S = mma_desc(BF16, T, T, false), DESC_Q = mma_desc(BF16, T, DP, true);
        auto kt = [&](int x) { return base + L::X + (x % L::XS) * L::TILE; };
        // S and dP of step x
        auto scores = [&](int x) {
            ok = __all_sync(0xffffffffu, bar_wait(k_full + 8 * (x % L::XS), (x / L::XS) & 1, &stalled));
            if (!ok) return;
            fence_after();
            if (one) {                                // this S: its last dS went into dQ(x - 2), issued before
                mul_values<DP>(tmem + 128 * (x & 1), base + L::A, kt(x), DESC_S);
                mma_commit(s_full + 8 * (x & 1));
            }
            ok = bar_wait(v_full + 8 * (x % L::YS), (x / L::YS) & 1, &stalled);
            if (x > 0) ok = bar_wait(dp_free, (x - 1) & 1, &stalled) && ok;
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) return;
            fence_after();
            if (one) {
                mul_values<DP>(tmem + 256, base + L::B, base + L::Y + (x % L::YS) * L::TILE, DESC_S);
                mma_commit(dp_full);
                mma_commit(v_empty + 8 * (x % L::YS));
            }
        };
        for (Items<false> it(queue); it.more() && ok; it.next()) {
            const DqItem w(a, it.at);
            if (w.n == 0) continue;
            ok = __all_sync(0xffffffffu, bar_wait(q_full, t & 1, &stalled));
            if (ok) scores(c);
            for (int i = 0; i < w.n && ok; ++i, ++c) {
                if (i + 1 < w.n) scores(c + 1);
                if (i == max(w.n - 2, 0) && ok && one) mma_commit(q_empty);       // Q and dO have met all their keys
                if (ok) ok = bar_wait(ds_full, c & 1, &stalled);
                if (i == 0 && t > 0) ok = bar_wait(dq_empty, (t - 1) & 1, &stalled) && ok;      // the last item's dQ has been read
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                fence_after();
                if (one) {
                    mul_rows(tmem + 384, tmem + 128 * (c & 1), kt(c), DESC_Q, i > 0);
                    mma_commit(k_empty + 8 * (c % L::XS));
                    if (i + 1 == w.n) mma_commit(done);
                }
            }
            ++t;
        }
        __syncwarp();
    } else if (warp == 10) {
        // -lse in units of log2, -delta and the scale of dS of each item's rows
        cudaGridDependencySynchronize();              // delta and the norms; nobody else here reads what the first kernel writes
        cudaTriggerProgrammaticLaunchCompletion();
        for (Items<false> it(queue); it.more() && ok; it.next()) {
            const DqItem w(a, it.at);
            if (w.n == 0) continue;
            const int st = t % L::SS;
            const int64_t at = ((int64_t)w.b * a.q_heads + w.h) * a.q_len;
            float l[4], d[4], up = 1.f;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int r = w.r0 + lane + 32 * x;
                l[x] = r < w.s.nq ? -a.lse[at + r] * LOG2E : 0.f;
                d[x] = r < w.s.nq ? -a.delta[at + r] : 0.f;
            }
            if constexpr (!BF16) up = ds_scale(a, norms, w.b, w.h, w.h + 1, w.g);
            if (t >= L::SS) ok = __all_sync(0xffffffffu, bar_wait(st_empty + 8 * st, (t / L::SS - 1) & 1, &stalled));
            ++t;
            if (!ok) break;
            float *to = stats + st * L::STAT;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                to[lane + 32 * x] = l[x];
                to[T + lane + 32 * x] = d[x];
            }
            if (lane == 0) to[2 * T] = up;
            bar_arrive(st_full + 8 * st);
        }
    } else if (warp < 8) {
        const int half = warp >> 2;                   // columns [64 half, 64 half + 64)
        const int lane_row = threadIdx.x & 127;
        const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
        const float mul = a.scale * LOG2E;
        const bool vec = rows16(a.dq, a.dim);
        for (Items<false> it(queue); it.more() && ok; it.next()) {
            const DqItem w(a, it.at);
            const AttnSeq &s = w.s;
            const int r = w.r0 + lane_row;
            const bool row = r < s.nq;
            const int lo = row ? attn_lo(a, s, r) : 0, hi = row ? attn_hi(a, s, r) : 0;
            // key tiles inside [whole_lo, whole_hi) are seen whole by every row
            const bool whole = w.r0 + T <= s.nq;
            const int whole_lo = whole ? attn_lo(a, s, w.r0 + T - 1) : s.nk, whole_hi = attn_hi(a, s, w.r0);
            float neg_lse = 0.f, neg_delta = 0.f, up = 1.f;
            if (w.n > 0) {
                const int st = t % L::SS;
                ok = __all_sync(0xffffffffu, bar_wait(st_full + 8 * st, (t / L::SS) & 1, &stalled));
                neg_lse = stats[st * L::STAT + lane_row];
                neg_delta = stats[st * L::STAT + T + lane_row];
                if constexpr (!BF16) up = stats[st * L::STAT + 2 * T];
                bar_arrive(st_empty + 8 * st);
            }
            for (int i = 0; i < w.n && ok; ++i, ++c) {
                ok = __all_sync(0xffffffffu, bar_wait(s_full + 8 * (c & 1), (c >> 1) & 1, &stalled) &&
                                                 bar_wait(dp_full, c & 1, &stalled));
                if (!ok) break;
                fence_after();
                float x[64], dp[64];
                const uint32_t ts = tmem + lanes + 128 * (c & 1) + 64 * half, td = tmem + lanes + 256 + 64 * half;
                tmem_ld32(td, reinterpret_cast<uint32_t *>(dp));
                tmem_ld32(td + 32, reinterpret_cast<uint32_t *>(dp) + 32);
                tmem_ld32(ts, reinterpret_cast<uint32_t *>(x));
                tmem_ld32(ts + 32, reinterpret_cast<uint32_t *>(x) + 32);
                wait_ld();
                fence_before();
                bar_arrive(dp_free);
                const int j0 = (w.first + i) * T;
#pragma unroll
                for (int k = 0; k < 64; k += 2) {
                    const float2 e = fma2(make_float2(x[k], x[k + 1]), make_float2(mul, mul), make_float2(neg_lse, neg_lse));
                    float2 p = make_float2(exp2_fast(e.x), exp2_fast(e.y));
                    if constexpr (!BF16) p = mul2(p, make_float2(up, up));
                    const float2 d = mul2(p, add2(make_float2(dp[k], dp[k + 1]), make_float2(neg_delta, neg_delta)));
                    x[k] = d.x;
                    x[k + 1] = d.y;
                }
                if (j0 < whole_lo || j0 + T > whole_hi) {
                    const int c0 = lo - j0 - 64 * half, c1 = hi - j0 - 64 * half;
#pragma unroll
                    for (int k = 0; k < 64; ++k) x[k] = k >= c0 && k < c1 ? x[k] : 0.f;
                }
                uint32_t u[32];
#pragma unroll
                for (int k = 0; k < 32; ++k) u[k] = pack2<BF16>(x[2 * k], x[2 * k + 1]);
                tmem_st32(ts, u);
                wait_st();
                fence_before();
                bar_arrive(ds_full);
            }
            if (ok && w.n > 0) ok = __all_sync(0xffffffffu, bar_wait(done, t & 1, &stalled));
            fence_after();
            const float factor = row && w.n > 0 ? a.scale / up : 0.f;
            uint16_t *out = reinterpret_cast<uint16_t *>(a.dq.p) + w.b * a.dq.sb + (int64_t)r * a.dq.sl + w.h * a.dq.sh;
            NanSums total;     // whether one of the row's values is NaN
#pragma unroll
            for (int k = 0; k < DP / 2; k += 32) {    // each half of the warps stores half of the columns
                float o[32];
                __syncwarp();
                if (w.n > 0 && ok) {
                    tmem_ld32(tmem + lanes + 384 + half * (DP / 2) + k, reinterpret_cast<uint32_t *>(o));
                    wait_ld();
                    if (k + 32 == DP / 2) {
                        fence_before();
                        bar_arrive(dq_empty);
                    }
                    total.add(o);
                }
                if (r < a.q_len) store32<BF16>(out, half * (DP / 2) + k, a.dim, vec, o, factor);
            }
            if (__any_sync(0xffffffffu, row && total.found())) {
                const int r32 = w.r0 + 32 * (warp & 3);
                again::query_gradients<typename Tensor16<BF16>::T>(a, w.b, w.h, r32, r32 + 32, half * (DP / 2), (half + 1) * (DP / 2));
            }
            if (w.n > 0) ++t;
        }
    }

    fence_before();
    __syncthreads();
    fence_after();
    if (stalled) drain_stalled(stalls);
    if (warp == 8) tmem_free(tmem, 512);
}

struct KvItem {
    AttnSeq s;
    int b, g, j0;
    int first, per_head, n;                                     // query tiles; steps: query heads of the group x their tiles
    __device__ __forceinline__ KvItem(const AttnArgs &a, uint32_t i)
    {
        const uint32_t heads = (uint32_t)a.batch * a.kv_heads, tile = i / heads, bg = i - tile * heads;
        g = (int)(bg / (uint32_t)a.batch);                    // neighbours in the list are other sequences: lengths mix
        b = (int)(bg - (uint32_t)g * (uint32_t)a.batch);
        s = attn_seq(a, b);
        j0 = (int)tile * T;                                     // the first keys of a causal bound have most queries
        first = per_head = 0;
        if (j0 < s.nk) {
            const int lo = attn_q_first(a, s, j0), hi = attn_q_last(a, s, min(j0 + T, s.nk));
            if (lo < hi) {
                first = lo / T;
                per_head = (hi + T - 1) / T - first;
            }
        }
        n = per_head * a.group;
    }
    // step i: query head and first row
    __device__ __forceinline__ int head(const AttnArgs &a, int i) const { return g * a.group + i / per_head; }
    __device__ __forceinline__ int row(int i) const { return (first + i % per_head) * T; }
};

template <bool BF16, int DP>
__global__ void __launch_bounds__(THREADS, 1)
attn_tc_dkdv_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ BwdMaps maps, const BwdNorms norms,
                    uint32_t count, unsigned long long *stalls)
{
    using L = BwdSmem<DP>;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    float *stats = reinterpret_cast<float *>(smem + L::STATS);
    volatile int &stalled = *reinterpret_cast<volatile int *>(smem + L::WORDS);
    uint32_t &tmem_base = *reinterpret_cast<uint32_t *>(smem + L::WORDS + 4);
    const uint32_t bars = base + L::BARS;
    const uint32_t kv_full = bars, kv_empty = bars + 8, fix = bars + 16, s_full = bars + 32, dp_full = bars + 40, p_full = bars + 48,
                   ds_full = bars + 56, done = bars + 64, acc_empty = bars + 72, q_full = bars + 96, q_empty = q_full + 8 * L::XS,
                   do_full = q_empty + 8 * L::XS, do_empty = do_full + 8 * L::YS,
                   st_full = do_empty + 8 * L::YS, st_empty = st_full + 8 * L::SS;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const ItemQueue queue{count, base + L::QUEUE, base + L::QUEUE + 32, base + L::QUEUE + 48, &stalled};

    if (threadIdx.x == 0) {
        stalled = 0;
        queue.init(10);
        bar_init(kv_full, 1);
        bar_init(kv_empty, 1);
        bar_init(fix, 1);
        bar_init(fix + 8, 1);
        bar_init(s_full, 1);
        bar_init(dp_full, 1);
        bar_init(p_full, 256);
        bar_init(ds_full, 256);
        bar_init(done, 1);
        bar_init(acc_empty, 256);
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

    // c counts a block's steps over all its items, t the items that have any
    bool ok = true;
    int c = 0, t = 0;
    if (warp == 9) {
        uint32_t patched = 0;
        for (Items<true> it(queue); it.more() && ok; it.next()) {
            const KvItem w(a, it.at);
            if (w.n == 0) continue;
            if (t > 0) ok = __all_sync(0xffffffffu, bar_wait(kv_empty, (t - 1) & 1, &stalled));
            ++t;
            if (ok && lane == 0) {
                bar_expect(kv_full, 2 * L::TILE);
                load_tile<DP>(base + L::A, &maps.k, kv_full, w.j0, w.g, w.b);
                load_tile<DP>(base + L::B, &maps.v, kv_full, w.j0, w.g, w.b);
            }
            for (int i = 0; i < w.n && ok; ++i, ++c) {
                const int qst = c % L::XS, ost = c % L::YS, r0 = w.row(i), h = w.head(a, i);
                const uint32_t qt = base + L::X + qst * L::TILE, dt = base + L::Y + ost * L::TILE;
                const bool patch = w.s.nq < a.q_len && r0 + T > w.s.nq;    // both are summed over their rows
                if (c >= L::XS) ok = __all_sync(0xffffffffu, bar_wait(q_empty + 8 * qst, (c / L::XS - 1) & 1, &stalled));
                if (!ok) break;
                if (lane == 0) {
                    const uint32_t bar = patch ? fix : q_full + 8 * qst;
                    bar_expect(bar, L::TILE);
                    load_tile<DP>(qt, &maps.q, bar, r0, h, w.b);
                }
                if (c >= L::YS) ok = __all_sync(0xffffffffu, bar_wait(do_empty + 8 * ost, (c / L::YS - 1) & 1, &stalled));
                if (!ok) break;
                if (lane == 0) {
                    const uint32_t bar = patch ? fix + 8 : do_full + 8 * ost;
                    bar_expect(bar, L::TILE);
                    load_tile<DP>(dt, &maps.dout, bar, r0, h, w.b);
                }
                if (patch) {
                    ok = patch_tile<DP>(qt, w.s.nq - r0, fix, patched, q_full + 8 * qst, &stalled) &&
                         patch_tile<DP>(dt, w.s.nq - r0, fix + 8, patched, do_full + 8 * ost, &stalled);
                    patched ^= 1;
                }
            }
        }
    } else if (warp == 8) {
        const bool one = elect_one();
        constexpr uint32_t DESC_S = mma_desc(BF16, T, T, false), DESC_G = mma_desc(BF16, T, DP, true);
        auto qt = [&](int x) { return base + L::X + (x % L::XS) * L::TILE; };
        auto dt = [&](int x) { return base + L::Y + (x % L::YS) * L::TILE; };
        auto scores = [&](int x) {                                  // S^T of step x
            ok = __all_sync(0xffffffffu, bar_wait(q_full + 8 * (x % L::XS), (x / L::XS) & 1, &stalled));
            if (!ok) return;
            fence_after();
            if (one) {
                mul_values<DP>(tmem, base + L::A, qt(x), DESC_S);
                mma_commit(s_full);
            }
        };
        auto dscores = [&](int x) {                                 // dP^T of step x
            ok = __all_sync(0xffffffffu, bar_wait(do_full + 8 * (x % L::YS), (x / L::YS) & 1, &stalled));
            if (!ok) return;
            fence_after();
            if (one) {
                mul_values<DP>(tmem + 128, base + L::B, dt(x), DESC_S);
                mma_commit(dp_full);
            }
        };
        for (Items<false> it(queue); it.more() && ok; it.next()) {
            const KvItem w(a, it.at);
            if (w.n == 0) continue;
            ok = __all_sync(0xffffffffu, bar_wait(kv_full, t & 1, &stalled));
            if (ok) scores(c);
            if (ok) dscores(c);
            if (w.n == 1 && ok && one) mma_commit(kv_empty);
            for (int i = 0; i < w.n && ok; ++i, ++c) {
                ok = bar_wait(p_full, c & 1, &stalled);
                if (i == 0 && t > 0) ok = bar_wait(acc_empty, (t - 1) & 1, &stalled) && ok;     // the last item's dV, dK have been read
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                fence_after();
                if (one) {
                    mul_rows(tmem + 256, tmem, dt(c), DESC_G, i > 0);
                    mma_commit(do_empty + 8 * (c % L::YS));
                }
                if (i + 1 < w.n) scores(c + 1);
                if (ok) ok = __all_sync(0xffffffffu, bar_wait(ds_full, c & 1, &stalled));
                if (!ok) break;
                fence_after();
                if (one) {
                    mul_rows(tmem + 384, tmem + 128, qt(c), DESC_G, i > 0);
                    mma_commit(q_empty + 8 * (c % L::XS));
                    if (i + 1 == w.n) mma_commit(done);
                }
                if (i + 1 < w.n) dscores(c + 1);
                if (i + 2 == w.n && ok && one) mma_commit(kv_empty);       // K and V have met all their queries
            }
            ++t;
        }
        __syncwarp();
    } else if (warp == 10) {
        // -lse (in units of log2; -inf where p is to be 0) and -delta of each step's 128 queries
        for (Items<false> it(queue); it.more() && ok; it.next()) {
            const KvItem w(a, it.at);
            float up = 1.f;
            if constexpr (!BF16) {
                if (w.n > 0) up = ds_scale(a, norms, w.b, w.g * a.group, (w.g + 1) * a.group, w.g);
            }
            for (int i = 0; i < w.n && ok; ++i, ++c) {
                const int st = c % L::SS, r0 = w.row(i);
                const int64_t at = ((int64_t)w.b * a.q_heads + w.head(a, i)) * a.q_len;
                float l[4], d[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int r = r0 + lane + 32 * x;
                    l[x] = r < w.s.nq ? -a.lse[at + r] * LOG2E : -INFINITY;
                    d[x] = r < w.s.nq ? -a.delta[at + r] : 0.f;
                    if (l[x] == INFINITY) l[x] = -INFINITY;          // a row that sees nothing
                }
                if (c >= L::SS) ok = __all_sync(0xffffffffu, bar_wait(st_empty + 8 * st, (c / L::SS - 1) & 1, &stalled));
                if (!ok) break;
                float *to = stats + st * L::STAT;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    to[lane + 32 * x] = l[x];
                    to[T + lane + 32 * x] = d[x];
                }
                if (lane == 0) to[2 * T] = up;
                bar_arrive(st_full + 8 * st);
            }
        }
    } else if (warp < 8) {
        const int half = warp >> 2;                                 // queries [64 half, 64 half + 64) of a tile
        const int lane_row = threadIdx.x & 127;
        const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
        const float mul = a.scale * LOG2E;
        const uint32_t ts = tmem + lanes + 64 * half, td = ts + 128;
        const AttnTensor &to = half == 0 ? a.dv : a.dk;             // the first four warps store dV, the others dK
        const bool vec = rows16(to, a.dim);
        for (Items<false> it(queue); it.more() && ok; it.next()) {
            const KvItem w(a, it.at);
            const AttnSeq &s = w.s;
            const int j = w.j0 + lane_row;
            const bool row = j < s.nk;
            const int lo = row ? attn_q_first(a, s, j) : 0, hi = row ? attn_q_last(a, s, j + 1) : 0;
            // query tiles inside [whole_lo, whole_hi) are seen whole by every key of this block
            const int whole_lo = attn_q_first(a, s, min(w.j0 + T, s.nk) - 1), whole_hi = attn_q_last(a, s, w.j0 + 1);
            float up = 1.f;
            int tile = 0;                                           // of the head: i % per_head
            for (int i = 0; i < w.n && ok; ++i, ++c) {
                const int st = c % L::SS, r0 = (w.first + tile) * T;
                if (++tile == w.per_head) tile = 0;
                const float *neg_lse = stats + st * L::STAT + 64 * half, *neg_delta = neg_lse + T;
                ok = __all_sync(0xffffffffu, bar_wait(st_full + 8 * st, (c / L::SS) & 1, &stalled) &&
                                                 bar_wait(s_full, c & 1, &stalled));
                if (!ok) break;
                fence_after();
                float x[64];
                tmem_ld32(ts, reinterpret_cast<uint32_t *>(x));
                tmem_ld32(ts + 32, reinterpret_cast<uint32_t *>(x) + 32);
                wait_ld();
#pragma unroll
                for (int k = 0; k < 64; k += 4) {
                    const float4 l = *reinterpret_cast<const float4 *>(neg_lse + k);
                    const float2 e = fma2(make_float2(x[k], x[k + 1]), make_float2(mul, mul), make_float2(l.x, l.y));
                    const float2 f = fma2(make_float2(x[k + 2], x[k + 3]), make_float2(mul, mul), make_float2(l.z, l.w));
                    x[k] = exp2_fast(e.x);
                    x[k + 1] = exp2_fast(e.y);
                    x[k + 2] = exp2_fast(f.x);
                    x[k + 3] = exp2_fast(f.y);
                }
                if (r0 < whole_lo || r0 + T > whole_hi) {
                    const int c0 = lo - r0 - 64 * half, c1 = hi - r0 - 64 * half;
#pragma unroll
                    for (int k = 0; k < 64; ++k) x[k] = k >= c0 && k < c1 ? x[k] : 0.f;
                }
                {
                    uint32_t u[32];
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        u[k] = BF16 ? pack2<BF16>(x[2 * k], x[2 * k + 1]) : pack2<BF16>(x[2 * k] * 32768.f, x[2 * k + 1] * 32768.f);
                    tmem_st32(ts, u);
                }
                wait_st();
                fence_before();
                bar_arrive(p_full);
                if constexpr (!BF16) up = stats[st * L::STAT + 2 * T];
                ok = __all_sync(0xffffffffu, bar_wait(dp_full, c & 1, &stalled));
                if (!ok) break;
                fence_after();
                uint32_t u[32];
#pragma unroll
                for (int k0 = 0; k0 < 64; k0 += 32) {
                    float dp[32];
                    tmem_ld32(td + k0, reinterpret_cast<uint32_t *>(dp));
                    wait_ld();
#pragma unroll
                    for (int k = 0; k < 32; k += 4) {
                        const float4 dl = *reinterpret_cast<const float4 *>(neg_delta + k0 + k);
                        float2 p = make_float2(x[k0 + k], x[k0 + k + 1]), q = make_float2(x[k0 + k + 2], x[k0 + k + 3]);
                        if constexpr (!BF16) {
                            p = mul2(p, make_float2(up, up));
                            q = mul2(q, make_float2(up, up));
                        }
                        p = mul2(p, add2(make_float2(dp[k], dp[k + 1]), make_float2(dl.x, dl.y)));
                        q = mul2(q, add2(make_float2(dp[k + 2], dp[k + 3]), make_float2(dl.z, dl.w)));
                        u[(k0 + k) / 2] = pack2<BF16>(p.x, p.y);
                        u[(k0 + k) / 2 + 1] = pack2<BF16>(q.x, q.y);
                    }
                }
                tmem_st32(td, u);
                wait_st();
                fence_before();
                bar_arrive(ds_full);
                bar_arrive(st_empty + 8 * st);
            }
            if (ok && w.n > 0) ok = __all_sync(0xffffffffu, bar_wait(done, t & 1, &stalled));
            fence_after();
            float factor = half == 0 ? (BF16 ? 1.f : 1.f / 32768.f) : a.scale / up;
            if (!row || w.n == 0) factor = 0.f;
            uint16_t *out = reinterpret_cast<uint16_t *>(to.p) + w.b * to.sb + (int64_t)j * to.sl + w.g * to.sh;
            NanSums total;                   // whether one of the row's values is NaN
#pragma unroll
            for (int k = 0; k < DP; k += 32) {
                float o[32];
                __syncwarp();
                if (w.n > 0 && ok) {
                    tmem_ld32(tmem + lanes + 256 + 128 * half + k, reinterpret_cast<uint32_t *>(o));
                    wait_ld();
                    if (k + 32 == DP) {
                        fence_before();
                        bar_arrive(acc_empty);
                    }
                    total.add(o);
                }
                if (j < a.k_len) store32<BF16>(out, k, a.dim, vec, o, factor);
            }
            if (__any_sync(0xffffffffu, row && total.found())) {
                const int j32 = w.j0 + 32 * (warp & 3);
                again::key_gradients<typename Tensor16<BF16>::T>(a, w.b, w.g, j32, j32 + 32, half == 1, half == 0);
            }
            if (w.n > 0) ++t;
        }
    }

    fence_before();
    __syncthreads();
    fence_after();
    if (stalled) drain_stalled(stalls);
    if (warp == 8) tmem_free(tmem, 512);
    // This kernel starts once every block of the dq kernel has seen the first kernel's end, and fills the SMs that they
    // leave; it is not to end before them.
    if (threadIdx.x == 0) cudaGridDependencySynchronize();
}

static int64_t tiles_of(int64_t n) { return (n + T - 1) / T; }

int64_t attn_tc_backward_work(int64_t batch, int32_t q_len, int32_t k_len, int32_t q_heads, int32_t kv_heads)
{
    return batch * q_heads * tiles_of(q_len) + batch * kv_heads * tiles_of(k_len);
}

bool attn_tc_backward_ok(const AttnArgs &a)
{
    return a.dtype != GS_TABLE_F32 && a.batch < ((int64_t)1 << 31) && attn_tma_ok(a.q, a.dtype, a.batch, a.q_len, a.q_heads) &&
           attn_tma_ok(a.dout, a.dtype, a.batch, a.q_len, a.q_heads) && attn_tma_ok(a.k, a.dtype, a.batch, a.k_len, a.kv_heads) &&
           attn_tma_ok(a.v, a.dtype, a.batch, a.k_len, a.kv_heads);
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
    const int64_t sms = sm_count();
    attn_tc_prepare_kernel<BF16, DP><<<(unsigned)(q_blocks + (BF16 ? 0 : k_blocks)), 256, 0, st>>>(a, norms);
    GS_CUDA_TRY(cudaGetLastError());
    constexpr int smem = BwdSmem<DP>::BYTES;
    static SharedRecord record[2];
    gs_status s;
    if ((s = allow_shared(attn_tc_dq_kernel<BF16, DP>, smem, record[0])) != GS_OK ||
        (s = allow_shared(attn_tc_dkdv_kernel<BF16, DP>, smem, record[1])) != GS_OK)
        return s;
    auto launch = [&](auto kernel, int64_t items) {
        const bool asked = items_asked(a, items);
        return launch_after(kernel, (int)(asked || items < sms ? items : sms), THREADS, smem, st, a, maps, norms,
                            asked ? 0u : (uint32_t)items, stalls);
    };
    GS_CUDA_TRY(launch(attn_tc_dq_kernel<BF16, DP>, q_blocks));
    GS_CUDA_TRY(launch(attn_tc_dkdv_kernel<BF16, DP>, k_blocks));
    return GS_OK;
}

gs_status attn_tc_backward(const AttnArgs &a, cudaStream_t st)
{
    const bool bf16 = a.dtype == GS_TABLE_BF16;
    BwdMaps m;
    gs_status s;
    if ((s = attn_tensor_map(&m.q, a.q, a.dtype, a.batch, a.q_len, a.q_heads, a.dim, 64, 128)) != GS_OK) return s;
    if ((s = attn_tensor_map(&m.dout, a.dout, a.dtype, a.batch, a.q_len, a.q_heads, a.dim, 64, 128)) != GS_OK) return s;
    if ((s = attn_tensor_map(&m.k, a.k, a.dtype, a.batch, a.k_len, a.kv_heads, a.dim, 64, 128)) != GS_OK) return s;
    if ((s = attn_tensor_map(&m.v, a.v, a.dtype, a.batch, a.k_len, a.kv_heads, a.dim, 64, 128)) != GS_OK) return s;
    BwdNorms nm;
    nm.dout = a.delta + a.batch * a.q_heads * (int64_t)a.q_len;
    nm.v = nm.dout + a.batch * a.q_heads * tiles_of(a.q_len);
    if (a.dim <= 64) return bf16 ? backward_t<true, 64>(a, m, nm, st) : backward_t<false, 64>(a, m, nm, st);
    return bf16 ? backward_t<true, 128>(a, m, nm, st) : backward_t<false, 128>(a, m, nm, st);
}

}  // namespace gs
