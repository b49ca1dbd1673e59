// Attention of short 16-bit sequences (up to 128 positions): walks.
//
// A walk's scores are a few 16 x 16 blocks, far less than a 128 x 128 tensor-core tile, and there are
// tens of thousands of walks: the bound is the traffic of q, k, v and the results.  So a unit - one head of one
// sequence - is brought to shared memory once, whole, and everything happens there and in registers:
// one warp per 16 rows, mma.sync m16n8k16 on 16 x 16 blocks, and only blocks that the window reaches.
// A block takes several units, so that its rows stay contiguous in memory over the heads of a walk, and several
// blocks share an SM, so that one's loads overlap another's arithmetic.
//
//  forward : scores of up to 64 keys at a time in registers, running maximum and sum over those
//  backward: dq by query rows, then dk and dv by key rows, both from the same copy in shared memory.  delta =
//            sum_j p_ij dp_ij comes from the probabilities themselves (a first walk over the row's blocks), so
//            the forward output is neither read nor is its rounding part of the gradient.
// Rows past a sequence's end are zeros in shared memory, never read from the tensors.
// P and dS are rounded to the tensors' type for their products.  For binary16 they are scaled by powers
// of two first, P by 2^14 (p <= 1), dS by the one that brings its bound |dS| <= max|dp| + |delta| below 2^15.
#include "gs_attn.cuh"
#include "gs_tc.cuh"

namespace gs {

using tc::exp2_fast;
using tc::pack2;
using tc::smem_u32;

static constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;
static constexpr int KEEP = 4;                    // blocks of 16 keys whose scores the forward pass holds

// byte offset of 16-byte chunk c of row r: rows of DP values, chunks permuted so that eight rows at one
// column fall into different banks
template <int DP>
__device__ __forceinline__ uint32_t at(int r, int c)
{
    constexpr int CH = DP / 8;                    // chunks per row
    const int x = CH >= 8 ? (r & 7) : CH == 4 ? ((r >> 1) & 3) : ((r >> 2) & 1);
    return (uint32_t)((r * CH + (c ^ x)) * 16);
}

__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <bool BF16>
__device__ __forceinline__ void mma(float *c, const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (BF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// A fragments of rows [r0, r0 + 16)
template <int DP>
__device__ __forceinline__ void load_a(uint32_t (&f)[DP / 16][4], uint32_t tile, int r0)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) ldm4(f[k], tile + at<DP>(r0 + (lane & 15), 2 * k + (lane >> 4)));
}

// s[16 x 16] = A B^T: rows j0..j0+15 of B are the columns.  s[0..3]: columns 0-7, s[4..7]: 8-15
template <bool BF16, int DP>
__device__ __forceinline__ void block_dot(float (&s)[8], const uint32_t (&a)[DP / 16][4], uint32_t b, int j0)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = 0.f;
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
        uint32_t f[4];
        ldm4(f, b + at<DP>(j0 + (lane & 7) + ((lane >> 4) << 3), 2 * k + ((lane >> 3) & 1)));
        mma<BF16>(s, a[k], f[0], f[1]);
        mma<BF16>(s + 4, a[k], f[2], f[3]);
    }
}

// acc[16 x DP] += p[16 x 16] B, rows j0..j0+15 of B summed over
template <bool BF16, int DP>
__device__ __forceinline__ void block_mul(float (&acc)[DP / 8][4], const uint32_t (&p)[4], uint32_t b, int j0)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int d = 0; d < DP / 16; ++d) {
        uint32_t f[4];
        ldm4t(f, b + at<DP>(j0 + (lane & 15), 2 * d + (lane >> 4)));
        mma<BF16>(acc[2 * d], p, f[0], f[1]);
        mma<BF16>(acc[2 * d + 1], p, f[2], f[3]);
    }
}

// the C layout of two 8-column blocks is the A layout of one 16-column block
template <bool BF16>
__device__ __forceinline__ void as_a(uint32_t (&p)[4], const float (&s)[8])
{
    p[0] = pack2<BF16>(s[0], s[1]);
    p[1] = pack2<BF16>(s[2], s[3]);
    p[2] = pack2<BF16>(s[4], s[5]);
    p[3] = pack2<BF16>(s[6], s[7]);
}

// column of value i of a 16 x 16 block (rows: lane / 4 for i & 2 == 0, + 8 otherwise)
__device__ __forceinline__ int col_of(int i) { return ((i >> 2) << 3) + 2 * (threadIdx.x & 3) + (i & 1); }

struct Lens {
    AttnSeq s;
    int64_t b;
    int h;
};

// rows [0, pad) of one head into shared memory: rows >= n and values >= dim are zeros
template <int DP>
__device__ __forceinline__ void load_head(uint32_t dst, const AttnTensor &t, int64_t b, int h, int n, int pad, int dim,
                                          bool vec, int tid, int threads)
{
    constexpr int CH = DP / 8;
    const uint16_t *base = reinterpret_cast<const uint16_t *>(t.p) + b * t.sb + h * t.sh;
    for (int e = tid; e < pad * CH; e += threads) {
        const int r = e / CH, c = e % CH;
        const uint32_t to = dst + at<DP>(r, c);
        if (vec) {
            const bool in = r < n && c * 8 < dim;
            const uint16_t *from = in ? base + (int64_t)r * t.sl + c * 8 : base;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(in ? 16 : 0) : "memory");
        } else {
            uint32_t u[4] = {};
            if (r < n) {
                const uint16_t *from = base + (int64_t)r * t.sl;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c * 8 + i < dim) u[i / 2] |= (uint32_t)from[c * 8 + i] << (16 * (i & 1));
            }
            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]) : "memory");
        }
    }
}
__device__ __forceinline__ void loads_done()
{
    asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
}

// the 16 x DP accumulator times its two row factors, in the tensors' type
template <bool BF16, int DP>
__device__ __forceinline__ void pack_tile(uint32_t (&u)[DP / 8][2], const float (&acc)[DP / 8][4], float f0, float f1)
{
#pragma unroll
    for (int c = 0; c < DP / 8; ++c) {
        u[c][0] = pack2<BF16>(acc[c][0] * f0, acc[c][1] * f0);
        u[c][1] = pack2<BF16>(acc[c][2] * f1, acc[c][3] * f1);
    }
}

// this warp's 16 x DP result, as pack_tile left it, to rows [r0, r0 + 16) of a tensor: through the
// 16 rows of `stage` in shared memory, which nobody else reads any more, for 16-byte stores.
// Rows >= n become zeros, rows >= len are not written.
template <int DP>
__device__ __forceinline__ void store_tile(const uint32_t (&u)[DP / 8][2], uint32_t stage, const AttnTensor &t,
                                           int64_t b, int h, int r0, int n, int len, int dim, bool vec)
{
    constexpr int CH = DP / 8;
    const int lane = threadIdx.x & 31, row = lane >> 2;
    const bool in0 = r0 + row < n, in1 = r0 + row + 8 < n;
    __syncwarp();
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const uint32_t lo = in0 ? u[c][0] : 0u, hi = in1 ? u[c][1] : 0u;
        asm volatile("st.shared.u32 [%0], %1;" ::"r"(stage + at<DP>(r0 + row, c) + 4 * (lane & 3)), "r"(lo) : "memory");
        asm volatile("st.shared.u32 [%0], %1;" ::"r"(stage + at<DP>(r0 + row + 8, c) + 4 * (lane & 3)), "r"(hi) : "memory");
    }
    __syncwarp();
    uint16_t *base = reinterpret_cast<uint16_t *>(t.p) + b * t.sb + h * t.sh;
    for (int e = lane; e < 16 * CH; e += 32) {
        const int r = r0 + e / CH, c = e % CH;
        if (r >= len || c * 8 >= dim) continue;
        uint4 u;
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "r"(stage + at<DP>(r, c)) : "memory");
        uint16_t *to = base + (int64_t)r * t.sl + c * 8;
        if (vec) {
            *reinterpret_cast<uint4 *>(to) = u;
        } else {
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c * 8 + i < dim) to[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
        }
    }
}

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

__device__ __forceinline__ Lens unit_of(const AttnArgs &a, int64_t u, int heads)
{
    Lens l;
    l.b = u / heads;
    l.h = (int)(u % heads);
    l.s = attn_seq(a, l.b);
    return l;
}

// `units` heads per block; qt, kt: 16-row tiles of the padded lengths; one warp per (unit, query tile)
// resident blocks of 256 threads that the register budget is set for
template <int DP> constexpr int blocks_per_sm() { return DP <= 32 ? 3 : DP == 64 ? 2 : 1; }

template <bool BF16, int DP>
__global__ void __launch_bounds__(256, blocks_per_sm<DP>())
attn_walk_forward_kernel(const __grid_constant__ AttnArgs a, int units, int qt, int kt, bool vec)
{
    extern __shared__ uint4 smem[];
    const uint32_t base = smem_u32(smem);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t total = a.batch * a.q_heads, u0 = (int64_t)blockIdx.x * units;
    const uint32_t q_bytes = qt * 16 * DP * 2, k_bytes = kt * 16 * DP * 2, unit_bytes = q_bytes + 2 * k_bytes;
    const int here = (int)min((int64_t)units, total - u0);
    const int mine = warp / qt;                               // the unit that this warp's group of qt warps works on
    if (mine < here) {
        const Lens l = unit_of(a, u0 + mine, a.q_heads);
        const uint32_t at0 = base + mine * unit_bytes;
        const int tid = threadIdx.x - mine * qt * 32;
        load_head<DP>(at0, a.q, l.b, l.h, l.s.nq, qt * 16, a.dim, vec, tid, qt * 32);
        load_head<DP>(at0 + q_bytes, a.k, l.b, l.h / a.group, l.s.nk, kt * 16, a.dim, vec, tid, qt * 32);
        load_head<DP>(at0 + q_bytes + k_bytes, a.v, l.b, l.h / a.group, l.s.nk, kt * 16, a.dim, vec, tid, qt * 32);
    }
    loads_done();
    __syncthreads();
    if (mine >= here) return;
    const Lens l = unit_of(a, u0 + mine, a.q_heads);
    const uint32_t Q = base + mine * unit_bytes, K = Q + q_bytes, V = K + k_bytes;
    const int r0 = (warp % qt) * 16, ra = r0 + (lane >> 2), rb = ra + 8;
    const int lo_a = attn_lo(a, l.s, ra), hi_a = attn_hi(a, l.s, ra), lo_b = attn_lo(a, l.s, rb), hi_b = attn_hi(a, l.s, rb);
    float acc[DP / 8][4] = {};
    float top_a = -INFINITY, top_b = -INFINITY, sum_a = 0.f, sum_b = 0.f;
    const int r_end = min(r0 + 16, l.s.nq);
    const int j_begin = attn_lo(a, l.s, r0) / 16, j_end = r_end > r0 ? (attn_hi(a, l.s, r_end - 1) + 15) / 16 : 0;
    const float mul = a.scale * LOG2E;
    if (j_begin < j_end) {
        uint32_t qf[DP / 16][4];
        load_a<DP>(qf, Q, r0);
        for (int j = j_begin; j < j_end; j += KEEP) {
            float s[KEEP][8];
            float m_a = top_a, m_b = top_b;
#pragma unroll
            for (int x = 0; x < KEEP; ++x) {
                if (j + x >= j_end) break;
                block_dot<BF16, DP>(s[x], qf, K, (j + x) * 16);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int c = (j + x) * 16 + col_of(i);
                    const bool in = i & 2 ? (c >= lo_b && c < hi_b) : (c >= lo_a && c < hi_a);
                    s[x][i] = in ? s[x][i] * mul : -INFINITY;
                    if (i & 2) m_b = fmaxf(m_b, s[x][i]);
                    else m_a = fmaxf(m_a, s[x][i]);
                }
            }
            m_a = quad_max(m_a);
            m_b = quad_max(m_b);
            const float base_a = m_a == -INFINITY ? 0.f : m_a, base_b = m_b == -INFINITY ? 0.f : m_b;
            if (j > j_begin) {
                const float keep_a = exp2_fast(top_a - base_a), keep_b = exp2_fast(top_b - base_b);
                sum_a *= keep_a;
                sum_b *= keep_b;
#pragma unroll
                for (int d = 0; d < DP / 8; ++d) {
                    acc[d][0] *= keep_a;
                    acc[d][1] *= keep_a;
                    acc[d][2] *= keep_b;
                    acc[d][3] *= keep_b;
                }
            }
            top_a = m_a;
            top_b = m_b;
#pragma unroll
            for (int x = 0; x < KEEP; ++x) {
                if (j + x >= j_end) break;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    s[x][i] = exp2_fast(s[x][i] - (i & 2 ? base_b : base_a));
                    if (i & 2) sum_b += s[x][i];
                    else sum_a += s[x][i];
                }
                uint32_t p[4];
                as_a<BF16>(p, s[x]);
                block_mul<BF16, DP>(acc, p, V, (j + x) * 16);
            }
        }
    }
    sum_a = quad_sum(sum_a);
    sum_b = quad_sum(sum_b);
    if ((lane & 3) == 0) {
        float *lse = a.lse + (l.b * a.q_heads + l.h) * a.q_len;
        if (ra < a.q_len) lse[ra] = sum_a == 0.f ? -INFINITY : (top_a + log2f(sum_a)) * LN2;
        if (rb < a.q_len) lse[rb] = sum_b == 0.f ? -INFINITY : (top_b + log2f(sum_b)) * LN2;
    }
    uint32_t out[DP / 8][2];
    pack_tile<BF16, DP>(out, acc, sum_a == 0.f ? 0.f : 1.f / sum_a, sum_b == 0.f ? 0.f : 1.f / sum_b);
    store_tile<DP>(out, Q, a.out, l.b, l.h, r0, l.s.nq, a.q_len, a.dim, vec);
}

// power of two that brings a bound below 2^15 (binary16 only)
template <bool BF16>
__device__ __forceinline__ float lift(float bound)
{
    if (BF16 || !(bound > 0.f) || !isfinite(bound)) return 1.f;
    const int e = (int)((__float_as_uint(bound) >> 23) & 255) - 126;       // bound < 2^e
    return __uint_as_float((uint32_t)(min(max(15 - e, -100), 100) + 127) << 23);
}

// `units` key/value heads per block, `tiles` = max(qt, kt) warps per unit
// SHARED: several query heads per key/value head
template <bool BF16, int DP, bool SHARED>
__global__ void __launch_bounds__(256, blocks_per_sm<DP>())
attn_walk_backward_kernel(const __grid_constant__ AttnArgs a, int units, int qt, int kt, bool vec)
{
    extern __shared__ uint4 smem[];
    const uint32_t base = smem_u32(smem);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tiles = max(qt, kt);
    const int64_t total = a.batch * a.kv_heads, u0 = (int64_t)blockIdx.x * units;
    const uint32_t q_bytes = qt * 16 * DP * 2, k_bytes = kt * 16 * DP * 2;
    const uint32_t unit_bytes = 2 * q_bytes + 2 * k_bytes + 3 * qt * 16 * 4;
    const int here = (int)min((int64_t)units, total - u0);
    const int mine = warp / tiles, tile = warp % tiles, tid = threadIdx.x - mine * tiles * 32;
    const bool active = mine < here;
    const Lens l = unit_of(a, u0 + (active ? mine : 0), a.kv_heads);
    const AttnSeq s = l.s;
    const uint32_t Q = base + mine * unit_bytes, DO = Q + q_bytes, K = DO + q_bytes, V = K + k_bytes;
    // per query row: lse in units of log2, delta, bound of |dS|
    float *lse2 = reinterpret_cast<float *>(reinterpret_cast<char *>(smem) + mine * unit_bytes + 2 * q_bytes + 2 * k_bytes);
    float *delta = lse2 + qt * 16, *bound = delta + qt * 16;
    const float mul = a.scale * LOG2E;
    float dk[DP / 8][4] = {}, dv[DP / 8][4] = {};
    float up_k = 1.f;

    const int group = SHARED ? a.group : 1;
    for (int x = 0; x < group; ++x) {
        const int h = l.h * group + x;
        if (x > 0) __syncthreads();
        if (active) {
            load_head<DP>(Q, a.q, l.b, h, s.nq, qt * 16, a.dim, vec, tid, tiles * 32);
            load_head<DP>(DO, a.dout, l.b, h, s.nq, qt * 16, a.dim, vec, tid, tiles * 32);
            if (x == 0) {
                load_head<DP>(K, a.k, l.b, l.h, s.nk, kt * 16, a.dim, vec, tid, tiles * 32);
                load_head<DP>(V, a.v, l.b, l.h, s.nk, kt * 16, a.dim, vec, tid, tiles * 32);
            }
            const float *lse = a.lse + (l.b * a.q_heads + h) * a.q_len;
            for (int r = tid; r < qt * 16; r += tiles * 32) {
                const float v = r < s.nq ? lse[r] * LOG2E : -INFINITY;
                lse2[r] = v == -INFINITY ? INFINITY : v;      // p = 0 in rows that see nothing
            }
        }
        loads_done();
        __syncthreads();

        // ---- dq of 16 query rows
        uint32_t dq[DP / 8][2] = {};
        const int r0 = tile * 16, ra = r0 + (lane >> 2), rb = ra + 8;
        if (active && tile < qt) {
            const int lo_a = attn_lo(a, s, ra), hi_a = attn_hi(a, s, ra), lo_b = attn_lo(a, s, rb), hi_b = attn_hi(a, s, rb);
            const int r_end = min(r0 + 16, s.nq);
            const int j_begin = attn_lo(a, s, r0) / 16, j_end = r_end > r0 ? (attn_hi(a, s, r_end - 1) + 15) / 16 : 0;
            const float l_a = lse2[ra], l_b = lse2[rb];
            uint32_t qf[DP / 16][4], df[DP / 16][4];
            load_a<DP>(qf, Q, r0);
            load_a<DP>(df, DO, r0);
            float d_a = 0.f, d_b = 0.f, m_a = 0.f, m_b = 0.f;
            auto scores = [&](int j, float (&p)[8], float (&dp)[8]) {
                block_dot<BF16, DP>(p, qf, K, j * 16);
                block_dot<BF16, DP>(dp, df, V, j * 16);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int c = j * 16 + col_of(i);
                    const bool in = i & 2 ? (c >= lo_b && c < hi_b) : (c >= lo_a && c < hi_a);
                    p[i] = in ? exp2_fast(fmaf(p[i], mul, -(i & 2 ? l_b : l_a))) : 0.f;
                    dp[i] = in ? dp[i] : 0.f;
                }
            };
            for (int j = j_begin; j < j_end; ++j) {
                float p[8], dp[8];
                scores(j, p, dp);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (i & 2) {
                        d_b = fmaf(p[i], dp[i], d_b);
                        m_b = fmaxf(m_b, fabsf(dp[i]));
                    } else {
                        d_a = fmaf(p[i], dp[i], d_a);
                        m_a = fmaxf(m_a, fabsf(dp[i]));
                    }
                }
            }
            d_a = quad_sum(d_a);
            d_b = quad_sum(d_b);
            if constexpr (!BF16) {
                m_a = quad_max(m_a) + fabsf(d_a);
                m_b = quad_max(m_b) + fabsf(d_b);
            }
            if ((lane & 3) == 0) {
                delta[ra] = d_a;
                delta[rb] = d_b;
                bound[ra] = m_a;
                bound[rb] = m_b;
            }
            const float up_a = lift<BF16>(m_a), up_b = lift<BF16>(m_b);
            float acc[DP / 8][4] = {};
            for (int j = j_begin; j < j_end; ++j) {
                float p[8], dp[8];
                scores(j, p, dp);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    p[i] *= dp[i] - (i & 2 ? d_b : d_a);
                    if constexpr (!BF16) p[i] *= i & 2 ? up_b : up_a;
                }
                uint32_t w[4];
                as_a<BF16>(w, p);
                block_mul<BF16, DP>(acc, w, K, j * 16);
            }
            pack_tile<BF16, DP>(dq, acc, a.scale / up_a, a.scale / up_b);
        }
        __syncthreads();

        // ---- dk, dv of 16 key rows
        if (active && tile < kt) {
            const int j0 = tile * 16, ja = j0 + (lane >> 2), jb = ja + 8;
            const int lo_a = attn_q_first(a, s, ja), hi_a = ja < s.nk ? attn_q_last(a, s, ja + 1) : 0;
            const int lo_b = attn_q_first(a, s, jb), hi_b = jb < s.nk ? attn_q_last(a, s, jb + 1) : 0;
            const int j_end = min(j0 + 16, s.nk);
            const int q_begin = attn_q_first(a, s, j0) / 16, q_end = j_end > j0 ? (attn_q_last(a, s, j_end) + 15) / 16 : 0;
            float up = 1.f;
            if constexpr (!BF16) {                           // one scale per head: dk sums over its queries
                float m = 0.f;
                for (int r = lane; r < qt * 16; r += 32) m = fmaxf(m, bound[r]);
#pragma unroll
                for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
                up = lift<BF16>(m);
                // a shared head's sums are carried from one query head's scale to the next one's
                if (x > 0 && up != up_k) {
#pragma unroll
                    for (int d = 0; d < DP / 8; ++d)
#pragma unroll
                        for (int i = 0; i < 4; ++i) dk[d][i] *= up / up_k;
                }
                up_k = up;
            }
            if (q_begin < q_end) {
                uint32_t kf[DP / 16][4], vf[DP / 16][4];
                load_a<DP>(kf, K, j0);
                load_a<DP>(vf, V, j0);
                for (int q = q_begin; q < q_end; ++q) {
                    float p[8], dp[8];
                    block_dot<BF16, DP>(p, kf, Q, q * 16);
                    block_dot<BF16, DP>(dp, vf, DO, q * 16);
                    const int c0 = q * 16 + 2 * (lane & 3);
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        const float2 ls = *reinterpret_cast<const float2 *>(lse2 + c0 + 8 * n);
                        const float2 de = *reinterpret_cast<const float2 *>(delta + c0 + 8 * n);
#pragma unroll
                        for (int i = 4 * n; i < 4 * n + 4; ++i) {
                            const int c = c0 + 8 * n + (i & 1);
                            const bool in = i & 2 ? (c >= lo_b && c < hi_b) : (c >= lo_a && c < hi_a);
                            p[i] = in ? exp2_fast(fmaf(p[i], mul, -(i & 1 ? ls.y : ls.x))) : 0.f;
                            dp[i] = in ? p[i] * (dp[i] - (i & 1 ? de.y : de.x)) : 0.f;
                            if constexpr (!BF16) {
                                dp[i] *= up;
                                p[i] *= 16384.f;
                            }
                        }
                    }
                    uint32_t w[4];
                    as_a<BF16>(w, p);
                    block_mul<BF16, DP>(dv, w, DO, q * 16);
                    as_a<BF16>(w, dp);
                    block_mul<BF16, DP>(dk, w, Q, q * 16);
                }
            }
        }
        __syncthreads();                                     // nobody reads Q, dO (and K, V after the last head) any more
        if (active && tile < qt)
            store_tile<DP>(dq, Q, a.dq, l.b, h, r0, s.nq, a.q_len, a.dim, vec);
    }
    if (active && tile < kt) {
        const float f = a.scale / up_k, g = BF16 ? 1.f : 1.f / 16384.f;
        uint32_t u[DP / 8][2];
        pack_tile<BF16, DP>(u, dk, f, f);
        store_tile<DP>(u, K, a.dk, l.b, l.h, tile * 16, s.nk, a.k_len, a.dim, vec);
        pack_tile<BF16, DP>(u, dv, g, g);
        store_tile<DP>(u, V, a.dv, l.b, l.h, tile * 16, s.nk, a.k_len, a.dim, vec);
    }
}

// 16-byte accesses need every row of every tensor aligned to eight values
static bool rows_of_eight(const AttnArgs &a, bool backward)
{
    auto ok = [](const AttnTensor &t) { return (uintptr_t)t.p % 16 == 0 && (t.sb | t.sl | t.sh) % 8 == 0; };
    bool v = a.dim % 8 == 0 && ok(a.q) && ok(a.k) && ok(a.v);
    if (backward) return v && ok(a.dout) && ok(a.dq) && ok(a.dk) && ok(a.dv);
    return v && ok(a.out);
}

template <bool BF16, int DP, bool BWD>
static gs_status launch(const AttnArgs &a, cudaStream_t st)
{
    const int qt = (a.q_len + 15) / 16, kt = (a.k_len + 15) / 16, tiles = BWD ? (qt > kt ? qt : kt) : qt;
    const int64_t total = a.batch * (BWD ? a.kv_heads : a.q_heads);
    const int unit_bytes = (BWD ? 2 : 1) * qt * 16 * DP * 2 + 2 * kt * 16 * DP * 2 + (BWD ? 3 * qt * 16 * 4 : 0);
    int units = 8 / tiles;                                    // eight warps a block, or one unit
    while (units > 1 && units * unit_bytes > 48 * 1024) --units;
    if (units < 1) units = 1;
    const int64_t blocks = (total + units - 1) / units;
    if (blocks == 0) return GS_OK;
    if (blocks > 0x7FFFFFFF) {
        set_error("attention of %lld blocks exceeds one launch", (long long)blocks);
        return GS_ERR_UNSUPPORTED;
    }
    auto kernel = !BWD ? attn_walk_forward_kernel<BF16, DP>
                       : a.group > 1 ? attn_walk_backward_kernel<BF16, DP, true> : attn_walk_backward_kernel<BF16, DP, false>;
    const int smem = units * unit_bytes;
    GS_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    kernel<<<(unsigned)blocks, units * tiles * 32, smem, st>>>(a, units, qt, kt, rows_of_eight(a, BWD));
    GS_CUDA_TRY(cudaGetLastError());
    return GS_OK;
}

template <bool BF16, bool BWD>
static gs_status by_dim(const AttnArgs &a, cudaStream_t st)
{
    if (a.dim <= 16) return launch<BF16, 16, BWD>(a, st);
    if (a.dim <= 32) return launch<BF16, 32, BWD>(a, st);
    if (a.dim <= 64) return launch<BF16, 64, BWD>(a, st);
    return launch<BF16, 128, BWD>(a, st);
}

bool attn_walk_ok(const AttnArgs &a)
{
    return a.dtype != GS_TABLE_F32 && a.q_len > 0 && a.k_len > 0 && a.q_len <= 128 && a.k_len <= 128;
}
gs_status attn_walk_forward(const AttnArgs &a, cudaStream_t st)
{
    return a.dtype == GS_TABLE_BF16 ? by_dim<true, false>(a, st) : by_dim<false, false>(a, st);
}
gs_status attn_walk_backward(const AttnArgs &a, cudaStream_t st)
{
    return a.dtype == GS_TABLE_BF16 ? by_dim<true, true>(a, st) : by_dim<false, true>(a, st);
}

}  // namespace gs
