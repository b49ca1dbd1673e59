// Attention of fp32 tensors on the tensor cores, forward beyond 128 positions and backward, with up to 64 columns, from 65
// positions where blocks of 64 rows fill the device one and a half times: every product as three of tf32
// (mma.sync m16n8k8; a tcgen05 product would need both parts of every operand in shared memory, P and dS included).
//
// A block of four warps owns 64 rows - queries for the output and dq, keys for dk and dv - and the rows of the other
// side come by in tiles, by cp.async into one buffer while the other one is worked on.  A warp has 16 of the
// rows: its scores, probabilities and score gradients never leave its registers, since a lane holds them in the order
// in which the A operand of the next product wants them.  Only tiles that one of the block's rows sees are
// fetched, and only those that one of the warp's rows sees are computed.
//  forward : running maximum and sum over the key tiles
//  backward: delta by a small kernel ahead; then, in one launch, blocks of keys make dk and dv and blocks of queries dq,
//            both from p = exp(s - lse).  A block of keys goes through the query heads of its group one after the
//            other, so shared heads are summed in a fixed order without atomics.
// A product of 16 x 8 x 8 needs about as many instructions to fetch and split its operands as tensor instructions, and an
// SM holds 12 warps: neither the tensor pipe (53 % busy forward, 50 % backward; 64 heads of 1024 x 64) nor the issue
// slots (52 and 48 %) are full, each product waits for its operands' conversion.  16 heads of 4096 x 64, all visible:
// forward 1381 us (50 TFLOP/s), backward 5048 us.
// The tensor cores round towards zero as they add, so sums over positions start from zero in every tile and the tiles'
// sums are added by the CUDA cores, rounded to nearest.
#include "gs_attn_again.cuh"
#include "gs_tc.cuh"

namespace gs {

using namespace tc;

namespace {

constexpr int OWN = 64, THREADS = 128;

// Rows are DP + 8 floats apart: four rows whose numbers differ modulo 4 then lie in different groups of 8 banks.  The
// lanes (g, t) = (lane / 4, lane % 4) read pairs of floats, 16 lanes at a time, without a conflict:
//  along rows   : row g's columns 2t, 2t + 1 as the elements t and t + 4 of a step of eight columns
//  along columns: columns 2g, 2g + 1, for two products at once, of rows t and other(t)
// Of eight rows on the other side, scores are computed in the order row_of_8, which gives a lane the scores of rows
// t and other(t): elements t and t + 4 of the next product.
template <int DP> constexpr int STRIDE = DP + 8;
__device__ __forceinline__ int other(int t) { return 4 + ((t + 2) & 3); }
__device__ __forceinline__ int row_of_8(int g) { return g & 1 ? other(g >> 1) : g >> 1; }

__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
struct Operand {                                          // 16 x 8 values
    uint32_t hi[4], lo[4];
    __device__ __forceinline__ void set(float a0, float a1, float a2, float a3)
    {
        split(a0, hi[0], lo[0]);
        split(a1, hi[1], lo[1]);
        split(a2, hi[2], lo[2]);
        split(a3, hi[3], lo[3]);
    }
};
__device__ __forceinline__ void mma3(float (&c)[4], const Operand &a, float y0, float y1)
{
    uint32_t h0, l0, h1, l1;
    split(y0, h0, l0);
    split(y1, h1, l1);
    mma(c, a.lo, h0, h1);
    mma(c, a.hi, l0, l1);
    mma(c, a.hi, h0, h1);
}

template <int N>
__device__ __forceinline__ void clear(float (&c)[N][4])
{
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) c[n][i] = 0.f;
}

__device__ __forceinline__ void copy16(float *dst, const float *src, bool in)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(smem_u32(dst)), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy4(float *dst, const float *src, bool in)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" :: "r"(smem_u32(dst)), "l"(src), "r"(in ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }

__device__ __forceinline__ float *row_of(const AttnTensor &t, int64_t b, int64_t pos, int64_t head)
{
    return reinterpret_cast<float *>(t.p) + b * t.sb + pos * t.sl + head * t.sh;
}

// rows [r0, r0 + ROWS) of one head; rows >= n and columns >= dim become zeros, whatever the tensor holds there
template <int ROWS, int DP>
__device__ __forceinline__ void copy_rows(float *dst, const AttnTensor &t, int64_t b, int head, int r0, int n, int dim, bool vec)
{
    const float *base = row_of(t, b, 0, head);
#pragma unroll
    for (int k = 0; k < ROWS * DP / 4 / THREADS; ++k) {
        const int e = threadIdx.x + k * THREADS, r = r0 + e / (DP / 4), c = e % (DP / 4) * 4;
        float *to = dst + e / (DP / 4) * STRIDE<DP> + c;
        const float *from = base + (int64_t)r * t.sl + c;
        if (vec) {
            const bool in = r < n && c < dim;
            copy16(to, in ? from : base, in);
        } else {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const bool in = r < n && c + x < dim;
                copy4(to + x, in ? from + x : base, in);
            }
        }
    }
}

// c[n][.] = own rows . rows of a tile, over the columns; `own` points to the warp's rows
template <int N, int DP>
__device__ __forceinline__ void dot(float (&c)[N][4], const float *own, const float *tile)
{
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const float *x = own + g * STRIDE<DP> + 2 * t, *y = tile + row_of_8(g) * STRIDE<DP> + 2 * t;
    clear(c);
#pragma unroll
    for (int k = 0; k < DP / 8; ++k) {
        const float2 u = *reinterpret_cast<const float2 *>(x + 8 * k);
        const float2 w = *reinterpret_cast<const float2 *>(x + 8 * STRIDE<DP> + 8 * k);
        Operand a;
        a.set(u.x, w.x, u.y, w.y);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const float2 z = *reinterpret_cast<const float2 *>(y + 8 * n * STRIDE<DP> + 8 * k);
            mma3(c[n], a, z.x, z.y);
        }
    }
}

// acc += p . tile, over the tile's 8 N rows.  A lane's acc[2m], acc[2m + 1] hold columns 16m + 4t .. + 3 of its rows.
template <int N, int DP>
__device__ __forceinline__ void mul(float (&acc)[DP / 8][4], const float (&p)[N][4], const float *tile)
{
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const float *y0 = tile + t * STRIDE<DP> + 2 * g, *y1 = tile + other(t) * STRIDE<DP> + 2 * g;
    Operand a[N];
#pragma unroll
    for (int n = 0; n < N; ++n) a[n].set(p[n][0], p[n][2], p[n][1], p[n][3]);
#pragma unroll
    for (int m = 0; m < DP / 16; ++m) {
        float c[2][4];
        clear(c);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const float2 u = *reinterpret_cast<const float2 *>(y0 + 8 * n * STRIDE<DP> + 16 * m);
            const float2 w = *reinterpret_cast<const float2 *>(y1 + 8 * n * STRIDE<DP> + 16 * m);
            mma3(c[0], a[n], u.x, w.x);
            mma3(c[1], a[n], u.y, w.y);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            acc[2 * m][i] += c[0][i];
            acc[2 * m + 1][i] += c[1][i];
        }
    }
}

// row `half` (0: g, 1: g + 8) of the accumulators, times a factor
template <int DP>
__device__ __forceinline__ void store_row(float *row, const float (&acc)[DP / 8][4], int half, float by, int dim, bool vec)
{
    const int t = threadIdx.x & 3;
#pragma unroll
    for (int m = 0; m < DP / 16; ++m) {
        const int c = 16 * m + 4 * t;
        const float v[4] = {acc[2 * m][2 * half] * by, acc[2 * m + 1][2 * half] * by, acc[2 * m][2 * half + 1] * by,
                            acc[2 * m + 1][2 * half + 1] * by};
        if (vec) {
            if (c < dim) *reinterpret_cast<float4 *>(row + c) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (c + x < dim) row[c + x] = v[x];
        }
    }
}

// whether this thread's part of a result holds a NaN: a sum of it does
template <int N>
__device__ __forceinline__ bool has_nan(const float (&acc)[N][4])
{
    float t = 0.f;
#pragma unroll
    for (int n = 0; n < N; ++n) t += (acc[n][0] + acc[n][1]) + (acc[n][2] + acc[n][3]);
    return t != t;
}

// What 16 rows see of a tile [x0, x0 + len): row r sees [lo(r), hi(r)), both rising with r
enum See { NOTHING, PART, ALL };
__device__ __forceinline__ See see(int lo_first, int lo_last, int hi_first, int hi_last, int x0, int len)
{
    if (hi_last <= x0 || lo_first >= x0 + len) return NOTHING;
    return lo_last <= x0 && hi_first >= x0 + len ? ALL : PART;
}

constexpr int ROWS = 32, N = ROWS / 8;                     // of a tile
template <int DP> constexpr int fwd_shared() { return 4 * STRIDE<DP> * (OWN + 4 * ROWS); }

template <int DP>
__global__ void __launch_bounds__(THREADS, DP <= 64 ? 3 : 2) attn_f32_forward_kernel(const __grid_constant__ AttnArgs a, int tiles, bool vec)
{
    constexpr int TILE = ROWS * STRIDE<DP>;
    extern __shared__ float4 smem4[];
    float *own = reinterpret_cast<float *>(smem4), *stream = own + OWN * STRIDE<DP>;      // K, V of one tile, then of the other
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g8 = lane >> 2, t = lane & 3;
    const int64_t heads = a.batch * a.q_heads;
    // the row tiles run from the last: under a causal bound the longest go first
    const int tile = tiles - 1 - (int)(blockIdx.x / heads);
    const int64_t bh = blockIdx.x % heads, b = bh / a.q_heads;
    const int h = (int)(bh % a.q_heads), g = h / a.group;
    const AttnSeq s = attn_seq(a, b);
    const int r0 = tile * OWN, w0 = r0 + 16 * warp;
    const int last = min(r0 + OWN, s.nq) - 1;
    const int j_end = last >= r0 ? attn_hi(a, s, last) : 0;
    const int j_begin = attn_lo(a, s, r0) / ROWS * ROWS;

    const int lo[2] = {attn_lo(a, s, w0 + g8), attn_lo(a, s, w0 + g8 + 8)};
    const int hi[2] = {attn_hi(a, s, w0 + g8), attn_hi(a, s, w0 + g8 + 8)};
    const int w_last = min(w0 + 16, s.nq) - 1;
    const int w_lo = attn_lo(a, s, w0), w_lo_last = attn_lo(a, s, w0 + 15), w_hi = attn_hi(a, s, w0);
    const int w_end = w_last >= w0 ? attn_hi(a, s, w_last) : 0;
    const bool whole = w_last == w0 + 15;
    float acc[DP / 8][4], top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};      // top in powers of two
    clear(acc);
    const float mul2e = a.scale * LOG2E;
    auto fetch = [&](int j0, int at) {
        copy_rows<ROWS, DP>(stream + at * 2 * TILE, a.k, b, g, j0, s.nk, a.dim, vec);
        copy_rows<ROWS, DP>(stream + at * 2 * TILE + TILE, a.v, b, g, j0, s.nk, a.dim, vec);
        copies_commit();
    };
    if (j_begin < j_end) {
        copy_rows<OWN, DP>(own, a.q, b, h, r0, s.nq, a.dim, vec);
        fetch(j_begin, 0);
    }
    int at = 0;
    for (int j0 = j_begin; j0 < j_end; j0 += ROWS, at ^= 1) {
        copies_wait();
        __syncthreads();                                   // the tile is here, and everyone is done with the one before
        if (j0 + ROWS < j_end) fetch(j0 + ROWS, at ^ 1);
        const See what = see(w_lo, w_lo_last, w_hi, w_end, j0, ROWS);
        if (what == NOTHING) continue;
        const float *K = stream + at * 2 * TILE, *V = K + TILE;
        float p[N][4];
        dot<N, DP>(p, own + 16 * warp * STRIDE<DP>, K);
        if (what == PART || !whole) {
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = j0 + 8 * n + (i & 1 ? other(t) : t);
                    if (j < lo[i >> 1] || j >= hi[i >> 1]) p[n][i] = -INFINITY;
                }
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float m = -INFINITY;
#pragma unroll
            for (int n = 0; n < N; ++n) m = fmaxf(m, fmaxf(p[n][2 * r], p[n][2 * r + 1]));
            m = fmaxf(top[r], quad_max(m) * mul2e);
            const float base = m == -INFINITY ? 0.f : m;               // no visible key so far: every term is 0
            const float keep = exp2_fast(top[r] - base);
            float part = 0.f;
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int i = 2 * r; i < 2 * r + 2; ++i) {
                    p[n][i] = exp2_fast(fmaf(p[n][i], mul2e, -base));
                    part += p[n][i];
                }
            sum[r] = fmaf(sum[r], keep, part);             // this lane's share; the lanes' shares are added at the end
            top[r] = m;
#pragma unroll
            for (int n = 0; n < DP / 8; ++n) {
                acc[n][2 * r] *= keep;
                acc[n][2 * r + 1] *= keep;
            }
        }
        mul<N, DP>(acc, p, V);
    }
    bool nan = has_nan(acc);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int i = w0 + g8 + 8 * r;
        const float total = quad_sum(sum[r]), by = again::row_factor(top[r], 1.f / total);
        nan = nan || again::is_nan(by);
        if (i >= a.q_len) continue;
        store_row<DP>(row_of(a.out, b, i, h), acc, r, by, a.dim, vec);
        if (t == 0) a.lse[bh * a.q_len + i] = again::row_lse(top[r], by, log2f(total));
    }
    if (__any_sync(0xffffffffu, nan)) again::outputs<float>(a, b, h, w0, w0 + 16);
}

// delta_i = dO_i . out_i; 16 lanes a row, heads of a position one after the other
__global__ void __launch_bounds__(256) attn_f32_delta_kernel(const __grid_constant__ AttnArgs a, bool vec)
{
    cudaTriggerProgrammaticLaunchCompletion();             // the next kernel's blocks may start and fetch their inputs
    const int lane = threadIdx.x & 15;
    const int64_t x = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4), per = (int64_t)a.q_len * a.q_heads;
    if (x >= a.batch * per) return;
    const int64_t b = x / per;
    const int i = (int)(x % per / a.q_heads), h = (int)(x % a.q_heads);
    float d = 0.f;
    if (i < attn_seq(a, b).nq) {
        const float *y = row_of(a.dout, b, i, h), *o = row_of(a.out, b, i, h);
        if (vec) {
            for (int c = 4 * lane; c < a.dim; c += 64) {
                const float4 u = __ldg(reinterpret_cast<const float4 *>(y + c)), w = __ldg(reinterpret_cast<const float4 *>(o + c));
                d = fmaf(u.x, w.x, fmaf(u.y, w.y, fmaf(u.z, w.z, fmaf(u.w, w.w, d))));
            }
        } else {
            for (int c = lane; c < a.dim; c += 16) d = fmaf(y[c], o[c], d);
        }
    }
#pragma unroll
    for (int o = 8; o; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o, 16);
    if (lane == 0) a.delta[(b * a.q_heads + h) * a.q_len + i] = d;
}

template <int DP> constexpr int bwd_shared()
{
    return 4 * (STRIDE<DP> * (2 * OWN + 4 * ROWS) + 4 * ROWS);
}

template <int DP>
__device__ __forceinline__ void dq_block(const AttnArgs &a, float *smem, int tile, int64_t bh, bool vec)
{
    constexpr int TILE = ROWS * STRIDE<DP>;
    float *Q = smem, *DO = Q + OWN * STRIDE<DP>, *stream = DO + OWN * STRIDE<DP>;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g8 = lane >> 2, t = lane & 3;
    const int64_t b = bh / a.q_heads;
    const int h = (int)(bh % a.q_heads), g = h / a.group;
    const AttnSeq s = attn_seq(a, b);
    const int r0 = tile * OWN, w0 = r0 + 16 * warp;
    const int last = min(r0 + OWN, s.nq) - 1;
    const int j_end = last >= r0 ? attn_hi(a, s, last) : 0;
    const int j_begin = attn_lo(a, s, r0) / ROWS * ROWS;
    auto fetch = [&](int j0, int at) {
        copy_rows<ROWS, DP>(stream + at * 2 * TILE, a.k, b, g, j0, s.nk, a.dim, vec);
        copy_rows<ROWS, DP>(stream + at * 2 * TILE + TILE, a.v, b, g, j0, s.nk, a.dim, vec);
        copies_commit();
    };
    if (j_begin < j_end) {
        copy_rows<OWN, DP>(Q, a.q, b, h, r0, s.nq, a.dim, vec);
        copy_rows<OWN, DP>(DO, a.dout, b, h, r0, s.nq, a.dim, vec);
        fetch(j_begin, 0);
    }
    const int w_last = min(w0 + 16, s.nq) - 1;
    const int w_lo = attn_lo(a, s, w0), w_lo_last = attn_lo(a, s, w0 + 15), w_hi = attn_hi(a, s, w0);
    const int w_end = w_last >= w0 ? attn_hi(a, s, w_last) : 0;
    const bool whole = w_last == w0 + 15;
    int lo[2], hi[2];
    float lse2[2], delta[2];
    cudaGridDependencySynchronize();                       // delta is ready
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int i = w0 + g8 + 8 * r;
        lo[r] = attn_lo(a, s, i);
        hi[r] = attn_hi(a, s, i);
        lse2[r] = i < s.nq ? a.lse[bh * a.q_len + i] * LOG2E : 0.f;
        delta[r] = i < s.nq ? a.delta[bh * a.q_len + i] : 0.f;
    }
    const float mul2e = a.scale * LOG2E;
    float acc[DP / 8][4];
    clear(acc);
    int at = 0;
    for (int j0 = j_begin; j0 < j_end; j0 += ROWS, at ^= 1) {
        copies_wait();
        __syncthreads();
        if (j0 + ROWS < j_end) fetch(j0 + ROWS, at ^ 1);
        const See what = see(w_lo, w_lo_last, w_hi, w_end, j0, ROWS);
        if (what == NOTHING) continue;
        const float *K = stream + at * 2 * TILE, *V = K + TILE;
        float p[N][4], dp[N][4];
        dot<N, DP>(p, Q + 16 * warp * STRIDE<DP>, K);
        dot<N, DP>(dp, DO + 16 * warp * STRIDE<DP>, V);
        const bool all = what == ALL && whole;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = j0 + 8 * n + (i & 1 ? other(t) : t);
                const float e = exp2_fast(fmaf(p[n][i], mul2e, -lse2[i >> 1])) * (dp[n][i] - delta[i >> 1]);
                dp[n][i] = all || (j >= lo[i >> 1] && j < hi[i >> 1]) ? e : 0.f;
            }
        mul<N, DP>(acc, dp, K);
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int i = w0 + g8 + 8 * r;
        if (i < a.q_len) store_row<DP>(row_of(a.dq, b, i, h), acc, r, a.scale, a.dim, vec);
    }
    if (__any_sync(0xffffffffu, has_nan(acc))) again::query_gradients_here<float>(a, b, h, w0, w0 + 16, 0, a.dim);
}

template <int DP>
__device__ __forceinline__ void dkdv_block(const AttnArgs &a, float *smem, int tile, int64_t bg, bool vec)
{
    constexpr int TILE = ROWS * STRIDE<DP>;
    float *K = smem, *V = K + OWN * STRIDE<DP>, *stream = V + OWN * STRIDE<DP>, *stats = stream + 4 * TILE;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g8 = lane >> 2, t = lane & 3;
    const int64_t b = bg / a.kv_heads;
    const int g = (int)(bg % a.kv_heads);
    const AttnSeq s = attn_seq(a, b);
    const int j0 = tile * OWN, w0 = j0 + 16 * warp;
    const int q_end = j0 < s.nk ? attn_q_last(a, s, min(j0 + OWN, s.nk)) : 0;
    const int q_begin = attn_q_first(a, s, j0) / ROWS * ROWS;
    const int per_head = q_begin < q_end ? (q_end - q_begin + ROWS - 1) / ROWS : 0;
    const int64_t steps = (int64_t)per_head * a.group;
    int next_h = g * a.group, next_r = q_begin;            // the tile that is fetched next
    auto fetch = [&](int at) {
        copy_rows<ROWS, DP>(stream + at * 2 * TILE, a.q, b, next_h, next_r, s.nq, a.dim, vec);
        copy_rows<ROWS, DP>(stream + at * 2 * TILE + TILE, a.dout, b, next_h, next_r, s.nq, a.dim, vec);
        if (threadIdx.x < 2 * ROWS) {
            const int x = threadIdx.x % ROWS;
            const float *from = (threadIdx.x < ROWS ? a.lse : a.delta) + (b * a.q_heads + next_h) * a.q_len;
            const bool in = next_r + x < s.nq;
            copy4(stats + at * 2 * ROWS + threadIdx.x, in ? from + next_r + x : from, in);
        }
        copies_commit();
        next_r += ROWS;
        if (next_r >= q_end) {
            next_r = q_begin;
            ++next_h;
        }
    };
    if (steps) {
        copy_rows<OWN, DP>(K, a.k, b, g, j0, s.nk, a.dim, vec);
        copy_rows<OWN, DP>(V, a.v, b, g, j0, s.nk, a.dim, vec);
    }
    cudaGridDependencySynchronize();                       // delta is ready
    if (steps) fetch(0);
    const int w_last = min(w0 + 16, s.nk) - 1;
    const bool whole = w_last == w0 + 15;
    // queries that a key sees, [lo, hi); none for a key past the sequence's end
    const int w_lo = attn_q_first(a, s, w0), w_lo_last = attn_q_first(a, s, w0 + 15);
    const int w_hi = attn_q_last(a, s, w0 + 1), w_end = w_last >= w0 ? attn_q_last(a, s, w_last + 1) : 0;
    int lo[2], hi[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int j = w0 + g8 + 8 * r;
        lo[r] = attn_q_first(a, s, j);
        hi[r] = j < s.nk ? attn_q_last(a, s, j + 1) : 0;
    }
    const float mul2e = a.scale * LOG2E;
    float dk[DP / 8][4], dv[DP / 8][4];
    clear(dk);
    clear(dv);
    int at = 0, r0 = q_begin;
    for (int64_t x = 0; x < steps; ++x, at ^= 1) {
        copies_wait();
        __syncthreads();
        if (x + 1 < steps) fetch(at ^ 1);
        const int i0 = r0;
        r0 = r0 + ROWS >= q_end ? q_begin : r0 + ROWS;
        const See what = see(w_lo, w_lo_last, w_hi, w_end, i0, ROWS);
        if (what == NOTHING) continue;
        const float *Q = stream + at * 2 * TILE, *DO = Q + TILE, *lse = stats + at * 2 * ROWS, *delta = lse + ROWS;
        float p[N][4], dp[N][4];
        dot<N, DP>(p, K + 16 * warp * STRIDE<DP>, Q);
        dot<N, DP>(dp, V + 16 * warp * STRIDE<DP>, DO);
        const bool all = what == ALL && whole;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int q = 8 * n + (c ? other(t) : t);
                const float l = lse[q] * LOG2E, d = delta[q];
#pragma unroll
                for (int i = c; i < 4; i += 2) {
                    const bool in = all || (i0 + q >= lo[i >> 1] && i0 + q < hi[i >> 1]);
                    const float e = exp2_fast(fmaf(p[n][i], mul2e, -l));
                    p[n][i] = in ? e : 0.f;
                    dp[n][i] = in ? e * (dp[n][i] - d) : 0.f;
                }
            }
        mul<N, DP>(dv, p, DO);
        mul<N, DP>(dk, dp, Q);
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int j = w0 + g8 + 8 * r;
        if (j >= a.k_len) continue;
        store_row<DP>(row_of(a.dk, b, j, g), dk, r, a.scale, a.dim, vec);
        store_row<DP>(row_of(a.dv, b, j, g), dv, r, 1.f, a.dim, vec);
    }
    if (__any_sync(0xffffffffu, has_nan(dk) || has_nan(dv))) again::key_gradients_here<float>(a, b, g, w0, w0 + 16, true, true);
}

// blocks [0, k_blocks) make dk and dv, the others dq.  Each kind starts with its longest: under a causal bound
// the first keys have most queries and the last queries most keys.
template <int DP>
__global__ void __launch_bounds__(THREADS, 3) attn_f32_backward_kernel(const __grid_constant__ AttnArgs a, int64_t k_blocks, int q_tiles, bool vec)
{
    extern __shared__ float4 smem4[];
    float *smem = reinterpret_cast<float *>(smem4);
    if (blockIdx.x < k_blocks) {
        const int64_t heads = a.batch * a.kv_heads;
        dkdv_block<DP>(a, smem, (int)(blockIdx.x / heads), blockIdx.x % heads, vec);
    } else {
        const int64_t heads = a.batch * a.q_heads, x = blockIdx.x - k_blocks;
        dq_block<DP>(a, smem, q_tiles - 1 - (int)(x / heads), x % heads, vec);
    }
}

template <int DP>
gs_status forward_t(const AttnArgs &a, cudaStream_t st)
{
    static SharedRecord record;
    const int tiles = (a.q_len + OWN - 1) / OWN;
    const int64_t blocks = a.batch * a.q_heads * tiles;
    gs_status s;
    if ((s = blocks_ok(blocks)) != GS_OK || (s = allow_shared(attn_f32_forward_kernel<DP>, fwd_shared<DP>(), record)) != GS_OK) return s;
    attn_f32_forward_kernel<DP><<<(unsigned)blocks, THREADS, fwd_shared<DP>(), st>>>(a, tiles, rows_of_four(a, 4, false));
    GS_CUDA_TRY(cudaGetLastError());
    return GS_OK;
}

template <int DP>
gs_status backward_t(const AttnArgs &a, cudaStream_t st)
{
    static SharedRecord record;
    const bool vec = rows_of_four(a, 4, true);
    const int q_tiles = (a.q_len + OWN - 1) / OWN, k_tiles = (a.k_len + OWN - 1) / OWN;
    const int64_t k_blocks = a.batch * a.kv_heads * k_tiles, blocks = k_blocks + a.batch * a.q_heads * q_tiles;
    const int64_t delta_blocks = (a.batch * a.q_heads * a.q_len + 15) / 16;
    gs_status s;
    if ((s = blocks_ok(blocks)) != GS_OK || (s = blocks_ok(delta_blocks)) != GS_OK ||
        (s = allow_shared(attn_f32_backward_kernel<DP>, bwd_shared<DP>(), record)) != GS_OK)
        return s;
    attn_f32_delta_kernel<<<(unsigned)delta_blocks, 256, 0, st>>>(a, vec);
    GS_CUDA_TRY(cudaGetLastError());
    GS_CUDA_TRY(launch_after(attn_f32_backward_kernel<DP>, (int)blocks, THREADS, bwd_shared<DP>(), st, a, k_blocks, q_tiles, vec));
    return GS_OK;
}

}  // namespace

gs_status attn_f32_forward(const AttnArgs &a, cudaStream_t st)
{
    if (a.dim <= 32) return forward_t<32>(a, st);
    return a.dim <= 64 ? forward_t<64>(a, st) : forward_t<128>(a, st);
}

// head_dim up to 64: dk and dv of 128 columns do not fit a thread's registers
gs_status attn_f32_backward(const AttnArgs &a, cudaStream_t st)
{
    return a.dim <= 32 ? backward_t<32>(a, st) : backward_t<64>(a, st);
}

}  // namespace gs
