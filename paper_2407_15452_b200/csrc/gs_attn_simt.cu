// Attention on the CUDA cores, everything in fp32 (products included): fp32 tensors that the tensor cores do not take
// (short ones, and backward few or wide heads), and long 16-bit tensors that TMA cannot address.
//
// A block of 4 * BT threads works on BT x BT tiles of scores; thread (ty, tx) holds 4 rows x BT/16
// columns of a tile and 4 rows x DP/16 columns of an accumulator, DP = head_dim padded to 32, 64 or
// 128 with zeros.  Operands sit in shared memory row-major with 4 floats of padding: 16-byte reads
// of consecutive rows then fall into different banks, and the same copy serves the products over
// the head dimension (row . row) and those over positions (column blocks of rows).  The bound is the rate of
// fp32 multiply-adds (35.5e12 a second measured); they are issued in pairs, which is no faster by itself but
// leaves issue slots for the shared-memory reads, and the next tile's rows travel to registers meanwhile.
//  forward : one block per BT query rows, running maximum and sum over the key tiles
//  backward: a sequence that fits one tile has its dq, dk and dv from one block (delta from the probabilities).
//            Longer ones: blocks of BT query rows make dq, blocks of BT key rows dk and dv, in one launch; each
//            computes p = exp(s - lse) and the delta it needs.  A key block loops over the query heads of
//            its group and their query tiles, so shared heads are summed in a fixed order without atomics.
#include "gs_attn_again.cuh"
#include "gs_tc.cuh"

namespace gs {

using tc::fma2;
using tc::mul2;

template <typename T>
__device__ __forceinline__ T *row_of(const AttnTensor &t, int64_t b, int64_t pos, int64_t head)
{
    return reinterpret_cast<T *>(t.p) + b * t.sb + pos * t.sl + head * t.sh;
}

// Rows [r0, r0 + BT) of one head, this thread's share of them; rows >= n and columns >= dim are zeros
// (whatever the padding of the input holds, NaN included, is not read)
template <typename T, int BT, int DP>
__device__ __forceinline__ void fetch_rows(float4 (&x)[DP / 16], const AttnTensor &t, int64_t b, int64_t head,
                                           int r0, int n, int dim, bool vec)
{
    const T *base = row_of<T>(t, b, 0, head);
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
        const int e = threadIdx.x + k * BT * 4, r = r0 + e / (DP / 4), c = (e % (DP / 4)) * 4;
        float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r < n && c < dim) {
            const T *p = base + (int64_t)r * t.sl + c;
            if (vec) {
                if constexpr (sizeof(T) == 4) {
                    f = __ldg(reinterpret_cast<const float4 *>(p));
                } else {
                    const uint2 u = __ldg(reinterpret_cast<const uint2 *>(p));
                    T h[4];
                    *reinterpret_cast<uint2 *>(h) = u;
                    f = make_float4(to_f(h[0]), to_f(h[1]), to_f(h[2]), to_f(h[3]));
                }
            } else {
                f.x = to_f(p[0]);
                if (c + 1 < dim) f.y = to_f(p[1]);
                if (c + 2 < dim) f.z = to_f(p[2]);
                if (c + 3 < dim) f.w = to_f(p[3]);
            }
        }
        x[k] = f;
    }
}
template <int BT, int DP>
__device__ __forceinline__ void put_rows(float (*dst)[DP + 4], const float4 (&x)[DP / 16])
{
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
        const int e = threadIdx.x + k * BT * 4;
        *reinterpret_cast<float4 *>(&dst[e / (DP / 4)][(e % (DP / 4)) * 4]) = x[k];
    }
}
template <typename T, int BT, int DP>
__device__ __forceinline__ void load_rows(float (*dst)[DP + 4], const AttnTensor &t, int64_t b, int64_t head,
                                          int r0, int n, int dim, bool vec)
{
    float4 x[DP / 16];
    fetch_rows<T, BT, DP>(x, t, b, head, r0, n, dim, vec);
    put_rows<BT, DP>(dst, x);
}

// s[i][j] = a[4 ty + i] . b[tx + 16 j]; even and odd columns summed apart
template <int BT, int DP>
__device__ __forceinline__ void dot_rows(float (&s)[4][BT / 16], const float (*a)[DP + 4], const float (*b)[DP + 4],
                                         int ty, int tx)
{
    float2 t[4][BT / 16];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < BT / 16; ++j) t[i][j] = make_float2(0.f, 0.f);
#pragma unroll 4
    for (int c = 0; c < DP; c += 4) {
        float4 x[4], y[BT / 16];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const float4 *>(&a[4 * ty + i][c]);
#pragma unroll
        for (int j = 0; j < BT / 16; ++j) y[j] = *reinterpret_cast<const float4 *>(&b[tx + 16 * j][c]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < BT / 16; ++j) {
                t[i][j] = fma2(make_float2(x[i].x, x[i].y), make_float2(y[j].x, y[j].y), t[i][j]);
                t[i][j] = fma2(make_float2(x[i].z, x[i].w), make_float2(y[j].z, y[j].w), t[i][j]);
            }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < BT / 16; ++j) s[i][j] = t[i][j].x + t[i][j].y;
}

// this thread's DP/16 columns of a row, as pairs: columns 4 tx.. of every 64 (2 tx.. if DP is 32)
template <int DP>
__device__ __forceinline__ void load_cols(float2 (&y)[DP / 32], const float *row, int tx)
{
    if constexpr (DP >= 64) {
#pragma unroll
        for (int m = 0; m < DP / 64; ++m) {
            const float4 v = *reinterpret_cast<const float4 *>(row + 64 * m + 4 * tx);
            y[2 * m] = make_float2(v.x, v.y);
            y[2 * m + 1] = make_float2(v.z, v.w);
        }
    } else {
        y[0] = *reinterpret_cast<const float2 *>(row + 2 * tx);
    }
}

// acc[i][:] += sum_j p[4 ty + i][j] x[j][:]
template <int BT, int DP>
__device__ __forceinline__ void mul_rows(float2 (&acc)[4][DP / 32], const float (*p)[BT + 4], const float (*x)[DP + 4],
                                         int ty, int tx)
{
#pragma unroll 2
    for (int j = 0; j < BT; j += 4) {
        float w[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<float4 *>(w[i]) = *reinterpret_cast<const float4 *>(&p[4 * ty + i][j]);
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
            float2 y[DP / 32];
            load_cols<DP>(y, x[j + jj], tx);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < DP / 32; ++c) acc[i][c] = fma2(make_float2(w[i][jj], w[i][jj]), y[c], acc[i][c]);
        }
    }
}

// acc[i][:] += sum_r p[r][4 ty + i] x[r][:]
template <int BT, int DP>
__device__ __forceinline__ void mul_cols(float2 (&acc)[4][DP / 32], const float (*p)[BT + 4], const float (*x)[DP + 4],
                                         int ty, int tx)
{
#pragma unroll 4
    for (int r = 0; r < BT; ++r) {
        float w[4];
        float2 y[DP / 32];
        *reinterpret_cast<float4 *>(w) = *reinterpret_cast<const float4 *>(&p[r][4 * ty]);
        load_cols<DP>(y, x[r], tx);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < DP / 32; ++c) acc[i][c] = fma2(make_float2(w[i], w[i]), y[c], acc[i][c]);
    }
}

template <int N>
__device__ __forceinline__ void clear(float2 (&acc)[4][N])
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < N; ++c) acc[i][c] = make_float2(0.f, 0.f);
}

template <typename T, int DP>
__device__ __forceinline__ void store_row(T *row, const float2 (&acc)[DP / 32], float mul, int tx, int dim, bool vec)
{
    constexpr int CW = DP >= 64 ? 4 : 2;
#pragma unroll
    for (int m = 0; m < DP / (16 * CW); ++m) {
        const int c = 16 * CW * m + CW * tx;
        float v[CW];
#pragma unroll
        for (int x = 0; x < CW / 2; ++x) {
            v[2 * x] = acc[m * CW / 2 + x].x * mul;
            v[2 * x + 1] = acc[m * CW / 2 + x].y * mul;
        }
        if constexpr (sizeof(T) == 4 && CW == 4) {
            if (vec) {
                if (c < dim) *reinterpret_cast<float4 *>(row + c) = make_float4(v[0], v[1], v[2], v[3]);
                continue;
            }
        }
#pragma unroll
        for (int x = 0; x < CW; ++x)
            if (c + x < dim) row[c + x] = from_f<T>(v[x]);
    }
}

// first of the eight rows of a tile that this thread's warp has
__device__ __forceinline__ int warp_rows() { return (int)(threadIdx.x >> 5) * 8; }

template <int N>
__device__ __forceinline__ bool has_nan(const float2 (&acc)[N])
{
    float t = 0.f;
#pragma unroll
    for (int c = 0; c < N; ++c) t += acc[c].x + acc[c].y;
    return t != t;
}
__device__ __forceinline__ float half_warp_max(float v)
{
#pragma unroll
    for (int o = 8; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float half_warp_sum(float v)
{
#pragma unroll
    for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

template <typename T, int BT, int DP>
__global__ void __launch_bounds__(BT * 4, BT == 64 && DP <= 64 ? 2 : 1) attn_simt_forward_kernel(const __grid_constant__ AttnArgs a, int tiles, bool vec)
{
    extern __shared__ float4 smem4[];
    float(*Q)[DP + 4] = reinterpret_cast<float(*)[DP + 4]>(smem4);
    float(*KV)[DP + 4] = Q + BT;                          // holds K, then V of the same tile
    float(*P)[BT + 4] = reinterpret_cast<float(*)[BT + 4]>(KV + BT);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int64_t heads = a.batch * a.q_heads;
    // row tiles are the slowest index and run from the last: under a causal bound the longest go first
    const int tile = tiles - 1 - (int)(blockIdx.x / heads);
    const int64_t bh = blockIdx.x % heads, b = bh / a.q_heads;
    const int h = (int)(bh % a.q_heads), g = h / a.group;
    const AttnSeq s = attn_seq(a, b);
    const int r0 = tile * BT, r1 = min(r0 + BT, a.q_len);

    float2 acc[4][DP / 32];
    float top[4], sum[4];
    int lo[4], hi[4];
    clear(acc);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        top[i] = -INFINITY;
        sum[i] = 0.f;
        lo[i] = attn_lo(a, s, r0 + 4 * ty + i);
        hi[i] = attn_hi(a, s, r0 + 4 * ty + i);
    }
    const int last = min(r1, s.nq) - 1;
    const int j_end = last >= r0 ? attn_hi(a, s, last) : 0;
    const int j_begin = attn_lo(a, s, r0) / BT * BT;
    float4 next_k[DP / 16], next_v[DP / 16];
    if (j_begin < j_end) {
        fetch_rows<T, BT, DP>(next_k, a.k, b, g, j_begin, s.nk, a.dim, vec);
        load_rows<T, BT, DP>(Q, a.q, b, h, r0, s.nq, a.dim, vec);
    }
    for (int j0 = j_begin; j0 < j_end; j0 += BT) {
        put_rows<BT, DP>(KV, next_k);
        fetch_rows<T, BT, DP>(next_v, a.v, b, g, j0, s.nk, a.dim, vec);
        __syncthreads();
        float sc[4][BT / 16];
        dot_rows<BT, DP>(sc, Q, KV, ty, tx);
        __syncthreads();
        put_rows<BT, DP>(KV, next_v);
        if (j0 + BT < j_end) fetch_rows<T, BT, DP>(next_k, a.k, b, g, j0 + BT, s.nk, a.dim, vec);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float m = top[i];
#pragma unroll
            for (int j = 0; j < BT / 16; ++j) {
                const int c = j0 + tx + 16 * j;
                sc[i][j] = c >= lo[i] && c < hi[i] ? sc[i][j] * a.scale : -INFINITY;
                m = fmaxf(m, sc[i][j]);
            }
            m = half_warp_max(m);
            const float base = m == -INFINITY ? 0.f : m;       // no visible key so far: every term is exp(-inf) = 0
            const float keep = expf(top[i] - base);
            float part = 0.f;
#pragma unroll
            for (int j = 0; j < BT / 16; ++j) {
                const float p = expf(sc[i][j] - base);
                part += p;
                P[4 * ty + i][tx + 16 * j] = p;
            }
            sum[i] = sum[i] * keep + half_warp_sum(part);
            top[i] = m;
#pragma unroll
            for (int c = 0; c < DP / 32; ++c) acc[i][c] = mul2(acc[i][c], make_float2(keep, keep));
        }
        __syncthreads();
        mul_rows<BT, DP>(acc, P, KV, ty, tx);
        __syncthreads();
    }
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + 4 * ty + i;
        nan = nan || has_nan(acc[i]);
        if (r >= a.q_len) continue;
        store_row<T, DP>(row_of<T>(a.out, b, r, h), acc[i], sum[i] > 0.f || sum[i] != sum[i] ? 1.f / sum[i] : 0.f, tx, a.dim, vec);
        if (tx == 0) a.lse[bh * a.q_len + r] = sum[i] == 0.f ? -INFINITY : top[i] + logf(sum[i]);
    }
    if (__any_sync(0xffffffffu, nan)) again::outputs<T>(a, b, h, r0 + warp_rows(), r0 + warp_rows() + 8);
}

// dk and dv of the keys j0 + 4 ty..
template <typename T, int BT, int DP>
__device__ __forceinline__ void store_keys(const AttnArgs &a, int64_t b, int g, int j0, const float2 (&dk)[4][DP / 32],
                                           const float2 (&dv)[4][DP / 32], int tx, int ty, bool vec)
{
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = j0 + 4 * ty + i;
        nan = nan || has_nan(dk[i]) || has_nan(dv[i]);
        if (j >= a.k_len) continue;
        store_row<T, DP>(row_of<T>(a.dk, b, j, g), dk[i], a.scale, tx, a.dim, vec);
        store_row<T, DP>(row_of<T>(a.dv, b, j, g), dv[i], 1.f, tx, a.dim, vec);
    }
    if (__any_sync(0xffffffffu, nan)) again::key_gradients<T>(a, b, g, j0 + warp_rows(), j0 + warp_rows() + 8, true, true);
}

template <int BT, int DP>
struct BwdTiles {                                          // shared memory of the backward kernels
    float a[BT][DP + 4], b[BT][DP + 4], c[BT][DP + 4], d[BT][DP + 4];
    float p[BT][BT + 4], s[BT][BT + 4];
    float lse[BT], delta[BT];
};

// p and, in place of dp, ds = p (dp - delta) of a tile whose rows are queries r0.. and columns keys j0..
template <int BT>
__device__ __forceinline__ void p_and_ds(float (&p)[4][BT / 16], float (&dp)[4][BT / 16], const float (&lse)[4], const float (&delta)[4],
                                         const int (&lo)[4], const int (&hi)[4], float scale, int j0, int tx)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < BT / 16; ++j) {
            const int c = j0 + tx + 16 * j;
            const bool in = c >= lo[i] && c < hi[i];
            p[i][j] = in ? expf(p[i][j] * scale - lse[i]) : 0.f;
            dp[i][j] = in ? p[i][j] * (dp[i][j] - delta[i]) : 0.f;
        }
}

// sequences of up to BT queries and keys; one block per key/value head
template <typename T, int BT, int DP>
__global__ void __launch_bounds__(BT * 4) attn_simt_backward_one_kernel(const __grid_constant__ AttnArgs a, bool vec)
{
    extern __shared__ float4 smem4[];
    BwdTiles<BT, DP> &t = *reinterpret_cast<BwdTiles<BT, DP> *>(smem4);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int64_t b = blockIdx.x / a.kv_heads;
    const int g = (int)(blockIdx.x % a.kv_heads);
    const AttnSeq s = attn_seq(a, b);
    float2 dk[4][DP / 32], dv[4][DP / 32];
    clear(dk);
    clear(dv);
    load_rows<T, BT, DP>(t.a, a.k, b, g, 0, s.nk, a.dim, vec);
    load_rows<T, BT, DP>(t.b, a.v, b, g, 0, s.nk, a.dim, vec);
    int lo[4], hi[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        lo[i] = attn_lo(a, s, 4 * ty + i);
        hi[i] = attn_hi(a, s, 4 * ty + i);
    }
    bool nan = false;
    for (int h = g * a.group; h < (g + 1) * a.group; ++h) {
        const float *lse_at = a.lse + (b * a.q_heads + h) * a.q_len;
        float lse[4], delta[4] = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) lse[i] = 4 * ty + i < s.nq ? lse_at[4 * ty + i] : 0.f;
        __syncthreads();
        load_rows<T, BT, DP>(t.c, a.q, b, h, 0, s.nq, a.dim, vec);
        load_rows<T, BT, DP>(t.d, a.dout, b, h, 0, s.nq, a.dim, vec);
        __syncthreads();
        float p[4][BT / 16], dp[4][BT / 16];
        dot_rows<BT, DP>(p, t.c, t.a, ty, tx);
        dot_rows<BT, DP>(dp, t.d, t.b, ty, tx);
        // the whole row is here: delta = sum_j p dp, and then ds = p dp - p delta
        p_and_ds<BT>(p, dp, lse, delta, lo, hi, a.scale, 0, tx);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float d = 0.f;
#pragma unroll
            for (int j = 0; j < BT / 16; ++j) d += dp[i][j];
            d = half_warp_sum(d);
#pragma unroll
            for (int j = 0; j < BT / 16; ++j) {
                t.p[4 * ty + i][tx + 16 * j] = p[i][j];
                t.s[4 * ty + i][tx + 16 * j] = fmaf(-p[i][j], d, dp[i][j]);
            }
        }
        __syncthreads();
        float2 dq[4][DP / 32];
        clear(dq);
        mul_rows<BT, DP>(dq, t.s, t.a, ty, tx);
        mul_cols<BT, DP>(dv, t.p, t.d, ty, tx);
        mul_cols<BT, DP>(dk, t.s, t.c, ty, tx);
#pragma unroll
        for (int i = 0; i < 4; ++i)
        {
            nan = nan || has_nan(dq[i]);
            if (4 * ty + i < a.q_len) store_row<T, DP>(row_of<T>(a.dq, b, 4 * ty + i, h), dq[i], a.scale, tx, a.dim, vec);
        }
    }
    store_keys<T, BT, DP>(a, b, g, 0, dk, dv, tx, ty, vec);
    if (__any_sync(0xffffffffu, nan))
        for (int h = g * a.group; h < (g + 1) * a.group; ++h) again::query_gradients<T>(a, b, h, warp_rows(), warp_rows() + 8, 0, a.dim);
}

// this thread's part (every 16th group of four columns) of the dot products of rows 4 ty.. of dO, in shared
// memory, with the output's rows in global memory; summed over tx
template <typename T, int DP>
__device__ __forceinline__ void row_deltas(float (&delta)[4], const float (*DO)[DP + 4], const AttnArgs &a, int64_t b, int h, int r0,
                                           int n, int ty, int tx, bool vec)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + 4 * ty + i;
        float d = 0.f;
        if (r < n) {
            const T *o = row_of<T>(a.out, b, r, h);
            for (int c = 4 * tx; c < a.dim; c += 64) {
                const float4 x = *reinterpret_cast<const float4 *>(&DO[4 * ty + i][c]);
                if (sizeof(T) == 4 && vec) {
                    const float4 y = __ldg(reinterpret_cast<const float4 *>(o + c));
                    d = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, d))));
                } else {
                    d = fmaf(x.x, to_f(o[c]), d);
                    if (c + 1 < a.dim) d = fmaf(x.y, to_f(o[c + 1]), d);
                    if (c + 2 < a.dim) d = fmaf(x.z, to_f(o[c + 2]), d);
                    if (c + 3 < a.dim) d = fmaf(x.w, to_f(o[c + 3]), d);
                }
            }
        }
        delta[i] = half_warp_sum(d);
    }
}

template <typename T, int BT, int DP>
__device__ __forceinline__ void dq_block(const AttnArgs &a, BwdTiles<BT, DP> &t, int tile, int64_t bh, bool vec)
{
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int64_t b = bh / a.q_heads;
    const int h = (int)(bh % a.q_heads), g = h / a.group;
    const AttnSeq s = attn_seq(a, b);
    const int r0 = tile * BT, r1 = min(r0 + BT, a.q_len);
    const int last = min(r1, s.nq) - 1;
    const int j_begin = attn_lo(a, s, r0) / BT * BT, j_end = last >= r0 ? attn_hi(a, s, last) : 0;
    float2 acc[4][DP / 32];
    clear(acc);
    if (j_begin < j_end) {
        float4 next_k[DP / 16], next_v[DP / 16];
        fetch_rows<T, BT, DP>(next_k, a.k, b, g, j_begin, s.nk, a.dim, vec);
        fetch_rows<T, BT, DP>(next_v, a.v, b, g, j_begin, s.nk, a.dim, vec);
        load_rows<T, BT, DP>(t.a, a.q, b, h, r0, s.nq, a.dim, vec);
        load_rows<T, BT, DP>(t.b, a.dout, b, h, r0, s.nq, a.dim, vec);
        __syncthreads();
        float lse[4], delta[4];
        int lo[4], hi[4];
        row_deltas<T, DP>(delta, t.b, a, b, h, r0, s.nq, ty, tx, vec);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = r0 + 4 * ty + i;
            lo[i] = attn_lo(a, s, r);
            hi[i] = attn_hi(a, s, r);
            lse[i] = r < s.nq ? a.lse[bh * a.q_len + r] : 0.f;
        }
        for (int j0 = j_begin; j0 < j_end; j0 += BT) {
            put_rows<BT, DP>(t.c, next_k);
            put_rows<BT, DP>(t.d, next_v);
            __syncthreads();
            if (j0 + BT < j_end) {
                fetch_rows<T, BT, DP>(next_k, a.k, b, g, j0 + BT, s.nk, a.dim, vec);
                fetch_rows<T, BT, DP>(next_v, a.v, b, g, j0 + BT, s.nk, a.dim, vec);
            }
            float p[4][BT / 16], ds[4][BT / 16];
            dot_rows<BT, DP>(p, t.a, t.c, ty, tx);
            dot_rows<BT, DP>(ds, t.b, t.d, ty, tx);
            p_and_ds<BT>(p, ds, lse, delta, lo, hi, a.scale, j0, tx);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < BT / 16; ++j) t.s[4 * ty + i][tx + 16 * j] = ds[i][j];
            __syncwarp();                                  // a row of ds is written and read by one half warp
            mul_rows<BT, DP>(acc, t.s, t.c, ty, tx);
            __syncthreads();
        }
    }
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + 4 * ty + i;
        nan = nan || has_nan(acc[i]);
        if (r < a.q_len) store_row<T, DP>(row_of<T>(a.dq, b, r, h), acc[i], a.scale, tx, a.dim, vec);
    }
    if (__any_sync(0xffffffffu, nan)) again::query_gradients<T>(a, b, h, r0 + warp_rows(), r0 + warp_rows() + 8, 0, a.dim);
}

template <typename T, int BT, int DP>
__device__ __forceinline__ void dkdv_block(const AttnArgs &a, BwdTiles<BT, DP> &t, int tile, int64_t bg, bool vec)
{
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int64_t b = bg / a.kv_heads;
    const int g = (int)(bg % a.kv_heads);
    const AttnSeq s = attn_seq(a, b);
    const int j0 = tile * BT;
    float2 dk[4][DP / 32], dv[4][DP / 32];
    clear(dk);
    clear(dv);
    const int q_end = j0 < s.nk ? attn_q_last(a, s, min(j0 + BT, s.nk)) : 0;
    const int q_begin = attn_q_first(a, s, j0) / BT * BT;
    if (q_begin < q_end) {
        const int per_head = (q_end - q_begin + BT - 1) / BT, n = per_head * a.group;
        float4 next_q[DP / 16], next_o[DP / 16];
        fetch_rows<T, BT, DP>(next_q, a.q, b, g * a.group, q_begin, s.nq, a.dim, vec);
        fetch_rows<T, BT, DP>(next_o, a.dout, b, g * a.group, q_begin, s.nq, a.dim, vec);
        load_rows<T, BT, DP>(t.a, a.k, b, g, j0, s.nk, a.dim, vec);
        load_rows<T, BT, DP>(t.b, a.v, b, g, j0, s.nk, a.dim, vec);
        for (int x = 0; x < n; ++x) {
            const int h = g * a.group + x / per_head, r0 = q_begin + (x % per_head) * BT;
            put_rows<BT, DP>(t.c, next_q);
            put_rows<BT, DP>(t.d, next_o);
            __syncthreads();
            if (x + 1 < n) {
                const int h1 = g * a.group + (x + 1) / per_head, r1 = q_begin + ((x + 1) % per_head) * BT;
                fetch_rows<T, BT, DP>(next_q, a.q, b, h1, r1, s.nq, a.dim, vec);
                fetch_rows<T, BT, DP>(next_o, a.dout, b, h1, r1, s.nq, a.dim, vec);
            }
            float lse[4], delta[4];
            int lo[4], hi[4];
            row_deltas<T, DP>(delta, t.d, a, b, h, r0, s.nq, ty, tx, vec);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = r0 + 4 * ty + i;
                lo[i] = attn_lo(a, s, r);
                hi[i] = attn_hi(a, s, r);
                lse[i] = r < s.nq ? a.lse[(b * a.q_heads + h) * a.q_len + r] : 0.f;
            }
            float p[4][BT / 16], ds[4][BT / 16];
            dot_rows<BT, DP>(p, t.c, t.a, ty, tx);
            dot_rows<BT, DP>(ds, t.d, t.b, ty, tx);
            p_and_ds<BT>(p, ds, lse, delta, lo, hi, a.scale, j0, tx);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < BT / 16; ++j) {
                    t.p[4 * ty + i][tx + 16 * j] = p[i][j];
                    t.s[4 * ty + i][tx + 16 * j] = ds[i][j];
                }
            __syncthreads();
            mul_cols<BT, DP>(dv, t.p, t.d, ty, tx);
            mul_cols<BT, DP>(dk, t.s, t.c, ty, tx);
            __syncthreads();
        }
    }
    store_keys<T, BT, DP>(a, b, g, j0, dk, dv, tx, ty, vec);
}

// blocks [0, k_blocks) make dk and dv, the others dq.  Each kind starts with its longest: under a causal bound
// the first keys have most queries and the last queries most keys.
template <typename T, int BT, int DP>
__global__ void __launch_bounds__(BT * 4, DP <= 64 ? 2 : 1) attn_simt_backward_kernel(const __grid_constant__ AttnArgs a, int64_t k_blocks, int q_tiles, bool vec)
{
    extern __shared__ float4 smem4[];
    BwdTiles<BT, DP> &t = *reinterpret_cast<BwdTiles<BT, DP> *>(smem4);
    if (blockIdx.x < k_blocks) {
        const int64_t heads = a.batch * a.kv_heads;
        dkdv_block<T, BT, DP>(a, t, (int)(blockIdx.x / heads), blockIdx.x % heads, vec);
    } else {
        const int64_t heads = a.batch * a.q_heads, x = blockIdx.x - k_blocks;
        dq_block<T, BT, DP>(a, t, q_tiles - 1 - (int)(x / heads), x % heads, vec);
    }
}

template <typename T, int BT, int DP>
static gs_status forward_t(const AttnArgs &a, cudaStream_t st)
{
    static SharedRecord record;
    const int smem = sizeof(float) * (2 * BT * (DP + 4) + BT * (BT + 4)), tiles = (a.q_len + BT - 1) / BT;
    const int64_t blocks = a.batch * a.q_heads * tiles;
    auto kernel = attn_simt_forward_kernel<T, BT, DP>;
    gs_status s;
    if ((s = blocks_ok(blocks)) != GS_OK || (s = allow_shared(kernel, smem, record)) != GS_OK) return s;
    kernel<<<(unsigned)blocks, BT * 4, smem, st>>>(a, tiles, rows_of_four(a, sizeof(T), false));
    GS_CUDA_TRY(cudaGetLastError());
    return GS_OK;
}

template <typename T, int BT, int DP>
static gs_status backward_t(const AttnArgs &a, cudaStream_t st)
{
    static SharedRecord record[2];
    const bool vec = rows_of_four(a, sizeof(T), true);
    const int smem = sizeof(BwdTiles<BT, DP>);
    gs_status s;
    if (BT == 16 || (a.q_len <= BT && a.k_len <= BT)) {     // by_shape gives 16-row tiles to nothing longer
        auto kernel = attn_simt_backward_one_kernel<T, BT, DP>;
        const int64_t blocks = a.batch * a.kv_heads;
        if ((s = blocks_ok(blocks)) != GS_OK || (s = allow_shared(kernel, smem, record[0])) != GS_OK) return s;
        kernel<<<(unsigned)blocks, BT * 4, smem, st>>>(a, vec);
    } else if constexpr (BT >= 32) {
        auto kernel = attn_simt_backward_kernel<T, BT, DP>;
        const int q_tiles = (a.q_len + BT - 1) / BT, k_tiles = (a.k_len + BT - 1) / BT;
        const int64_t k_blocks = a.batch * a.kv_heads * k_tiles, blocks = k_blocks + a.batch * a.q_heads * q_tiles;
        if ((s = blocks_ok(blocks)) != GS_OK || (s = allow_shared(kernel, smem, record[1])) != GS_OK) return s;
        kernel<<<(unsigned)blocks, BT * 4, smem, st>>>(a, k_blocks, q_tiles, vec);
    }
    GS_CUDA_TRY(cudaGetLastError());
    return GS_OK;
}

template <typename T, bool BWD>
static gs_status by_shape(const AttnArgs &a, cudaStream_t st)
{
    // one 16 x 16 or 32 x 32 tile holds all scores of a short sequence's head
    const int n = a.q_len > a.k_len ? a.q_len : a.k_len;
#define GS_SIMT_CASE(BT, DP) return BWD ? backward_t<T, BT, DP>(a, st) : forward_t<T, BT, DP>(a, st)
    if constexpr (sizeof(T) == 4) {                        // 16-bit tensors come here beyond 128 positions only
        if (n <= 16) {
            if constexpr (BWD) {                           // forward, narrower heads are done whole elsewhere
                if (a.dim <= 32) GS_SIMT_CASE(16, 32);
                if (a.dim <= 64) GS_SIMT_CASE(16, 64);
            }
            GS_SIMT_CASE(16, 128);
        }
    }
    // Tiles of 64 rows do more with what they read, tiles of 32 waste less of a causal bound and make four times the
    // blocks for a device that 64-row tiles fill less than one and a half times (two blocks of an SM, one with 128
    // columns).  Backward, 64 | 32 rows: 8 x 4 heads of 333 x 64 104 | 83 us, 16 x 8 heads 327 | 313, 4 x 8 heads of
    // 1024 507 | 579, 8 heads of 1500 x 128 1041 | 1166.  Up to 64 rows one block has all of a head.
    const int64_t blocks64 = (n + 63) / 64 * a.batch * (BWD ? a.q_heads + a.kv_heads : a.q_heads);
    const int64_t slots = (a.dim <= 64 ? 2 : 1) * (int64_t)sm_count();
    if (n <= 32 || (n > 64 && 2 * blocks64 < 3 * slots)) {
        if (a.dim <= 32) GS_SIMT_CASE(32, 32);
        if (a.dim <= 64) GS_SIMT_CASE(32, 64);
        GS_SIMT_CASE(32, 128);
    }
    if (a.dim <= 32) GS_SIMT_CASE(64, 32);
    if (a.dim <= 64) GS_SIMT_CASE(64, 64);
    GS_SIMT_CASE(64, 128);
#undef GS_SIMT_CASE
}

gs_status attn_simt_forward(const AttnArgs &a, cudaStream_t st)
{
    if (a.dtype == GS_TABLE_F16) return by_shape<__half, false>(a, st);
    if (a.dtype == GS_TABLE_BF16) return by_shape<__nv_bfloat16, false>(a, st);
    return by_shape<float, false>(a, st);
}

gs_status attn_simt_backward(const AttnArgs &a, cudaStream_t st)
{
    if (a.dtype == GS_TABLE_F16) return by_shape<__half, true>(a, st);
    if (a.dtype == GS_TABLE_BF16) return by_shape<__nv_bfloat16, true>(a, st);
    return by_shape<float, true>(a, st);
}

}  // namespace gs
