// Attention on the CUDA cores, everything in fp32 (products included).
//
// A block of 4 * BT threads works on BT x BT tiles of scores; thread (ty, tx) holds 4 rows x BT/16
// columns of a tile and 4 rows x DP/16 columns of an accumulator, DP = head_dim padded to 32, 64 or
// 128 with zeros.  Operands sit in shared memory row-major with 4 floats of padding: 16-byte reads
// of consecutive rows then fall into different banks, and the same copy serves the products over
// the head dimension (row . row) and those over positions (column blocks of rows).
//  forward: one block per BT query rows, running maximum and sum over the key tiles
//  dq     : one block per BT query rows; recomputes p = exp(s - lse), also leaves delta for dk/dv
//  dk, dv : one block per BT key rows and key/value head; loops over the query heads of its group
//           and their query tiles, so shared heads are summed in a fixed order without atomics
#include "gs_attn.cuh"

namespace gs {

template <typename T> __device__ __forceinline__ float to_f(T x);
template <> __device__ __forceinline__ float to_f<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_f<__half>(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ float from_f<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_f<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

template <typename T>
__device__ __forceinline__ T *row_of(const AttnTensor &t, int64_t b, int64_t pos, int64_t head)
{
    return reinterpret_cast<T *>(t.p) + b * t.sb + pos * t.sl + head * t.sh;
}

template <int BT, int DP>
struct Tile {
    static constexpr int LD = DP + 4, LP = BT + 4, NT = BT * 4, NC = BT / 16;
    static constexpr int CW = DP >= 64 ? 4 : 2, CN = DP / (16 * CW);    // accumulator columns: CN groups of CW
    float x[BT][LD];
};

// rows [r0, r0 + BT) of one head into shared memory; rows >= n and columns >= dim become zero
// (whatever the padding of the input holds, NaN included, is not read)
template <typename T, int BT, int DP>
__device__ __forceinline__ void load_rows(float (*dst)[DP + 4], const AttnTensor &t, int64_t b, int64_t head,
                                          int r0, int n, int dim, bool vec)
{
    for (int e = threadIdx.x; e < BT * (DP / 4); e += BT * 4) {
        const int r = e / (DP / 4), c = (e % (DP / 4)) * 4;
        float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r0 + r < n && c < dim) {
            const T *p = row_of<T>(t, b, r0 + r, head) + c;
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
        *reinterpret_cast<float4 *>(&dst[r][c]) = f;
    }
}

// s[i][j] = a[4 ty + i] . b[tx + 16 j]
template <int BT, int DP>
__device__ __forceinline__ void dot_rows(float (&s)[4][BT / 16], const float (*a)[DP + 4], const float (*b)[DP + 4],
                                         int ty, int tx)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < BT / 16; ++j) s[i][j] = 0.f;
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
                s[i][j] = fmaf(x[i].x, y[j].x, s[i][j]);
                s[i][j] = fmaf(x[i].y, y[j].y, s[i][j]);
                s[i][j] = fmaf(x[i].z, y[j].z, s[i][j]);
                s[i][j] = fmaf(x[i].w, y[j].w, s[i][j]);
            }
    }
}

template <int DP>
__device__ __forceinline__ void load_cols(float (&y)[DP / 16], const float *row, int tx)
{
    if constexpr (DP >= 64) {
#pragma unroll
        for (int m = 0; m < DP / 64; ++m)
            *reinterpret_cast<float4 *>(&y[4 * m]) = *reinterpret_cast<const float4 *>(row + 64 * m + 4 * tx);
    } else {
        *reinterpret_cast<float2 *>(&y[0]) = *reinterpret_cast<const float2 *>(row + 2 * tx);
    }
}

// acc[i][:] += sum_j p[4 ty + i][j] x[j][:]
template <int BT, int DP>
__device__ __forceinline__ void mul_rows(float (&acc)[4][DP / 16], const float (*p)[BT + 4], const float (*x)[DP + 4],
                                         int ty, int tx)
{
#pragma unroll 2
    for (int j = 0; j < BT; j += 4) {
        float w[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<float4 *>(w[i]) = *reinterpret_cast<const float4 *>(&p[4 * ty + i][j]);
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
            float y[DP / 16];
            load_cols<DP>(y, x[j + jj], tx);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < DP / 16; ++c) acc[i][c] = fmaf(w[i][jj], y[c], acc[i][c]);
        }
    }
}

// acc[i][:] += sum_r p[r][4 ty + i] x[r][:]
template <int BT, int DP>
__device__ __forceinline__ void mul_cols(float (&acc)[4][DP / 16], const float (*p)[BT + 4], const float (*x)[DP + 4],
                                         int ty, int tx)
{
#pragma unroll 4
    for (int r = 0; r < BT; ++r) {
        float w[4], y[DP / 16];
        *reinterpret_cast<float4 *>(w) = *reinterpret_cast<const float4 *>(&p[r][4 * ty]);
        load_cols<DP>(y, x[r], tx);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < DP / 16; ++c) acc[i][c] = fmaf(w[i], y[c], acc[i][c]);
    }
}

template <typename T, int DP>
__device__ __forceinline__ void store_row(T *row, const float (&acc)[DP / 16], float mul, int tx, int dim, bool vec)
{
    constexpr int CW = DP >= 64 ? 4 : 2;
#pragma unroll
    for (int m = 0; m < DP / (16 * CW); ++m) {
        const int c = 16 * CW * m + CW * tx;
        if constexpr (sizeof(T) == 4 && CW == 4) {
            if (vec) {
                if (c < dim)
                    *reinterpret_cast<float4 *>(row + c) = make_float4(acc[4 * m] * mul, acc[4 * m + 1] * mul,
                                                                       acc[4 * m + 2] * mul, acc[4 * m + 3] * mul);
                continue;
            }
        }
#pragma unroll
        for (int x = 0; x < CW; ++x)
            if (c + x < dim) row[c + x] = from_f<T>(acc[CW * m + x] * mul);
    }
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
__global__ void __launch_bounds__(BT * 4) attn_simt_forward_kernel(const AttnArgs a, int tiles, bool vec)
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

    float acc[4][DP / 16] = {}, top[4], sum[4];
    int lo[4], hi[4];
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
    load_rows<T, BT, DP>(Q, a.q, b, h, r0, s.nq, a.dim, vec);
    for (int j0 = j_begin; j0 < j_end; j0 += BT) {
        load_rows<T, BT, DP>(KV, a.k, b, g, j0, s.nk, a.dim, vec);
        __syncthreads();
        float sc[4][BT / 16];
        dot_rows<BT, DP>(sc, Q, KV, ty, tx);
        __syncthreads();
        load_rows<T, BT, DP>(KV, a.v, b, g, j0, s.nk, a.dim, vec);
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
            for (int c = 0; c < DP / 16; ++c) acc[i][c] *= keep;
        }
        __syncthreads();
        mul_rows<BT, DP>(acc, P, KV, ty, tx);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + 4 * ty + i;
        if (r >= a.q_len) continue;
        store_row<T, DP>(row_of<T>(a.out, b, r, h), acc[i], sum[i] > 0.f || sum[i] != sum[i] ? 1.f / sum[i] : 0.f, tx, a.dim, vec);
        if (tx == 0) a.lse[bh * a.q_len + r] = sum[i] == 0.f ? -INFINITY : top[i] + logf(sum[i]);
    }
}

template <typename T, int BT, int DP>
__global__ void __launch_bounds__(BT * 4) attn_simt_dq_kernel(const AttnArgs a, int tiles, bool vec)
{
    extern __shared__ float4 smem4[];
    float(*Q)[DP + 4] = reinterpret_cast<float(*)[DP + 4]>(smem4);
    float(*DO)[DP + 4] = Q + BT;
    float(*K)[DP + 4] = DO + BT;
    float(*V)[DP + 4] = K + BT;
    float(*S)[BT + 4] = reinterpret_cast<float(*)[BT + 4]>(V + BT);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int64_t heads = a.batch * a.q_heads;
    const int tile = tiles - 1 - (int)(blockIdx.x / heads);
    const int64_t bh = blockIdx.x % heads, b = bh / a.q_heads;
    const int h = (int)(bh % a.q_heads), g = h / a.group;
    const AttnSeq s = attn_seq(a, b);
    const int r0 = tile * BT, r1 = min(r0 + BT, a.q_len);

    load_rows<T, BT, DP>(Q, a.q, b, h, r0, s.nq, a.dim, vec);
    load_rows<T, BT, DP>(DO, a.dout, b, h, r0, s.nq, a.dim, vec);
    load_rows<T, BT, DP>(V, a.out, b, h, r0, s.nq, a.dim, vec);       // the output rows, for delta only
    __syncthreads();
    float acc[4][DP / 16] = {}, lse[4], delta[4];
    int lo[4], hi[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + 4 * ty + i;
        float x[DP / 16], y[DP / 16], d = 0.f;
        load_cols<DP>(x, DO[4 * ty + i], tx);
        load_cols<DP>(y, V[4 * ty + i], tx);
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) d = fmaf(x[c], y[c], d);
        delta[i] = half_warp_sum(d);
        lo[i] = attn_lo(a, s, r);
        hi[i] = attn_hi(a, s, r);
        lse[i] = r < s.nq ? a.lse[bh * a.q_len + r] : 0.f;
        if (tx == 0 && r < a.q_len) a.delta[bh * a.q_len + r] = delta[i];
    }
    const int last = min(r1, s.nq) - 1;
    const int j_end = last >= r0 ? attn_hi(a, s, last) : 0;
    for (int j0 = attn_lo(a, s, r0) / BT * BT; j0 < j_end; j0 += BT) {
        __syncthreads();
        load_rows<T, BT, DP>(K, a.k, b, g, j0, s.nk, a.dim, vec);
        load_rows<T, BT, DP>(V, a.v, b, g, j0, s.nk, a.dim, vec);
        __syncthreads();
        float sc[4][BT / 16], dp[4][BT / 16];
        dot_rows<BT, DP>(sc, Q, K, ty, tx);
        dot_rows<BT, DP>(dp, DO, V, ty, tx);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < BT / 16; ++j) {
                const int c = j0 + tx + 16 * j;
                float ds = 0.f;
                if (c >= lo[i] && c < hi[i]) ds = expf(sc[i][j] * a.scale - lse[i]) * (dp[i][j] - delta[i]);
                S[4 * ty + i][tx + 16 * j] = ds;
            }
        __syncthreads();
        mul_rows<BT, DP>(acc, S, K, ty, tx);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + 4 * ty + i;
        if (r < a.q_len) store_row<T, DP>(row_of<T>(a.dq, b, r, h), acc[i], a.scale, tx, a.dim, vec);
    }
}

template <typename T, int BT, int DP>
__global__ void __launch_bounds__(BT * 4) attn_simt_dkdv_kernel(const AttnArgs a, int tiles, bool vec)
{
    extern __shared__ float4 smem4[];
    float(*K)[DP + 4] = reinterpret_cast<float(*)[DP + 4]>(smem4);
    float(*V)[DP + 4] = K + BT;
    float(*Q)[DP + 4] = V + BT;
    float(*DO)[DP + 4] = Q + BT;
    float(*P)[BT + 4] = reinterpret_cast<float(*)[BT + 4]>(DO + BT);
    float(*S)[BT + 4] = P + BT;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int64_t heads = a.batch * a.kv_heads;
    const int tile = (int)(blockIdx.x / heads);           // under a causal bound the first tiles are the longest
    const int64_t bg = blockIdx.x % heads, b = bg / a.kv_heads;
    const int g = (int)(bg % a.kv_heads);
    const AttnSeq s = attn_seq(a, b);
    const int j0 = tile * BT;

    load_rows<T, BT, DP>(K, a.k, b, g, j0, s.nk, a.dim, vec);
    load_rows<T, BT, DP>(V, a.v, b, g, j0, s.nk, a.dim, vec);
    float dk[4][DP / 16] = {}, dv[4][DP / 16] = {};
    const int q_end = j0 < s.nk ? attn_q_last(a, s, min(j0 + BT, s.nk)) : 0;
    const int q_begin = attn_q_first(a, s, j0) / BT * BT;
    for (int h = g * a.group; h < (g + 1) * a.group; ++h) {
        const int64_t bh = b * a.q_heads + h;
        for (int r0 = q_begin; r0 < q_end; r0 += BT) {
            __syncthreads();
            load_rows<T, BT, DP>(Q, a.q, b, h, r0, s.nq, a.dim, vec);
            load_rows<T, BT, DP>(DO, a.dout, b, h, r0, s.nq, a.dim, vec);
            __syncthreads();
            float sc[4][BT / 16], dp[4][BT / 16];
            dot_rows<BT, DP>(sc, Q, K, ty, tx);
            dot_rows<BT, DP>(dp, DO, V, ty, tx);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = r0 + 4 * ty + i;
                const int lo = attn_lo(a, s, r), hi = attn_hi(a, s, r);
                const float lse = r < s.nq ? a.lse[bh * a.q_len + r] : 0.f;
                const float delta = r < s.nq ? a.delta[bh * a.q_len + r] : 0.f;
#pragma unroll
                for (int j = 0; j < BT / 16; ++j) {
                    const int c = j0 + tx + 16 * j;
                    float p = 0.f, ds = 0.f;
                    if (c >= lo && c < hi) {
                        p = expf(sc[i][j] * a.scale - lse);
                        ds = p * (dp[i][j] - delta);
                    }
                    P[4 * ty + i][tx + 16 * j] = p;
                    S[4 * ty + i][tx + 16 * j] = ds;
                }
            }
            __syncthreads();
            mul_cols<BT, DP>(dv, P, DO, ty, tx);
            mul_cols<BT, DP>(dk, S, Q, ty, tx);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = j0 + 4 * ty + i;
        if (j >= a.k_len) continue;
        store_row<T, DP>(row_of<T>(a.dk, b, j, g), dk[i], a.scale, tx, a.dim, vec);
        store_row<T, DP>(row_of<T>(a.dv, b, j, g), dv[i], 1.f, tx, a.dim, vec);
    }
}

// 4-element vector accesses need every row of every tensor aligned to four elements
static bool rows_of_four(const AttnArgs &a, size_t es, bool backward)
{
    auto ok = [&](const AttnTensor &t) {
        return ((uintptr_t)t.p % (4 * es)) == 0 && (t.sb | t.sl | t.sh) % 4 == 0;
    };
    bool v = a.dim % 4 == 0 && ok(a.q) && ok(a.k) && ok(a.v) && ok(a.out);
    if (backward) v = v && ok(a.dout) && ok(a.dq) && ok(a.dk) && ok(a.dv);
    return v;
}

template <typename K>
static gs_status launch(K kernel, const AttnArgs &a, int64_t heads, int32_t len, int bt, size_t smem, bool vec,
                        SharedRecord &record, cudaStream_t st)
{
    const int tiles = (len + bt - 1) / bt;
    const int64_t blocks = heads * tiles;
    if (blocks == 0) return GS_OK;
    if (blocks > 0x7FFFFFFF) {
        set_error("attention of %lld row tiles exceeds one launch", (long long)blocks);
        return GS_ERR_UNSUPPORTED;
    }
    gs_status s = allow_shared(kernel, (int)smem, record);
    if (s != GS_OK) return s;
    kernel<<<(unsigned)blocks, bt * 4, smem, st>>>(a, tiles, vec);
    GS_CUDA_TRY(cudaGetLastError());
    return GS_OK;
}

template <typename T, int BT, int DP>
static gs_status forward_t(const AttnArgs &a, cudaStream_t st)
{
    const size_t smem = sizeof(float) * (2 * BT * (DP + 4) + BT * (BT + 4));
    static SharedRecord record;
    return launch(attn_simt_forward_kernel<T, BT, DP>, a, a.batch * a.q_heads, a.q_len, BT, smem,
                  rows_of_four(a, sizeof(T), false), record, st);
}

template <typename T, int BT, int DP>
static gs_status backward_t(const AttnArgs &a, cudaStream_t st)
{
    const bool vec = rows_of_four(a, sizeof(T), true);
    const size_t rows = sizeof(float) * 4 * BT * (DP + 4), tile = sizeof(float) * BT * (BT + 4);
    static SharedRecord record[2];
    gs_status s = launch(attn_simt_dq_kernel<T, BT, DP>, a, a.batch * a.q_heads, a.q_len, BT, rows + tile, vec, record[0], st);
    if (s != GS_OK) return s;
    return launch(attn_simt_dkdv_kernel<T, BT, DP>, a, a.batch * a.kv_heads, a.k_len, BT, rows + 2 * tile, vec, record[1], st);
}

template <typename T, bool BWD>
static gs_status by_shape(const AttnArgs &a, cudaStream_t st)
{
    const bool small = a.q_len <= 16 && a.k_len <= 16;     // one 16 x 16 tile holds all scores of a head
#define GS_SIMT_CASE(BT, DP) return BWD ? backward_t<T, BT, DP>(a, st) : forward_t<T, BT, DP>(a, st)
    if (small) {
        if (a.dim <= 32) GS_SIMT_CASE(16, 32);
        if (a.dim <= 64) GS_SIMT_CASE(16, 64);
        GS_SIMT_CASE(16, 128);
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
