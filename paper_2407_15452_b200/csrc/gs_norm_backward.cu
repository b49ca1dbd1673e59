// Layer norm, backward: dx = rstd (g - mean(g) - xh mean(g xh)) with g = dy weight, and the gradients of weight and bias, sums of
// dy xh and dy over all rows.
//
// x (or its 8-bit form) and dy are read once.  A thread adds up the weights' gradients of its columns over the rows of its team;
// the teams of a block are joined through shared memory, the blocks' sums by a second kernel, always in the same order.  Bound:
// memory traffic.
#include "gs_norm.cuh"

namespace gs {

// x of a row as it travels: T, or 8 bits and their scale
template <typename T, int VEC, bool KEPT> struct Source {
    typename Piece<T, VEC>::raw r;
    __device__ __forceinline__ void load(const NormArgs &a, const RowAt &at, int c)
    {
        r = load_piece<T, VEC>(row_of<T>(a.x, at), c, a.columns, at.live);
    }
    __device__ __forceinline__ void get(float (&f)[VEC]) const { Piece<T, VEC>::get(r, f); }
};
template <typename T, int VEC> struct Source<T, VEC, true> {
    typename Kept<VEC>::raw r;
    float scale;
    __device__ __forceinline__ void load(const NormArgs &a, const RowAt &at, int c)
    {
        const bool on = at.live && c < a.columns;
        r = on ? *reinterpret_cast<const typename Kept<VEC>::raw *>(a.packed + at.row * a.columns + c) : Kept<VEC>::none();
        scale = on ? a.scales[at.row * a.kept_blocks + c / KEPT_BLOCK] : 0.0f;
    }
    __device__ __forceinline__ void get(float (&f)[VEC]) const
    {
        int q[VEC];
        Kept<VEC>::get(r, q);
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = kept_value(q[e], scale);
    }
};

template <typename T, typename S, bool KEPT>
__global__ void __launch_bounds__(S::THREADS) norm_backward_kernel(const __grid_constant__ NormArgs a)
{
    constexpr int VEC = S::VEC, NV = S::NV;
    typedef Piece<T, VEC> P;
    __shared__ float2 places[2][16];
    extern __shared__ float2 shared_sums[];                        // FAR: [NV * VEC][threads]; teams in a warp: [team][column]
    PairSums sums = {places, 0};
    const float inverse = 1.0f / (float)a.columns;

    float w[S::FAR ? 1 : NV][VEC];
    float2 acc[S::FAR ? 1 : NV][VEC];                              // dweight, dbias
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        if (!S::FAR) vector_piece<T, VEC>(a.weight, a.weight_f32, S::column(v), a.columns, 1.0f, w[S::FAR ? 0 : v]);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            if (S::FAR) shared_sums[(v * VEC + e) * blockDim.x + threadIdx.x] = make_float2(0.0f, 0.0f);
            else acc[S::FAR ? 0 : v][e] = make_float2(0.0f, 0.0f);
        }
    }

    const int64_t step = (int64_t)gridDim.x * S::teams();
    int64_t base = (int64_t)blockIdx.x * S::teams();
    RowAt next = row_at(a, base + S::index());
    typename P::raw rdy[NV];
    Source<T, VEC, KEPT> rx[NV];
    float2 stats = next.live ? reinterpret_cast<const float2 *>(a.stats)[next.row] : make_float2(0.0f, 0.0f);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        rx[v].load(a, next, S::column(v));
        rdy[v] = load_piece<T, VEC>(row_of<T>(a.dy, next), S::column(v), a.columns, next.live);
    }
    for (; base < a.rows; base += step) {
        const RowAt at = next;
        const float rstd = stats.y, mean = stats.x;
        float xh[NV][VEC], g[NV][VEC];
        float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            rx[v].get(xh[v]);
            P::get(rdy[v], g[v]);
            if (S::column(v) < a.columns) {
                float wv[VEC];
                if (S::FAR) vector_piece<T, VEC>(a.weight, a.weight_f32, S::column(v), a.columns, 1.0f, wv);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float h = (xh[v][e] - mean) * rstd, d = g[v][e];
                    if (S::FAR) {
                        float2 &c = shared_sums[(v * VEC + e) * blockDim.x + threadIdx.x];
                        c = make_float2(fmaf(d, h, c.x), c.y + d);
                    } else {
                        float2 &c = acc[S::FAR ? 0 : v][e];
                        c.x = fmaf(d, h, c.x);
                        c.y += d;
                    }
                    xh[v][e] = h;
                    g[v][e] = d * (S::FAR ? wv[e] : w[S::FAR ? 0 : v][e]);
                    s.x += g[v][e];
                    s.y = fmaf(g[v][e], h, s.y);
                }
            }
        }
        next = row_at(a, base + step + S::index());
        stats = next.live ? reinterpret_cast<const float2 *>(a.stats)[next.row] : make_float2(0.0f, 0.0f);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            rx[v].load(a, next, S::column(v));
            rdy[v] = load_piece<T, VEC>(row_of<T>(a.dy, next), S::column(v), a.columns, next.live);
        }
        s = team_sum<S>(s, sums);
        s.x *= inverse;
        s.y *= inverse;
        if (at.there) {
            T *to = row_of<T>(a.dx, at);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = S::column(v);
                if (c < a.columns) {
                    float o[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) o[e] = at.live ? rstd * (g[v][e] - s.x - xh[v][e] * s.y) : 0.0f;
                    *reinterpret_cast<typename P::raw *>(to + c) = P::put(o);
                }
            }
        }
    }
    if (!a.partial) return;
    // [block][2][columns]
    float *dw = a.partial + (int64_t)blockIdx.x * 2 * a.columns, *db = dw + a.columns;
    if (S::BLOCK) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = S::column(v);
            if (c < a.columns)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float2 t = S::FAR ? shared_sums[(v * VEC + e) * blockDim.x + threadIdx.x] : acc[S::FAR ? 0 : v][e];
                    dw[c + e] = t.x;
                    db[c + e] = t.y;
                }
        }
    } else {
        constexpr int WIDTH = (S::BLOCK ? 32 : S::LANES) * NV * VEC;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < VEC; ++e) shared_sums[S::index() * WIDTH + S::column(v) + e] = acc[S::FAR ? 0 : v][e];
        __syncthreads();
        for (int c = threadIdx.x; c < a.columns; c += NORM_THREADS) {
            float2 t = make_float2(0.0f, 0.0f);
            for (int i = 0; i < S::teams(); ++i) {
                t.x += shared_sums[i * WIDTH + c].x;
                t.y += shared_sums[i * WIDTH + c].y;
            }
            dw[c] = t.x;
            db[c] = t.y;
        }
    }
}

// Sums of the blocks' partial sums: a block has 32 neighbouring values of [2][columns], warp w adds up every eighth block's
__global__ void __launch_bounds__(256) norm_join_kernel(const float *partial, int blocks, int columns, void *dweight, void *dbias, int type)
{
    __shared__ float part[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
    cudaGridDependencySynchronize();
    float s = 0.0f;
    if (i < 2 * columns)
#pragma unroll 8
        for (int k = warp; k < blocks; k += 8) s += partial[(int64_t)k * 2 * columns + i];
    part[warp][lane] = s;
    __syncthreads();
    if (warp || i >= 2 * columns) return;
#pragma unroll
    for (int w = 1; w < 8; ++w) s += part[w][lane];
    void *to = i < columns ? dweight : dbias;
    const int c = i < columns ? i : i - columns;
    if (!to) return;
    if (type == GS_TABLE_F32) static_cast<float *>(to)[c] = s;
    else if (type == GS_TABLE_F16) static_cast<__half *>(to)[c] = from_float<__half>(s);
    else static_cast<__nv_bfloat16 *>(to)[c] = from_float<__nv_bfloat16>(s);
}

template <typename T, typename S, bool KEPT>
static gs_status launch(const NormArgs &args, int threads, int32_t weight_type, void *dweight, void *dbias, cudaStream_t st)
{
    NormArgs a = args;
    const int teams = S::BLOCK ? 1 : NORM_THREADS / S::LANES;
    int per_sm = 1024 / threads;
    if (per_sm < 1) per_sm = 1;
    if (per_sm > NORM_PARTIALS) per_sm = NORM_PARTIALS;
    const int64_t blocks = (a.rows + teams - 1) / teams, most = (int64_t)sm_count() * per_sm;
    const int grid = (int)(blocks < most ? blocks : most);
    const bool sums = dweight || dbias;
    if (!sums) a.partial = nullptr;
    const size_t shared = (S::FAR ? (size_t)S::NV * S::VEC * threads : S::BLOCK ? 0 : (size_t)NORM_THREADS * S::NV * S::VEC) * sizeof(float2);
    static SharedRecord record;
    gs_status s = allow_shared(norm_backward_kernel<T, S, KEPT>, (int)shared, record);
    if (s != GS_OK) return s;
    norm_backward_kernel<T, S, KEPT><<<grid, threads, shared, st>>>(a);
    GS_CUDA_TRY(cudaGetLastError());
    if (sums)
        GS_CUDA_TRY(launch_after(norm_join_kernel, (2 * a.columns + 31) / 32, 256, 0, st, a.partial, grid, a.columns, dweight, dbias,
                                 weight_type));
    return GS_OK;
}

gs_status norm_backward(const NormArgs &a, int32_t dtype, bool aligned, void *dweight, void *dbias, cudaStream_t st)
{
    return with_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        return with_team<T>(a.columns, aligned, [&](auto team, int threads) {
            typedef decltype(team) S;
            const int32_t wt = a.weight_f32 ? GS_TABLE_F32 : dtype;
            return a.packed ? launch<T, S, true>(a, threads, wt, dweight, dbias, st) : launch<T, S, false>(a, threads, wt, dweight, dbias, st);
        });
    });
}

}  // namespace gs
