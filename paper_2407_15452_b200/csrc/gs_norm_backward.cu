// Layer norm, backward: dx = rstd (g - mean(g) - xh mean(g xh)) with g = dy weight, and the gradients of weight and bias, sums of
// dy xh and dy over all rows.
//
// x (or its 8-bit form) and dy are read once.  A thread adds up the weights' gradients of its columns over the rows of its team;
// the teams of a block are joined through shared memory, the blocks' sums by a second kernel, always in the same order.
//
// Bound: memory traffic in fp32 (400000 x 128 108 us, 5.7 TB/s), and nearly so in bf16 (61 us, 5.1 TB/s; 16384 x 4096 91 us, 4.4 TB/s: a thread
// has 8 columns there, since their sums and weights are 24 registers and two blocks of 512 threads have to fit; with 16 columns 107 us).
#include "gs_norm.cuh"

namespace gs {

// x of a row as it travels: T, or 8 bits and their scale
template <typename T, int VEC, bool KEPT> struct Source {
    typename Piece<T, VEC>::raw r;
    __device__ __forceinline__ void load(const NormArgs &, const RowAt &, const T *at, int, bool on) { r = load_piece<T, VEC>(at, on); }
    template <typename F, int N> __device__ __forceinline__ void get(F (&f)[N]) const { Piece<T, VEC>::get(r, f); }
};
template <typename T, int VEC> struct Source<T, VEC, true> {
    typename Kept<VEC>::raw r;
    float scale;
    __device__ __forceinline__ void load(const NormArgs &a, const RowAt &at, const T *, int c, bool on)
    {
        r = on ? *reinterpret_cast<const typename Kept<VEC>::raw *>(a.packed + at.row * a.columns + c) : Kept<VEC>::none();
        scale = on ? a.scales[at.row * a.kept_blocks + c / KEPT_BLOCK] : 0.0f;
    }
    template <typename F, int N> __device__ __forceinline__ void get(F (&f)[N]) const { Kept<VEC>::get(r, scale, f); }
};

template <typename T, typename S, bool KEPT>
__global__ void __launch_bounds__(S::THREADS, S::RESIDENT) norm_backward_kernel(const __grid_constant__ NormArgs a)
{
    constexpr int VEC = S::VEC, NV = S::NV, N = S::N, V = S::V;
    typedef Piece<T, VEC> P;
    typedef typename Vec<V>::type F;
    __shared__ float2 places[2][16];
    extern __shared__ float shared_sums[];                         // FAR: [dweight, dbias][column]; teams in a warp: [team][2][column]
    TeamSums sums = {places, 0};
    const float inverse = 1.0f / (float)a.columns;
    constexpr int WIDTH = (S::BLOCK ? 32 : S::LANES) * NV * VEC;   // of a warp's teams

    F w[S::FAR ? 1 : NV][N], dw[S::FAR ? 1 : NV][N], db[S::FAR ? 1 : NV][N];
    F *const far_dw = reinterpret_cast<F *>(shared_sums) + threadIdx.x, *const far_db = far_dw + (S::FAR ? NV * N * blockDim.x : 0);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        if (!S::FAR) vector_piece<T, VEC>(a, a.weight, S::column(v), S::in(v, a.columns), 1.0f, w[S::FAR ? 0 : v]);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if (S::FAR) far_dw[(v * N + e) * blockDim.x] = far_db[(v * N + e) * blockDim.x] = all_of<V>(0.0f);
            else dw[S::FAR ? 0 : v][e] = db[S::FAR ? 0 : v][e] = all_of<V>(0.0f);
        }
    }

    int64_t base = (int64_t)blockIdx.x * S::teams();
    RowAt next(a, base + S::index());
    typename P::raw rdy[NV];
    Source<T, VEC, KEPT> rx[NV];
    float2 stats;
    Line<T> x(a.x, next, S::column(0)), dy(a.dy, next, S::column(0)), dx(a.dx, next, S::column(0));
    auto load = [&]() {
        stats = next.live ? reinterpret_cast<const float2 *>(a.stats)[next.row] : make_float2(0.0f, 0.0f);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const bool on = next.live && S::in(v, a.columns);
            rx[v].load(a, next, x.at() + S::apart(v), S::column(v), on);
            rdy[v] = load_piece<T, VEC>(dy.at() + S::apart(v), on);
        }
    };
    load();
    for (; base < a.rows; base += a.step) {
        const RowAt at = next;
        const float rstd = stats.y;
        const F by = all_of<V>(rstd), minus_mean = all_of<V>(-stats.x);
        F xh[NV][N], g[NV][N], s1 = all_of<V>(0.0f), s2 = all_of<V>(0.0f);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            rx[v].get(xh[v]);
            P::get(rdy[v], g[v]);
            if (S::in(v, a.columns)) {
                F wv[N];
                if (S::FAR) vector_piece<T, VEC>(a, a.weight, S::column(v), true, 1.0f, wv);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const F h = mul_of(add_of(xh[v][e], minus_mean), by), d = g[v][e];
                    F &sum_w = S::FAR ? far_dw[(v * N + e) * blockDim.x] : dw[S::FAR ? 0 : v][e];
                    F &sum_b = S::FAR ? far_db[(v * N + e) * blockDim.x] : db[S::FAR ? 0 : v][e];
                    sum_w = fma_of(d, h, sum_w);
                    sum_b = add_of(sum_b, d);
                    xh[v][e] = h;
                    g[v][e] = mul_of(d, S::FAR ? wv[e] : w[S::FAR ? 0 : v][e]);
                    s1 = add_of(s1, g[v][e]);
                    s2 = fma_of(g[v][e], h, s2);
                }
            }
        }
        const bool wrapped = next.next(a);
        if (!KEPT) x.next(a.x, wrapped);
        dy.next(a.dy, wrapped);
        load();
        const float2 s = team_sum<S>(make_float2(sum_of(s1), sum_of(s2)), sums);
        if (at.there) {
            const F less = all_of<V>(-s.x * inverse), along = all_of<V>(-s.y * inverse);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (S::in(v, a.columns)) {
                    F o[N];
#pragma unroll
                    for (int e = 0; e < N; ++e) o[e] = mul_of(by, fma_of(xh[v][e], along, add_of(g[v][e], less)));
                    *reinterpret_cast<typename P::raw *>(dx.at() + S::apart(v)) = at.live ? P::put(o) : P::none();
                }
            }
        }
        dx.next(a.dx, wrapped);
    }
    if (!a.partial) return;
    // [block][2][columns]
    float *to_dw = a.partial + (int64_t)blockIdx.x * 2 * a.columns, *to_db = to_dw + a.columns;
    if (!S::BLOCK) {
        // the teams' sums, side by side
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                float *team = shared_sums + S::index() * 2 * WIDTH + S::column(v) + e;
                team[0] = reinterpret_cast<const float *>(dw[S::FAR ? 0 : v])[e];
                team[WIDTH] = reinterpret_cast<const float *>(db[S::FAR ? 0 : v])[e];
            }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * a.columns; i += NORM_THREADS) {
            const float *from = shared_sums + (i < a.columns ? i : WIDTH + i - a.columns);
            float t = 0.0f;
            for (int k = 0; k < S::teams(); ++k) t += from[k * 2 * WIDTH];
            to_dw[i] = t;
        }
        return;
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = S::column(v);
        if (c >= a.columns) continue;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const F sum_w = S::FAR ? far_dw[(v * N + e / V) * blockDim.x] : dw[S::FAR ? 0 : v][e / V];
            const F sum_b = S::FAR ? far_db[(v * N + e / V) * blockDim.x] : db[S::FAR ? 0 : v][e / V];
            to_dw[c + e] = reinterpret_cast<const float *>(&sum_w)[e % V];
            to_db[c + e] = reinterpret_cast<const float *>(&sum_b)[e % V];
        }
    }
}

// Sums of the blocks' partial sums: a block has 32 neighbouring values of [2][columns], warp w adds up every 32nd block's (of 8 warps each
// takes four times as many, one after another: 20000 x 1001 f16 backward 58 us in all, 53 with 32)
static constexpr int JOIN_WARPS = 32;
__global__ void __launch_bounds__(32 * JOIN_WARPS) norm_join_kernel(const float *partial, int blocks, int columns, void *dweight, void *dbias, int type)
{
    __shared__ float part[JOIN_WARPS][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
    cudaGridDependencySynchronize();
    float s = 0.0f;
    if (i < 2 * columns)
#pragma unroll 8
        for (int k = warp; k < blocks; k += JOIN_WARPS) s += partial[(int64_t)k * 2 * columns + i];
    part[warp][lane] = s;
    __syncthreads();
    if (warp || i >= 2 * columns) return;
#pragma unroll
    for (int w = 1; w < JOIN_WARPS; ++w) s += part[w][lane];
    void *to = i < columns ? dweight : dbias;
    const int c = i < columns ? i : i - columns;
    if (!to) return;
    if (type == GS_TABLE_F32) static_cast<float *>(to)[c] = s;
    else if (type == GS_TABLE_F16) static_cast<__half *>(to)[c] = from_float<__half>(s);
    else static_cast<__nv_bfloat16 *>(to)[c] = from_float<__nv_bfloat16>(s);
}

// Blocks of a launch: one for every so many rows, at most what the device holds at once
template <typename S>
static int grid_of(int64_t rows, int threads)
{
    const int teams = S::BLOCK ? 1 : NORM_THREADS / S::LANES;
    int per_sm = S::ON_SM / threads;
    if (per_sm > NORM_PARTIALS) per_sm = NORM_PARTIALS;
    const int64_t blocks = (rows + teams - 1) / teams, most = (int64_t)sm_count() * per_sm;
    return (int)(blocks < most ? blocks : most);
}

template <typename T, typename S, bool KEPT>
static gs_status launch(const NormArgs &args, int threads, int32_t weight_type, void *dweight, void *dbias, cudaStream_t st)
{
    NormArgs a = args;
    const int grid = grid_of<S>(a.rows, threads);
    set_step(a, (int64_t)grid * (S::BLOCK ? 1 : NORM_THREADS / S::LANES), sizeof(T));
    const bool sums = dweight || dbias;
    if (!sums) a.partial = nullptr;
    const size_t shared = (S::FAR ? (size_t)S::NV * S::VEC * threads : S::BLOCK ? 0 : (size_t)NORM_THREADS * S::NV * S::VEC) * sizeof(float2);
    static SharedRecord record;
    gs_status s = allow_shared(norm_backward_kernel<T, S, KEPT>, (int)shared, record);
    if (s != GS_OK) return s;
    norm_backward_kernel<T, S, KEPT><<<grid, threads, shared, st>>>(a);
    GS_CUDA_TRY(cudaGetLastError());
    if (sums)
        GS_CUDA_TRY(launch_after(norm_join_kernel, (2 * a.columns + 31) / 32, 32 * JOIN_WARPS, 0, st, a.partial, grid, a.columns, dweight, dbias,
                                 weight_type));
    return GS_OK;
}

int64_t norm_backward_partials(int64_t rows, int32_t columns, int32_t dtype)
{
    int most = 0;
    with_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        auto count = [&](auto team, int threads) {
            const int grid = grid_of<decltype(team)>(rows, threads);
            if (grid > most) most = grid;
            return GS_OK;
        };
        if (columns % Wide<T>::N == 0) with_team<T>(columns, true, count);
        return with_team<T>(columns, false, count);
    });
    return most;
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
