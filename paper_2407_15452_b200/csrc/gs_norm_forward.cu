// Layer norm, forward: y = (x - mean) rstd weight + bias, and on request x in 8 bits beside it.
//
// The mean is taken first and the squares of what differs from it second, both from registers; the differences' own mean, what rounding left
// of the first, is taken with them, so that a mean far from zero costs no digits.  Bound: memory traffic, one read and one write of
// every value.
#include "gs_norm.cuh"

namespace gs {

// KEEP: x is kept in 8 bits as well
template <typename T, typename S, bool KEEP>
__global__ void __launch_bounds__(S::THREADS, S::BLOCK ? 1 : 2) norm_forward_kernel(const __grid_constant__ NormArgs a)
{
    constexpr int VEC = S::VEC, NV = S::NV, N = S::N, V = S::V;
    typedef Piece<T, VEC> P;
    typedef typename Vec<V>::type F;
    __shared__ float2 places[2][16];
    TeamSums sums = {places, 0};
    const float inverse = 1.0f / (float)a.columns;

    F w[S::FAR ? 1 : NV][N], b[S::FAR ? 1 : NV][N];
    if (!S::FAR)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            vector_piece<T, VEC>(a.weight, a.weight_f32, S::column(v), a.columns, 1.0f, w[v]);
            vector_piece<T, VEC>(a.bias, a.weight_f32, S::column(v), a.columns, 0.0f, b[v]);
        }

    int64_t base = (int64_t)blockIdx.x * S::teams();
    RowAt next(a, base + S::index());
    typename P::raw raw[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) raw[v] = load_piece<T, VEC>(next.of<const T>(a.x), S::column(v), a.columns, next.live);
    for (; base < a.rows; base += a.step) {
        const RowAt at = next;
        F f[NV][N], s = all_of<V>(0.0f);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            P::get(raw[v], f[v]);
#pragma unroll
            for (int e = 0; e < N; ++e) s = add_of(s, f[v][e]);
        }
        next.next(a);
        const T *row = next.of<const T>(a.x);
#pragma unroll
        for (int v = 0; v < NV; ++v) raw[v] = load_piece<T, VEC>(row, S::column(v), a.columns, next.live);

        if constexpr (KEEP) {
#pragma unroll
            for (int v0 = 0; v0 < NV; v0 += S::KEPT_PIECES) {
                uint32_t top = 0;
#pragma unroll
                for (int v = v0; v < v0 + S::KEPT_PIECES; ++v)
#pragma unroll
                    for (int e = 0; e < N; ++e) top = max(top, magnitude(f[v][e]));
                const KeptScale scale(largest<S::KEPT_LANES>(top));
#pragma unroll
                for (int v = v0; v < v0 + S::KEPT_PIECES; ++v) {
                    uint32_t q[VEC];
                    scale.of(f[v], q);
                    const int c = S::column(v);
                    if (at.there && c < a.columns) {
                        *reinterpret_cast<typename Kept<VEC>::raw *>(a.packed + at.row * a.columns + c) = Kept<VEC>::put(q);
                        if (c % KEPT_BLOCK == 0) a.scales[at.row * a.kept_blocks + c / KEPT_BLOCK] = scale.s;
                    }
                }
            }
        }

        const float mean = team_sum<S>(sum_of(s), sums) * inverse;
        F rest = all_of<V>(0.0f), squares = all_of<V>(0.0f);
        const F minus_mean = all_of<V>(-mean);
#pragma unroll
        for (int v = 0; v < NV; ++v)
            if (S::column(v) < a.columns)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    f[v][e] = add_of(f[v][e], minus_mean);
                    rest = add_of(rest, f[v][e]);
                    squares = fma_of(f[v][e], f[v][e], squares);
                }
        float2 t = team_sum<S>(make_float2(sum_of(rest), sum_of(squares)), sums);
        t.x *= inverse;
        const float rstd = rsqrtf(fmaxf(fmaf(-t.x, t.x, t.y * inverse), 0.0f) + a.eps);
        if (at.there) {
            T *to = at.of<T>(a.y);
            const F by = all_of<V>(rstd), less = all_of<V>(-t.x);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = S::column(v);
                if (c < a.columns) {
                    F wv[N], bv[N], o[N];
                    if (S::FAR) {
                        vector_piece<T, VEC>(a.weight, a.weight_f32, c, a.columns, 1.0f, wv);
                        vector_piece<T, VEC>(a.bias, a.weight_f32, c, a.columns, 0.0f, bv);
                    }
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        o[e] = fma_of(mul_of(add_of(f[v][e], less), by), S::FAR ? wv[e] : w[S::FAR ? 0 : v][e],
                                      S::FAR ? bv[e] : b[S::FAR ? 0 : v][e]);
                    *reinterpret_cast<typename P::raw *>(to + c) = at.live ? P::put(o) : P::none();
                }
            }
            if (a.stats && S::member() == 0)
                reinterpret_cast<float2 *>(a.stats)[at.row] = at.live ? make_float2(mean + t.x, rstd) : make_float2(0.0f, 0.0f);
        }
    }
}

gs_status norm_forward(const NormArgs &a, int32_t dtype, bool aligned, cudaStream_t st)
{
    return with_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        return with_team<T>(a.columns, aligned, [&](auto team, int threads) {
            typedef decltype(team) S;
            const int teams = S::BLOCK ? 1 : NORM_THREADS / S::LANES;
            const int64_t blocks = (a.rows + teams - 1) / teams, most = (int64_t)sm_count() * (2048 / threads) * 2;
            const int64_t grid = blocks < most ? blocks : most;
            NormArgs b = a;
            set_step(b, grid * teams);
            if constexpr (S::VEC > 1)
                if (a.packed) {
                    norm_forward_kernel<T, S, true><<<(unsigned)grid, threads, 0, st>>>(b);
                    GS_CUDA_TRY(cudaGetLastError());
                    return GS_OK;
                }
            norm_forward_kernel<T, S, false><<<(unsigned)grid, threads, 0, st>>>(b);
            GS_CUDA_TRY(cudaGetLastError());
            return GS_OK;
        });
    });
}

}  // namespace gs
