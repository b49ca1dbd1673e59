// Layer norm, forward: y = (x - mean) rstd weight + bias, and on request x in 8 bits beside it.
//
// The mean is taken first and the squares of what differs from it second, both from registers; the differences' own mean, what rounding left
// of the first, is taken with them, so that a mean far from zero costs no digits.  Bound: memory traffic, one read and one write of
// every value.
#include "gs_norm.cuh"

namespace gs {

template <typename T, typename S>
__global__ void __launch_bounds__(S::THREADS) norm_forward_kernel(const __grid_constant__ NormArgs a)
{
    constexpr int VEC = S::VEC, NV = S::NV;
    typedef Piece<T, VEC> P;
    __shared__ float2 places[2][16];
    PairSums sums = {places, 0};
    const float inverse = 1.0f / (float)a.columns;

    float w[S::FAR ? 1 : NV][VEC], b[S::FAR ? 1 : NV][VEC];
    if (!S::FAR)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            vector_piece<T, VEC>(a.weight, a.weight_f32, S::column(v), a.columns, 1.0f, w[v]);
            vector_piece<T, VEC>(a.bias, a.weight_f32, S::column(v), a.columns, 0.0f, b[v]);
        }

    const int64_t step = (int64_t)gridDim.x * S::teams();
    int64_t base = (int64_t)blockIdx.x * S::teams();
    RowAt next = row_at(a, base + S::index());
    typename P::raw raw[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) raw[v] = load_piece<T, VEC>(row_of<T>(a.x, next), S::column(v), a.columns, next.live);
    for (; base < a.rows; base += step) {
        const RowAt at = next;
        float f[NV][VEC];
        float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            P::get(raw[v], f[v]);
#pragma unroll
            for (int e = 0; e < VEC; ++e) s.x += f[v][e];
        }
        next = row_at(a, base + step + S::index());
#pragma unroll
        for (int v = 0; v < NV; ++v) raw[v] = load_piece<T, VEC>(row_of<T>(a.x, next), S::column(v), a.columns, next.live);

        if (VEC > 1 && a.packed) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                uint32_t top = 0;
#pragma unroll
                for (int e = 0; e < VEC; ++e) top = max(top, magnitude(f[v][e]));
                const KeptScale scale(largest<S::KEPT_LANES>(top));
                int q[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) q[e] = scale.of(f[v][e]);
                const int c = S::column(v);
                if (at.there && c < a.columns) {
                    *reinterpret_cast<typename Kept<VEC>::raw *>(a.packed + at.row * a.columns + c) = Kept<VEC>::put(q);
                    if (c % KEPT_BLOCK == 0) a.scales[at.row * a.kept_blocks + c / KEPT_BLOCK] = scale.s;
                }
            }
        }

        const float mean = team_sum<S>(s, sums).x * inverse;
        s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int v = 0; v < NV; ++v)
            if (S::column(v) < a.columns)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    f[v][e] -= mean;
                    s.x += f[v][e];
                    s.y = fmaf(f[v][e], f[v][e], s.y);
                }
        s = team_sum<S>(s, sums);
        const float rest = s.x * inverse, rstd = rsqrtf(fmaxf(fmaf(-rest, rest, s.y * inverse), 0.0f) + a.eps);
        if (at.there) {
            T *to = row_of<T>(a.y, at);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = S::column(v);
                if (c < a.columns) {
                    float wv[VEC], bv[VEC], o[VEC];
                    if (S::FAR) {
                        vector_piece<T, VEC>(a.weight, a.weight_f32, c, a.columns, 1.0f, wv);
                        vector_piece<T, VEC>(a.bias, a.weight_f32, c, a.columns, 0.0f, bv);
                    }
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float y = fmaf((f[v][e] - rest) * rstd, S::FAR ? wv[e] : w[S::FAR ? 0 : v][e],
                                             S::FAR ? bv[e] : b[S::FAR ? 0 : v][e]);
                        o[e] = at.live ? y : 0.0f;
                    }
                    *reinterpret_cast<typename P::raw *>(to + c) = P::put(o);
                }
            }
            if (a.stats && S::member() == 0)
                reinterpret_cast<float2 *>(a.stats)[at.row] = at.live ? make_float2(mean + rest, rstd) : make_float2(0.0f, 0.0f);
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
            norm_forward_kernel<T, S><<<(unsigned)(blocks < most ? blocks : most), threads, 0, st>>>(a);
            GS_CUDA_TRY(cudaGetLastError());
            return GS_OK;
        });
    });
}

}  // namespace gs
