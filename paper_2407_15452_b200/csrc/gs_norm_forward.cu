// Layer norm, forward: y = (x - mean) rstd weight + bias, and on request x in 8 bits beside it.
//
// The mean is taken first and the squares of what differs from it second, both from registers; the differences' own mean, what rounding left
// of the first, is taken with them, so that a mean far from zero costs no digits.  A block's warps do so each for its own columns and
// then join: the squares about their means, and the squares of the means about the row's.
//
// Every value is read and written once, and memory traffic is the bound of fp32 rows and of short ones: 400000 x 128 take 68 us in fp32 (6.0 TB/s)
// and 44 in bf16 (4.7).  Wide 16-bit rows take 25 instructions a value, which keep the issue slots busy for two thirds of the time; the rest are the steps of a block's sums,
// shuffles and a barrier with few rows under way at once: 16384 x 4096 bf16 71 us (3.8 TB/s), fp32 96 (5.6), keeping 8 bits and the backward pass from them 215 and 271; with 32 columns a thread and the weights in shared memory 84, a warp for every row 95.
#include "gs_norm.cuh"

namespace gs {

// KEEP: x is kept in 8 bits as well
template <typename T, typename S, bool KEEP>
__global__ void __launch_bounds__(S::THREADS, S::RESIDENT) norm_forward_kernel(const __grid_constant__ NormArgs a)
{
    constexpr int VEC = S::VEC, NV = S::NV, N = S::N, V = S::V;
    typedef Piece<T, VEC> P;
    typedef typename Vec<V>::type F;
    __shared__ float4 places[2][16];                               // of a block's warps, in turn: mean, what it lacks, squares, columns
    int turn = 0;
    const float inverse = 1.0f / (float)a.columns;
    // columns of the lanes that reduce by shuffles, and 1 / that
    float in_group = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) in_group += S::in(v, a.columns) ? (float)VEC : 0.0f;
    in_group = group_sum<S>(in_group);
    const float of_group = in_group > 0.0f ? 1.0f / in_group : 0.0f;

    F w[S::FAR ? 1 : NV][N], b[S::FAR ? 1 : NV][N];
    if (!S::FAR)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            vector_piece<T, VEC>(a, a.weight, S::column(v), S::in(v, a.columns), 1.0f, w[v]);
            vector_piece<T, VEC>(a, a.bias, S::column(v), S::in(v, a.columns), 0.0f, b[v]);
        }

    int64_t base = (int64_t)blockIdx.x * S::teams();
    RowAt next(a, base + S::index());
    Line<T> x(a.x, next, S::column(0)), y(a.y, next, S::column(0));
    typename P::raw raw[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) raw[v] = load_piece<T, VEC>(x.at() + S::apart(v), next.live && S::in(v, a.columns));
    for (; base < a.rows; base += a.step) {
        const RowAt at = next;
        F f[NV][N], s = all_of<V>(0.0f);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            P::get(raw[v], f[v]);
#pragma unroll
            for (int e = 0; e < N; ++e) s = add_of(s, f[v][e]);
        }
        const bool wrapped = next.next(a);
        x.next(a.x, wrapped);
#pragma unroll
        for (int v = 0; v < NV; ++v) raw[v] = load_piece<T, VEC>(x.at() + S::apart(v), next.live && S::in(v, a.columns));

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
                    if (at.there && S::in(v, a.columns)) {
                        *reinterpret_cast<typename Kept<VEC>::raw *>(a.packed + at.row * a.columns + c) = Kept<VEC>::put(q);
                        if (c % KEPT_BLOCK == 0) a.scales[at.row * a.kept_blocks + c / KEPT_BLOCK] = scale.s;
                    }
                }
            }
        }

        // a warp's own mean and squares about it, then the warps' together
        const float mean = group_sum<S>(sum_of(s)) * of_group;
        F rest = all_of<V>(0.0f), squares = all_of<V>(0.0f);
        const F minus_mean = all_of<V>(-mean);
#pragma unroll
        for (int v = 0; v < NV; ++v)
            if (S::in(v, a.columns))
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    f[v][e] = add_of(f[v][e], minus_mean);
                    rest = add_of(rest, f[v][e]);
                    squares = fma_of(f[v][e], f[v][e], squares);
                }
        float2 t = group_sum<S>(make_float2(sum_of(rest), sum_of(squares)));
        t.x *= of_group;                                             // the mean's own rounding
        float less = t.x, m2 = t.y - in_group * t.x * t.x, whole = mean + t.x;
        if (S::BLOCK) {
            // means as what they differ by from the first warp's, which keeps their digits
            float4 *place = places[turn];
            turn ^= 1;
            if ((threadIdx.x & 31) == 0) place[threadIdx.x >> 5] = make_float4(mean, t.x, m2, in_group);
            __syncthreads();
            const int other = threadIdx.x & 15;                      // at most 16 warps
            const float first = place[0].x;
            const float4 its = other < (int)blockDim.x >> 5 ? place[other] : make_float4(first, 0.0f, 0.0f, 0.0f);
            const float d = its.x - first + its.y;
            float2 all = make_float2(d * its.w, fmaf(d * d, its.w, its.z));
#pragma unroll
            for (int o = 8; o; o >>= 1)
                all = add_of(all, make_float2(__shfl_xor_sync(0xffffffffu, all.x, o), __shfl_xor_sync(0xffffffffu, all.y, o)));
            const float off = all.x * inverse;
            m2 = fmaf(-off, all.x, all.y);
            less = first - mean + off;
            whole = first + off;
        }
        const float variance = m2 * inverse;
        const float rstd = rsqrtf((variance < 0.0f ? 0.0f : variance) + a.eps);     // a NaN stays one, which a maximum would let go
        if (at.there) {
            const F by = all_of<V>(rstd), minus_less = all_of<V>(-less);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (S::in(v, a.columns)) {
                    F wv[N], bv[N], o[N];
                    if (S::FAR) {
                        vector_piece<T, VEC>(a, a.weight, S::column(v), true, 1.0f, wv);
                        vector_piece<T, VEC>(a, a.bias, S::column(v), true, 0.0f, bv);
                    }
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        o[e] = fma_of(mul_of(add_of(f[v][e], minus_less), by), S::FAR ? wv[e] : w[S::FAR ? 0 : v][e],
                                      S::FAR ? bv[e] : b[S::FAR ? 0 : v][e]);
                    *reinterpret_cast<typename P::raw *>(y.at() + S::apart(v)) = at.live ? P::put(o) : P::none();
                }
            }
            if (a.stats && S::member() == 0)
                reinterpret_cast<float2 *>(a.stats)[at.row] = at.live ? make_float2(whole, rstd) : make_float2(0.0f, 0.0f);
        }
        y.next(a.y, wrapped);
    }
}

template <typename K>
static gs_status launch(K kernel, const NormArgs &args, int threads, int teams, int64_t most, int64_t element, cudaStream_t st)
{
    NormArgs a = args;
    const int64_t blocks = (a.rows + teams - 1) / teams, grid = blocks < most ? blocks : most;
    set_step(a, grid * teams, element);
    kernel<<<(unsigned)grid, threads, 0, st>>>(a);
    GS_CUDA_TRY(cudaGetLastError());
    return GS_OK;
}

gs_status norm_forward(const NormArgs &a, int32_t dtype, bool aligned, cudaStream_t st)
{
    return with_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        return with_team<T>(a.columns, aligned, [&](auto team, int threads) {
            typedef decltype(team) S;
            auto kernel = norm_forward_kernel<T, S, false>;
            if constexpr (S::VEC > 1)
                if (a.packed) kernel = norm_forward_kernel<T, S, true>;
            return launch(kernel, a, threads, S::BLOCK ? 1 : NORM_THREADS / S::LANES, (int64_t)sm_count() * (S::ON_SM / threads), sizeof(T), st);
        });
    });
}

}  // namespace gs
