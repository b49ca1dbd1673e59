// One row of a result again, by one warp, from nothing but what the row sees.
//
// The tile kernels multiply whole tiles: a key that a row does not see has a factor of zero there, and zero times an
// infinity or a NaN is NaN.  fp32 products as three of tf32 turn an infinite factor into a NaN as well (its low part is
// inf - inf).  Either way the row's result holds a NaN, so a warp that meets one among its results has those rows, once
// they are stored, done again here, in fp32 and term by term: infinities give what the formulas in gs_attn.cuh give for
// them, hidden positions give nothing, and a NaN that the row does see stays a NaN.  A tile kernel pays one addition per
// result to know.  Of finite inputs only rows with scores beyond 10^7 come here (row_factor).
//
// Scores are made by one lane per position, sums over positions by lanes that own the columns lane, lane + 32, ..; the
// loop ends at the first NaN that reaches every column.
#pragma once

#include "gs_attn.cuh"

namespace gs {
namespace again {

static constexpr unsigned ALL_LANES = 0xffffffffu;

template <typename T>
__device__ __forceinline__ T *row_at(const AttnTensor &t, int64_t b, int64_t pos, int64_t head)
{
    return reinterpret_cast<T *>(t.p) + b * t.sb + pos * t.sl + head * t.sh;
}
// by one lane; rows of whole, aligned 16 bytes are read so (8 heads of 4096 x 128, bf16, causal, a NaN in one column of v that
// every row sees: forward 83 ms value by value and 21 ms so)
template <typename T>
__device__ __forceinline__ float dot(const T *x, const T *y, int n)
{
    constexpr int PER = 16 / (int)sizeof(T);
    float s = 0.f;
    if (n % PER == 0 && ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y)) & 15) == 0) {
#pragma unroll 4
        for (int c = 0; c < n; c += PER) {
            const uint4 u = __ldg(reinterpret_cast<const uint4 *>(x + c)), w = __ldg(reinterpret_cast<const uint4 *>(y + c));
            const T *f = reinterpret_cast<const T *>(&u), *g = reinterpret_cast<const T *>(&w);
#pragma unroll
            for (int i = 0; i < PER; ++i) s = fmaf(to_f(f[i]), to_f(g[i]), s);
        }
    } else {
        for (int c = 0; c < n; ++c) s = fmaf(to_f(x[c]), to_f(y[c]), s);
    }
    return s;
}
// acc += sum over the first n lanes' w times their rows, which lie `stride` values apart
template <typename T>
__device__ __forceinline__ void add_rows(float (&acc)[4], float w, const T *rows, int64_t stride, int n, int dim)
{
    const int lane = threadIdx.x & 31;
#pragma unroll 8
    for (int j = 0; j < n; ++j) {
        const float f = __shfl_sync(ALL_LANES, w, j);
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (lane + 32 * x < dim) acc[x] = fmaf(f, to_f(rows[j * stride + lane + 32 * x]), acc[x]);
    }
}
template <typename T>
__device__ __forceinline__ void put_row(T *row, const float (&acc)[4], float by, int c0, int c1)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const int c = lane + 32 * x;
        if (c >= c0 && c < c1) row[c] = from_f<T>(acc[x] * by);
    }
}
// whether a stored row holds a NaN; past L1, where rows that left through TMA have never been
__device__ __forceinline__ bool is_nan(float x) { return x != x; }
template <typename T>
__device__ __forceinline__ bool nan_in(const T *row, int c0, int c1)
{
    bool found = false;
    for (int c = c0 + (int)(threadIdx.x & 31); c < c1; c += 32) found = found || is_nan(to_f(__ldcg(row + c)));
    return __any_sync(ALL_LANES, found);
}
template <typename T>
__device__ __forceinline__ void zero_row(T *row, int c0, int c1)
{
    for (int c = c0 + (int)(threadIdx.x & 31); c < c1; c += 32) row[c] = from_f<T>(0.f);
}
__device__ __forceinline__ void fill(float (&acc)[4], float v)
{
#pragma unroll
    for (int x = 0; x < 4; ++x) acc[x] = v;
}

// What the accumulators of a row are multiplied by at the end, `top` being the base of its exponents in powers of two and
// `inverse` that of its sum.  Exponents are formed as s * mul - top in one operation, of which top has been rounded; that is
// one factor for the whole row as long as it is a few powers of two, but beyond 2^31 the largest probability itself becomes
// zero or infinite (in binary16 beyond 2^28).  From 2^24 on, where it may be half a power, the row is marked
// to be done again, where the exponents are differences of scores.
__device__ __forceinline__ float row_factor(float top, float inverse)
{
    if (fabsf(top) < 16777216.f) return inverse;
    return top == -INFINITY && !is_nan(inverse) ? 0.f : NAN;       // 0: nothing visible, or nothing above -infinity
}
// the row's lse, from the same and the sum's logarithm in powers of two
__device__ __forceinline__ float row_lse(float top, float factor, float log2_sum)
{
    return factor == 0.f ? -INFINITY : is_nan(factor) ? NAN : (top + log2_sum) * LN2;
}

// output and lse of query row i < n_q
template <typename T>
__device__ __forceinline__ void output(const AttnArgs &a, int64_t b, int h, int i)
{
    const AttnSeq s = attn_seq(a, b);
    const int lane = threadIdx.x & 31, lo = attn_lo(a, s, i), hi = attn_hi(a, s, i), g = h / a.group;
    const T *q = row_at<T>(a.q, b, i, h);
    float *lse = a.lse + (b * a.q_heads + h) * a.q_len + i;
    const bool known = !is_nan(__ldcg(lse));               // the tile kernel's scores held no NaN: its lse stands
    float acc[4] = {}, top = -INFINITY, sum = 0.f;
    for (int j0 = lo; j0 < hi; j0 += 32) {
        const bool in = j0 + lane < hi;
        const float x = in ? a.scale * dot(q, row_at<T>(a.k, b, j0 + lane, g), a.dim) : -INFINITY;
        if (__any_sync(ALL_LANES, x != x)) {
            fill(acc, NAN);
            top = sum = NAN;
            break;
        }
        float m = x;
#pragma unroll
        for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(ALL_LANES, m, o));
        m = fmaxf(m, top);
        const float base = m == -INFINITY ? 0.f : m, keep = expf(top - base), p = in ? expf(x - base) : 0.f;
        float part = p;
#pragma unroll
        for (int o = 16; o; o >>= 1) part += __shfl_xor_sync(ALL_LANES, part, o);
        sum = fmaf(sum, keep, part);
        top = m;
#pragma unroll
        for (int x = 0; x < 4; ++x) acc[x] *= keep;
        add_rows(acc, p, row_at<T>(a.v, b, j0, g), a.v.sl, min(32, hi - j0), a.dim);
        bool over = known;                                 // every column is NaN already
#pragma unroll
        for (int x = 0; x < 4; ++x) over = over && (lane + 32 * x >= a.dim || is_nan(acc[x]));
        if (__all_sync(ALL_LANES, over)) break;
    }
    // a score of +infinity: lse is infinite and every quotient exp(s - lse) of it is NaN
    put_row(row_at<T>(a.out, b, i, h), acc, sum == 0.f ? 0.f : 1.f / sum, 0, a.dim);
    if (lane == 0 && !known) *lse = sum == 0.f ? -INFINITY : top == INFINITY ? top : top + logf(sum);
}

// columns [c0, c1) of dq of query row i < n_q
template <typename T>
__device__ __forceinline__ void query_gradient(const AttnArgs &a, int64_t b, int h, int i, int c0, int c1)
{
    const AttnSeq s = attn_seq(a, b);
    const int lane = threadIdx.x & 31, lo = attn_lo(a, s, i), hi = attn_hi(a, s, i), g = h / a.group;
    const T *q = row_at<T>(a.q, b, i, h), *d = row_at<T>(a.dout, b, i, h);
    const float lse = a.lse[(b * a.q_heads + h) * a.q_len + i], delta = dot(d, row_at<T>(a.out, b, i, h), a.dim);
    float acc[4] = {};
    for (int j0 = lo; j0 < hi && lse != -INFINITY; j0 += 32) {
        float ds = 0.f;
        if (j0 + lane < hi) {
            const float p = expf(a.scale * dot(q, row_at<T>(a.k, b, j0 + lane, g), a.dim) - lse);
            ds = p * (dot(d, row_at<T>(a.v, b, j0 + lane, g), a.dim) - delta);
        }
        if (__any_sync(ALL_LANES, ds != ds)) {
            fill(acc, NAN);
            break;
        }
        add_rows(acc, ds, row_at<T>(a.k, b, j0, g), a.k.sl, min(32, hi - j0), a.dim);
    }
    put_row(row_at<T>(a.dq, b, i, h), acc, a.scale, c0, c1);
}

// dk and dv of key row j < n_k, or one of them
template <typename T>
__device__ __forceinline__ void key_gradient(const AttnArgs &a, int64_t b, int g, int j, bool want_k, bool want_v)
{
    const AttnSeq s = attn_seq(a, b);
    const int lane = threadIdx.x & 31, lo = attn_q_first(a, s, j), hi = attn_q_last(a, s, j + 1);
    const T *k = row_at<T>(a.k, b, j, g), *v = row_at<T>(a.v, b, j, g);
    float dk[4] = {}, dv[4] = {};
    bool over = false;                                     // nothing that is to come can change a result
    for (int h = g * a.group; h < (g + 1) * a.group && !over; ++h)
        for (int i0 = lo; i0 < hi && !over; i0 += 32) {
            float p = 0.f, ds = 0.f;
            bool in = i0 + lane < hi;
            const float lse = in ? a.lse[(b * a.q_heads + h) * a.q_len + i0 + lane] : -INFINITY;
            in = lse != -INFINITY;                         // a row that sees nothing gives no gradient
            if (in) {
                const T *q = row_at<T>(a.q, b, i0 + lane, h), *d = row_at<T>(a.dout, b, i0 + lane, h);
                p = expf(a.scale * dot(q, k, a.dim) - lse);
                ds = p * (dot(d, v, a.dim) - dot(d, row_at<T>(a.out, b, i0 + lane, h), a.dim));
            }
            const bool no_v = __any_sync(ALL_LANES, p != p), no_k = __any_sync(ALL_LANES, ds != ds);
            if (no_v) fill(dv, NAN);
            if (no_k) fill(dk, NAN);
            over = (no_v || !want_v) && (no_k || !want_k);
            // rows without a part are left out, as they are of the sums above: their factor of zero may meet a NaN
            unsigned some = over ? 0 : __ballot_sync(ALL_LANES, in);
            while (some) {                                 // a run of rows at a time: mostly all of them
                const int x = __ffs(some) - 1, run = __ffs(~(some >> x)) - 1, n = run < 0 ? 32 : run;
                add_rows(dv, __shfl_sync(ALL_LANES, p, (x + lane) & 31), row_at<T>(a.dout, b, i0 + x, h), a.dout.sl, n, a.dim);
                add_rows(dk, __shfl_sync(ALL_LANES, ds, (x + lane) & 31), row_at<T>(a.q, b, i0 + x, h), a.q.sl, n, a.dim);
                some = x + n < 32 ? some >> (x + n) << (x + n) : 0;
            }
        }
    if (want_k) put_row(row_at<T>(a.dk, b, j, g), dk, a.scale, 0, a.dim);
    if (want_v) put_row(row_at<T>(a.dv, b, j, g), dv, 1.f, 0, a.dim);
}

// What a warp calls, whole, behind its own stores: those of rows [r0, r1) that hold a NaN.  Rows past a sequence's end
// are zeros.
template <typename T>
static __device__ __noinline__ void outputs(const AttnArgs &a, int64_t b, int h, int r0, int r1)
{
    __syncwarp();
    const int n = attn_seq(a, b).nq;
    r1 = min(r1, a.q_len);
    for (int r = r0; r < r1; ++r) {
        if (!nan_in(row_at<T>(a.out, b, r, h), 0, a.dim)) continue;
        if (r < n) output<T>(a, b, h, r);
        else zero_row(row_at<T>(a.out, b, r, h), 0, a.dim);
    }
}
// columns [c0, c1) of dq: another warp has the others
template <typename T>
__device__ __forceinline__ void query_gradients_here(const AttnArgs &a, int64_t b, int h, int r0, int r1, int c0, int c1)
{
    __syncwarp();
    const int n = attn_seq(a, b).nq;
    r1 = min(r1, a.q_len);
    c1 = min(c1, a.dim);
    for (int r = r0; r < r1; ++r) {
        if (!nan_in(row_at<T>(a.dq, b, r, h), c0, c1)) continue;
        if (r < n) query_gradient<T>(a, b, h, r, c0, c1);
        else zero_row(row_at<T>(a.dq, b, r, h), c0, c1);
    }
}
// dk and dv, or one of them
template <typename T>
__device__ __forceinline__ void key_gradients_here(const AttnArgs &a, int64_t b, int g, int j0, int j1, bool want_k, bool want_v)
{
    __syncwarp();
    const int n = attn_seq(a, b).nk;
    j1 = min(j1, a.k_len);
    for (int j = j0; j < j1; ++j) {
        const bool k = want_k && nan_in(row_at<T>(a.dk, b, j, g), 0, a.dim), v = want_v && nan_in(row_at<T>(a.dv, b, j, g), 0, a.dim);
        if (!k && !v) continue;
        if (j < n) {
            key_gradient<T>(a, b, g, j, k, v);
        } else {
            if (k) zero_row(row_at<T>(a.dk, b, j, g), 0, a.dim);
            if (v) zero_row(row_at<T>(a.dv, b, j, g), 0, a.dim);
        }
    }
}


// Called or in place, as suits a kernel's registers.  Backward, called | in place, us: fp32 tiles 16 x 8 heads of 333 x 64 246 |
// 227, 64 x 4 of 200 x 32 82 | 78; 16384 walks of 40 655 | 663, 8192 of 80 433 | 444, 4096 heads of 100 x 128 349 | 357.
template <typename T>
static __device__ __noinline__ void query_gradients(const AttnArgs &a, int64_t b, int h, int r0, int r1, int c0, int c1)
{
    query_gradients_here<T>(a, b, h, r0, r1, c0, c1);
}
template <typename T>
static __device__ __noinline__ void key_gradients(const AttnArgs &a, int64_t b, int g, int j0, int j1, bool want_k, bool want_v)
{
    key_gradients_here<T>(a, b, g, j0, j1, want_k, want_v);
}

}  // namespace again
}  // namespace gs
