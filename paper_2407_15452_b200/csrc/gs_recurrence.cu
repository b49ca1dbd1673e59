// Gated linear recurrence along the positions of a sequence, and its gradient.
//
//   a_t = sigmoid(z_t), h_t = a_t h_(t-1) + (1 - a_t) x_t;   g_t = dout_t + r_(t+1), r_t = a_t g_t,
//   dx_t = (1 - a_t) g_t, dz_t = a_t (1 - a_t) (h_(t-1) - x_t) g_t.
//
// Over a stretch of positions the state is an affine function of the state before it, h_end = P h_start + B with
// P the product of the a_t, and r_start = P r_end + R with the same P, so stretches can be computed side by side and joined.
// A warp has a stretch of up to 16 positions of 32 (or 64) channels, a block 8 stretches one after another, SPAN positions,
// and sequences longer than that are a cluster's: its blocks take neighbouring spans, exchange the (P, B) of theirs through
// distributed shared memory and go on to the next window of spans with the state that all of them know.  Every input is read once and every
// output written once; the joins are made in a fixed order.  The backward pass reads the state before each span, which the
// forward pass left, computes h again (one stream fewer than reading it, and in fp32) and joins only r.
#include <math.h>

#include <type_traits>

#include "gs_layers.cuh"

namespace gs {

static constexpr int STEPS = 16, WARPS = 8, SPAN = STEPS * WARPS, MOST_BLOCKS = 8;
// Blocks of an SM: what their registers and the shared memory that the next inputs wait in allow
static constexpr int FORWARD_BLOCKS = 3, BACKWARD_BLOCKS = 2;

struct ScanTensor {
    void *p;
    int64_t sb, st;                       // strides in elements: sequence, position
};

struct ScanArgs {
    ScanTensor gate, x, out, dout, dgate, dx;
    const float *h0, *dfinal;
    float *final_state, *dh0, *states;
    const int32_t *lens;
    Divider by_slabs;
    int64_t batch, channels, chains;      // chains = batch * slabs
    int32_t length, slabs, spans;         // slabs of 32 * V channels; spans = ceil(length / SPAN)
    int32_t stretches, steps;             // warps that share a span, positions of each
    int32_t blocks;                       // blocks of a cluster
};

// V neighbouring channels of a lane as they travel: a register each
template <typename T, int V> struct Lane;
template <> struct Lane<float, 1> {
    typedef float raw;
    static __device__ __forceinline__ void get(raw r, float (&f)[1]) { f[0] = r; }
    static __device__ __forceinline__ raw put(const float (&f)[1]) { return f[0]; }
};
template <typename T> struct Lane<T, 1> {
    typedef T raw;
    static __device__ __forceinline__ void get(raw r, float (&f)[1]) { f[0] = to_float(r); }
    static __device__ __forceinline__ raw put(const float (&f)[1]) { return from_float<T>(f[0]); }
};
template <typename T> struct Lane<T, 2> {
    typedef uint32_t raw;
    static __device__ __forceinline__ void get(raw r, float (&f)[2]) { unpack2<T>(r, f[0], f[1]); }
    static __device__ __forceinline__ raw put(const float (&f)[2]) { return pack2<T>(f[0], f[1]); }
};
// the same value in all of a lane's channels
template <typename T, int V> __device__ __forceinline__ typename Lane<T, V>::raw all_of(float x)
{
    float f[V];
#pragma unroll
    for (int v = 0; v < V; ++v) f[v] = x;
    return Lane<T, V>::put(f);
}

// Powers of two and reciprocals as the special-function units have them, 2^-22 and 2^-23 of the result; below 2^-126 they are zero.
__device__ __forceinline__ float power_of_two(float y)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
    return r;
}
__device__ __forceinline__ float reciprocal(float y)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
    return r;
}
// exp(z) = 2^y, y = z log2(e).  Rounding y costs |z| 2^-24 of the result, which tensors of 16 bits do not see; fp32 tensors get the first
// term of what it left out back.
template <typename T> __device__ __forceinline__ float exp_of(float z) { return power_of_two(1.44269504f * z); }
template <> __device__ __forceinline__ float exp_of<float>(float z)
{
    asm("min.NaN.f32 %0, %0, 0f42C80000;\n\tmax.NaN.f32 %0, %0, 0fC2C80000;" : "+f"(z));    // to [-100, 100]: infinities have no remainder
    const float y = 1.44269504f * z, rest = fmaf(1.44269504f, z, -y) + 1.92596299e-8f * z;
    return power_of_two(y) * fmaf(0.693147181f, rest, 1.0f);
}
// 1 - a = 1 / (1 + exp(z)), to a few units of its own last place however small it is: from a rounded a it would have no
// digits left where a channel remembers for long.
template <typename T> __device__ __forceinline__ float shut_of(float z) { return reciprocal(1.0f + exp_of<T>(z)); }

// a h + (1 - a) x from u = 1 - a: h - u h is rounded once, so a state that is kept for long loses nothing to a rounded a, and
// one that is given up (u = 1) leaves nothing behind
__device__ __forceinline__ float advance(float u, float h, float x) { return fmaf(u, x, fmaf(-u, h, h)); }

// What the backward pass keeps of a gate: the smaller of a and 1 - a, with the sign bit set where that is a.  Both factors of a (1 - a) are then
// at hand with all their digits, also where one of them is nearly 1.
template <typename T>
__device__ __forceinline__ float gate_of(float z, float &u)
{
    const float e = exp_of<T>(-fabsf(z)), larger = reciprocal(1.0f + e), m = e * larger;
    const bool shut = signbit(z);
    u = shut ? larger : m;
    return shut ? -m : m;
}

struct Place {                            // what a warp works on: positions [t0, t0 + rows) of a chain, `valid` of them valid
    int64_t b;                            // sequence
    uint32_t c;                           // the lane's first channel
    bool on, writes;                      // the warp has a chain; the lane has a channel (one that has none reads another's)
    int k, t0, rows, valid;               // k: the span
};

template <int V>
__device__ __forceinline__ Place place_of(const ScanArgs &a, int64_t chain, int lane, int k, int warp)
{
    Place p;
    p.on = chain < a.chains;
    p.b = p.on ? a.by_slabs.of(chain) : 0;
    p.c = p.on ? (uint32_t)(chain - p.b * a.slabs) * (32 * V) + lane * V : 0;
    p.writes = p.on && p.c < a.channels;
    if (!p.writes) p.c = 0;
    p.k = k;
    p.t0 = k * SPAN + warp * a.steps;
    p.rows = p.on ? min(max(a.length - p.t0, 0), a.steps) : 0;
    const int len = a.lens && p.on ? min(max(__ldg(a.lens + p.b), 0), a.length) : a.length;
    p.valid = min(p.rows, max(len - p.t0, 0));
    return p;
}

// A lane's channels of one tensor at position t0 + s.  The warp's part of the address is the same in all its lanes, so the
// accesses of a stretch need one register of each.
template <typename T, int V>
struct Walker {
    typedef typename Lane<T, V>::raw raw;
    char *p;                              // of the warp
    int64_t step;
    uint32_t lane;
    __device__ __forceinline__ Walker(const ScanTensor &t, const Place &at)
        : p(static_cast<char *>(t.p) + (at.b * t.sb + at.t0 * t.st) * (int64_t)sizeof(T)), step(t.st * (int64_t)sizeof(T)),
          lane(at.c * (uint32_t)sizeof(T))
    {
    }
    __device__ __forceinline__ raw &operator[](int s) const { return *reinterpret_cast<raw *>(p + s * step + lane); }
};

// Inputs wait in shared memory, each in a place that only the lane that asked for it reads again: no registers are held while they are on
// their way, and no barrier is needed when they have come.  In the places of positions that are not valid stands `without`, a gate that is open
// (a = 1) or a zero, so that what is computed from them changes nothing and needs no test.
template <typename R>
struct Stage {
    R (*place)[32];                       // [step][lane]
    int lane;
    template <typename W>
    __device__ __forceinline__ void fetch(const W &from, int valid, R without)
    {
        if constexpr (sizeof(R) == 4) {
            const uint32_t to = (uint32_t)__cvta_generic_to_shared(&place[0][lane]);
            if (valid == STEPS) {
#pragma unroll
                for (int s = 0; s < STEPS; ++s) copy(to + s * 128, &from[s]);
            } else {
#pragma unroll
                for (int s = 0; s < STEPS; ++s)
                    if (s < valid) copy(to + s * 128, &from[s]);
                    else place[s][lane] = without;
            }
        } else {                          // two bytes are less than such a copy moves
            R r[STEPS];
#pragma unroll
            for (int s = 0; s < STEPS; ++s) r[s] = s < valid ? from[s] : without;
#pragma unroll
            for (int s = 0; s < STEPS; ++s) place[s][lane] = r[s];
        }
    }
    static __device__ __forceinline__ void copy(uint32_t to, const R *from)
    {
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
    }
    __device__ __forceinline__ R operator[](int s) const { return place[s][lane]; }
};
__device__ __forceinline__ void fetches_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// all but the latest group of this thread's fetches have come
__device__ __forceinline__ void fetches_wait() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// stores a pair into the shared memory of another block of the cluster, at the place that `local` has in this one
__device__ __forceinline__ void store_remote(const float2 *local, uint32_t rank, float2 v)
{
    uint32_t there;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"((uint32_t)__cvta_generic_to_shared(local)), "r"(rank));
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there), "f"(v.x), "f"(v.y) : "memory");
}

// Joins of stretches, (P, B) each.  BACK: the chain runs from the last stretch to the first.  A block's pairs are published, read by
// all its warps after a barrier, and may be overwritten after the next one (of the block or the cluster) that `join` ends with.
template <int V, bool CLUSTER, bool BACK>
struct Joins {
    float2 (*part)[32 * V];                          // [stretch][channel]: of this block
    float2 (*span)[MOST_BLOCKS][32 * V];             // [2 in turn][rank][channel]: of the cluster's blocks
    float (*ahead)[32 * V];                          // [stretch][channel]: B of the stretches in the other direction
    int stretches, blocks, rank, warp, lane, first;  // first: index of the block's warp that has this chain's first stretch
    int turn;

    // p, b: of this warp's stretch; carry: into the window, moved over it; into: into this stretch.  With `ahead`: h, the state
    // before the block's span, and hb, its B over this stretch; h becomes the state before the stretch.
    __device__ __forceinline__ void join(const float (&p)[V], const float (&b)[V], float (&carry)[V], float (&into)[V],
                                         const float (&hb)[V], float (&h)[V])
    {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            part[first + warp][v * 32 + lane] = make_float2(p[v], b[v]);
            if (BACK) ahead[first + warp][v * 32 + lane] = hb[v];
        }
        __syncthreads();
        const int before = BACK ? stretches - 1 - warp : warp;
        if (BACK)
            for (int i = 0; i < warp; ++i)
#pragma unroll
                for (int v = 0; v < V; ++v)
                    h[v] = fmaf(part[first + i][v * 32 + lane].x, h[v], ahead[first + i][v * 32 + lane]);
        if (!CLUSTER) {
#pragma unroll
            for (int v = 0; v < V; ++v) into[v] = carry[v];
            for (int i = 0; i < before; ++i) {
                const int w = first + (BACK ? stretches - 1 - i : i);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float2 s = part[w][v * 32 + lane];
                    into[v] = fmaf(s.x, into[v], s.y);
                }
            }
            __syncthreads();
            return;
        }
        // the block's span, which every warp joins for itself (and what comes before its stretch on the way); each of
        // them hands it to one block
        float2 all[V], own[V];
#pragma unroll
        for (int v = 0; v < V; ++v) own[v] = all[v] = make_float2(1.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < WARPS; ++i) {
            const int w = BACK ? WARPS - 1 - i : i;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float2 s = part[w][v * 32 + lane];
                if (i == before) own[v] = all[v];
                all[v].y = fmaf(s.x, all[v].y, s.y);
                all[v].x *= s.x;
            }
        }
        if (warp < blocks)
#pragma unroll
            for (int v = 0; v < V; ++v) store_remote(&span[turn][rank][v * 32 + lane], warp, all[v]);
        cluster_arrive();
        cluster_wait();
        for (int i = 0; CLUSTER && i < blocks; ++i) {
            const int k = BACK ? blocks - 1 - i : i;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float2 s = span[turn][k][v * 32 + lane];
                if (k == rank) into[v] = fmaf(own[v].x, carry[v], own[v].y);
                carry[v] = fmaf(s.x, carry[v], s.y);
            }
        }
        turn ^= 1;                        // written again two windows later, behind a barrier that follows every read
    }
};

// A warp's items: a cluster has one chain and goes through its windows; a block of short chains goes from one group of chains to
// another, as long as there are some.
template <bool CLUSTER, bool BACK>
struct Items {
    int64_t chain, stride;                           // of the present item
    int window, windows;
    __device__ __forceinline__ bool next(const ScanArgs &a)
    {
        if (!CLUSTER) {
            chain += stride;
            return chain - chain_offset < a.chains;
        }
        window += BACK ? -1 : 1;
        return BACK ? window >= 0 : window < windows;
    }
    int64_t chain_offset;                            // of the warp's group in its block: all warps of a block take the same number of items
};
template <bool CLUSTER, bool BACK>
__device__ __forceinline__ Items<CLUSTER, BACK> first_item(const ScanArgs &a, int group, int groups)
{
    Items<CLUSTER, BACK> it;
    it.windows = (a.spans + a.blocks - 1) / a.blocks;
    it.window = CLUSTER && BACK ? it.windows - 1 : 0;
    it.chain = CLUSTER ? blockIdx.x / a.blocks : (int64_t)blockIdx.x * groups + group;
    it.chain_offset = group;
    it.stride = (int64_t)gridDim.x * groups;
    return it;
}

template <typename T, int V, bool CLUSTER>
__global__ void __launch_bounds__(32 * WARPS, CLUSTER ? 2 : FORWARD_BLOCKS) scan_forward_kernel(const __grid_constant__ ScanArgs a)
{
    typedef typename Lane<T, V>::raw raw;
    __shared__ float2 part[WARPS][32 * V];
    __shared__ float2 span[CLUSTER ? 2 : 1][CLUSTER ? MOST_BLOCKS : 1][32 * V];
    extern __shared__ uint32_t room[];                               // [2 in turn][gate, x][warp][step][lane]
    const int lane = threadIdx.x & 31, index = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    const int group = CLUSTER ? 0 : index / a.stretches, warp = CLUSTER ? index : index - group * a.stretches;
    const int rank = CLUSTER ? (int)cluster_rank() : 0, groups = CLUSTER ? 1 : (blockDim.x >> 5) / a.stretches;
    raw (*stages)[32] = reinterpret_cast<raw(*)[32]>(room) + index * STEPS;
    constexpr int ROWS = WARPS * STEPS;
    if (CLUSTER) cluster_arrive();                      // completed by the wait before the first remote store

    auto item = first_item<CLUSTER, false>(a, group, groups);
    Place next = place_of<V>(a, item.chain, lane, item.window * a.blocks + rank, warp);
    auto fetch = [&](const Place &p, int turn) {
        Stage<raw>{stages + (2 * turn) * ROWS, lane}.fetch(Walker<T, V>(a.gate, p), p.valid, all_of<T, V>(INFINITY));
        Stage<raw>{stages + (2 * turn + 1) * ROWS, lane}.fetch(Walker<T, V>(a.x, p), p.valid, all_of<T, V>(0.0f));
    };
    fetch(next, 0);
    fetches_end();

    Joins<V, CLUSTER, false> joins = {part, reinterpret_cast<float2(*)[MOST_BLOCKS][32 * V]>(span), nullptr,
                                      a.stretches, a.blocks, rank, warp, lane, group * a.stretches, 0};
    float carry[V], into[V];
    if (CLUSTER) {
#pragma unroll
        for (int v = 0; v < V; ++v) carry[v] = a.h0 ? a.h0[next.b * a.channels + next.c + v] : 0.0f;
        cluster_wait();
    }
    bool more;
    int turn = 0;
    do {
        const Place p = next;
        more = item.next(a);
        if (more) {
            next = place_of<V>(a, item.chain, lane, item.window * a.blocks + rank, warp);
            fetch(next, turn ^ 1);
        }
        fetches_end();
        if (!CLUSTER)
#pragma unroll
            for (int v = 0; v < V; ++v) carry[v] = a.h0 ? a.h0[p.b * a.channels + p.c + v] : 0.0f;
        fetches_wait();
        const Stage<raw> z = {stages + (2 * turn) * ROWS, lane}, x = {stages + (2 * turn + 1) * ROWS, lane};
        turn ^= 1;
        float u[STEPS][V], h[V], pn[V];
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = 0.0f, pn[v] = 1.0f;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            float zf[V], xf[V];
            Lane<T, V>::get(z[s], zf);
            Lane<T, V>::get(x[s], xf);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                u[s][v] = shut_of<T>(zf[v]);
                h[v] = advance(u[s][v], h[v], xf[v]);
                pn[v] = fmaf(-u[s][v], pn[v], pn[v]);
            }
        }
        if (CLUSTER || a.stretches > 1) {
            joins.join(pn, h, carry, into, h, h);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) into[v] = carry[v];
        }
        const Walker<T, V> out(a.out, p);
        auto write = [&](auto full_stretch) {
            constexpr bool whole = decltype(full_stretch)::value;
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                float o[V];
                Lane<T, V>::get(x[s], o);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    o[v] = into[v] = advance(u[s][v], into[v], o[v]);
                    if (!whole && s >= p.valid) o[v] = 0.0f;
                }
                if (whole || s < p.rows) out[s] = Lane<T, V>::put(o);
            }
        };
        if (p.writes) {
            if (p.valid == STEPS) write(std::true_type());
            else write(std::false_type());
        }
        if (p.writes && warp == a.stretches - 1 && p.k < a.spans) {
            float *to = p.k < a.spans - 1 ? (a.states ? a.states + (p.b * (a.spans - 1) + p.k) * a.channels : nullptr)
                                          : (a.final_state ? a.final_state + p.b * a.channels : nullptr);
            if (to)
#pragma unroll
                for (int v = 0; v < V; ++v) to[p.c + v] = into[v];
        }
    } while (more);
}

template <typename T, int V, bool CLUSTER>
__global__ void __launch_bounds__(32 * WARPS, BACKWARD_BLOCKS) scan_backward_kernel(const __grid_constant__ ScanArgs a)
{
    typedef typename Lane<T, V>::raw raw;
    __shared__ float2 part[WARPS][32 * V];
    __shared__ float ahead[WARPS][32 * V];
    __shared__ float2 span[CLUSTER ? 2 : 1][CLUSTER ? MOST_BLOCKS : 1][32 * V];
    extern __shared__ uint32_t room[];                               // [2 in turn][gate, x, dout][warp][step][lane]
    const int lane = threadIdx.x & 31, index = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    const int group = CLUSTER ? 0 : index / a.stretches, warp = CLUSTER ? index : index - group * a.stretches;
    const int rank = CLUSTER ? (int)cluster_rank() : 0, groups = CLUSTER ? 1 : (blockDim.x >> 5) / a.stretches;
    raw (*stages)[32] = reinterpret_cast<raw(*)[32]>(room) + index * STEPS;
    constexpr int ROWS = WARPS * STEPS;
    if (CLUSTER) cluster_arrive();

    auto item = first_item<CLUSTER, true>(a, group, groups);
    Place next = place_of<V>(a, item.chain, lane, item.window * a.blocks + rank, warp);
    auto fetch = [&](const Place &p, int turn) {
        Stage<raw>{stages + (3 * turn) * ROWS, lane}.fetch(Walker<T, V>(a.gate, p), p.valid, all_of<T, V>(INFINITY));
        Stage<raw>{stages + (3 * turn + 1) * ROWS, lane}.fetch(Walker<T, V>(a.x, p), p.valid, all_of<T, V>(0.0f));
        Stage<raw>{stages + (3 * turn + 2) * ROWS, lane}.fetch(Walker<T, V>(a.dout, p), a.dout.p ? p.valid : 0, all_of<T, V>(0.0f));
    };
    fetch(next, 0);
    fetches_end();

    Joins<V, CLUSTER, true> joins = {part, reinterpret_cast<float2(*)[MOST_BLOCKS][32 * V]>(span), ahead,
                                     a.stretches, a.blocks, rank, warp, lane, group * a.stretches, 0};
    float carry[V], into[V];
    if (CLUSTER) {
#pragma unroll
        for (int v = 0; v < V; ++v) carry[v] = a.dfinal ? a.dfinal[next.b * a.channels + next.c + v] : 0.0f;
        cluster_wait();
    }
    bool more;
    int turn = 0;
    do {
        const Place p = next;
        more = item.next(a);
        if (more) {
            next = place_of<V>(a, item.chain, lane, item.window * a.blocks + rank, warp);
            fetch(next, turn ^ 1);
        }
        fetches_end();
        float h[V];                                                  // the state before the block's span
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int64_t at = p.b * a.channels + p.c + v;
            if (!CLUSTER) carry[v] = a.dfinal ? a.dfinal[at] : 0.0f;
            h[v] = 0.0f;
            if (CLUSTER && p.k > 0 && p.k < a.spans) h[v] = a.states[(p.b * (a.spans - 1) + p.k - 1) * a.channels + p.c + v];
            else if (p.k == 0 && a.h0) h[v] = a.h0[at];
        }
        fetches_wait();
        const Stage<raw> z = {stages + (3 * turn) * ROWS, lane}, x = {stages + (3 * turn + 1) * ROWS, lane},
                         g = {stages + (3 * turn + 2) * ROWS, lane};
        turn ^= 1;
        float u[STEPS][V], hn[V], pn[V], rn[V];                      // u: first as gate_of has it, then 1 - a
#pragma unroll
        for (int v = 0; v < V; ++v) hn[v] = 0.0f, pn[v] = 1.0f, rn[v] = 0.0f;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            float zf[V], xf[V], gf[V];
            Lane<T, V>::get(z[s], zf);
            Lane<T, V>::get(x[s], xf);
            Lane<T, V>::get(g[s], gf);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float shut;
                u[s][v] = gate_of<T>(zf[v], shut);
                hn[v] = advance(shut, hn[v], xf[v]);
                pn[v] = fmaf(-shut, pn[v], pn[v]);
                rn[v] = fmaf(pn[v], gf[v], rn[v]);
            }
        }
        if (CLUSTER || a.stretches > 1) {
            joins.join(pn, rn, carry, into, hn, h);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) into[v] = carry[v];
        }
        float d[STEPS][V];                                           // a (1 - a) (h_(t-1) - x_t)
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            float xf[V];
            Lane<T, V>::get(x[s], xf);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float m = fabsf(u[s][v]);
                u[s][v] = signbit(u[s][v]) ? 1.0f - m : m;
                d[s][v] = fmaf(-m, m, m) * (h[v] - xf[v]);
                h[v] = advance(u[s][v], h[v], xf[v]);
            }
        }
        const Walker<T, V> at_dx(a.dx, p), at_dz(a.dgate, p);
        auto write = [&](auto full_stretch) {
            constexpr bool whole = decltype(full_stretch)::value;
#pragma unroll
            for (int s = STEPS - 1; s >= 0; --s) {
                float gf[V], dx[V], dz[V];
                Lane<T, V>::get(g[s], gf);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float full = gf[v] + into[v];
                    dx[v] = u[s][v] * full;
                    into[v] = full - dx[v];
                    dz[v] = d[s][v] * full;
                    if (!whole && s >= p.valid) dx[v] = dz[v] = 0.0f;
                }
                if (whole || s < p.rows) {
                    at_dx[s] = Lane<T, V>::put(dx);
                    at_dz[s] = Lane<T, V>::put(dz);
                }
            }
        };
        if (p.writes) {
            if (p.valid == STEPS) write(std::true_type());
            else write(std::false_type());
        }
        if (a.dh0 && p.writes && p.k == 0 && warp == 0)
#pragma unroll
            for (int v = 0; v < V; ++v) a.dh0[p.b * a.channels + p.c + v] = into[v];
    } while (more);
}

template <typename T, int V>
static gs_status launch(const ScanArgs &args, bool backward, cudaStream_t st)
{
    ScanArgs a = args;
    a.slabs = (int32_t)((a.channels + 32 * V - 1) / (32 * V));
    a.by_slabs = Divider(a.slabs);
    a.chains = a.batch * a.slabs;
    a.spans = (a.length + SPAN - 1) / SPAN;
    const bool cluster = a.spans > 1;
    static SharedRecord records[4];
    auto kernel = backward ? cluster ? scan_backward_kernel<T, V, true> : scan_backward_kernel<T, V, false>
                           : cluster ? scan_forward_kernel<T, V, true> : scan_forward_kernel<T, V, false>;
    SharedRecord &record = records[2 * backward + cluster];
    const size_t shared = (size_t)2 * (backward ? 3 : 2) * SPAN * 32 * sizeof(typename Lane<T, V>::raw);
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr = {};
    int64_t grid;
    if (cluster) {
        // as few windows as a cluster of MOST_BLOCKS allows, and no more blocks than these need
        const int windows = (a.spans + MOST_BLOCKS - 1) / MOST_BLOCKS;
        a.blocks = (a.spans + windows - 1) / windows;
        a.stretches = WARPS;
        a.steps = STEPS;
        grid = a.chains * a.blocks;
        cfg.blockDim = dim3(32 * WARPS);
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = (unsigned)a.blocks;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
    } else {
        // several chains a block where one needs few warps
        a.blocks = 1;
        a.stretches = a.length > STEPS ? (a.length + STEPS - 1) / STEPS : 1;
        a.steps = (a.length + a.stretches - 1) / a.stretches;
        const int groups = WARPS / a.stretches > 0 ? WARPS / a.stretches : 1;
        cfg.blockDim = dim3(32 * groups * a.stretches);
        const int64_t most = (int64_t)sm_count() * (backward ? BACKWARD_BLOCKS : FORWARD_BLOCKS);
        grid = (a.chains + groups - 1) / groups;
        if (grid > most) grid = most;
    }
    if (grid > 0x7FFFFFFF) {
        set_error("a recurrence of %lld blocks exceeds one launch", (long long)grid);
        return GS_ERR_UNSUPPORTED;
    }
    gs_status s = allow_shared(kernel, (int)shared, record);
    if (s != GS_OK) return s;
    cfg.gridDim = dim3((unsigned)grid);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = st;
    GS_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, a));
    return GS_OK;
}

// an empty sequence ends with the state that it starts with
static gs_status copy_states(const float *from, float *to, int64_t n, cudaStream_t st)
{
    if (!to || to == from) return GS_OK;
    if (from) GS_CUDA_TRY(cudaMemcpyAsync(to, from, n * sizeof(float), cudaMemcpyDeviceToDevice, st));
    else GS_CUDA_TRY(cudaMemsetAsync(to, 0, n * sizeof(float), st));
    return GS_OK;
}

static gs_status check(const gs_recurrence_config *c, ScanArgs *a)
{
    if (!c) return bad("config is NULL");
    if (!known_type(c->dtype)) return bad("dtype must be GS_TABLE_F32, GS_TABLE_F16 or GS_TABLE_BF16");
    if (c->batch < 0 || c->length < 0 || c->channels <= 0) return bad("negative batch or length, or no channels");
    if (c->length > (1 << 30) || c->channels > ((int64_t)1 << 30) || (c->batch > 0 && c->channels > ((int64_t)1 << 40) / c->batch)) {
        set_error("recurrences of up to 2^30 positions, 2^30 channels and 2^40 states are supported");
        return GS_ERR_UNSUPPORTED;
    }
    *a = ScanArgs{};
    a->batch = c->batch;
    a->channels = c->channels;
    a->length = c->length;
    a->lens = c->d_lens;
    return GS_OK;
}

static ScanTensor tensor(const void *p, const int64_t (&stride)[2])
{
    return {const_cast<void *>(p), stride[0], stride[1]};
}

static gs_status run(ScanArgs &a, int32_t dtype, const ScanTensor *const *t, int n, int outputs, bool backward, cudaStream_t st)
{
    const uintptr_t es = size_of(dtype);
    bool pairs = dtype != GS_TABLE_F32 && a.channels % 2 == 0;
    for (int i = 0; i < n; ++i) {
        if (!t[i]->p) return bad("null pointer");
        if ((uintptr_t)t[i]->p % es) return bad("tensor not aligned to its element size");
        if (i < outputs && ((a.batch > 1 && t[i]->sb == 0) || (a.length > 1 && t[i]->st == 0)))
            return bad("an output has a zero stride");
        pairs = pairs && (uintptr_t)t[i]->p % 4 == 0 && (t[i]->sb | t[i]->st) % 2 == 0;
    }
    pairs = pairs && a.channels > 32;                   // one channel a lane where two would leave half the lanes idle
    if (dtype == GS_TABLE_F32) return launch<float, 1>(a, backward, st);
    if (dtype == GS_TABLE_F16) return pairs ? launch<__half, 2>(a, backward, st) : launch<__half, 1>(a, backward, st);
    return pairs ? launch<__nv_bfloat16, 2>(a, backward, st) : launch<__nv_bfloat16, 1>(a, backward, st);
}

}  // namespace gs

using namespace gs;

extern "C" {

int64_t gs_recurrence_states(const gs_recurrence_config *cfg)
{
    ScanArgs a;
    if (check(cfg, &a) != GS_OK) return -1;
    return a.length > 0 ? a.batch * a.channels * ((a.length - 1) / SPAN) : 0;
}

gs_status gs_recurrence_forward(const gs_recurrence_config *cfg, const void *d_gate, const void *d_x, const float *d_h0,
                                void *d_out, float *d_final, float *d_states, void *stream)
{
    ScanArgs a;
    gs_status s = check(cfg, &a);
    if (s != GS_OK || a.batch == 0) return s;
    a.h0 = d_h0;
    a.final_state = d_final;
    a.states = d_states;
    if (a.length == 0) return copy_states(d_h0, d_final, a.batch * a.channels, (cudaStream_t)stream);
    a.gate = tensor(d_gate, cfg->gate_stride);
    a.x = tensor(d_x, cfg->x_stride);
    a.out = tensor(d_out, cfg->out_stride);
    const ScanTensor *all[3] = {&a.out, &a.gate, &a.x};
    return run(a, cfg->dtype, all, 3, 1, false, (cudaStream_t)stream);
}

gs_status gs_recurrence_backward(const gs_recurrence_config *cfg, const void *d_dout, const float *d_dfinal,
                                 const void *d_gate, const void *d_x, const float *d_h0, const float *d_states,
                                 void *d_dgate, void *d_dx, float *d_dh0, void *stream)
{
    ScanArgs a;
    gs_status s = check(cfg, &a);
    if (s != GS_OK || a.batch == 0) return s;
    a.h0 = d_h0;
    a.dfinal = d_dfinal;
    a.dh0 = d_dh0;
    a.states = const_cast<float *>(d_states);
    if (a.length == 0) return copy_states(d_dfinal, d_dh0, a.batch * a.channels, (cudaStream_t)stream);
    if (a.length > SPAN && !d_states) return bad("d_states is NULL");
    a.gate = tensor(d_gate, cfg->gate_stride);
    a.x = tensor(d_x, cfg->x_stride);
    a.dgate = tensor(d_dgate, cfg->dgate_stride);
    a.dx = tensor(d_dx, cfg->dx_stride);
    a.dout = tensor(d_dout, cfg->dout_stride);
    const ScanTensor *all[5] = {&a.dgate, &a.dx, &a.gate, &a.x, &a.dout};
    return run(a, cfg->dtype, all, d_dout ? 5 : 4, 2, true, (cudaStream_t)stream);
}

}  // extern "C"
