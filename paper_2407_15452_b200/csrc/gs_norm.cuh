// Layer norm: what the forward and the backward kernels share.
//
// A row is held by a team, the lanes of a part of a warp or all threads of a block, in registers from its only read to its only
// write: thread i of the team has NV pieces of VEC neighbouring columns, piece v at column (v * team + i) * VEC.  A thread's
// columns are the same in every row, so weights, and in the backward pass the sums for their gradients, stay in registers while the team goes
// through its rows; the next row's values are on their way while the present one is summed.
#pragma once

#include "gs_layers.cuh"

namespace gs {

static constexpr int NORM_THREADS = 256;              // of blocks that hold several teams
static constexpr int NORM_MOST_COLUMNS = 16384;
static constexpr int NORM_PARTIALS = 8;               // blocks of a backward launch per SM, at most

struct NormRows {
    void *p;
    int64_t sb, st;                                   // strides in elements: sequence, position
    int64_t hop, wrap;                                // bytes from a team's row to its next, and more where that is another sequence's
};

struct NormArgs {
    NormRows x, y, dy, dx;
    const void *weight, *bias;
    float *stats, *scales, *partial;
    int8_t *packed;
    const int32_t *lens;
    Divider by_length;
    int64_t rows, length;
    int64_t step, step_b, step_t;                     // from a team's row to its next: rows, and the same in sequences and positions
    int32_t columns, kept_blocks;                     // kept_blocks = ceil(columns / KEPT_BLOCK)
    int32_t weight_f32, vectors_wide;                 // vectors_wide: weight and bias can be read 16 bytes at a time
    float eps;
};

// A team's place among the rows, from one to the next without a division: `there`: the row exists; `live`: its position is valid
struct RowAt {
    int64_t row, b, t;
    bool there, live;

    __device__ __forceinline__ RowAt(const NormArgs &a, int64_t first) : row(first)
    {
        b = a.by_length.of(first);
        t = first - b * a.length;
        look(a);
    }
    __device__ __forceinline__ void look(const NormArgs &a)
    {
        there = row < a.rows;
        live = there && (!a.lens || t < __ldg(a.lens + b));
    }
    // true if the next row is in another sequence than the steps have it
    __device__ __forceinline__ bool next(const NormArgs &a)
    {
        row += a.step;
        b += a.step_b;
        t += a.step_t;
        const bool wrapped = t >= a.length;
        if (wrapped) {
            t -= a.length;
            ++b;
        }
        look(a);
        return wrapped;
    }
};
// A team's place in a tensor, at the column of the thread's first piece
template <typename T>
struct Line {
    char *p;
    __device__ __forceinline__ Line(const NormRows &r, const RowAt &at, int column)
        : p(reinterpret_cast<char *>(static_cast<T *>(r.p) + at.b * r.sb + at.t * r.st + column))
    {
    }
    __device__ __forceinline__ void next(const NormRows &r, bool wrapped) { p += wrapped ? r.hop + r.wrap : r.hop; }
    __device__ __forceinline__ T *at() const { return reinterpret_cast<T *>(p); }
};
// the steps of a launch whose teams are `step` rows apart
inline void set_step(NormArgs &a, int64_t step, int64_t element)
{
    a.step = step;
    a.step_b = step / a.length;
    a.step_t = step % a.length;
    for (NormRows *r : {&a.x, &a.y, &a.dy, &a.dx}) {
        r->hop = (a.step_b * r->sb + a.step_t * r->st) * element;
        r->wrap = (r->sb - a.length * r->st) * element;
    }
}

// The shape of a team.  LANES 2 to 32: part of a warp; more: the block; 0: the block, of up to 512 threads.  FAR: the rows' weights (and sums)
// do not fit the threads' registers: weights are read again for every row, sums live in shared memory.  FULL: every thread's every piece lies in
// the row.
template <int VEC_, int NV_, int LANES_, bool FULL_ = false, bool FAR_ = false>
struct Team {
    static constexpr int VEC = VEC_, NV = NV_, LANES = LANES_;
    static constexpr int V = VEC % 2 == 0 ? 2 : 1, N = VEC / V;       // a piece in fp32: N times V values
    static constexpr bool FULL = FULL_, FAR = FAR_, BLOCK = LANES_ == 0 || LANES_ > 32;
    static constexpr int GROUP = BLOCK ? 32 : LANES;                  // lanes that reduce by shuffles
    static constexpr int KEPT_LANES = GROUP < KEPT_BLOCK / VEC ? GROUP : KEPT_BLOCK / VEC;   // that hold a scale's columns,
    static constexpr int KEPT_PIECES = KEPT_BLOCK / VEC / KEPT_LANES < NV ? KEPT_BLOCK / VEC / KEPT_LANES : NV;    // and their pieces
    static constexpr int THREADS = !BLOCK ? NORM_THREADS : LANES ? LANES : 512;       // at most
    // threads of an SM that the registers have to allow, and blocks of these
    static constexpr int ON_SM = BLOCK && NV * VEC <= 8 ? 1024 : 512, RESIDENT = ON_SM / THREADS;
    static __device__ __forceinline__ int size() { return LANES ? LANES : blockDim.x; }
    static __device__ __forceinline__ int member() { return BLOCK ? threadIdx.x : threadIdx.x % LANES; }
    static __device__ __forceinline__ int teams() { return BLOCK ? 1 : NORM_THREADS / LANES; }
    static __device__ __forceinline__ int index() { return BLOCK ? 0 : threadIdx.x / LANES; }
    static __device__ __forceinline__ int column(int v) { return (v * size() + member()) * VEC; }
    static __device__ __forceinline__ bool in(int v, int columns) { return FULL || column(v) < columns; }
    // from a thread's first piece to its others, in elements
    static __device__ __forceinline__ int apart(int v) { return v * size() * VEC; }
};

// Sums over the lanes of a team that lie in one warp
template <typename S>
__device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int o = S::GROUP / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <typename S>
__device__ __forceinline__ float2 group_sum(float2 v)
{
#pragma unroll
    for (int o = S::GROUP / 2; o; o >>= 1)
        v = add_of(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
    return v;
}
// Sums over a team, two at a time.  The warps of a block leave theirs in one of two places in turn, so that one barrier a sum is enough:
// a place is written again two sums later, when every thread has met the barrier in between.
struct TeamSums {
    float2 (*place)[16];
    int turn;
};
template <typename S>
__device__ __forceinline__ float2 team_sum(float2 v, TeamSums &sums)
{
    v = group_sum<S>(v);
    if (!S::BLOCK) return v;
    float2 *place = sums.place[sums.turn];
    sums.turn ^= 1;
    if ((threadIdx.x & 31) == 0) place[threadIdx.x >> 5] = v;
    __syncthreads();
    const int w = threadIdx.x & 15;                                // at most 16 warps
    v = w < (int)blockDim.x >> 5 ? place[w] : make_float2(0.0f, 0.0f);
#pragma unroll
    for (int o = 8; o; o >>= 1)
        v = add_of(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
    return v;
}

// a piece of a row, all of which lies in the row or nothing (VEC > 1 only where columns % VEC == 0)
template <typename T, int VEC>
__device__ __forceinline__ typename Piece<T, VEC>::raw load_piece(const T *at, bool on)
{
    if (on) return *reinterpret_cast<const typename Piece<T, VEC>::raw *>(at);
    return Piece<T, VEC>::none();
}
// the same of a weight or bias, `without` where there is none
template <typename T, int VEC, typename F, int N>
__device__ __forceinline__ void vector_piece(const NormArgs &a, const void *p, int c, bool on, float without, F (&f)[N])
{
    float *one = reinterpret_cast<float *>(f);
    if (!p || !on) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) one[e] = without;
    } else if (VEC > 1 && a.vectors_wide) {
        if (!a.weight_f32) {
            if constexpr (VEC == 8) Piece<T, VEC>::get(*reinterpret_cast<const typename Piece<T, VEC>::raw *>(static_cast<const T *>(p) + c), f);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; e += 4) {
                const float4 q = *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + c + e);
                one[e] = q.x;
                if constexpr (VEC > 1) one[e + 1] = q.y, one[e + 2] = q.z, one[e + 3] = q.w;
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) one[e] = a.weight_f32 ? static_cast<const float *>(p)[c + e] : to_float(static_cast<const T *>(p)[c + e]);
    }
}

// Calls launch(Team, threads) with the team for rows of `columns` values: 16 columns a thread, as few threads as that takes up to a warp (fewer steps
// to a sum; 400000 x 128 bf16 forward by 8 threads 51 us, by 16 68), a block beyond, with 8 columns a thread up to 4096 (16384 x 4096 bf16 backward 91 us
// against 107 with 16; forward, which takes the same teams, 70 against 67, and keeping 8 bits with the backward pass from them 215 against 208, 65536 x 768 159
// against 184) and 32 beyond 8192.  Rows that 16-byte accesses do not fit go one value at a time, by blocks whose size the compiler knows (20000 x 1001
// bf16 backward 55 us, by blocks of any size 75).
template <int VEC, int PER_THREAD, int LANES, typename F>
static gs_status full_or_not(int columns, int threads, F &&launch)
{
    if (columns == PER_THREAD * (LANES ? LANES : threads)) return launch(Team<VEC, PER_THREAD / VEC, LANES, true>(), threads);
    return launch(Team<VEC, PER_THREAD / VEC, LANES, false>(), threads);
}
template <typename T, typename F>
static gs_status with_team(int columns, bool aligned, F &&launch)
{
    constexpr int W = Wide<T>::N;
    auto block = [&](int per_thread) { return (columns + 32 * per_thread - 1) / (32 * per_thread) * 32; };
    if (aligned) {
        if (columns <= 32) return full_or_not<W, 16, 2>(columns, NORM_THREADS, launch);
        if (columns <= 64) return full_or_not<W, 16, 4>(columns, NORM_THREADS, launch);
        if (columns <= 128) return full_or_not<W, 16, 8>(columns, NORM_THREADS, launch);
        if (columns <= 256) return full_or_not<W, 16, 16>(columns, NORM_THREADS, launch);
        if (columns <= 512) return full_or_not<W, 16, 32>(columns, NORM_THREADS, launch);
        if (columns <= 4096) return full_or_not<W, 8, 0>(columns, block(8), launch);
        if (columns <= 8192) return full_or_not<W, 16, 0>(columns, block(16), launch);
        return launch(Team<W, 32 / W, 0, false, true>(), block(32));
    }
    if (columns <= 32) return launch(Team<1, 2, 16>(), NORM_THREADS);
    if (columns <= 64) return launch(Team<1, 4, 16>(), NORM_THREADS);
    if (columns <= 128) return launch(Team<1, 8, 16>(), NORM_THREADS);
    if (columns <= 256) return launch(Team<1, 8, 32>(), NORM_THREADS);
    if (columns <= 512) return launch(Team<1, 16, 32>(), NORM_THREADS);
    if (columns <= 1024) return launch(Team<1, 16, 64>(), 64);
    if (columns <= 2048) return launch(Team<1, 16, 128>(), 128);
    if (columns <= 4096) return launch(Team<1, 16, 256>(), 256);
    if (columns <= 8192) return launch(Team<1, 16, 512>(), 512);
    return launch(Team<1, 32, 512, false, true>(), 512);
}

// gs_norm_forward.cu, gs_norm_backward.cu
gs_status norm_forward(const NormArgs &a, int32_t dtype, bool aligned, cudaStream_t st);
gs_status norm_backward(const NormArgs &a, int32_t dtype, bool aligned, void *dweight, void *dbias, cudaStream_t st);
// blocks that leave sums of their rows for another kernel: as many as any alignment of the tensors takes
int64_t norm_backward_partials(int64_t rows, int32_t columns, int32_t dtype);
// gs_checkpoint.cu
gs_status checkpoint_pack(int32_t dtype, const NormRows &x, const int32_t *lens, int64_t batch, int64_t length, int64_t columns,
                          int8_t *packed, float *scales, cudaStream_t st);

}  // namespace gs
