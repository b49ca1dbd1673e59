// Gated linear recurrence along the positions of a sequence, and its gradient.
//
//   a_t = sigmoid(z_t), h_t = a_t h_(t-1) + (1 - a_t) x_t;   g_t = dout_t + r_(t+1), r_t = a_t g_t,
//   dx_t = (1 - a_t) g_t, dz_t = a_t (1 - a_t) (h_(t-1) - x_t) g_t.
//
// Over a stretch of positions the state is an affine function of the state before it, h_end = P h_start + B with
// P the product of the a_t, and r_start = P r_end + R with the same P, so stretches can be computed side by side and joined.
// A warp has a stretch of up to 16 positions of 32 channels (64 of 16-bit tensors, two an instruction), a block 8 stretches one after
// another, SPAN positions; sequences no longer than that share blocks, which go from one group of them to the next.  A longer sequence is a cluster's: its blocks take neighbouring
// spans, send each other the (P, B) of theirs through distributed shared memory and go on to the next window of spans with the state that all of them
// know by then.  Where that leaves the device idle, several clusters share a sequence.  A stretch is gone through twice, for its function and for its results, from gates held
// in registers; the next one's inputs arrive in shared memory meanwhile (rows of 16 bits that are
// aligned to two bytes only come through registers, before the joins).  Every input is read once and every output written once; the joins are made in
// a fixed order.  The backward pass reads the state before each span, which the forward pass left, computes h again (one stream fewer than reading it,
// and in fp32) and joins only r.
//
// Bound: memory traffic and, for 16 bits, the time that the dozen instructions of an element and the joins take beside it.  Long sequences, 4 x 8192 x 2048
// bf16: forward 93 us (4.3 TB/s; without the joins 76, with loads and stores alone 66), backward 145 to 155 (4.3 to 4.6).  Walks of 40 x 128 bf16, 16384 of
// them: 97 to 105 us (4.6 to 4.9 TB/s), 8192 of 80 f16 backward 151 to 169 (4.7 to 5.3); fp32 walks of 100 x 256, 4096 of them, forward 211 us (6.0 TB/s), backward 353
// (6.0).  (Ranges: several devices and runs.)  Rows aligned to four bytes only: 3 x 5003 x 777 fp32 backward 117 us (3 x 5000 x 776: 69); to two: 4 x 8192 x
// 2047 bf16 254 us forward and 337 backward (2046 channels 126 and 264), 16384 walks of 40 x 127 223 and 434 (128 channels 99 and 171).
#include <math.h>

#include <type_traits>

#include "gs_layers.cuh"

namespace gs {

static constexpr int STEPS = 16, WARPS = 8, SPAN = STEPS * WARPS, MOST_BLOCKS = 8;
// Windows of a chain from which on clusters may share it: 8192 positions of 64 channels bf16 alone | shared forward 22 | 19 us, backward 29 | 20; 4096
// positions 18 | 20 and 18 | 20
static constexpr int LEAST_WINDOWS = 8;
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
    int32_t stretches;                    // warps that share a span; a block has as many chains as that leaves room for
    int32_t blocks;                       // blocks of a cluster
    int32_t parts, windows_of_part;       // clusters that share a chain, and windows that each of them has
    float *sums;                          // where there are several: what each chain's parts amount to, see scan_sums_kernel
    unsigned long long *stalls;           // where blocks whose waits ran out are counted
};

// V neighbouring channels of a lane as they travel, and in fp32
template <typename T, int V> struct Lane;
template <typename T> struct Lane<T, 1> {
    typedef T raw;
    static __device__ __forceinline__ float get(raw r) { return to_float(r); }
    static __device__ __forceinline__ raw at_most_88(raw r)
    {
        if constexpr (sizeof(T) == 4) return r;       // exp_of does it
        else return __hmin_nan(r, from_float<T>(88.0f));
    }
    static __device__ __forceinline__ raw put(float f) { return from_float<T>(f); }
    static __device__ __forceinline__ raw put_negative(float f) { return from_float<T>(-f); }
};
template <typename T> struct Lane<T, 2> {
    typedef uint32_t raw;
    static __device__ __forceinline__ float2 get(raw r)
    {
        float2 f;
        unpack2<T>(r, f.x, f.y);
        return f;
    }
    static __device__ __forceinline__ raw at_most_88(raw r)
    {
        typedef typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type two;
        const uint32_t most = pack2<T>(88.0f, 88.0f);
        const two m = __hmin2_nan(*reinterpret_cast<const two *>(&r), *reinterpret_cast<const two *>(&most));
        return *reinterpret_cast<const uint32_t *>(&m);
    }
    static __device__ __forceinline__ raw put(float2 f) { return pack2<T>(f.x, f.y); }
    static __device__ __forceinline__ raw put_negative(float2 f) { return put(f) ^ 0x80008000u; }
};

// exp(z) = 2^y, y = z log2(e).  Rounding y costs |z| 2^-24 of the result, which tensors of 16 bits do not see; fp32 tensors get the first
// term of what it left out back.  Where products follow that have no use for an infinity, z is held to 88 (Lane::at_most_88,
// in the words that it travels in); 1 / (1 + exp(88)) is zero already, as all that is below 2^-126.  NaN stays NaN.
static constexpr float LOG2_E = 1.44269504f, LOG2_E_REST = 1.92596299e-8f, LN_2 = 0.693147181f;
template <typename T> __device__ __forceinline__ float exp_of_one(float z, float y)
{
    if constexpr (sizeof(T) == 4) {
        asm("min.NaN.f32 %0, %0, 0f42B00000;\n\tmax.NaN.f32 %0, %0, 0fC2C80000;" : "+f"(z));                   // to [-100, 88]
        y = LOG2_E * z;
        const float rest = fmaf(LOG2_E, z, -y) + LOG2_E_REST * z;
        return tc::exp2_fast(y) * fmaf(LN_2, rest, 1.0f);
    }
    return tc::exp2_fast(y);
}
template <typename T> __device__ __forceinline__ float exp_of(float z) { return exp_of_one<T>(z, LOG2_E * z); }
template <typename T> __device__ __forceinline__ float2 exp_of(float2 z)
{
    const float2 y = mul_of(z, make_float2(LOG2_E, LOG2_E));
    return make_float2(exp_of_one<T>(z.x, y.x), exp_of_one<T>(z.y, y.y));
}
__device__ __forceinline__ float reciprocal(float x) { return tc::rcp_fast(x); }
__device__ __forceinline__ float2 reciprocal(float2 x) { return make_float2(tc::rcp_fast(x.x), tc::rcp_fast(x.y)); }

// -(1 - a) = 1 / (-1 - e), e = exp(z), to a few units of its own last place however small it is: from a rounded a it would have no digits
// left where a channel remembers for long.  Negative, because that is what multiply-adds take.
template <typename F>
__device__ __forceinline__ F minus_shut(F e)
{
    const F one = all_of<sizeof(F) / 4>(-1.0f);
    return reciprocal(fma_of(e, one, one));
}
// States travel negated, -h: -(a h + (1 - a) x) = (-h) + n (-h) + n x with n = -(1 - a).  (-h) + n (-h) is rounded once, so a state that is
// kept for long loses nothing to a rounded a, and one that is given up (n = -1) leaves nothing behind.
template <typename F> __device__ __forceinline__ F advance(F n, F minus_h, F x) { return fma_of(n, x, fma_of(n, minus_h, minus_h)); }

struct Place {                            // what a warp works on: positions [t0, t0 + rows) of a chain, `valid` of them valid
    int64_t b, c;                         // sequence; the warp's first channel
    int len;                              // valid positions of the sequence
    int k, t0, rows, valid;               // k: the span
    bool there, on;                       // the warp has a chain; and the lane a channel

    __device__ __forceinline__ void stretch(const ScanArgs &a, int span, int warp)
    {
        k = span;
        t0 = k * SPAN + warp * STEPS;
        rows = there ? min(max(a.length - t0, 0), STEPS) : 0;
        valid = min(rows, max(len - t0, 0));
    }
};
template <int V>
__device__ __forceinline__ Place place_of(const ScanArgs &a, int64_t chain, int lane)
{
    Place p;
    p.there = chain < a.chains;
    p.b = p.there ? a.by_slabs.of(chain) : 0;
    p.c = p.there ? (chain - p.b * a.slabs) * (32 * V) : 0;
    p.on = p.there && p.c + lane * V < a.channels;
    p.len = a.lens && p.there ? min(max(__ldg(a.lens + p.b), 0), a.length) : a.length;
    return p;
}

// A warp's stretch of one tensor in shared memory, [step][lane].  Lanes bring (and take away) CHUNK bytes each, 16 where the tensors' rows are
// aligned to that, so that a stretch is four copies of a warp; each lane computes with its own channels of every position.  Copies of 4 and 16
// bytes hold no registers while they are on their way; there are none of 2, so those are loads that the warp waits for before it goes on.  In the places of positions that are not valid stands `without`, a gate that is open (a = 1) or a zero, so that
// what is computed from them changes nothing and needs no test.
template <typename T, int V, int CHUNK>
struct Stage {
    typedef typename Lane<T, V>::raw raw;
    static constexpr int ROW = 32 * (int)sizeof(raw), ACROSS = ROW / CHUNK, AT_ONCE = 32 / ACROSS, ROUNDS = STEPS / AT_ONCE;
    static constexpr int BYTES = STEPS * ROW;
    char *room;
    int lane;

    __device__ __forceinline__ raw &operator[](int s) const { return *reinterpret_cast<raw *>(room + s * ROW + lane * sizeof(raw)); }
    // where the lane's first chunk of a stretch lies in a tensor; the others follow AT_ONCE positions apart
    static __device__ __forceinline__ char *chunk(const ScanTensor &t, const Place &p, int lane)
    {
        return static_cast<char *>(t.p) + (p.b * t.sb + (p.t0 + lane / ACROSS) * t.st + p.c) * (int64_t)sizeof(T) + lane % ACROSS * CHUNK;
    }
    static __device__ __forceinline__ bool inside(const ScanArgs &a, const Place &p, int lane)
    {
        return p.c + lane % ACROSS * (CHUNK / (int)sizeof(T)) < a.channels;
    }
    static __device__ __forceinline__ int64_t round(const ScanTensor &t) { return AT_ONCE * t.st * (int64_t)sizeof(T); }

    static __device__ __forceinline__ void copy(uint32_t to, const char *from, int on)
    {
        if constexpr (CHUNK == 4)
            asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %2, 0;\n\t@p cp.async.ca.shared.global [%0], [%1], 4;\n\t}"
                         ::"r"(to), "l"(from), "r"(on) : "memory");
        else
            asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %2, 0;\n\t@p cp.async.cg.shared.global [%0], [%1], 16;\n\t}"
                         ::"r"(to), "l"(from), "r"(on) : "memory");
    }
    __device__ __forceinline__ void fetch(const char *from, int64_t step, bool in, int valid, uint32_t without) const
    {
        char *to = room + lane * CHUNK;
        const int row = lane / ACROSS;
        if constexpr (CHUNK == 2) {
#pragma unroll
            for (int i = 0; i < ROUNDS; ++i, from += step, to += 32 * CHUNK)
                *reinterpret_cast<uint16_t *>(to) = in && i < valid ? *reinterpret_cast<const uint16_t *>(from) : (uint16_t)without;
            return;
        }
        const uint32_t at = (uint32_t)__cvta_generic_to_shared(to);
        if constexpr (CHUNK == 4) {
            if (valid == STEPS) {                    // a row a round: no test of each (3 x 5003 x 777 fp32 backward 109 -> 104 us)
                if (in)
#pragma unroll
                    for (int i = 0; i < ROUNDS; ++i, from += step) copy(at + i * 32 * CHUNK, from, true);
                return;
            }
        }
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i, from += step) copy(at + i * 32 * CHUNK, from, in && i * AT_ONCE + row < valid);
        if (valid < STEPS)
#pragma unroll
            for (int i = 0; i < ROUNDS; ++i, to += 32 * CHUNK)
                if (i * AT_ONCE + row >= valid) {
                    if constexpr (CHUNK == 4) *reinterpret_cast<uint32_t *>(to) = without;
                    else *reinterpret_cast<uint4 *>(to) = make_uint4(without, without, without, without);
                }
    }
    // positions that are not valid are written as zeros
    __device__ __forceinline__ void write(char *to, int64_t step, bool in, const Place &p) const
    {
        typedef typename std::conditional<CHUNK == 2, uint16_t, typename std::conditional<CHUNK == 4, uint32_t, uint4>::type>::type word;
        const char *from = room + lane * CHUNK;
        const int row = lane / ACROSS;
        word w[ROUNDS];
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) w[i] = *reinterpret_cast<const word *>(from + i * 32 * CHUNK);
        if (CHUNK == 4 && p.valid == STEPS) {
            if (in)
#pragma unroll
                for (int i = 0; i < ROUNDS; ++i, to += step) *reinterpret_cast<word *>(to) = w[i];
            return;
        }
        if (p.valid < STEPS) {
#pragma unroll
            for (int i = 0; i < ROUNDS; ++i)
                if (i * AT_ONCE + row >= p.valid) w[i] = word{};
        }
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i, to += step)
            if (in && i * AT_ONCE + row < p.rows) *reinterpret_cast<word *>(to) = w[i];
    }
};
// a value as the words that its tensor holds
template <typename T> __device__ __forceinline__ uint32_t words_of(float x)
{
    if constexpr (sizeof(T) == 4) return __float_as_uint(x);
    else return pack2<T>(x, x);
}
__device__ __forceinline__ void fetches_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// all but the latest LATER groups of the warp's fetches have come
template <int LATER>
__device__ __forceinline__ void fetches_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(LATER) : "memory");
    __syncwarp();
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// A lane's share of the affine function of a stretch, x -> p x + b
template <int V> struct alignas(8 * V) Affine {
    typedef typename Vec<V>::type F;
    F p, b;
    __device__ __forceinline__ void before(const Affine &next)          // this one, then `next`
    {
        b = fma_of(next.p, b, next.b);
        p = mul_of(next.p, p);
    }
    __device__ __forceinline__ F of(F x) const { return fma_of(p, x, b); }
};
__device__ __forceinline__ uint32_t in_block(uint32_t address, uint32_t rank)
{
    uint32_t there;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(address), "r"(rank));
    return there;
}
// stores into the shared memory of another block of the cluster, at the place that `to` is in this one, and counts the bytes on that block's
// barrier `bar`
template <int V>
__device__ __forceinline__ void store_remote(uint32_t to, uint32_t bar, uint32_t rank, const Affine<V> &f)
{
    if constexpr (V == 2)
        asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                     ::"r"(in_block(to, rank)), "f"(f.p.x), "f"(f.p.y), "f"(f.b.x), "f"(f.b.y), "r"(in_block(bar, rank)) : "memory");
    else
        asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];"
                     ::"r"(in_block(to, rank)), "f"(f.p), "f"(f.b), "r"(in_block(bar, rank)) : "memory");
}

// The functions of a window's stretches, and of a cluster's spans, where the warps that need them find them.  BACK: the chain runs
// from the last stretch to the first, and beside it h from the first to the last (with the same p, and `ahead` for its b).
//
// A cluster's blocks send each other their spans' functions, which a barrier of the receiver counts in (`come`), without waiting for one another: the
// places of a window are written again two windows later, and who sends then has the functions of the window between from all blocks, which
// these sent when all of their warps had read the window before.  Places of the stretches are written again when the block's warps have counted their
// reads on `read` (clusters), or in turn (blocks, whose warps meet at a barrier in every window).
template <int V, bool CLUSTER, bool BACK>
struct Board {
    static constexpr int TURNS = CLUSTER ? 1 : 2;
    Affine<V> stretch[TURNS][WARPS][32];
    typename Vec<V>::type ahead[BACK ? TURNS : 1][BACK ? WARPS : 1][32];
    Affine<V> span[CLUSTER ? 2 : 1][CLUSTER ? MOST_BLOCKS : 1][32];
    unsigned long long come[2], read;
    int stalled;
};
template <int V, bool CLUSTER, bool BACK>
struct Joins {
    typedef typename Vec<V>::type F;
    Board<V, CLUSTER, BACK> &board;
    int stretches, blocks, rank, warp, lane, first;  // first: index of the block's warp that has this chain's first stretch
    int window;                                      // counted from the first that is worked on
    Affine<V> ahead;                                 // of what lies between the block's edge and this warp's stretch

    static __device__ __forceinline__ uint32_t address(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
    // before any other use, by all threads of the cluster
    __device__ __forceinline__ void open()
    {
        if (!CLUSTER) return;
        if (threadIdx.x == 0) {
            board.stalled = 0;
            tc::bar_init(address(&board.come[0]), 1);
            tc::bar_init(address(&board.come[1]), 1);
            tc::bar_init(address(&board.read), WARPS);
            tc::fence_barrier_init();
        }
        __syncwarp();
        cluster_arrive();
    }
    // no block leaves while another may still send to it, whatever became of the waits
    __device__ __forceinline__ void close(unsigned long long *stalls)
    {
        if (!CLUSTER) return;
        __syncwarp();
        cluster_arrive();
        cluster_wait();
        if (threadIdx.x == 0 && stalls && *(volatile int *)&board.stalled) atomicAdd_system(stalls, 1ull);
    }

    // Gives away the function of this warp's stretch and hb, the b of h over it; h moves from the state before the block's first stretch to
    // that before this one.
    __device__ __forceinline__ void give(const Affine<V> &own, F hb, F &h)
    {
        const int place = CLUSTER ? 0 : window & 1;
        if (CLUSTER && window > 0) tc::bar_wait(address(&board.read), (window - 1) & 1, &board.stalled);
        board.stretch[place][first + warp][lane] = own;
        if (BACK) board.ahead[BACK ? place : 0][BACK ? first + warp : 0][lane] = hb;
        __syncthreads();
        if (BACK)
#pragma unroll 1
            for (int i = 0; i < warp; ++i)
                h = fma_of(board.stretch[place][first + i][lane].p, h, board.ahead[BACK ? place : 0][BACK ? first + i : 0][lane]);
        ahead.p = all_of<V>(1.0f);
        ahead.b = all_of<V>(0.0f);
        const int count = BACK ? stretches - 1 - warp : warp, edge = BACK ? first + stretches - 1 : first;
        // one turn after another: all at once, 7 of them with a test each, take as long where most are due (4 x 8192 x 2048 bf16 forward 91 | 92 us, backward
        // 146 | 144) and longer where few are (walks of 40 101 | 97)
#pragma unroll 1
        for (int i = 0; i < count; ++i) ahead.before(board.stretch[place][BACK ? edge - i : edge + i][lane]);
        if (!CLUSTER) return;
        __syncwarp();
        if (lane == 0) tc::bar_arrive(address(&board.read));
        const uint32_t bar = address(&board.come[window & 1]);
        if (count == WARPS - 1) {                    // this stretch ends the block's span
            if (lane == 0) tc::bar_expect(bar, blocks * (int)sizeof(board.span[0][0]));
            Affine<V> all = ahead;
            all.before(own);
            for (int r = 0; r < blocks; ++r) store_remote(address(&board.span[window & 1][rank][lane]), bar, r, all);
        }
    }
    // carry: the state (or r) at the window's edge, moved over the window; returns that at this stretch's
    __device__ __forceinline__ F take(F &carry)
    {
        F into = carry;
        if (CLUSTER) {
            const int place = window & 1;
            tc::bar_wait(address(&board.come[place]), (window >> 1) & 1, &board.stalled);
#pragma unroll 1
            for (int i = 0; i < blocks; ++i) {
                const int k = BACK ? blocks - 1 - i : i;
                const Affine<V> f = board.span[CLUSTER ? place : 0][CLUSTER ? k : 0][lane];
                if (BACK ? k > rank : k < rank) into = f.of(into);
                carry = f.of(carry);
            }
        }
        ++window;
        return ahead.of(into);
    }
};

template <int V>
__device__ __forceinline__ typename Vec<V>::type load_state(const float *from, int64_t row, int64_t channels, const Place &p, int lane)
{
    if (!from || !p.on) return all_of<V>(0.0f);
    from += row * channels + p.c + lane * V;
    if constexpr (V == 1) return from[0];
    else return make_float2(from[0], from[1]);
}
template <int V>
__device__ __forceinline__ void store_state(float *to, int64_t row, int64_t channels, const Place &p, int lane, typename Vec<V>::type h)
{
    if (!to || !p.on) return;
    to += row * channels + p.c + lane * V;
    if constexpr (V == 1) to[0] = h;
    else {
        to[0] = h.x;
        to[1] = h.y;
    }
}

// What both directions need to know about their warp
template <bool CLUSTER>
struct Seat {
    int lane, index, group, warp, rank, groups;
    __device__ __forceinline__ explicit Seat(const ScanArgs &a)
    {
        lane = threadIdx.x & 31;
        index = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
        group = CLUSTER ? 0 : index / a.stretches;
        warp = CLUSTER ? index : index - group * a.stretches;
        rank = CLUSTER ? (int)cluster_rank() : 0;
        groups = CLUSTER ? 1 : (blockDim.x >> 5) / a.stretches;
    }
};

// A warp's items one after another: a cluster's windows of its chain (BACK: the last first), or the groups of chains that a block of short chains has.
// All warps of a block have the same number of them.
template <typename T, int V, int CHUNK, bool CLUSTER, bool BACK>
struct Items {
    typedef Stage<T, V, CHUNK> S;
    const ScanArgs &a;
    const Seat<CLUSTER> &seat;
    Place place;
    bool in;                                         // the lane's chunks lie in the tensors
    int64_t chain;
    int part, window, first, last;                   // windows: the present one, and the part's

    __device__ __forceinline__ Items(const ScanArgs &args, const Seat<CLUSTER> &s) : a(args), seat(s)
    {
        part = first = last = 0;
        if (CLUSTER) {
            chain = blockIdx.x / a.blocks;
            if (a.parts > 1) {
                const int64_t whole = chain / a.parts;
                part = (int)(chain - whole * a.parts);
                chain = whole;
            }
            const int windows = (a.spans + a.blocks - 1) / a.blocks;
            first = part * a.windows_of_part;
            last = min(first + a.windows_of_part, windows) - 1;
        } else {
            chain = (int64_t)blockIdx.x * seat.groups + seat.group;
        }
        window = CLUSTER && BACK ? last : first;
        settle();
    }
    __device__ __forceinline__ void settle()
    {
        place = place_of<V>(a, chain, seat.lane);
        in = S::inside(a, place, seat.lane);
        place.stretch(a, CLUSTER ? window * a.blocks + seat.rank : 0, seat.warp);
    }
    __device__ __forceinline__ bool next()
    {
        if (CLUSTER) {
            window += BACK ? -1 : 1;
            if (BACK ? window < first : window > last) return false;
            place.stretch(a, window * a.blocks + seat.rank, seat.warp);
        } else {
            chain += (int64_t)gridDim.x * seat.groups;
            if (chain - seat.group >= a.chains) return false;
            settle();
        }
        return true;
    }
    // of a line that was at the item before
    __device__ __forceinline__ void follow(char *&line, const ScanTensor &t) const
    {
        if (CLUSTER) line += (BACK ? -1 : 1) * (int64_t)a.blocks * SPAN * t.st * (int64_t)sizeof(T);
        else line = S::chunk(t, place, seat.lane);
    }
};

// Few chains, long ones: several clusters share a chain, each with a part of its windows, and a kernel ahead of theirs sums the parts up: a block for every `windows_of_part` spans, with as
// many stretches one after another in each of its warps, leaves the function of its positions.  Entry 0 of a chain is its state before everything (a
// function that takes no notice of what comes before), which the clusters read here and not from h0: one of them may have written the final state there.
// BACK: of r, and entry 0 is what comes from behind the end.
template <typename T, int V, bool BACK>
__global__ void __launch_bounds__(32 * WARPS) scan_sums_kernel(const __grid_constant__ ScanArgs a)
{
    typedef Lane<T, V> L;
    typedef typename Vec<V>::type F;
    __shared__ Affine<V> stretch[WARPS][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, each = a.parts * a.blocks;
    const int64_t chain = blockIdx.x / each;
    const int entry = (int)(blockIdx.x - chain * each);
    Place p = place_of<V>(a, chain, lane);
    Affine<V> own = {all_of<V>(1.0f), all_of<V>(0.0f)};
    const ScanTensor &other = BACK ? a.dout : a.x;
    for (int j = 0; j < a.windows_of_part; ++j) {
        // this warp's positions follow one another, so that the order of the sums is the order of the positions
        const int64_t t0 = ((int64_t)entry * WARPS + warp) * a.windows_of_part * STEPS + j * STEPS;
        const int valid = (int)min((int64_t)STEPS, max((int64_t)p.len - t0, (int64_t)0));
        if (valid == 0) break;
        const int64_t at = p.c + (p.on ? lane * V : 0);
        const char *gate = static_cast<const char *>(a.gate.p) + (p.b * a.gate.sb + t0 * a.gate.st + at) * (int64_t)sizeof(T);
        const char *from = static_cast<const char *>(other.p) + (p.b * other.sb + t0 * other.st + at) * (int64_t)sizeof(T);
        typename L::raw z[STEPS], x[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
            if (s < valid) {
                z[s] = *reinterpret_cast<const typename L::raw *>(gate + s * a.gate.st * (int64_t)sizeof(T));
                x[s] = other.p ? *reinterpret_cast<const typename L::raw *>(from + s * other.st * (int64_t)sizeof(T)) : L::put(all_of<V>(0.0f));
            }
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
            if (s < valid) {
                const F n = minus_shut(exp_of<T>(L::get(z[s])));
                if (!BACK) own.b = advance(n, own.b, L::get(x[s]));
                own.p = fma_of(n, own.p, own.p);
                if (BACK) own.b = fma_of(own.p, L::get(x[s]), own.b);
            }
    }
    stretch[warp][lane] = own;
    __syncthreads();
    if (warp) return;
    Affine<V> all = stretch[BACK ? WARPS - 1 : 0][lane];
    for (int i = 1; i < WARPS; ++i) all.before(stretch[BACK ? WARPS - 1 - i : i][lane]);
    Affine<V> *to = reinterpret_cast<Affine<V> *>(a.sums) + chain * (each + 1) * 32 + lane;
    to[(BACK ? each - entry : 1 + entry) * 32] = all;
    if (entry == 0) {
        const F h = load_state<V>(BACK ? a.dfinal : a.h0, p.b, a.channels, p, lane);
        to[0] = {all_of<V>(0.0f), BACK ? h : mul_of(h, all_of<V>(-1.0f))};
    }
}
// the state before a part (BACK: r behind it), from the sums of those before
template <int V, bool BACK>
__device__ __forceinline__ typename Vec<V>::type part_start(const ScanArgs &a, int64_t chain, int part, int lane)
{
    const int each = a.parts * a.blocks, entries = 1 + (BACK ? a.parts - 1 - part : part) * a.blocks;
    const Affine<V> *from = reinterpret_cast<const Affine<V> *>(a.sums) + chain * (each + 1) * 32 + lane;
    typename Vec<V>::type carry = all_of<V>(0.0f);
#pragma unroll 8
    for (int i = 0; i < entries; ++i) carry = from[(int64_t)i * 32].of(carry);
    return carry;
}

template <typename T, int V, int CHUNK, bool CLUSTER>
__global__ void __launch_bounds__(32 * WARPS, FORWARD_BLOCKS) scan_forward_kernel(const __grid_constant__ ScanArgs a)
{
    typedef Stage<T, V, CHUNK> S;
    typedef Lane<T, V> L;
    typedef typename Vec<V>::type F;
    __shared__ Board<V, CLUSTER, false> board;
    extern __shared__ uint4 room[];                                  // [warp][gate, x, the next x]
    const Seat<CLUSTER> seat(a);
    Joins<V, CLUSTER, false> joins = {board, a.stretches, a.blocks, seat.rank, seat.warp, seat.lane, seat.group * a.stretches, 0};
    // Where the final state takes the place of the first (d_final = d_h0) the first is read before the cluster's barrier: the last block writes
    // once it has the functions of the others, which would not by itself tell it that their reads are done.  Elsewhere the barrier's
    // latency passes behind the first copies (64 x 512 x 1024 bf16 43.7 us, after them 46.5; 64 x 129 x 1024 23.1 | 24.7).
    const bool in_place = a.h0 && a.h0 == a.final_state;
    if (!in_place) joins.open();

    Items<T, V, CHUNK, CLUSTER, false> item(a, seat);
    char *const stages = reinterpret_cast<char *>(room) + seat.index * 3 * S::BYTES;
    const S z = {stages, seat.lane};
    S x = {stages + S::BYTES, seat.lane}, spare = {stages + 2 * S::BYTES, seat.lane};
    char *line_z = S::chunk(a.gate, item.place, seat.lane), *line_x = S::chunk(a.x, item.place, seat.lane),
         *line_out = S::chunk(a.out, item.place, seat.lane);
    z.fetch(line_z, S::round(a.gate), item.in, item.place.valid, words_of<T>(INFINITY));
    x.fetch(line_x, S::round(a.x), item.in, item.place.valid, 0u);
    fetches_end();

    const F minus = all_of<V>(-1.0f);
    F next_h = load_state<V>(CLUSTER && a.parts > 1 ? nullptr : a.h0, item.place.b, a.channels, item.place, seat.lane);
    if (in_place) joins.open();
    F carry = mul_of(next_h, minus);
    if (CLUSTER && a.parts > 1) carry = part_start<V, false>(a, item.chain, item.part, seat.lane);
    if (CLUSTER) cluster_wait();
    bool more;
    do {
        const Place p = item.place;
        const bool in = item.in;
        if (!CLUSTER) carry = mul_of(next_h, minus);                 // negated, as all states are
        fetches_wait<0>();
        F n[STEPS];
        Affine<V> own = {all_of<V>(1.0f), all_of<V>(0.0f)};
        if (p.valid > 0) {                                           // else nothing happens in this stretch
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                n[s] = minus_shut(exp_of<T>(L::get(z[s])));
                own.b = advance(n[s], own.b, L::get(x[s]));
                own.p = fma_of(n[s], own.p, own.p);
            }
        }
        // the gates' stage is free again, and the results will take the place of x
        more = item.next();
        __syncwarp();
        if (more) {
            item.follow(line_z, a.gate);
            item.follow(line_x, a.x);
            z.fetch(line_z, S::round(a.gate), item.in, item.place.valid, words_of<T>(INFINITY));
            spare.fetch(line_x, S::round(a.x), item.in, item.place.valid, 0u);
            if (!CLUSTER) next_h = load_state<V>(a.h0, item.place.b, a.channels, item.place, seat.lane);
        }
        fetches_end();
        F into = carry;
        if (CLUSTER || a.stretches > 1) {
            joins.give(own, own.b, own.b);
            into = joins.take(carry);
        }
        if (p.valid > 0) {
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                into = advance(n[s], into, L::get(x[s]));
                x[s] = L::put_negative(into);
            }
        }
        __syncwarp();
        x.write(line_out, S::round(a.out), in, p);
        if (seat.warp == a.stretches - 1) {
            if (p.k < a.spans - 1) store_state<V>(a.states, p.b * (a.spans - 1) + p.k, a.channels, p, seat.lane, mul_of(into, minus));
            else if (p.k == a.spans - 1) store_state<V>(a.final_state, p.b, a.channels, p, seat.lane, mul_of(into, minus));
        }
        item.follow(line_out, a.out);
        const S was = x;
        x = spare;
        spare = was;
    } while (more);
    joins.close(a.stalls);
}

template <typename T, int V, int CHUNK, bool CLUSTER>
__global__ void __launch_bounds__(32 * WARPS, BACKWARD_BLOCKS) scan_backward_kernel(const __grid_constant__ ScanArgs a)
{
    typedef Stage<T, V, CHUNK> S;
    typedef Lane<T, V> L;
    typedef typename Vec<V>::type F;
    __shared__ Board<V, CLUSTER, true> board;
    extern __shared__ uint4 room[];                                  // [warp][2 in turn][gate, x, dout]
    const Seat<CLUSTER> seat(a);
    Joins<V, CLUSTER, true> joins = {board, a.stretches, a.blocks, seat.rank, seat.warp, seat.lane, seat.group * a.stretches, 0};
    joins.open();

    Items<T, V, CHUNK, CLUSTER, true> item(a, seat);
    char *const stages = reinterpret_cast<char *>(room) + seat.index * 6 * S::BYTES;
    char *line_z = S::chunk(a.gate, item.place, seat.lane), *line_x = S::chunk(a.x, item.place, seat.lane),
         *line_g = S::chunk(a.dout, item.place, seat.lane), *line_dx = S::chunk(a.dx, item.place, seat.lane),
         *line_dz = S::chunk(a.dgate, item.place, seat.lane);
    auto fetch = [&](int turn) {
        char *const to = stages + turn * 3 * S::BYTES;
        S{to, seat.lane}.fetch(line_z, S::round(a.gate), item.in, item.place.valid, words_of<T>(INFINITY));
        S{to + S::BYTES, seat.lane}.fetch(line_x, S::round(a.x), item.in, item.place.valid, 0u);
        S{to + 2 * S::BYTES, seat.lane}.fetch(line_g, S::round(a.dout), item.in, a.dout.p ? item.place.valid : 0, 0u);
    };
    fetch(0);
    fetches_end();

    // the state before the item's span, and r behind its end: asked for with the inputs
    auto state_before = [&](const Place &p) {
        if (p.k == 0) return load_state<V>(a.h0, p.b, a.channels, p, seat.lane);
        return load_state<V>(p.k < a.spans ? a.states : nullptr, p.b * (a.spans - 1) + p.k - 1, a.channels, p, seat.lane);
    };
    F next_h = state_before(item.place), carry = load_state<V>(a.dfinal, item.place.b, a.channels, item.place, seat.lane), next_carry = carry;
    if (CLUSTER && a.parts > 1) carry = part_start<V, true>(a, item.chain, item.part, seat.lane);
    if (CLUSTER) cluster_wait();
    bool more;
    int turn = 0;
    do {
        const Place p = item.place;
        const bool in = item.in;
        F h = mul_of(next_h, all_of<V>(-1.0f));                      // negated, as all states are
        if (!CLUSTER) carry = next_carry;
        more = item.next();
        if (more) {
            item.follow(line_z, a.gate);
            item.follow(line_x, a.x);
            item.follow(line_g, a.dout);
            fetch(turn ^ 1);
            next_h = state_before(item.place);
            if (!CLUSTER) next_carry = load_state<V>(a.dfinal, item.place.b, a.channels, item.place, seat.lane);
        }
        fetches_end();
        fetches_wait<1>();
        char *const at = stages + turn * 3 * S::BYTES;
        const S z = {at, seat.lane}, x = {at + S::BYTES, seat.lane}, g = {at + 2 * S::BYTES, seat.lane};
        turn ^= 1;
        F n[STEPS], d[STEPS], hb = all_of<V>(0.0f);                  // d: -a (1 - a), then that times x_t - h_(t-1)
        Affine<V> own = {all_of<V>(1.0f), all_of<V>(0.0f)};
        if (p.valid > 0) {                                           // else nothing happens in this stretch
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const F e = exp_of<T>(L::get(L::at_most_88(z[s])));
                n[s] = minus_shut(e);
                d[s] = mul_of(mul_of(e, n[s]), n[s]);                // -a times -(1 - a)
                hb = advance(n[s], hb, L::get(x[s]));
                own.p = fma_of(n[s], own.p, own.p);
                own.b = fma_of(own.p, L::get(g[s]), own.b);
            }
        }
        const bool joined = CLUSTER || a.stretches > 1;
        if (joined) joins.give(own, hb, h);
        if (p.valid > 0) {
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const F xf = L::get(x[s]);
                d[s] = mul_of(d[s], add_of(h, xf));                  // a (1 - a) (x_t - h_(t-1))
                h = advance(n[s], h, xf);
            }
        }
        F into = joined ? joins.take(carry) : carry;
        if (p.valid > 0) {
#pragma unroll
            for (int s = STEPS - 1; s >= 0; --s) {
                const F full = add_of(L::get(g[s]), into);
                x[s] = L::put_negative(mul_of(n[s], full));
                into = fma_of(n[s], full, full);
                z[s] = L::put_negative(mul_of(d[s], full));
            }
        }
        __syncwarp();
        x.write(line_dx, S::round(a.dx), in, p);
        z.write(line_dz, S::round(a.dgate), in, p);
        item.follow(line_dx, a.dx);
        item.follow(line_dz, a.dgate);
        if (p.k == 0 && seat.warp == 0) store_state<V>(a.dh0, p.b, a.channels, p, seat.lane, into);
        __syncwarp();                                                // before the stage is filled again
    } while (more);
    joins.close(a.stalls);
}

template <typename T, int V, int CHUNK>
static gs_status launch(const ScanArgs &args, bool backward, cudaStream_t st)
{
    ScanArgs a = args;
    a.slabs = (int32_t)((a.channels + 32 * V - 1) / (32 * V));
    a.by_slabs = Divider(a.slabs);
    a.chains = a.batch * a.slabs;
    a.spans = (a.length + SPAN - 1) / SPAN;
    const bool cluster = a.spans > 1;
    static SharedRecord records[4];
    auto kernel = backward ? cluster ? scan_backward_kernel<T, V, CHUNK, true> : scan_backward_kernel<T, V, CHUNK, false>
                           : cluster ? scan_forward_kernel<T, V, CHUNK, true> : scan_forward_kernel<T, V, CHUNK, false>;
    SharedRecord &record = records[2 * backward + cluster];
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr = {};
    // a block's warps, and how many such blocks the device holds at once by registers and shared memory
    a.stretches = a.length >= SPAN ? WARPS : a.length > STEPS ? (a.length + STEPS - 1) / STEPS : 1;
    const int groups = WARPS / a.stretches, warps = groups * a.stretches;
    const size_t shared = (size_t)(backward ? 6 : 3) * warps * Stage<T, V, CHUNK>::BYTES;
    const size_t board = backward ? cluster ? sizeof(Board<V, true, true>) : sizeof(Board<V, false, true>)
                                  : cluster ? sizeof(Board<V, true, false>) : sizeof(Board<V, false, false>);
    const int by_registers = (backward ? BACKWARD_BLOCKS : FORWARD_BLOCKS) * WARPS / warps, by_shared = (int)((size_t)228 * 1024 / (shared + board + 1024));
    const int64_t slots = (int64_t)sm_count() * (by_registers < by_shared ? by_registers : by_shared);
    cfg.blockDim = dim3(32 * warps);
    int64_t grid;
    if (cluster) {
        a.stalls = stall_counter();
        gs_status s = stalled_before();
        if (s != GS_OK) return s;
        // Clusters as small as fill the device: their blocks wait for one another in every window.  Measured with 1, 2, 4, 8 blocks:
        // 4 x 8192 x 2048 bf16 forward (rule: 4) 127, 91, 93, 100 us, backward (4) 179, 139, 144, 160; 3 x 5003 x 777 fp32 backward (4)
        // 164, 109, 117, 109.  Counts between (3, 7) lay between these or above.
        a.blocks = 1;
        while (a.blocks < MOST_BLOCKS && a.blocks < a.spans && a.chains * a.blocks < slots) a.blocks *= 2;
        // Parts of a chain, where its clusters alone leave most of the device idle: each part's windows come one after another, the parts'
        // side by side, for a second reading of two inputs.  Alone | shared, bf16: 32768 x 64 forward 74 | 29 us, backward 99 | 29; 200000 x 64
        // 427 | 77 and 582 | 64; 32768 x 512 74 | 64 (6 parts) and 101 | 72 (4); 32768 x 1024 97 | 108 (3) and 146 | 127 (2); fp32 2 x 16384 x
        // 256 41 | 56 (3) and 64 | 62 (2)
        const int windows = (a.spans + a.blocks - 1) / a.blocks;
        a.parts = 1;
        a.windows_of_part = windows;
        const int64_t most = slots / (a.chains * a.blocks);
        if (a.sums && a.blocks == MOST_BLOCKS && windows >= LEAST_WINDOWS && most >= (backward ? 2 : 4)) {
            a.windows_of_part = (int)((windows + most - 1) / most);
            a.parts = (windows + a.windows_of_part - 1) / a.windows_of_part;
        }
        grid = a.chains * a.parts * a.blocks;
        if (a.parts > 1) {
            if (backward) scan_sums_kernel<T, V, true><<<(unsigned)grid, 32 * WARPS, 0, st>>>(a);
            else scan_sums_kernel<T, V, false><<<(unsigned)grid, 32 * WARPS, 0, st>>>(a);
            GS_CUDA_TRY(cudaGetLastError());
        }
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = (unsigned)a.blocks;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
    } else {
        a.blocks = 1;
        grid = (a.chains + groups - 1) / groups;
        if (grid > slots) grid = slots;
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
    const int64_t es = (int64_t)size_of(dtype);
    if ((uintptr_t)a.sums % 16) return bad("d_work must be aligned to 16 bytes");
    for (const void *p : {(const void *)a.h0, (const void *)a.dfinal, (const void *)a.final_state, (const void *)a.dh0, (const void *)a.states})
        if ((uintptr_t)p % 4) return bad("a state is not aligned to its element size");
    bool pairs = es == 2 && a.channels % 2 == 0, wide = a.channels * es % 16 == 0;
    for (int i = 0; i < n; ++i) {
        if (!t[i]->p) return bad("null pointer");
        if ((uintptr_t)t[i]->p % es) return bad("tensor not aligned to its element size");
        if (i < outputs && ((a.batch > 1 && t[i]->sb == 0) || (a.length > 1 && t[i]->st == 0)))
            return bad("an output has a zero stride");
        pairs = pairs && (uintptr_t)t[i]->p % 4 == 0 && (t[i]->sb | t[i]->st) % 2 == 0;
        wide = wide && (uintptr_t)t[i]->p % 16 == 0 && (t[i]->sb * es | t[i]->st * es) % 16 == 0;
    }
    pairs = pairs && a.channels > 32;                   // one channel a lane where two would leave half the lanes idle
    return with_type(dtype, [&](auto type) {
        typedef decltype(type) T;
        if constexpr (sizeof(T) == 4) return wide ? launch<T, 1, 16>(a, backward, st) : launch<T, 1, 4>(a, backward, st);
        else {
            if (pairs) return wide ? launch<T, 2, 16>(a, backward, st) : launch<T, 2, 4>(a, backward, st);
            return wide ? launch<T, 1, 16>(a, backward, st) : launch<T, 1, 2>(a, backward, st);
        }
    });
}

}  // namespace gs

using namespace gs;

extern "C" {

int64_t gs_recurrence_work(const gs_recurrence_config *cfg)
{
    ScanArgs a;
    if (check(cfg, &a) != GS_OK) return -1;
    if (a.length <= (LEAST_WINDOWS - 1) * MOST_BLOCKS * SPAN) return 0;
    // a block's function for each of the blocks that the device holds at once, and one more a chain, of which there are fewer: 64 channels of two numbers
    return (int64_t)sm_count() * FORWARD_BLOCKS * 2 * 64 * 2;
}

int64_t gs_recurrence_states(const gs_recurrence_config *cfg)
{
    ScanArgs a;
    if (check(cfg, &a) != GS_OK) return -1;
    return a.length > 0 ? a.batch * a.channels * ((a.length - 1) / SPAN) : 0;
}

gs_status gs_recurrence_forward(const gs_recurrence_config *cfg, const void *d_gate, const void *d_x, const float *d_h0,
                                void *d_out, float *d_final, float *d_states, float *d_work, void *stream)
{
    ScanArgs a;
    gs_status s = check(cfg, &a);
    if (s != GS_OK || a.batch == 0) return s;
    a.h0 = d_h0;
    a.final_state = d_final;
    a.states = d_states;
    a.sums = d_work;
    if (a.length == 0) return copy_states(d_h0, d_final, a.batch * a.channels, (cudaStream_t)stream);
    a.gate = tensor(d_gate, cfg->gate_stride);
    a.x = tensor(d_x, cfg->x_stride);
    a.out = tensor(d_out, cfg->out_stride);
    const ScanTensor *all[3] = {&a.out, &a.gate, &a.x};
    return run(a, cfg->dtype, all, 3, 1, false, (cudaStream_t)stream);
}

gs_status gs_recurrence_backward(const gs_recurrence_config *cfg, const void *d_dout, const float *d_dfinal,
                                 const void *d_gate, const void *d_x, const float *d_h0, const float *d_states,
                                 void *d_dgate, void *d_dx, float *d_dh0, float *d_work, void *stream)
{
    ScanArgs a;
    gs_status s = check(cfg, &a);
    if (s != GS_OK || a.batch == 0) return s;
    a.h0 = d_h0;
    a.dfinal = d_dfinal;
    a.dh0 = d_dh0;
    a.sums = d_work;
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
