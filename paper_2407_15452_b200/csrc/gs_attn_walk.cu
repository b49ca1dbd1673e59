// Attention of short sequences (up to 128 positions): walks.
//
// A walk's scores are a few 16 x 16 blocks, far less than a 128 x 128 tensor-core tile, and there are
// tens of thousands of walks: the bound is the traffic of q, k, v and the results.  So a unit - one head of one
// sequence - is brought to shared memory once, whole, and everything happens there and in registers:
// one warp per 16 rows, mma.sync on 16 x 16 blocks (fp32 as three tf32 products), and only blocks that the window
// reaches.
// The grid is as large as fits the device; a block goes through its share of the units, several at a time, and
// TMA brings the next ones into a second set of tiles meanwhile.  Results leave through TMA too, from the
// tiles whose rows they replace.  Tensors that TMA cannot address (odd strides or addresses) are copied by
// the threads, and results stored by them.
//  forward : scores of up to 48 keys at a time in registers, running maximum and sum over those
//  backward: dq by query rows, then dk and dv by key rows, both from the same copy in shared memory.  delta =
//            sum_j p_ij dp_ij comes from the probabilities themselves (a first walk over the row's blocks), so
//            the forward output is neither read nor is its rounding part of the gradient (but in rows done again).
// Rows past a sequence's end are zeros in shared memory, whatever the tensors hold there.
// The window enters as the value that the scores' accumulators start from, 0 or -infinity: what a 16 x 16 block
// shows depends on its distance from the diagonal only, and the few distances with a partly visible block
// have their starting values in shared memory (a comparison and a select per score were a third of the
// instructions, and instructions are what these kernels run out of first).
// P and dS are rounded to 16-bit tensors' type for their products.  For binary16 they are scaled by powers
// of two first, P by 2^14 (p <= 1), dS by the one that brings its bound |dS| <= max|dp| + |delta| below 2^15.
#include <type_traits>

#include "gs_attn_again.cuh"
#include "gs_attn_tc.cuh"

namespace gs {

using namespace tc;

static constexpr int KEEP = 3;                    // blocks of 16 keys whose scores the forward pass holds

enum Kind { F16, BF16, F32 };
template <int K> struct TypeOf { using T = float; };
template <> struct TypeOf<F16> { using T = __half; };
template <> struct TypeOf<BF16> { using T = __nv_bfloat16; };

// A tile holds the padded rows of one head as TMA writes them: rows of DP values, in pieces of at most 128 bytes a
// row (one after the other), whose 16-byte chunks are permuted within 8 rows, so that eight rows at one
// column fall into different banks.
template <int K, int DP>
struct Row {
    static constexpr int SIZE = K == F32 ? 4 : 2, PIECES = DP * SIZE > 128 ? DP * SIZE / 128 : 1;
    static constexpr int VALUES = DP / PIECES, BYTES = VALUES * SIZE, CHUNKS = BYTES / 16;
    static constexpr int FLIP = CHUNKS == 8 ? 0 : CHUNKS == 4 ? 1 : 2;         // row bits below the permutation
    static constexpr uint32_t BLOCK = 16 * BYTES;                             // 16 rows of a piece
    static constexpr int WORDS = K == F32 ? 4 : 2;                            // of a thread's four values in the tensors' type
    // byte offset of chunk c of row r within a piece
    static __device__ __forceinline__ uint32_t at(int r, int c) { return r * BYTES + ((c ^ ((r >> FLIP) & (CHUNKS - 1))) << 4); }
    static __host__ __device__ constexpr uint32_t tile(int rows16) { return PIECES * rows16 * BLOCK; }
};
// lse, delta and bound of the padded query rows
__host__ __device__ constexpr uint32_t stat_bytes(int qt) { return 3 * qt * 16 * 4; }

__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ float lds(uint32_t addr)
{
    float x;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(addr) : "memory");
    return x;
}
template <int K>
__device__ __forceinline__ void mma(float *c, const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (K == BF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else if constexpr (K == F16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void mma3(float *c, const uint32_t (&ah)[4], const uint32_t (&al)[4], float y0, float y1)
{
    uint32_t h0, l0, h1, l1;
    split(y0, h0, l0);
    split(y1, h1, l1);
    mma<F32>(c, al, h0, h1);
    mma<F32>(c, ah, l0, l1);
    mma<F32>(c, ah, h0, h1);
}

// A lane's offset in a block of 16 rows.  The permutation of a row's chunks depends on the row within its 16 rows
// only, and a later step of the columns is the first one with bits of its chunk flipped: a lane adds its offset to a
// block's address once and flips from there.
//  rows: as the A operand; dot: as the B operand of a product over columns; mul: of one over rows
// 16-bit values come by ldmatrix, fp32 values one by one: lane (g, t) = (lane / 4, lane % 4) holds rows g and
// g + 8, columns t and t + 4 of a step of eight, or for mul rows 2t and 2t + 1 - the order in which a thread holds
// its scores, so that they serve as A operand as they are - of column g.
template <int K, int DP> __device__ __forceinline__ uint32_t lane_dot()
{
    const int l = threadIdx.x & 31;
    if constexpr (K == F32) return Row<K, DP>::at(l >> 2, 0) + 4 * (l & 3);
    else return Row<K, DP>::at((l & 7) + ((l >> 4) << 3), (l >> 3) & 1);
}
template <int K, int DP> __device__ __forceinline__ uint32_t lane_mul()
{
    const int l = threadIdx.x & 31;
    if constexpr (K == F32) return Row<K, DP>::at(2 * (l & 3), l >> 4) + 4 * ((l >> 2) & 3);
    else return Row<K, DP>::at(l & 15, l >> 4);
}
template <int K, int DP> __device__ __forceinline__ uint32_t lane_rows()
{
    if constexpr (K == F32) return lane_dot<K, DP>();
    else return lane_mul<K, DP>();
}
// step k of the columns (32 bytes) of a row whose step 0 is at `block`; `piece`: bytes of a piece of a tile
template <int K, int DP>
__device__ __forceinline__ uint32_t step_at(uint32_t block, int k, uint32_t piece)
{
    constexpr int STEPS = Row<K, DP>::BYTES / 32;
    return (block ^ (32 * (k % STEPS))) + (Row<K, DP>::PIECES > 1 ? (k / STEPS) * piece : 0);
}

// The 16 rows that a warp multiplies with block after block: in registers (HELD), or from shared
// memory each time where they would crowd out the accumulators
template <int K, int DP, bool HELD = DP <= 32>
struct Rows {
    static constexpr int STEPS = DP * Row<K, DP>::SIZE / 32;                  // of 16 values, or of 8 fp32 values
    uint32_t f[HELD ? STEPS : 1][4], g[HELD && K == F32 ? STEPS : 1][4], block, piece;      // fp32: hi and lo
    __device__ __forceinline__ Rows(uint32_t b, uint32_t p) : block(b), piece(p)
    {
        if constexpr (HELD) {
#pragma unroll
            for (int k = 0; k < STEPS; ++k) load(f[k], g[K == F32 ? k : 0], k);
        }
    }
    __device__ __forceinline__ void load(uint32_t (&hi)[4], uint32_t (&lo)[4], int k) const
    {
        const uint32_t at = step_at<K, DP>(block, k, piece);
        if constexpr (K == F32) {
            split(lds(at), hi[0], lo[0]);
            split(lds(at + 8 * Row<K, DP>::BYTES), hi[1], lo[1]);
            split(lds(at ^ 16), hi[2], lo[2]);
            split(lds((at ^ 16) + 8 * Row<K, DP>::BYTES), hi[3], lo[3]);
        } else {
            ldm4(hi, at);
        }
    }
};

// s[16 x 16] += A B^T, the 16 rows of B are the columns; `block` includes lane_dot.  s[0..3]: columns 0-7, s[4..7]: 8-15
template <int K, int DP, bool HELD>
__device__ __forceinline__ void block_dot(float (&s)[8], const Rows<K, DP, HELD> &a, uint32_t block, uint32_t piece)
{
#pragma unroll
    for (int k = 0; k < Rows<K, DP, HELD>::STEPS; ++k) {
        uint32_t hi[4], lo[4];
        if constexpr (HELD) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                hi[i] = a.f[k][i];
                if constexpr (K == F32) lo[i] = a.g[k][i];
            }
        } else {
            a.load(hi, lo, k);
        }
        const uint32_t at = step_at<K, DP>(block, k, piece);
        if constexpr (K == F32) {
            mma3(s, hi, lo, lds(at), lds(at ^ 16));
            mma3(s + 4, hi, lo, lds(at + 8 * Row<K, DP>::BYTES), lds((at ^ 16) + 8 * Row<K, DP>::BYTES));
        } else {
            uint32_t f[4];
            ldm4(f, at);
            mma<K>(s, hi, f[0], f[1]);
            mma<K>(s + 4, hi, f[2], f[3]);
        }
    }
}

// acc[16 x DP] += p[16 x 16] B, the 16 rows of B summed over; `block` includes lane_mul.  The thread's values of p,
// eight columns of which are s[0..3] and s[4..7], are the A operand as they stand, rounded for 16-bit types.
// The tensor cores round towards zero as they add.  fp32 sums over positions therefore start from zero in every block
// and the blocks' sums are added to nearest: 200 heads of 128 x 64, root mean square error of the output 6.5e-7 of its own,
// one running sum 1.3e-6, everything in fp32 3.9e-7; 256 x 4 heads of 100 x 64 80 us instead of 78, backward 350 instead of 328.
template <int K, int DP>
__device__ __forceinline__ void block_mul(float (&acc)[DP / 8][4], const float (&s)[8], uint32_t block, uint32_t piece)
{
    if constexpr (K == F32) {
        uint32_t hi[2][4], lo[2][4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            split(s[4 * j], hi[j][0], lo[j][0]);
            split(s[4 * j + 2], hi[j][1], lo[j][1]);
            split(s[4 * j + 1], hi[j][2], lo[j][2]);
            split(s[4 * j + 3], hi[j][3], lo[j][3]);
        }
#pragma unroll
        for (int d = 0; d < DP / 8; ++d) {
            float c[4] = {};
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t at = step_at<K, DP>(block + j * 8 * Row<K, DP>::BYTES, d, piece);
                mma3(c, hi[j], lo[j], lds(at), lds(at ^ (Row<K, DP>::BYTES | 16)));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[d][i] += c[i];
        }
    } else {
        const uint32_t p[4] = {pack2<K == BF16>(s[0], s[1]), pack2<K == BF16>(s[2], s[3]), pack2<K == BF16>(s[4], s[5]),
                               pack2<K == BF16>(s[6], s[7])};
#pragma unroll
        for (int d = 0; d < DP / 16; ++d) {
            uint32_t f[4];
            ldm4t(f, step_at<K, DP>(block, d, piece));
            mma<K>(acc[2 * d], p, f[0], f[1]);
            mma<K>(acc[2 * d + 1], p, f[2], f[3]);
        }
    }
}

// offset of value i's column from the thread's first one (rows: lane / 4 for i & 2 == 0, + 8 otherwise)
__device__ __forceinline__ constexpr int step_of(int i) { return ((i >> 2) << 3) + (i & 1); }

struct Unit {
    AttnSeq s;
    int64_t b;
    int h;
};

__device__ __forceinline__ Unit unit_of(const AttnArgs &a, uint32_t u, uint32_t heads)
{
    Unit l;
    const uint32_t b = u / heads;
    l.b = b;
    l.h = (int)(u - b * heads);
    l.s = attn_seq(a, l.b);
    return l;
}

// Blocks whose distance from the diagonal (in blocks, -7..7, column block minus row block) makes them partly
// visible: their place among the starting values in shared memory; -1: wholly visible
struct WalkMask {
    signed char slot[16];
    signed char dist[4];              // of each place
    int n;
    int left, right;                  // columns before and after the row's own that are visible, < 0: all
};

// bytes of the starting values: two planes of four floats per lane, for each place
__host__ __device__ constexpr uint32_t mask_bytes(int n) { return n * 1024; }

__device__ __forceinline__ void fill_masks(float *to, const WalkMask &m)
{
    for (int e = threadIdx.x; e < m.n * 256; e += blockDim.x) {
        const int i = (e & 3) + ((e >> 7) & 1) * 4, lane = (e >> 2) & 31;
        const int row = (lane >> 2) + (i & 2 ? 8 : 0), col = 2 * (lane & 3) + step_of(i);
        const int at = 16 * m.dist[e >> 8] + col - row;
        to[e] = (m.left < 0 || at >= -m.left) && (m.right < 0 || at <= m.right) ? 0.f : -INFINITY;
    }
}

// starting values of the block `dist` blocks right of the diagonal.  shift != 0: rows and columns are shifted
// against each other (queries and keys of different lengths), and the values are worked out here.
__device__ __forceinline__ void start_scores(float (&s)[8], const WalkMask &m, uint32_t masks, int dist, int shift)
{
    const int lane = threadIdx.x & 31;
    if (shift == 0) {
        const int slot = m.slot[dist + 7];
        if (slot >= 0) {
            const uint32_t from = masks + slot * 1024 + lane * 16;
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(s[0]), "=f"(s[1]), "=f"(s[2]), "=f"(s[3]) : "r"(from) : "memory");
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(s[4]), "=f"(s[5]), "=f"(s[6]), "=f"(s[7]) : "r"(from + 512) : "memory");
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] = 0.f;
        return;
    }
    const int at = 16 * dist + 2 * (lane & 3) - (lane >> 2) - shift;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int d = at + step_of(i) - (i & 2 ? 8 : 0);
        s[i] = (m.left < 0 || d >= -m.left) && (m.right < 0 || d <= m.right) ? 0.f : -INFINITY;
    }
}

// columns >= n of a block are not visible: keys past the sequence's end
__device__ __forceinline__ void hide_from(float (&s)[8], int n)
{
    const int left = n - 2 * ((int)threadIdx.x & 3);
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = step_of(i) < left ? s[i] : -INFINITY;
}

// what the launcher settles
struct WalkPlan {
    int units;                        // heads that a block works on at a time
    int qt, kt;                       // 16-row tiles of the padded lengths
    bool tma;                         // loads and stores through TMA
    int stages;                       // sets of tiles: two if they fit (one without TMA)
    bool vec;                         // without it: 16-byte loads and stores
    WalkMask rows, cols;              // by query rows (columns: keys) and by key rows (columns: queries)
};
struct WalkMaps {                     // boxes of all rows for the inputs, of 16 rows for the results
    CUtensorMap q, k, v, dout, out, dk, dv;
};

// one head's rows through TMA (one thread)
template <int K, int DP>
__device__ __forceinline__ void tma_head(uint32_t dst, const CUtensorMap *map, uint32_t bar, int head, int64_t b, uint32_t piece)
{
#pragma unroll
    for (int x = 0; x < Row<K, DP>::PIECES; ++x) tma_load(dst + x * piece, map, bar, x * Row<K, DP>::VALUES, 0, head, (int)b);
}

// 16 bytes of a row from value c on in global memory, zeros from value dim on; and back
template <int K>
__device__ __forceinline__ uint4 read_chunk(const void *row, int c, int dim, bool vec)
{
    uint32_t u[4] = {};
    if (vec) {
        if (c < dim) return __ldg(reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(row) + c * (K == F32 ? 4 : 2)));
    } else if constexpr (K == F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i < dim) u[i] = reinterpret_cast<const uint32_t *>(row)[c + i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < dim) u[i / 2] |= (uint32_t) reinterpret_cast<const uint16_t *>(row)[c + i] << (16 * (i & 1));
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}
template <int K>
__device__ __forceinline__ void write_chunk(void *row, int c, int dim, bool vec, uint4 w)
{
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
    if (vec) {
        if (c < dim) *reinterpret_cast<uint4 *>(reinterpret_cast<char *>(row) + c * (K == F32 ? 4 : 2)) = w;
    } else if constexpr (K == F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i < dim) reinterpret_cast<uint32_t *>(row)[c + i] = v[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < dim) reinterpret_cast<uint16_t *>(row)[c + i] = (uint16_t)(v[i / 2] >> (16 * (i & 1)));
    }
}
template <int K>
__device__ __forceinline__ char *row_at(const AttnTensor &t, int64_t b, int h, int r)
{
    return reinterpret_cast<char *>(t.p) + (b * t.sb + h * t.sh + (int64_t)r * t.sl) * (K == F32 ? 4 : 2);
}

// rows [0, pad) of one head by `threads` threads: rows >= n and values >= dim are zeros
template <int K, int DP>
__device__ __forceinline__ void copy_head(uint32_t dst, const AttnTensor &t, int64_t b, int h, int n, int pad, int dim,
                                          bool vec, int tid, int threads)
{
    constexpr int CH = Row<K, DP>::CHUNKS * Row<K, DP>::PIECES, PER = 16 / Row<K, DP>::SIZE;
    for (int e = tid; e < pad * CH; e += threads) {
        const int r = e / CH, c = e % CH;
        const uint4 u = r < n ? read_chunk<K>(row_at<K>(t, b, h, r), c * PER, dim, vec) : make_uint4(0, 0, 0, 0);
        const uint32_t to = dst + (c / Row<K, DP>::CHUNKS) * pad * Row<K, DP>::BYTES + Row<K, DP>::at(r, c % Row<K, DP>::CHUNKS);
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(u.x), "r"(u.y), "r"(u.z), "r"(u.w) : "memory");
    }
}

// rows [n, pad) become zeros: they take part in sums over rows, where a zero probability must not meet a NaN
template <int K, int DP>
__device__ __forceinline__ void zero_rows(uint32_t tile, int n, int pad, int tid, int threads)
{
    for (int e = n * Row<K, DP>::CHUNKS + tid; e < pad * Row<K, DP>::CHUNKS; e += threads)
#pragma unroll
        for (int x = 0; x < Row<K, DP>::PIECES; ++x)
            asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(tile + x * pad * Row<K, DP>::BYTES + e * 16), "r"(0) : "memory");
}

// the 16 x DP accumulator times its two row factors, in the tensors' type
template <int K, int DP>
__device__ __forceinline__ void pack_tile(uint32_t (&u)[DP / 8][Row<K, DP>::WORDS], const float (&acc)[DP / 8][4], float f0, float f1)
{
#pragma unroll
    for (int c = 0; c < DP / 8; ++c) {
        if constexpr (K == F32) {
            u[c][0] = __float_as_uint(acc[c][0] * f0);
            u[c][1] = __float_as_uint(acc[c][1] * f0);
            u[c][2] = __float_as_uint(acc[c][2] * f1);
            u[c][3] = __float_as_uint(acc[c][3] * f1);
        } else {
            u[c][0] = pack2<K == BF16>(acc[c][0] * f0, acc[c][1] * f0);
            u[c][1] = pack2<K == BF16>(acc[c][2] * f1, acc[c][3] * f1);
        }
    }
}

// A sum whose only use is that it is NaN if one of the words' values is.  One of 16-bit values may also become NaN by
// running over; then rows are looked at for nothing.
template <int K>
struct NanSum {
    using Pair = typename std::conditional<K == F32, float, typename std::conditional<K == BF16, __nv_bfloat162, __half2>::type>::type;
    uint32_t t = 0;
    __device__ __forceinline__ uint32_t add(uint32_t w)        // passes the word on
    {
        Pair &s = reinterpret_cast<Pair &>(t);
        if constexpr (K == F32) s += __uint_as_float(w);
        else s = __hadd2(s, reinterpret_cast<const Pair &>(w));
        return w;
    }
    __device__ __forceinline__ bool found()
    {
        Pair &s = reinterpret_cast<Pair &>(t);
        if constexpr (K == F32) return s != s;
        else return __hisnan(__hadd(s.x, s.y));
    }
};

// This warp's 16 x DP result, as pack_tile left it, to rows [r0, r0 + 16) of one head: first into the 16
// rows at `stage` in shared memory, which nobody else reads any more, then in 16-byte pieces.
// Rows >= n become zeros, rows >= len are not written.  TMA reads the stage until tma_stores_read.  Returns whether this
// thread's part of rows < n holds a NaN (or may).
template <int K, int DP>
__device__ __forceinline__ bool store_tile(const uint32_t (&u)[DP / 8][Row<K, DP>::WORDS], uint32_t stage, uint32_t piece,
                                           const WalkPlan &plan, const CUtensorMap *map, const AttnTensor &t, int64_t b, int h,
                                           int r0, int n, int len, int dim)
{
    constexpr int CH = Row<K, DP>::CHUNKS, PER = 16 / Row<K, DP>::SIZE;
    const int lane = threadIdx.x & 31, row = lane >> 2, t4 = lane & 3;
    const bool in0 = r0 + row < n, in1 = r0 + row + 8 < n;
    NanSum<K> top, bottom;                                     // rows 0-7 and 8-15
    __syncwarp();
#pragma unroll
    for (int c = 0; c < DP / 8; ++c) {                       // the thread's columns 8c + 2 t4 and the next
        if constexpr (K == F32) {
            const int chunk = 2 * c;
            const uint32_t to = stage + (chunk / CH) * piece + Row<K, DP>::at(row, chunk % CH + (t4 >> 1)) + 8 * (t4 & 1);
            asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(to), "r"(top.add(in0 ? u[c][0] : 0u)), "r"(top.add(in0 ? u[c][1] : 0u)) : "memory");
            asm volatile("st.shared.v2.u32 [%0], {%1, %2};"
                         ::"r"(to + 8 * Row<K, DP>::BYTES), "r"(bottom.add(in1 ? u[c][2] : 0u)), "r"(bottom.add(in1 ? u[c][3] : 0u)) : "memory");
        } else {
            const uint32_t to = stage + (c / CH) * piece + Row<K, DP>::at(row, c % CH) + 4 * t4;
            asm volatile("st.shared.u32 [%0], %1;" ::"r"(to), "r"(top.add(in0 ? u[c][0] : 0u)) : "memory");
            asm volatile("st.shared.u32 [%0], %1;" ::"r"(to + 8 * Row<K, DP>::BYTES), "r"(bottom.add(in1 ? u[c][1] : 0u)) : "memory");   // row + 8: the same permutation
        }
    }
    top.add(bottom.t);
    const bool nan = top.found();
    if (plan.tma) {
        fence_async_shared();
        __syncwarp();
        if (lane == 0) {
#pragma unroll
            for (int x = 0; x < Row<K, DP>::PIECES; ++x) tma_store(map, stage + x * piece, x * Row<K, DP>::VALUES, r0, h, (int)b);
            tma_store_commit();
        }
        return nan;
    }
    __syncwarp();
    constexpr int ALL = CH * Row<K, DP>::PIECES;
    for (int e = lane; e < 16 * ALL; e += 32) {
        const int rr = e / ALL, c = e % ALL, r = r0 + rr;
        if (r >= len) continue;
        uint4 w;
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w)
                     : "r"(stage + (c / CH) * piece + Row<K, DP>::at(rr, c % CH)) : "memory");
        write_chunk<K>(row_at<K>(t, b, h, r), c * PER, dim, plan.vec, w);
    }
    return nan;
}

// Registers of a thread, and how many blocks of up to BLOCK_WARPS warps an SM is to hold with them.  Measured on
// 16384 walks of 40 with 4 heads of 32 (forward) and 8192 of 80 (backward): 80 registers and 8 warps 188 us, 64
// registers 208, 108 registers 264; backward 96 registers 448 us, 128 registers with p and dp of three blocks kept
// for the second walk over them 465, 80 registers 523.
template <int K, int DP, bool BWD> constexpr int registers()
{
    if (K == F32) return DP <= 32 && !BWD ? 128 : DP <= 64 ? 168 : 255;
    return DP <= 32 ? (BWD ? 96 : 80) : DP == 64 ? 128 : 255;
}
template <int K, int DP, bool BWD> constexpr int blocks_per_sm()
{
    if (K == F32) return DP <= 32 && !BWD ? 2 : 1;
    return DP <= 32 ? (BWD ? 4 : 3) : DP == 64 ? 2 : 1;
}
static constexpr int BLOCK_WARPS = 8;             // a head of 128 rows

// one warp per (unit, query tile)
template <int K, int DP>
__global__ void __maxnreg__((registers<K, DP, false>()))
attn_walk_forward_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ WalkPlan plan, const __grid_constant__ WalkMaps maps,
                         unsigned long long *stalls)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ __align__(8) uint64_t full[2];
    __shared__ volatile int stalled;
    __shared__ volatile int nan;                          // one of the block's results holds one
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, qt = plan.qt, kt = plan.kt;
    const uint32_t total = (uint32_t)a.batch * a.q_heads, step = gridDim.x * plan.units;
    const uint32_t q_half = qt * Row<K, DP>::BLOCK, k_half = kt * Row<K, DP>::BLOCK;
    const uint32_t q_bytes = Row<K, DP>::tile(qt), k_bytes = Row<K, DP>::tile(kt), unit_bytes = q_bytes + 2 * k_bytes;
    const int mine = (int)((uint32_t)warp / (uint32_t)qt), tile = warp - mine * qt;   // qt warps work on one unit
    const int tid = threadIdx.x - mine * qt * 32, threads = qt * 32;
    const uint32_t bars = smem_u32(full);
    const bool ragged = a.k_lens != nullptr && plan.tma;
    auto tiles_at = [&](int st) { return smem_u32(smem) + (st * plan.units + mine) * unit_bytes; };
    uint8_t *masks = smem + plan.stages * plan.units * unit_bytes;
    const uint32_t mask_rows = smem_u32(masks);
    fill_masks(reinterpret_cast<float *>(masks), plan.rows);
    auto load = [&](uint32_t u, int st) {              // the unit's first thread
        const uint32_t bar = bars + 8 * st, Q = tiles_at(st);
        if (u >= total) {
            bar_arrive(bar);
            return;
        }
        const uint32_t b = u / (uint32_t)a.q_heads;
        const int h = (int)(u - b * a.q_heads), g = h / a.group;
        bar_expect(bar, unit_bytes);
        tma_head<K, DP>(Q, &maps.q, bar, h, b, q_half);
        tma_head<K, DP>(Q + q_bytes, &maps.k, bar, g, b, k_half);
        tma_head<K, DP>(Q + q_bytes + k_bytes, &maps.v, bar, g, b, k_half);
    };
    if (threadIdx.x == 0) {
        stalled = nan = 0;
        bar_init(bars, plan.units);
        bar_init(bars + 8, plan.units);
        fence_barrier_init();
    }
    __syncthreads();
    uint32_t u = blockIdx.x * plan.units + mine;
    if (plan.tma && tid == 0) {
        load(u, 0);
        if (plan.stages == 2) load(u + step, 1);
    }
    const float mul = a.scale * LOG2E;
    for (uint32_t u0 = blockIdx.x * plan.units, n = 0; u0 < total; u0 += step, u += step, ++n) {
    const int st = n & (plan.stages - 1);
    const bool active = u < total;
    const Unit l = unit_of(a, active ? u : u0, a.q_heads);
    const uint32_t Q = tiles_at(st), Kt = Q + q_bytes, V = Kt + k_bytes;
    // Once a wait has run out all others return at once: the loop then goes on to its end without data and without
    // new loads, so that nobody is left alone at a barrier and no barrier is armed a second time.
    if (plan.tma) {
        bar_wait(bars + 8 * st, (n >> (plan.stages - 1)) & 1, &stalled);
        __syncwarp();
    } else if (active) {
        const int g = l.h / a.group;
        copy_head<K, DP>(Q, a.q, l.b, l.h, l.s.nq, qt * 16, a.dim, plan.vec, tid, threads);
        copy_head<K, DP>(Kt, a.k, l.b, g, l.s.nk, kt * 16, a.dim, plan.vec, tid, threads);
        copy_head<K, DP>(V, a.v, l.b, g, l.s.nk, kt * 16, a.dim, plan.vec, tid, threads);
    }
    if (ragged && l.s.nk < a.k_len) zero_rows<K, DP>(V, l.s.nk, kt * 16, tid, threads);
    if (ragged || !plan.tma) __syncthreads();           // rows that other threads have written
    if (active) {
    const int r0 = tile * 16, ra = r0 + (lane >> 2), rb = ra + 8;
    float acc[DP / 8][4] = {};
    float top_a = -INFINITY, top_b = -INFINITY, sum_a = 0.f, sum_b = 0.f;     // top: largest score, not yet scaled
    const int r_end = min(r0 + 16, l.s.nq);
    const int j_begin = attn_lo(a, l.s, r0) / 16, j_end = r_end > r0 ? (attn_hi(a, l.s, r_end - 1) + 15) / 16 : 0;
    if (j_begin < j_end) {
        const Rows<K, DP, (K != F32 || DP <= 32)> qf(Q + tile * Row<K, DP>::BLOCK + lane_rows<K, DP>(), q_half);
        const uint32_t kb = Kt + lane_dot<K, DP>(), vb = V + lane_mul<K, DP>();
        for (int j = j_begin; j < j_end; j += KEEP) {
            float s[KEEP][8];
            float m_a = top_a, m_b = top_b;
#pragma unroll
            for (int x = 0; x < KEEP; ++x) {
                if (j + x >= j_end) break;
                start_scores(s[x], plan.rows, mask_rows, j + x - tile, l.s.off);
                block_dot<K, DP>(s[x], qf, kb + (j + x) * Row<K, DP>::BLOCK, k_half);
                if ((j + x + 1) * 16 > l.s.nk) hide_from(s[x], l.s.nk - (j + x) * 16);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (i & 2) m_b = fmaxf(m_b, s[x][i]);
                    else m_a = fmaxf(m_a, s[x][i]);
                }
            }
            m_a = quad_max(m_a);
            m_b = quad_max(m_b);
            // nothing visible yet: every term is exp2(-inf) = 0
            const float base_a = m_a == -INFINITY ? 0.f : m_a * mul, base_b = m_b == -INFINITY ? 0.f : m_b * mul;
            if (j > j_begin) {
                const float keep_a = exp2_fast(top_a * mul - base_a), keep_b = exp2_fast(top_b * mul - base_b);
                sum_a *= keep_a;
                sum_b *= keep_b;
#pragma unroll
                for (int d = 0; d < DP / 8; ++d) {
                    acc[d][0] *= keep_a;
                    acc[d][1] *= keep_a;
                    acc[d][2] *= keep_b;
                    acc[d][3] *= keep_b;
                }
            }
            top_a = m_a;
            top_b = m_b;
#pragma unroll
            for (int x = 0; x < KEEP; ++x) {
                if (j + x >= j_end) break;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    s[x][i] = exp2_fast(fmaf(s[x][i], mul, i & 2 ? -base_b : -base_a));
                    if (i & 2) sum_b += s[x][i];
                    else sum_a += s[x][i];
                }
                block_mul<K, DP>(acc, s[x], vb + (j + x) * Row<K, DP>::BLOCK, k_half);
            }
        }
    }
    sum_a = quad_sum(sum_a);
    sum_b = quad_sum(sum_b);
    top_a *= mul;
    top_b *= mul;
    const float by_a = again::row_factor(top_a, rcp_fast(sum_a)), by_b = again::row_factor(top_b, rcp_fast(sum_b));
    if ((lane & 3) == 0) {
        float *lse = a.lse + (l.b * a.q_heads + l.h) * a.q_len;
        if (ra < a.q_len) lse[ra] = ra >= l.s.nq ? -INFINITY : again::row_lse(top_a, by_a, log2_fast(sum_a));
        if (rb < a.q_len) lse[rb] = rb >= l.s.nq ? -INFINITY : again::row_lse(top_b, by_b, log2_fast(sum_b));
    }
    uint32_t out[DP / 8][Row<K, DP>::WORDS];
    pack_tile<K, DP>(out, acc, by_a, by_b);
    if (store_tile<K, DP>(out, Q + tile * Row<K, DP>::BLOCK, q_half, plan, &maps.out, a.out, l.b, l.h, r0, l.s.nq, a.q_len, a.dim))
        nan = 1;
    }
    if (plan.tma) {
        if (lane == 0) tma_stores_read();
        if (ragged) fence_async_shared();               // zeroed rows, before TMA writes there again
    }
    __syncthreads();                                    // everybody is done with this set of tiles
    if (plan.tma && tid == 0 && !stalled && u0 + plan.stages * step < total) load(u + plan.stages * step, st);
    }
    if (stalled) drain_stalled(stalls);
    if (nan) {
        if (plan.tma && lane == 0) tma_stores_done();
        for (uint32_t v = blockIdx.x * plan.units + mine; v < total; v += step)
            again::outputs<typename TypeOf<K>::T>(a, v / (uint32_t)a.q_heads, (int)(v % (uint32_t)a.q_heads), tile * 16, tile * 16 + 16);
    }
}

// power of two that brings a bound below 2^15 (binary16 only)
template <int K>
__device__ __forceinline__ float lift(float bound)
{
    if (K != F16 || !(bound > 0.f) || !isfinite(bound)) return 1.f;
    const int e = (int)((__float_as_uint(bound) >> 23) & 255) - 126;       // bound < 2^e
    return __uint_as_float((uint32_t)(min(max(15 - e, -100), 100) + 127) << 23);
}

// `tiles` = max(qt, kt) warps per unit; a unit is a key/value head, gone through once per query head of its group.
// SHARED: several query heads per key/value head.
template <int K, int DP, bool SHARED>
__global__ void __maxnreg__((registers<K, DP, true>()))
attn_walk_backward_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ WalkPlan plan, const __grid_constant__ WalkMaps maps,
                          unsigned long long *stalls)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ __align__(8) uint64_t full[2];
    __shared__ volatile int stalled;
    __shared__ volatile int nan;                          // one of the block's results holds one
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, qt = plan.qt, kt = plan.kt, tiles = max(qt, kt);
    const uint32_t total = (uint32_t)a.batch * a.kv_heads, step = gridDim.x * plan.units;
    const uint32_t q_half = qt * Row<K, DP>::BLOCK, k_half = kt * Row<K, DP>::BLOCK;
    const uint32_t q_bytes = Row<K, DP>::tile(qt), k_bytes = Row<K, DP>::tile(kt), unit_bytes = 2 * q_bytes + 2 * k_bytes;
    const int mine = (int)((uint32_t)warp / (uint32_t)tiles), tile = warp - mine * tiles;
    const int tid = threadIdx.x - mine * tiles * 32, threads = tiles * 32;
    const uint32_t bars = smem_u32(full);
    const bool ragged = (a.q_lens != nullptr || a.k_lens != nullptr) && plan.tma;
    const int group = SHARED ? a.group : 1;
    // per query row: -lse in units of log2, -delta, bound of |dS|
    float *neg_lse = reinterpret_cast<float *>(smem + plan.stages * plan.units * unit_bytes + mine * stat_bytes(qt));
    float *neg_delta = neg_lse + qt * 16, *bound = neg_delta + qt * 16;
    uint8_t *masks = smem + plan.units * (plan.stages * unit_bytes + stat_bytes(qt));
    const uint32_t mask_rows = smem_u32(masks), mask_cols = mask_rows + mask_bytes(plan.rows.n);
    fill_masks(reinterpret_cast<float *>(masks), plan.rows);
    fill_masks(reinterpret_cast<float *>(masks + mask_bytes(plan.rows.n)), plan.cols);
    auto tiles_at = [&](int st) { return smem_u32(smem) + (st * plan.units + mine) * unit_bytes; };
    auto load = [&](uint32_t u, int x, int st) {       // the unit's first thread; x: query head of the group
        const uint32_t bar = bars + 8 * st, Q = tiles_at(st);
        if (u >= total) {
            bar_arrive(bar);
            return;
        }
        const uint32_t b = u / (uint32_t)a.kv_heads;
        const int g = (int)(u - b * a.kv_heads), h = g * group + x;
        bar_expect(bar, unit_bytes);
        tma_head<K, DP>(Q, &maps.q, bar, h, b, q_half);
        tma_head<K, DP>(Q + q_bytes, &maps.dout, bar, h, b, q_half);
        tma_head<K, DP>(Q + 2 * q_bytes, &maps.k, bar, g, b, k_half);
        tma_head<K, DP>(Q + 2 * q_bytes + k_bytes, &maps.v, bar, g, b, k_half);
    };
    if (threadIdx.x == 0) {
        stalled = nan = 0;
        bar_init(bars, plan.units);
        bar_init(bars + 8, plan.units);
        fence_barrier_init();
    }
    __syncthreads();
    uint32_t u = blockIdx.x * plan.units + mine;
    if (plan.tma && tid == 0) {
        load(u, 0, 0);
        if (plan.stages == 2) {
            if (group > 1) load(u, 1, 1);
            else load(u + step, 0, 1);
        }
    }
    const float mul = a.scale * LOG2E;
    uint32_t n = 0;
    for (uint32_t u0 = blockIdx.x * plan.units; u0 < total; u0 += step, u += step) {
    const bool active = u < total;
    const Unit l = unit_of(a, active ? u : u0, a.kv_heads);
    const AttnSeq s = l.s;
    float dk[DP / 8][4] = {}, dv[DP / 8][4] = {};
    float up_k = 1.f;
    for (int x = 0; x < group; ++x, ++n) {
        const int st = n & (plan.stages - 1);
        const int h = l.h * group + x;
        const uint32_t Q = tiles_at(st), DO = Q + q_bytes, Kt = DO + q_bytes, V = Kt + k_bytes;
        const float *lse = a.lse + (l.b * a.q_heads + h) * a.q_len;
        for (int r = tid; r < qt * 16; r += threads) {
            const float v = r < s.nq ? -lse[r] * LOG2E : -INFINITY;
            neg_lse[r] = v == INFINITY ? -INFINITY : v;       // p = 0 in rows that see nothing
        }
        // the dq rows of this thread
        const int r0 = tile * 16, ra = r0 + (lane >> 2), rb = ra + 8;
        float l_a = ra < s.nq ? -lse[ra] * LOG2E : -INFINITY, l_b = rb < s.nq ? -lse[rb] * LOG2E : -INFINITY;
        l_a = l_a == INFINITY ? -INFINITY : l_a;
        l_b = l_b == INFINITY ? -INFINITY : l_b;
        if (plan.tma) {                                       // as in the forward kernel, a wait that runs out ends no loop
            bar_wait(bars + 8 * st, (n >> (plan.stages - 1)) & 1, &stalled);
            __syncwarp();
        } else if (active) {
            copy_head<K, DP>(Q, a.q, l.b, h, s.nq, qt * 16, a.dim, plan.vec, tid, threads);
            copy_head<K, DP>(DO, a.dout, l.b, h, s.nq, qt * 16, a.dim, plan.vec, tid, threads);
            copy_head<K, DP>(Kt, a.k, l.b, l.h, s.nk, kt * 16, a.dim, plan.vec, tid, threads);
            copy_head<K, DP>(V, a.v, l.b, l.h, s.nk, kt * 16, a.dim, plan.vec, tid, threads);
        }
        if (ragged && s.nq < a.q_len) {
            zero_rows<K, DP>(Q, s.nq, qt * 16, tid, threads);
            zero_rows<K, DP>(DO, s.nq, qt * 16, tid, threads);
        }
        if (ragged && s.nk < a.k_len) {
            zero_rows<K, DP>(Kt, s.nk, kt * 16, tid, threads);
            zero_rows<K, DP>(V, s.nk, kt * 16, tid, threads);
        }
        if (ragged || !plan.tma) __syncthreads();             // rows that other threads have written

        // ---- dq of 16 query rows
        uint32_t dq[DP / 8][Row<K, DP>::WORDS] = {};
        if (active && tile < qt) {
            const int r_end = min(r0 + 16, s.nq);
            const int j_begin = attn_lo(a, s, r0) / 16, j_end = r_end > r0 ? (attn_hi(a, s, r_end - 1) + 15) / 16 : 0;
            const Rows<K, DP> qf(Q + tile * Row<K, DP>::BLOCK + lane_rows<K, DP>(), q_half), df(DO + tile * Row<K, DP>::BLOCK + lane_rows<K, DP>(), q_half);
            const uint32_t lb = lane_dot<K, DP>(), kb = Kt + lane_mul<K, DP>();
            float d_a = 0.f, d_b = 0.f, m_a = 0.f, m_b = 0.f;
            // p and dp of one block
            auto scores = [&](int j, float (&p)[8], float (&dp)[8]) {
                start_scores(p, plan.rows, mask_rows, j - tile, s.off);
                block_dot<K, DP>(p, qf, Kt + lb + j * Row<K, DP>::BLOCK, k_half);
                if ((j + 1) * 16 > s.nk) hide_from(p, s.nk - j * 16);
#pragma unroll
                for (int i = 0; i < 8; ++i) dp[i] = 0.f;
                block_dot<K, DP>(dp, df, V + lb + j * Row<K, DP>::BLOCK, k_half);
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] = exp2_fast(fmaf(p[i], mul, i & 2 ? l_b : l_a));
            };
            auto take = [&](const float (&p)[8], const float (&dp)[8]) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (i & 2) {
                        d_b = fmaf(p[i], dp[i], d_b);
                        if constexpr (K == F16) m_b = fmaxf(m_b, fabsf(dp[i]));
                    } else {
                        d_a = fmaf(p[i], dp[i], d_a);
                        if constexpr (K == F16) m_a = fmaxf(m_a, fabsf(dp[i]));
                    }
                }
            };
            float up_a = 1.f, up_b = 1.f;
            auto rows_known = [&] {
                d_a = quad_sum(d_a);
                d_b = quad_sum(d_b);
                if constexpr (K == F16) {
                    m_a = quad_max(m_a) + fabsf(d_a);
                    m_b = quad_max(m_b) + fabsf(d_b);
                    up_a = lift<K>(m_a);
                    up_b = lift<K>(m_b);
                }
                if ((lane & 3) == 0) {
                    neg_delta[ra] = -d_a;
                    neg_delta[rb] = -d_b;
                    if constexpr (K == F16) {                   // an infinity must not cost the head's other rows their scale
                        bound[ra] = m_a < INFINITY ? m_a : 0.f;
                        bound[rb] = m_b < INFINITY ? m_b : 0.f;
                    }
                }
            };
            float acc[DP / 8][4] = {}, nd_a = 0.f, nd_b = 0.f;                // nd: -delta, scaled
            auto add = [&](int j, float (&p)[8], const float (&dp)[8]) {
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] *= K != F16 ? dp[i] - (i & 2 ? d_b : d_a) : fmaf(dp[i], i & 2 ? up_b : up_a, i & 2 ? nd_b : nd_a);
                block_mul<K, DP>(acc, p, kb + j * Row<K, DP>::BLOCK, k_half);
            };
            float p[8], dp[8];
            for (int j = j_begin; j < j_end; ++j) {
                scores(j, p, dp);
                take(p, dp);
            }
            rows_known();
            nd_a = -d_a * up_a;
            nd_b = -d_b * up_b;
            for (int j = j_begin; j < j_end; ++j) {
                scores(j, p, dp);
                add(j, p, dp);
            }
            pack_tile<K, DP>(dq, acc, a.scale / up_a, a.scale / up_b);
        }
        __syncthreads();

        // ---- dk, dv of 16 key rows
        if (active && tile < kt) {
            const int j0 = tile * 16;
            const int j_end = min(j0 + 16, s.nk);
            const int q_begin = attn_q_first(a, s, j0) / 16, q_end = j_end > j0 ? (attn_q_last(a, s, j_end) + 15) / 16 : 0;
            float up_p = 1.f;                                 // of dp - delta, beside a p that is scaled itself
            if constexpr (K == F16) {                           // one scale per head: dk sums over its queries
                float m = 0.f;
                for (int r = lane; r < qt * 16; r += 32) m = fmaxf(m, bound[r]);
#pragma unroll
                for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
                const float up = lift<K>(m);
                // a shared head's sums are carried from one query head's scale to the next one's
                if (x > 0 && up != up_k) {
#pragma unroll
                    for (int d = 0; d < DP / 8; ++d)
#pragma unroll
                        for (int i = 0; i < 4; ++i) dk[d][i] *= up / up_k;
                }
                up_k = up;
                up_p = up / 16384.f;
            }
            if (q_begin < q_end) {
                const Rows<K, DP> kf(Kt + tile * Row<K, DP>::BLOCK + lane_rows<K, DP>(), k_half), vf(V + tile * Row<K, DP>::BLOCK + lane_rows<K, DP>(), k_half);
                const uint32_t lb = lane_dot<K, DP>(), la = lane_mul<K, DP>();
                for (int q = q_begin; q < q_end; ++q) {
                    const uint32_t qb = Q + q * Row<K, DP>::BLOCK, ob = DO + q * Row<K, DP>::BLOCK;
                    float p[8], dp[8];
                    // queries past the end: their lse makes p zero
                    start_scores(p, plan.cols, mask_cols, q - tile, -s.off);
                    block_dot<K, DP>(p, kf, qb + lb, q_half);
#pragma unroll
                    for (int i = 0; i < 8; ++i) dp[i] = 0.f;
                    block_dot<K, DP>(dp, vf, ob + lb, q_half);
                    const int c = q * 16 + 2 * (lane & 3);
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        float2 nl = *reinterpret_cast<const float2 *>(neg_lse + c + 8 * n);
                        float2 nd = *reinterpret_cast<const float2 *>(neg_delta + c + 8 * n);
                        if constexpr (K == F16) {                // p by 2^14, ds by up
                            nl.x += 14.f;
                            nl.y += 14.f;
                            nd.x *= up_p;
                            nd.y *= up_p;
                        }
#pragma unroll
                        for (int i = 4 * n; i < 4 * n + 4; ++i) {
                            p[i] = exp2_fast(fmaf(p[i], mul, i & 1 ? nl.y : nl.x));
                            dp[i] = p[i] * (K != F16 ? dp[i] + (i & 1 ? nd.y : nd.x) : fmaf(dp[i], up_p, i & 1 ? nd.y : nd.x));
                        }
                    }
                    block_mul<K, DP>(dv, p, ob + la, q_half);
                    block_mul<K, DP>(dk, dp, qb + la, q_half);
                }
            }
        }
        __syncthreads();                                      // nobody reads this set of tiles any more
        if (active && tile < qt &&
            store_tile<K, DP>(dq, Q + tile * Row<K, DP>::BLOCK, q_half, plan, &maps.out, a.dq, l.b, h, r0, s.nq, a.q_len, a.dim))
            nan = 1;
        if (active && tile < kt && x == group - 1) {
            const float f = a.scale / up_k, g = K != F16 ? 1.f : 1.f / 16384.f;
            uint32_t w[DP / 8][Row<K, DP>::WORDS];
            pack_tile<K, DP>(w, dk, f, f);
            bool found = store_tile<K, DP>(w, Kt + tile * Row<K, DP>::BLOCK, k_half, plan, &maps.dk, a.dk, l.b, l.h, tile * 16, s.nk, a.k_len, a.dim);
            pack_tile<K, DP>(w, dv, g, g);
            found |= store_tile<K, DP>(w, V + tile * Row<K, DP>::BLOCK, k_half, plan, &maps.dv, a.dv, l.b, l.h, tile * 16, s.nk, a.k_len, a.dim);
            if (found) nan = 1;
        }
        if (plan.tma) {
            if (lane == 0) tma_stores_read();
            if (ragged) fence_async_shared();                 // zeroed rows, before TMA writes there again
        }
        __syncthreads();
        if (plan.tma && tid == 0 && !stalled) {               // the step that uses these tiles next
            const int ahead = (x + plan.stages) / group, x2 = (x + plan.stages) % group;
            if (u0 + ahead * step < total) load(u + ahead * step, x2, st);
        }
    }
    }
    if (stalled) drain_stalled(stalls);
    if (nan) {
        using T = typename TypeOf<K>::T;
        if (plan.tma && lane == 0) tma_stores_done();
        for (uint32_t v = blockIdx.x * plan.units + mine; v < total; v += step) {
            const int64_t b = v / (uint32_t)a.kv_heads;
            const int g = (int)(v % (uint32_t)a.kv_heads);
            for (int x = 0; x < group; ++x) again::query_gradients<T>(a, b, g * group + x, tile * 16, tile * 16 + 16, 0, a.dim);
            again::key_gradients<T>(a, b, g, tile * 16, tile * 16 + 16, true, true);
        }
    }
}

// 16-byte accesses need every row of every tensor aligned to them
static bool rows_of_16_bytes(const AttnArgs &a, bool backward)
{
    const int n = a.dtype == GS_TABLE_F32 ? 4 : 8;
    auto ok = [&](const AttnTensor &t) { return (uintptr_t)t.p % 16 == 0 && (t.sb | t.sl | t.sh) % n == 0; };
    bool v = a.dim % n == 0 && ok(a.q) && ok(a.k) && ok(a.v);
    if (backward) return v && ok(a.dout) && ok(a.dq) && ok(a.dk) && ok(a.dv);
    return v && ok(a.out);
}

static bool all_tma(const AttnArgs &a, bool backward)
{
    auto on_q = [&](const AttnTensor &t) { return attn_tma_ok(t, a.dtype, a.batch, a.q_len, a.q_heads); };
    auto on_k = [&](const AttnTensor &t) { return attn_tma_ok(t, a.dtype, a.batch, a.k_len, a.kv_heads); };
    const bool v = a.dim % (a.dtype == GS_TABLE_F32 ? 4 : 8) == 0 && on_q(a.q) && on_k(a.k) && on_k(a.v);
    if (backward) return v && on_q(a.dout) && on_q(a.dq) && on_k(a.dk) && on_k(a.dv);
    return v && on_q(a.out);
}

static WalkMask mask_of(int left, int right)
{
    WalkMask m = {};
    m.left = left;
    m.right = right;
    for (int d = -7; d <= 7; ++d) {
        const int lo = 16 * d - 15, hi = 16 * d + 15;        // distances of the block's corners from the diagonal
        const bool whole = (left < 0 || lo >= -left) && (right < 0 || hi <= right);
        const bool some = (left < 0 || hi >= -left) && (right < 0 || lo <= right);
        m.slot[d + 7] = -1;
        if (some && !whole) {                                // at most two such blocks at each end of the window
            m.slot[d + 7] = (signed char)m.n;
            m.dist[m.n++] = (signed char)d;
        }
    }
    return m;
}

template <int K, int DP, bool BWD>
static gs_status launch(const AttnArgs &a, cudaStream_t st)
{
    WalkPlan plan;
    plan.rows = mask_of(a.left, a.right);
    plan.cols = mask_of(a.right, a.left);
    plan.qt = (a.q_len + 15) / 16;
    plan.kt = (a.k_len + 15) / 16;
    plan.tma = all_tma(a, BWD);
    plan.vec = rows_of_16_bytes(a, BWD);
    const int tiles = BWD && plan.kt > plan.qt ? plan.kt : plan.qt;
    const int64_t total = a.batch * (BWD ? a.kv_heads : a.q_heads);
    if (total == 0) return GS_OK;
    if (total > 0x3FFFFFFF) {
        set_error("attention of %lld sequence heads exceeds one launch", (long long)total);
        return GS_ERR_UNSUPPORTED;
    }
    WalkMaps m;
    if (plan.tma) {
        constexpr int BOX = Row<K, DP>::VALUES;
        auto on_q = [&](CUtensorMap *t, const AttnTensor &x, int rows) {
            return attn_tensor_map(t, x, a.dtype, a.batch, a.q_len, a.q_heads, a.dim, BOX, rows);
        };
        auto on_k = [&](CUtensorMap *t, const AttnTensor &x, int rows) {
            return attn_tensor_map(t, x, a.dtype, a.batch, a.k_len, a.kv_heads, a.dim, BOX, rows);
        };
        gs_status s = GS_OK;
        if ((s = on_q(&m.q, a.q, plan.qt * 16)) != GS_OK || (s = on_k(&m.k, a.k, plan.kt * 16)) != GS_OK ||
            (s = on_k(&m.v, a.v, plan.kt * 16)) != GS_OK || (s = on_q(&m.out, BWD ? a.dq : a.out, 16)) != GS_OK)
            return s;
        if (BWD && ((s = on_q(&m.dout, a.dout, plan.qt * 16)) != GS_OK || (s = on_k(&m.dk, a.dk, 16)) != GS_OK ||
                    (s = on_k(&m.dv, a.dv, 16)) != GS_OK))
            return s;
    }
    const int unit = (BWD ? 2 : 1) * (int)Row<K, DP>::tile(plan.qt) + 2 * (int)Row<K, DP>::tile(plan.kt);
    const int stats = BWD ? (int)stat_bytes(plan.qt) : 0;
    const int masks = (int)(mask_bytes(plan.rows.n) + (BWD ? mask_bytes(plan.cols.n) : 0));
    // two sets of tiles if one unit leaves room for the resident blocks, and as many units as the block's warps
    // and that room allow
    const int room = (227 * 1024) / blocks_per_sm<K, DP, BWD>() - 2048;
    plan.stages = plan.tma && 2 * unit + stats + masks <= room ? 2 : 1;
    const int per_unit = plan.stages * unit + stats;
    plan.units = BLOCK_WARPS / tiles;
    while (plan.units > 1 && plan.units * per_unit + masks > room) --plan.units;
    if (plan.units < 1) plan.units = 1;
    const int smem = plan.units * per_unit + masks;
    auto kernel = !BWD ? attn_walk_forward_kernel<K, DP>
                       : a.group > 1 ? attn_walk_backward_kernel<K, DP, true> : attn_walk_backward_kernel<K, DP, false>;
    static SharedRecord record[2];
    gs_status s = allow_shared(kernel, smem, record[BWD && a.group > 1]);
    if (s != GS_OK) return s;
    const int threads = plan.units * tiles * 32;
    // blocks that an SM holds, by shared memory (1 KB and the static variables on top) and by registers
    const int by_shared = 228 * 1024 / (smem + 2048), by_registers = 65536 / (registers<K, DP, BWD>() * threads);
    const int resident = by_shared < by_registers ? by_shared : by_registers;
    const int64_t blocks = (total + plan.units - 1) / plan.units, most = (int64_t)sm_count() * (resident > 0 ? resident : 1);
    kernel<<<(unsigned)(blocks < most ? blocks : most), threads, smem, st>>>(a, plan, m, stall_counter());
    GS_CUDA_TRY(cudaGetLastError());
    return GS_OK;
}

template <int K, bool BWD>
static gs_status by_dim(const AttnArgs &a, cudaStream_t st)
{
    if (K != F32 && a.dim <= 16) return launch<K, K == F32 ? 32 : 16, BWD>(a, st);
    if (a.dim <= 32) return launch<K, 32, BWD>(a, st);
    if (a.dim <= 64) return launch<K, 64, BWD>(a, st);
    return launch<K, 128, BWD>(a, st);
}

// bytes of one head's tiles, which have to fit one block (fp32 with 128 columns does up to 96 positions backward)
static int64_t head_bytes(const AttnArgs &a, bool backward)
{
    const int64_t row = (a.dtype == GS_TABLE_F32 ? 4 : 2) * (a.dim <= 32 ? 32 : a.dim <= 64 ? 64 : 128);
    return row * ((backward ? 2 : 1) * ((a.q_len + 15) / 16 * 16) + 2 * ((a.k_len + 15) / 16 * 16));
}

bool attn_walk_ok(const AttnArgs &a, bool backward)
{
    return a.q_len > 0 && a.k_len > 0 && a.q_len <= 128 && a.k_len <= 128 && head_bytes(a, backward) <= 208 * 1024;
}
gs_status attn_walk_forward(const AttnArgs &a, cudaStream_t st)
{
    if (a.dtype == GS_TABLE_F32) return by_dim<F32, false>(a, st);
    return a.dtype == GS_TABLE_BF16 ? by_dim<BF16, false>(a, st) : by_dim<F16, false>(a, st);
}
gs_status attn_walk_backward(const AttnArgs &a, cudaStream_t st)
{
    if (a.dtype == GS_TABLE_F32) return by_dim<F32, true>(a, st);
    return a.dtype == GS_TABLE_BF16 ? by_dim<BF16, true>(a, st) : by_dim<F16, true>(a, st);
}

}  // namespace gs
