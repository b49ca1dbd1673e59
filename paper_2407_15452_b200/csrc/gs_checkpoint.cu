// Activations in 8 bits: packing and unpacking.
//
// A block of 128 columns is held by 16 or 32 lanes, 16 bytes of values each (or, where rows are not aligned to that, by a warp,
// one value at a time), so that its largest magnitude is a few shuffles and every value is read once.  Bound: memory traffic; 16384 x 4096
// there and back take 110 us in fp32 (6.1 TB/s) and 75 in bf16 (5.4 TB/s; packing is the slower half, its issue slots 70 % busy).
#include "gs_norm.cuh"

namespace gs {

static constexpr int PACK_THREADS = 256, PACK_BLOCKS = 8;             // blocks of an SM

struct PackArgs {
    NormRows x;
    int8_t *packed;
    float *scales;
    const int32_t *lens;
    Divider by_blocks, by_length;
    int64_t rows, length, columns, blocks_of_row, blocks;              // blocks: of 128 columns, in all
};

// Lanes that hold a block of columns, and values of a lane's access.  FLAT: blocks follow one another in memory.
template <typename T, bool ALIGNED> struct Holders {
    static constexpr int VEC = ALIGNED ? Wide<T>::N : 1, LANES = ALIGNED ? KEPT_BLOCK / VEC : 32, PIECES = KEPT_BLOCK / VEC / LANES;
    static constexpr int N = VEC % 2 ? VEC : VEC / 2, AT_ONCE = ALIGNED ? 4 : 2;     // neighbouring blocks that a group of lanes has under way
};

struct BlockAt {
    int64_t i, row, k, b, t;                                           // k: of the row's blocks

    __device__ __forceinline__ BlockAt(const PackArgs &a, int64_t first) : i(first)
    {
        if (i >= a.blocks) i = a.blocks;
        row = a.by_blocks.of(i);
        k = i - row * a.blocks_of_row;
        b = a.by_length.of(row);
        t = row - b * a.length;
    }
    __device__ __forceinline__ void next(const PackArgs &a)
    {
        ++i;
        if (++k < a.blocks_of_row) return;
        k = 0;
        ++row;
        if (++t < a.length) return;
        t = 0;
        ++b;
    }
    __device__ __forceinline__ bool there(const PackArgs &a) const { return i < a.blocks; }
};

template <typename T, bool ALIGNED, bool FLAT>
__global__ void __launch_bounds__(PACK_THREADS) pack_kernel(const __grid_constant__ PackArgs a)
{
    typedef Holders<T, ALIGNED> H;
    typedef Piece<T, H::VEC> P;
    typedef typename P::raw raw;
    typedef typename Kept<H::VEC>::raw kept;
    const int member = threadIdx.x % H::LANES, at = member * H::VEC;
    const int64_t step = (int64_t)gridDim.x * (PACK_THREADS / H::LANES) * H::AT_ONCE;
    // the same number of rounds for all lanes of a warp: they reduce together
    for (int64_t i0 = (int64_t)blockIdx.x * (PACK_THREADS / H::LANES) * H::AT_ONCE; i0 < a.blocks; i0 += step) {
        const int64_t first = i0 + threadIdx.x / H::LANES * H::AT_ONCE;
        raw r[H::AT_ONCE][H::PIECES];
        BlockAt p(a, FLAT ? 0 : first);
#pragma unroll
        for (int u = 0; u < H::AT_ONCE; ++u) {
            if (FLAT) {
                const T *from = static_cast<const T *>(a.x.p) + first * KEPT_BLOCK + at;
                r[u][0] = first + u < a.blocks ? *reinterpret_cast<const raw *>(from + u * KEPT_BLOCK) : P::none();
                continue;
            }
            const bool live = p.there(a) && (!a.lens || p.t < __ldg(a.lens + p.b));
            const T *row = static_cast<const T *>(a.x.p) + p.b * a.x.sb + p.t * a.x.st;
#pragma unroll
            for (int k = 0; k < H::PIECES; ++k) {
                const int64_t c = p.k * KEPT_BLOCK + k * H::LANES * H::VEC + at;
                r[u][k] = live && c < a.columns ? *reinterpret_cast<const raw *>(row + c) : P::none();
            }
            p.next(a);
        }
        BlockAt w(a, FLAT ? 0 : first);
#pragma unroll
        for (int u = 0; u < H::AT_ONCE; ++u) {
            typename P::F f[H::PIECES][H::N];
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < H::PIECES; ++k) {
                P::get(r[u][k], f[k]);
#pragma unroll
                for (int e = 0; e < H::N; ++e) top = max(top, magnitude(f[k][e]));
            }
            const KeptScale scale(largest<H::LANES>(top));
            uint32_t q[H::PIECES][H::VEC];
#pragma unroll
            for (int k = 0; k < H::PIECES; ++k) scale.of(f[k], q[k]);
            if (FLAT) {
                if (first + u < a.blocks) {
                    *reinterpret_cast<kept *>(a.packed + (first + u) * KEPT_BLOCK + at) = Kept<H::VEC>::put(q[0]);
                    if (member == 0) a.scales[first + u] = scale.s;
                }
                continue;
            }
            if (w.there(a)) {
#pragma unroll
                for (int k = 0; k < H::PIECES; ++k) {
                    const int64_t c = w.k * KEPT_BLOCK + k * H::LANES * H::VEC + at;
                    if (c < a.columns) *reinterpret_cast<kept *>(a.packed + w.row * a.columns + c) = Kept<H::VEC>::put(q[k]);
                }
                if (member == 0) a.scales[w.i] = scale.s;
            }
            w.next(a);
        }
    }
}

template <typename T, bool ALIGNED, bool FLAT>
__global__ void __launch_bounds__(PACK_THREADS) unpack_kernel(const __grid_constant__ PackArgs a)
{
    typedef Holders<T, ALIGNED> H;
    typedef Piece<T, H::VEC> P;
    typedef typename P::raw raw;
    typedef typename Kept<H::VEC>::raw kept;
    const int at = threadIdx.x % H::LANES * H::VEC;
    const int64_t step = (int64_t)gridDim.x * (PACK_THREADS / H::LANES) * H::AT_ONCE;
    for (int64_t first = ((int64_t)blockIdx.x * (PACK_THREADS / H::LANES) + threadIdx.x / H::LANES) * H::AT_ONCE; first < a.blocks;
         first += step) {
        kept r[H::AT_ONCE][H::PIECES];
        float s[H::AT_ONCE];
        BlockAt p(a, FLAT ? 0 : first);
#pragma unroll
        for (int u = 0; u < H::AT_ONCE; ++u) {
            const bool on = first + u < a.blocks;
            s[u] = on ? a.scales[first + u] : 0.0f;
            if (FLAT) {
                r[u][0] = on ? *reinterpret_cast<const kept *>(a.packed + (first + u) * KEPT_BLOCK + at) : Kept<H::VEC>::none();
                continue;
            }
#pragma unroll
            for (int k = 0; k < H::PIECES; ++k) {
                const int64_t c = p.k * KEPT_BLOCK + k * H::LANES * H::VEC + at;
                r[u][k] = on && c < a.columns ? *reinterpret_cast<const kept *>(a.packed + p.row * a.columns + c) : Kept<H::VEC>::none();
            }
            p.next(a);
        }
        BlockAt w(a, FLAT ? 0 : first);
#pragma unroll
        for (int u = 0; u < H::AT_ONCE; ++u) {
            if (first + u >= a.blocks) break;
            T *row = static_cast<T *>(a.x.p) + (FLAT ? (first + u) * KEPT_BLOCK : w.row * a.x.st);
#pragma unroll
            for (int k = 0; k < H::PIECES; ++k) {
                const int64_t c = (FLAT ? 0 : w.k * KEPT_BLOCK) + k * H::LANES * H::VEC + at;
                typename P::F f[H::N];
                Kept<H::VEC>::get(r[u][k], s[u], f);
                if (FLAT || c < a.columns) *reinterpret_cast<raw *>(row + c) = P::put(f);
            }
            w.next(a);
        }
    }
}

template <typename T, bool ALIGNED, bool FLAT>
static gs_status launch(const PackArgs &a, bool pack, cudaStream_t st)
{
    typedef Holders<T, ALIGNED> H;
    const int64_t each = (int64_t)(PACK_THREADS / H::LANES) * H::AT_ONCE, blocks = (a.blocks + each - 1) / each;
    const int64_t most = (int64_t)sm_count() * PACK_BLOCKS * 4;
    const unsigned grid = (unsigned)(blocks < most ? blocks : most);
    if (pack) pack_kernel<T, ALIGNED, FLAT><<<grid, PACK_THREADS, 0, st>>>(a);
    else unpack_kernel<T, ALIGNED, FLAT><<<grid, PACK_THREADS, 0, st>>>(a);
    GS_CUDA_TRY(cudaGetLastError());
    return GS_OK;
}

static gs_status run(int32_t dtype, const NormRows &x, const int32_t *lens, int64_t batch, int64_t length, int64_t columns, int8_t *packed,
                     float *scales, bool pack, cudaStream_t st)
{
    PackArgs a = {};
    a.x = x;
    a.packed = packed;
    a.scales = scales;
    a.lens = lens;
    a.rows = batch * length;
    a.length = length;
    a.columns = columns;
    a.blocks_of_row = (columns + KEPT_BLOCK - 1) / KEPT_BLOCK;
    a.blocks = a.rows * a.blocks_of_row;
    a.by_blocks = Divider(a.blocks_of_row);
    a.by_length = Divider(length);
    const int64_t es = (int64_t)size_of(dtype);
    const bool aligned = columns * es % 16 == 0 && (uintptr_t)x.p % 16 == 0 && (x.sb * es | x.st * es) % 16 == 0 && (uintptr_t)packed % 8 == 0;
    const bool flat = aligned && columns % KEPT_BLOCK == 0 && !lens && (length <= 1 || x.st == columns) && (batch <= 1 || x.sb == length * columns);
    return with_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        return flat ? launch<T, true, true>(a, pack, st) : aligned ? launch<T, true, false>(a, pack, st) : launch<T, false, false>(a, pack, st);
    });
}

gs_status checkpoint_pack(int32_t dtype, const NormRows &x, const int32_t *lens, int64_t batch, int64_t length, int64_t columns,
                          int8_t *packed, float *scales, cudaStream_t st)
{
    return run(dtype, x, lens, batch, length, columns, packed, scales, true, st);
}

static gs_status entry(int32_t dtype, const void *x, int64_t rows, int64_t columns, int64_t row_stride, const int8_t *packed,
                       const float *scales, bool pack, void *stream)
{
    if (!known_type(dtype)) return bad("dtype must be GS_TABLE_F32, GS_TABLE_F16 or GS_TABLE_BF16");
    if (rows < 0 || columns < 0) return bad("negative number of rows or columns");
    if (rows > ((int64_t)1 << 40) || columns > 0x7FFFFFFF || (columns > 0 && rows > ((int64_t)1 << 46) / columns)) {
        set_error("checkpoints of up to 2^40 rows, 2^31 - 1 columns and 2^46 values are supported");
        return GS_ERR_UNSUPPORTED;
    }
    if (rows == 0 || columns == 0) return GS_OK;
    if (!x || !packed || !scales) return bad("null pointer");
    if ((uintptr_t)x % size_of(dtype) || (uintptr_t)scales % 4) return bad("tensor not aligned to its element size");
    if (!pack && rows > 1 && row_stride == 0) return bad("an output has a zero stride");
    const NormRows r = {const_cast<void *>(x), 0, row_stride, 0, 0};
    return run(dtype, r, nullptr, 1, rows, columns, const_cast<int8_t *>(packed), const_cast<float *>(scales), pack, (cudaStream_t)stream);
}

}  // namespace gs

using namespace gs;

extern "C" {

gs_status gs_checkpoint_pack(int32_t dtype, const void *d_x, int64_t rows, int64_t columns, int64_t row_stride, int8_t *d_packed,
                             float *d_scales, void *stream)
{
    return entry(dtype, d_x, rows, columns, row_stride, d_packed, d_scales, true, stream);
}

gs_status gs_checkpoint_unpack(int32_t dtype, const int8_t *d_packed, const float *d_scales, int64_t rows, int64_t columns,
                               int64_t row_stride, void *d_x, void *stream)
{
    return entry(dtype, d_x, rows, columns, row_stride, d_packed, d_scales, false, stream);
}

}  // extern "C"
