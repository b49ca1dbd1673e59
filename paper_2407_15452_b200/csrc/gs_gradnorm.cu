// Global gradient norm over many tensors, and clipping by it.
//
//   norm = sqrt(sum over all tensors and elements of g^2),  out = g * factor,
//   factor = max_norm / norm if norm > max_norm and norm is finite, else 1.
//
// The tensors travel in the kernel's parameters (no device-side list to upload or to keep).  All of
// them are cut into chunks of 4096 elements; the blocks of a grid take chunks round robin, so
// one large matrix and hundreds of small vectors load the SMs alike, and the order of every sum is
// fixed by the gradients' sizes, types and alignment (and the number of SMs), whatever they are scaled into: results are
// bitwise repeatable, and the norm alone is the clipping call's norm.  Squares are summed in fp32 over the 16 elements that
// a thread takes of a chunk (18 in a tensor's ragged first or last one) and in fp64 from there on.  Bound: memory
// traffic.  The second pass runs backwards and finds the last of the first's reads in L2.
#include <math.h>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gs_common.cuh"

namespace gs {

static constexpr int NT = 256, UNROLL = 4, CHUNK = NT * 4 * UNROLL;
// Resident blocks of an SM, and how many times as many the grids have: a pass in one round of blocks, each with its
// fixed share, waits for the slowest.  Measured over two fp32 tensors of 128M elements: one round 163 + 381 us, 4
// and 16 rounds 158 + 319 us (a copy of the same bytes: 317 us); the sums take fewer because each leaves a partial sum.
static constexpr int RESIDENT = 8, ROUNDS_SUM = 4, ROUNDS_SCALE = 16;

struct GradTensor {
    const void *in;
    void *out;
    int64_t n;
};

template <int CAP>
struct GradList {
    GradTensor t[CAP];
    int32_t first[CAP + 1];          // first chunk of each tensor; first[count] = number of chunks
    uint8_t in_type[CAP], out_type[CAP];
    uint8_t head[CAP];               // elements before what a pass accesses is 16-byte aligned; 255: never all of it
    int32_t count;
};

// Four elements a thread and access: 16 bytes of fp32 or 8 of a 16-bit type, so that a warp's access is one
// contiguous piece in either, also where gradients and outputs differ in type (eight elements a thread leave
// every second 16 bytes of an fp32 access to the next one: 394 instead of 331 us for a pass over 256M fp32 elements)
__device__ __forceinline__ void unpack4(const float *p, float (&f)[4])
{
    const float4 a = *reinterpret_cast<const float4 *>(p);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
}
__device__ __forceinline__ void unpack4(const __half *p, float (&f)[4])
{
    uint2 u = *reinterpret_cast<const uint2 *>(p);
    const float2 a = __half22float2(*reinterpret_cast<__half2 *>(&u.x)), b = __half22float2(*reinterpret_cast<__half2 *>(&u.y));
    f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y;
}
__device__ __forceinline__ void unpack4(const __nv_bfloat16 *p, float (&f)[4])
{
    const uint2 u = *reinterpret_cast<const uint2 *>(p);
    f[0] = __uint_as_float(u.x << 16); f[1] = __uint_as_float(u.x & 0xFFFF0000u);
    f[2] = __uint_as_float(u.y << 16); f[3] = __uint_as_float(u.y & 0xFFFF0000u);
}

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }

__device__ __forceinline__ void put(float *p, float x) { *p = x; }
__device__ __forceinline__ void put(__half *p, float x) { *p = __float2half_rn(x); }
__device__ __forceinline__ void put(__nv_bfloat16 *p, float x) { *p = __float2bfloat16_rn(x); }

__device__ __forceinline__ void pack4(float *p, const float (&f)[4])
{
    *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
}
__device__ __forceinline__ void pack4(__half *p, const float (&f)[4])
{
    __half2 h[2] = {__floats2half2_rn(f[0], f[1]), __floats2half2_rn(f[2], f[3])};
    *reinterpret_cast<uint2 *>(p) = *reinterpret_cast<uint2 *>(h);
}
__device__ __forceinline__ void pack4(__nv_bfloat16 *p, const float (&f)[4])
{
    __nv_bfloat162 h[2] = {__floats2bfloat162_rn(f[0], f[1]), __floats2bfloat162_rn(f[2], f[3])};
    *reinterpret_cast<uint2 *>(p) = *reinterpret_cast<uint2 *>(h);
}

// tensor of a chunk: the last one whose first chunk is <= c
template <int CAP>
__device__ __forceinline__ int tensor_of(const GradList<CAP> &l, int c)
{
    int lo = 0, hi = l.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (l.first[mid] <= c) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// sum of squares of this thread's share of chunk `c` of a tensor
template <typename T>
__device__ __forceinline__ double squares(const T *p, int64_t n, int head, int64_t c)
{
    float s = 0.f;
    if (c == 0 && (int)threadIdx.x < head && (int64_t)threadIdx.x < n) {
        const float x = as_float(p[threadIdx.x]);
        s = fmaf(x, x, s);
    }
    const T *q = p + head + c * CHUNK;
    const int64_t rest = n - head - c * CHUNK;
    if (rest >= CHUNK) {
        float f[UNROLL][4];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) unpack4(q + (u * NT + threadIdx.x) * 4, f[u]);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) s = fmaf(f[u][i], f[u][i], s);
    } else if (rest > 0) {
        const int m = (int)rest, groups = m >> 2;
        for (int e = threadIdx.x; e < groups; e += NT) {
            float f[4];
            unpack4(q + e * 4, f);
#pragma unroll
            for (int i = 0; i < 4; ++i) s = fmaf(f[i], f[i], s);
        }
        if ((int)threadIdx.x < (m & 3)) {
            const float x = as_float(q[groups * 4 + threadIdx.x]);
            s = fmaf(x, x, s);
        }
    }
    return (double)s;
}

__device__ __forceinline__ double block_sum(double v, double *sh)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    double t = 0.0;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) t += sh[w];
    __syncthreads();
    return t;
}

template <int CAP>
__global__ void __launch_bounds__(NT, RESIDENT) grad_squares_kernel(const __grid_constant__ GradList<CAP> l, double *partial)
{
    __shared__ double sh[NT / 32];
    cudaTriggerProgrammaticLaunchCompletion();           // the next kernel may take up its place and wait
    double s = 0.0;
    const int chunks = l.first[l.count];
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int t = tensor_of(l, c);
        const int64_t k = c - l.first[t];
        const int head = l.head[t];
        if (l.in_type[t] == GS_TABLE_F32) s += squares((const float *)l.t[t].in, l.t[t].n, head, k);
        else if (l.in_type[t] == GS_TABLE_F16) s += squares((const __half *)l.t[t].in, l.t[t].n, head, k);
        else s += squares((const __nv_bfloat16 *)l.t[t].in, l.t[t].n, head, k);
    }
    s = block_sum(s, sh);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// norm from the partial sums, in the same order in every block
__device__ __forceinline__ float norm_of(const double *partial, int n, double *sh)
{
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += NT) s += partial[i];
    return (float)sqrt(block_sum(s, sh));
}

__global__ void __launch_bounds__(NT) grad_norm_kernel(const double *partial, int n, float *norm)
{
    __shared__ double sh[NT / 32];
    cudaGridDependencySynchronize();
    const float v = norm_of(partial, n, sh);
    if (threadIdx.x == 0) *norm = v;
}

template <typename I, typename O>
__device__ __forceinline__ void scale_chunk(const I *p, O *o, int64_t n, int head, int64_t c, float factor)
{
    if (head == 255) {                                   // two sides that no shift aligns: element by element
        const int64_t at = c * CHUNK;
        const int m = (int)min((int64_t)CHUNK, n - at);
        for (int e = threadIdx.x; e < m; e += NT) put(o + at + e, as_float(p[at + e]) * factor);
        return;
    }
    if (c == 0 && (int)threadIdx.x < head && (int64_t)threadIdx.x < n)
        put(o + threadIdx.x, as_float(p[threadIdx.x]) * factor);
    const I *q = p + head + c * CHUNK;
    O *w = o + head + c * CHUNK;
    const int64_t rest = n - head - c * CHUNK;
    if (rest >= CHUNK) {
        float f[UNROLL][4];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) unpack4(q + (u * NT + threadIdx.x) * 4, f[u]);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[u][i] *= factor;
            pack4(w + (u * NT + threadIdx.x) * 4, f[u]);
        }
    } else if (rest > 0) {
        const int m = (int)rest, groups = m >> 2;
        for (int e = threadIdx.x; e < groups; e += NT) {
            float f[4];
            unpack4(q + e * 4, f);
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] *= factor;
            pack4(w + e * 4, f);
        }
        if ((int)threadIdx.x < (m & 3))
            put(w + groups * 4 + threadIdx.x, as_float(q[groups * 4 + threadIdx.x]) * factor);
    }
}

template <typename I>
__device__ __forceinline__ void scale_to(const I *p, void *o, int out_type, int64_t n, int head, int64_t c, float f)
{
    if (out_type == GS_TABLE_F32) scale_chunk(p, (float *)o, n, head, c, f);
    else if (out_type == GS_TABLE_F16) scale_chunk(p, (__half *)o, n, head, c, f);
    else scale_chunk(p, (__nv_bfloat16 *)o, n, head, c, f);
}

template <int CAP>
__global__ void __launch_bounds__(NT, RESIDENT) grad_scale_kernel(const __grid_constant__ GradList<CAP> l, const double *partial,
                                                        int n_partial, float max_norm, bool in_place, float *norm_out)
{
    __shared__ double sh[NT / 32];
    cudaGridDependencySynchronize();
    const float norm = norm_of(partial, n_partial, sh);
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
    const bool over = norm > max_norm && isfinite(norm);
    if (!over && in_place) return;
    const float factor = over ? max_norm / norm : 1.f;
    const int chunks = l.first[l.count];
    // backwards: the chunks that the sums read last are still in L2
    for (int c = chunks - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
        const int t = tensor_of(l, c);
        const int64_t k = c - l.first[t];
        const int head = l.head[t];
        const GradTensor &g = l.t[t];
        if (l.in_type[t] == GS_TABLE_F32) scale_to((const float *)g.in, g.out, l.out_type[t], g.n, head, k, factor);
        else if (l.in_type[t] == GS_TABLE_F16) scale_to((const __half *)g.in, g.out, l.out_type[t], g.n, head, k, factor);
        else scale_to((const __nv_bfloat16 *)g.in, g.out, l.out_type[t], g.n, head, k, factor);
    }
}

static size_t size_of(int32_t dtype) { return dtype == GS_TABLE_F32 ? 4 : 2; }

static int aligned_head(const gs_tensor &in, const gs_tensor &out)
{
    for (int h = 0; h < 8; ++h)
        if (((uintptr_t)in.d_data + h * size_of(in.dtype)) % 16 == 0 &&
            ((uintptr_t)out.d_data + h * size_of(out.dtype)) % 16 == 0)
            return h;
    return 255;
}

static constexpr int SMALL = 64, LARGE = 800;       // tensors per launch: 2.0 KB and 24.8 KB of parameters

// fills `l` from tensors [*at, n) for a pass from `in` to `out`, or over `in` alone if they are the same; advances *at.
// Returns the number of chunks.
template <int CAP>
static int fill(GradList<CAP> *l, const gs_tensor *in, const gs_tensor *out, int64_t n, int64_t *at)
{
    int64_t chunks = 0;
    l->count = 0;
    while (*at < n && l->count < CAP) {
        const gs_tensor &t = in[*at];
        const int64_t c = (t.numel + CHUNK - 1) / CHUNK;
        if (c > 0) {
            const int i = l->count++;
            l->t[i].in = t.d_data;
            l->t[i].out = out[*at].d_data;
            l->t[i].n = t.numel;
            l->in_type[i] = (uint8_t)t.dtype;
            l->out_type[i] = (uint8_t)out[*at].dtype;
            l->head[i] = (uint8_t)aligned_head(t, out[*at]);
            l->first[i] = (int32_t)chunks;
            chunks += c;
        }
        ++*at;
    }
    l->first[l->count] = (int32_t)chunks;
    return (int)chunks;
}

static int grid_for(int chunks, int rounds)
{
    const int cap = sm_count() * RESIDENT * rounds;
    return chunks < 1 ? 1 : chunks < cap ? chunks : cap;
}

static int64_t launches_of(int64_t n) { return n <= SMALL ? 1 : (n + LARGE - 1) / LARGE; }

template <int CAP>
static gs_status run(const gs_tensor *in, const gs_tensor *out, int64_t n, bool scale, float max_norm, double *work,
                     float *norm, cudaStream_t st)
{
    GradList<CAP> l;
    int64_t at = 0;
    int partials = 0;
    do {
        const int chunks = fill(&l, in, in, n, &at);
        const int grid = grid_for(chunks, ROUNDS_SUM);
        grad_squares_kernel<CAP><<<grid, NT, 0, st>>>(l, work + partials);
        GS_CUDA_TRY(cudaGetLastError());
        partials += grid;
    } while (at < n);
    if (!scale) {
        GS_CUDA_TRY(launch_after(grad_norm_kernel, 1, NT, 0, st, work, partials, norm));
        return GS_OK;
    }
    const bool in_place = in == out;
    at = 0;
    do {
        const int chunks = fill(&l, in, out, n, &at);
        const int grid = grid_for(chunks, ROUNDS_SCALE);
        GS_CUDA_TRY(launch_after(grad_scale_kernel<CAP>, grid, NT, 0, st, l, work, partials, max_norm, in_place, norm));
    } while (at < n);
    return GS_OK;
}

// Chunks of all tensors (2^42 elements): every index of a chunk, one grid past the last included, is an int
static constexpr int64_t MOST_CHUNKS = 1 << 30;

static gs_status check(const gs_tensor *t, int64_t n, const char *what)
{
    int64_t chunks = 0;
    for (int64_t i = 0; i < n; ++i) {
        const bool type_ok = t[i].dtype == GS_TABLE_F32 || t[i].dtype == GS_TABLE_F16 || t[i].dtype == GS_TABLE_BF16;
        if (!type_ok || t[i].numel < 0 || t[i].numel > MOST_CHUNKS * CHUNK || (t[i].numel > 0 && !t[i].d_data) ||
            (uintptr_t)t[i].d_data % size_of(t[i].dtype) != 0) {
            set_error("invalid argument: %s %lld has a bad type, size, pointer or alignment", what, (long long)i);
            return GS_ERR_INVALID_ARG;
        }
        chunks += (t[i].numel + CHUNK - 1) / CHUNK;
    }
    if (chunks > MOST_CHUNKS) {
        set_error("invalid argument: the tensors have more than 2^42 elements");
        return GS_ERR_INVALID_ARG;
    }
    return GS_OK;
}

static gs_status entry(const gs_tensor *in, const gs_tensor *out, int64_t n, bool scale, float max_norm, double *work,
                       float *norm, void *stream)
{
    if (n < 0 || n > (1 << 24) || (n > 0 && !in) || !work || !norm) {
        set_error("invalid argument: null pointer or a number of tensors outside [0, 2^24]");
        return GS_ERR_INVALID_ARG;
    }
    if (scale && !(max_norm >= 0.f && isfinite(max_norm))) {
        set_error("invalid argument: max_norm must be finite and >= 0");
        return GS_ERR_INVALID_ARG;
    }
    gs_status s = check(in, n, "gradient");
    if (s != GS_OK) return s;
    if (out) {
        if ((s = check(out, n, "output")) != GS_OK) return s;
        for (int64_t i = 0; i < n; ++i) {
            if (out[i].numel != in[i].numel) {
                set_error("invalid argument: output %lld has another size than its gradient", (long long)i);
                return GS_ERR_INVALID_ARG;
            }
            if (out[i].d_data == in[i].d_data && out[i].dtype != in[i].dtype && in[i].numel > 0) {
                set_error("invalid argument: output %lld is its gradient's buffer in another type", (long long)i);
                return GS_ERR_INVALID_ARG;
            }
        }
    }
    if (!out) out = in;
    if (n <= SMALL) return run<SMALL>(in, out, n, scale, max_norm, work, norm, (cudaStream_t)stream);
    return run<LARGE>(in, out, n, scale, max_norm, work, norm, (cudaStream_t)stream);
}

}  // namespace gs

using namespace gs;

extern "C" {

int64_t gs_gradient_norm_work(int64_t n_tensors)
{
    if (n_tensors < 0) return 0;
    return launches_of(n_tensors) * (int64_t)(sm_count() * RESIDENT * ROUNDS_SUM);
}

gs_status gs_gradient_norm(const gs_tensor *h_grads, int64_t n_tensors, double *d_work, float *d_norm, void *stream)
{
    return entry(h_grads, nullptr, n_tensors, false, 0.f, d_work, d_norm, stream);
}

gs_status gs_clip_gradients(const gs_tensor *h_grads, const gs_tensor *h_out, int64_t n_tensors, float max_norm,
                            double *d_work, float *d_norm, void *stream)
{
    return entry(h_grads, h_out, n_tensors, true, max_norm, d_work, d_norm, stream);
}

}  // extern "C"
