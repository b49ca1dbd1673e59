// Shared pieces of the layers around attention: element types, rows of [batch][length][columns] tensors, and
// the 8-bit form of activations.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "gs_common.cuh"
#include "gs_tc.cuh"

namespace gs {

inline gs_status bad(const char *what)
{
    set_error("invalid argument: %s", what);
    return GS_ERR_INVALID_ARG;
}
inline bool known_type(int32_t t) { return t == GS_TABLE_F32 || t == GS_TABLE_F16 || t == GS_TABLE_BF16; }
inline size_t size_of(int32_t t) { return t == GS_TABLE_F32 ? 4 : 2; }

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// two 16-bit values of a word, the first in its lower half
template <typename T> __device__ __forceinline__ void unpack2(uint32_t u, float &a, float &b);
template <> __device__ __forceinline__ void unpack2<__half>(uint32_t u, float &a, float &b)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&u));
    a = f.x;
    b = f.y;
}
template <> __device__ __forceinline__ void unpack2<__nv_bfloat16>(uint32_t u, float &a, float &b)
{
    a = __uint_as_float(u << 16);
    b = __uint_as_float(u & 0xFFFF0000u);
}
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// One value, or two neighbours that one instruction works on
template <int V> struct Vec;
template <> struct Vec<1> { typedef float type; };
template <> struct Vec<2> { typedef float2 type; };
__device__ __forceinline__ float fma_of(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ float2 fma_of(float2 a, float2 b, float2 c) { return tc::fma2(a, b, c); }
__device__ __forceinline__ float mul_of(float a, float b) { return a * b; }
__device__ __forceinline__ float2 mul_of(float2 a, float2 b) { return tc::mul2(a, b); }
__device__ __forceinline__ float add_of(float a, float b) { return a + b; }
__device__ __forceinline__ float2 add_of(float2 a, float2 b) { return tc::add2(a, b); }
__device__ __forceinline__ float sum_of(float a) { return a; }
__device__ __forceinline__ float sum_of(float2 a) { return a.x + a.y; }
template <int V> __device__ __forceinline__ typename Vec<V>::type all_of(float x)
{
    if constexpr (V == 1) return x;
    else return make_float2(x, x);
}

// N neighbouring elements as one access moves them, 16 bytes, or one element where rows are not aligned to that; in fp32 they are N / V
// pairs (or one value)
template <typename T, int N> struct Piece;
template <> struct Piece<float, 4> {
    typedef float4 raw;
    typedef float2 F;
    static __device__ __forceinline__ raw none() { return make_float4(0.f, 0.f, 0.f, 0.f); }
    static __device__ __forceinline__ void get(raw r, F (&f)[2])
    {
        f[0] = make_float2(r.x, r.y);
        f[1] = make_float2(r.z, r.w);
    }
    static __device__ __forceinline__ raw put(const F (&f)[2]) { return make_float4(f[0].x, f[0].y, f[1].x, f[1].y); }
};
template <typename T> struct Piece<T, 8> {
    typedef uint4 raw;
    typedef float2 F;
    static __device__ __forceinline__ raw none() { return make_uint4(0u, 0u, 0u, 0u); }
    static __device__ __forceinline__ void get(raw r, F (&f)[4])
    {
        unpack2<T>(r.x, f[0].x, f[0].y);
        unpack2<T>(r.y, f[1].x, f[1].y);
        unpack2<T>(r.z, f[2].x, f[2].y);
        unpack2<T>(r.w, f[3].x, f[3].y);
    }
    static __device__ __forceinline__ raw put(const F (&f)[4])
    {
        return make_uint4(pack2<T>(f[0].x, f[0].y), pack2<T>(f[1].x, f[1].y), pack2<T>(f[2].x, f[2].y), pack2<T>(f[3].x, f[3].y));
    }
};
template <typename T> struct Piece<T, 1> {
    typedef T raw;
    typedef float F;
    static __device__ __forceinline__ raw none() { return from_float<T>(0.f); }
    static __device__ __forceinline__ void get(raw r, F (&f)[1]) { f[0] = to_float(r); }
    static __device__ __forceinline__ raw put(const F (&f)[1]) { return from_float<T>(f[0]); }
};
template <typename T> struct Wide;                    // elements of a 16-byte access
template <> struct Wide<float> { static constexpr int N = 4; };
template <> struct Wide<__half> { static constexpr int N = 8; };
template <> struct Wide<__nv_bfloat16> { static constexpr int N = 8; };

// calls f(T()) with the type of a dtype
template <typename F>
static gs_status with_type(int32_t dtype, F &&f)
{
    if (dtype == GS_TABLE_F32) return f(float());
    if (dtype == GS_TABLE_F16) return f(__half());
    return f(__nv_bfloat16());
}

// ---- rows -------------------------------------------------------------------------------
// n / d for n < 2^31 as a multiplication: m = floor(2^(31+s) / d) + 1 with 2^s >= d, so that n m / 2^(31+s) exceeds
// n / d by less than n / 2^(31+s) <= 1 / d and has the same whole part.
struct Divider {
    uint32_t m, shift;
    int64_t d;
    Divider(int64_t by = 1) : m(0), shift(0), d(by)
    {
        if (by > 1 && by < ((int64_t)1 << 31)) {
            while (((int64_t)1 << shift) < by) ++shift;
            m = (uint32_t)((((uint64_t)1 << (31 + shift)) / (uint64_t)by) + 1);
        }
    }
    __device__ __forceinline__ int64_t of(int64_t n) const
    {
        if (d == 1) return n;
        if (m && n < ((int64_t)1 << 31)) return __umulhi((uint32_t)n, m) >> (shift - 1);
        return n / d;
    }
};

// ---- activations in 8 bits ------------------------------------------------------------------
static constexpr int KEPT_BLOCK = 128;                // columns that share a scale

// Largest magnitude of a block as bits of |x|: as whole numbers these order finite values like the values, and infinities and
// NaN above all of them, which a maximum of floats would let go.
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t magnitude(float2 x) { return max(magnitude(x.x), magnitude(x.y)); }
template <int LANES>
__device__ __forceinline__ uint32_t largest(uint32_t m)
{
    // a whole warp in one instruction (16384 x 4096 fp32 there and back 112 -> 110 us); of the halves of one, they take turns (bf16 75 -> 78)
    if constexpr (LANES == 32) return __reduce_max_sync(0xffffffffu, m);
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
}

// The whole number nearest to x / s, as the low byte of its sum with WHOLE (a sum in which the last place is one).  x times a rounded reciprocal,
// rounded to a whole number q, is at most one off; what remains, x - q s, is a multiple of the smaller operand's last place below s in magnitude
// and so exact in one multiply-add, and where it is not below s / 2 the slow way decides, ties to even: hardly ever.  The same way
// go blocks of magnitudes whose reciprocal is not finite or whose scale is subnormal (and q possibly beyond 127), scaled up by a power of two.
static constexpr float WHOLE = 12582912.0f;           // 1.5 * 2^23
struct KeptScale {
    float s, inverse, half;
    bool slow;
    __device__ __forceinline__ explicit KeptScale(uint32_t top)
    {
        const float t = __uint_as_float(top);
        // t / 127 towards zero: t times 1 / 127 as fp32 has it (2^-27 off) is one of the two neighbours of t / 127, and the exact sign of
        // 127 s - t tells which
        s = t * (1.0f / 127.0f);
        if (fmaf(s, 127.0f, -t) > 0.0f) s = __uint_as_float(__float_as_uint(s) - 1u);
        slow = top - 0x21800000u >= 0x5E000000u;      // below 2^-60, or not finite
        if (slow) s = top >= 0x7F800000u ? __uint_as_float(0x7FFFFFFFu) : __fdiv_rd(t, 127.0f);
        inverse = tc::rcp_fast(s);
        half = 0.5f * s;
    }
    __device__ __forceinline__ uint32_t slowly(float x) const
    {
        if (!(s > 0.0f)) return 0u;
        const float up = slow ? 1.20892582e24f : 1.0f, v = x * up, step = s * up;                  // 2^80
        float q = rintf(v * __frcp_rn(step));
        const float left = fmaf(-q, step, v), over = fabsf(left) - 0.5f * step;
        if (over > 0.0f || (over == 0.0f && ((int)q & 1))) q += copysignf(1.0f, left);
        return (uint32_t)(int)fminf(fmaxf(q, -127.0f), 127.0f);
    }
    // words whose low bytes are the numbers; returns the largest |x - q s|
    __device__ __forceinline__ float fast(float x, uint32_t (&q)[1]) const
    {
        const float t = fmaf(x, inverse, WHOLE);
        q[0] = __float_as_uint(t);
        return fabsf(fmaf(t - WHOLE, -s, x));
    }
    __device__ __forceinline__ float fast(float2 x, uint32_t (&q)[2]) const
    {
        const float2 t = tc::fma2(x, make_float2(inverse, inverse), make_float2(WHOLE, WHOLE));
        q[0] = __float_as_uint(t.x);
        q[1] = __float_as_uint(t.y);
        const float2 left = tc::fma2(tc::add2(t, make_float2(-WHOLE, -WHOLE)), make_float2(-s, -s), x);
        return fmaxf(fabsf(left.x), fabsf(left.y));
    }
    template <typename F, int N, int M>
    __device__ __forceinline__ void of(const F (&x)[N], uint32_t (&q)[M]) const
    {
        constexpr int V = M / N;
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint32_t w[V];
            most = fmaxf(most, fast(x[i], w));
#pragma unroll
            for (int v = 0; v < V; ++v) q[i * V + v] = w[v];
        }
        if (!slow && most < half) return;
        const float *one = reinterpret_cast<const float *>(x);
#pragma unroll
        for (int e = 0; e < M; ++e) q[e] = slowly(one[e]);
    }
};

// N neighbouring 8-bit values, and what they stand for
template <int N> struct Kept;
template <> struct Kept<4> {
    typedef uint32_t raw;
    static __device__ __forceinline__ raw none() { return 0u; }
    static __device__ __forceinline__ raw put(const uint32_t (&q)[4])
    {
        return __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
    }
    // a byte b under the exponent of 2^23 is 2^23 + b, and b = q + 128
    static __device__ __forceinline__ float2 two(uint32_t bytes, uint32_t first, float scale)
    {
        const float2 f = make_float2(__uint_as_float(__byte_perm(bytes, 0x4B000000u, 0x7440u | first)),
                                     __uint_as_float(__byte_perm(bytes, 0x4B000000u, 0x7440u | (first + 1))));
        return tc::mul2(tc::add2(f, make_float2(-8388736.0f, -8388736.0f)), make_float2(scale, scale));
    }
    static __device__ __forceinline__ void get(raw r, float scale, float2 (&f)[2])
    {
        const uint32_t bytes = r ^ 0x80808080u;
        f[0] = two(bytes, 0, scale);
        f[1] = two(bytes, 2, scale);
    }
};
template <> struct Kept<8> {
    typedef uint2 raw;
    static __device__ __forceinline__ raw none() { return make_uint2(0u, 0u); }
    static __device__ __forceinline__ raw put(const uint32_t (&q)[8])
    {
        return make_uint2(Kept<4>::put({q[0], q[1], q[2], q[3]}), Kept<4>::put({q[4], q[5], q[6], q[7]}));
    }
    static __device__ __forceinline__ void get(raw r, float scale, float2 (&f)[4])
    {
        const uint32_t a = r.x ^ 0x80808080u, b = r.y ^ 0x80808080u;
        f[0] = Kept<4>::two(a, 0, scale);
        f[1] = Kept<4>::two(a, 2, scale);
        f[2] = Kept<4>::two(b, 0, scale);
        f[3] = Kept<4>::two(b, 2, scale);
    }
};
template <> struct Kept<1> {
    typedef int8_t raw;
    static __device__ __forceinline__ raw none() { return 0; }
    static __device__ __forceinline__ raw put(const uint32_t (&q)[1]) { return (int8_t)q[0]; }
    static __device__ __forceinline__ void get(raw r, float scale, float (&f)[1]) { f[0] = (float)r * scale; }
};

}  // namespace gs
