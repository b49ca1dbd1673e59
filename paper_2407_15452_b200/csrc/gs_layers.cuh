// Shared pieces of the layers around attention: element types, rows of [batch][length][columns] tensors, and
// the 8-bit form of activations.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gs_common.cuh"

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

// N neighbouring elements as one access moves them: 16 bytes, or one element where rows are not aligned to that
template <typename T, int N> struct Piece;
template <> struct Piece<float, 4> {
    typedef float4 raw;
    static __device__ __forceinline__ raw none() { return make_float4(0.f, 0.f, 0.f, 0.f); }
    static __device__ __forceinline__ void get(raw r, float (&f)[4]) { f[0] = r.x; f[1] = r.y; f[2] = r.z; f[3] = r.w; }
    static __device__ __forceinline__ raw put(const float (&f)[4]) { return make_float4(f[0], f[1], f[2], f[3]); }
};
template <typename T> struct Piece<T, 8> {
    typedef uint4 raw;
    static __device__ __forceinline__ raw none() { return make_uint4(0u, 0u, 0u, 0u); }
    static __device__ __forceinline__ void get(raw r, float (&f)[8])
    {
        unpack2<T>(r.x, f[0], f[1]);
        unpack2<T>(r.y, f[2], f[3]);
        unpack2<T>(r.z, f[4], f[5]);
        unpack2<T>(r.w, f[6], f[7]);
    }
    static __device__ __forceinline__ raw put(const float (&f)[8])
    {
        return make_uint4(pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3]), pack2<T>(f[4], f[5]), pack2<T>(f[6], f[7]));
    }
};
template <typename T> struct Piece<T, 1> {
    typedef T raw;
    static __device__ __forceinline__ raw none() { return from_float<T>(0.f); }
    static __device__ __forceinline__ void get(raw r, float (&f)[1]) { f[0] = to_float(r); }
    static __device__ __forceinline__ raw put(const float (&f)[1]) { return from_float<T>(f[0]); }
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
template <int LANES>
__device__ __forceinline__ uint32_t largest(uint32_t m)
{
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
}

// The whole number nearest to x / s.  The quotient by a rounded reciprocal is at most one off; what remains, x - q s, is a
// multiple of the smaller operand's last place below s in magnitude and so exact in one multiply-add, and its comparison with s / 2
// decides, ties to even.  Blocks of small values are scaled up by a power of two first, so that the reciprocal is finite.
struct KeptScale {
    float s, up, scaled, inverse;
    __device__ __forceinline__ explicit KeptScale(uint32_t top)
    {
        const float t = __uint_as_float(top);
        s = top >= 0x7F800000u ? __uint_as_float(0x7FFFFFFFu) : __fdiv_rd(t, 127.0f);
        up = t < 8.67361738e-19f ? 1.20892582e24f : 1.0f;             // 2^-60: 2^80
        scaled = s * up;
        inverse = s > 0.0f ? __frcp_rn(scaled) : 0.0f;                // s NaN: 0 as well
    }
    __device__ __forceinline__ int of(float x) const
    {
        const float v = x * up;
        float q = rintf(v * inverse);
        const float left = fmaf(-q, scaled, v), over = fabsf(left) - 0.5f * scaled;
        if (over >= 0.0f && inverse > 0.0f && (over > 0.0f || ((int)q & 1))) q += copysignf(1.0f, left);
        return inverse > 0.0f ? (int)fminf(fmaxf(q, -127.0f), 127.0f) : 0;
    }
};
__device__ __forceinline__ float kept_value(int q, float s) { return (float)q * s; }

// N neighbouring 8-bit values
template <int N> struct Kept;
template <> struct Kept<8> {
    typedef uint2 raw;
    static __device__ __forceinline__ raw none() { return make_uint2(0u, 0u); }
    static __device__ __forceinline__ void get(raw r, int (&q)[8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            q[i] = (int)(r.x << (24 - 8 * i)) >> 24;
            q[4 + i] = (int)(r.y << (24 - 8 * i)) >> 24;
        }
    }
    static __device__ __forceinline__ raw put(const int (&q)[8])
    {
        uint2 r = make_uint2(0u, 0u);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            r.x |= (uint32_t)(q[i] & 255) << (8 * i);
            r.y |= (uint32_t)(q[4 + i] & 255) << (8 * i);
        }
        return r;
    }
};
template <> struct Kept<4> {
    typedef uint32_t raw;
    static __device__ __forceinline__ raw none() { return 0u; }
    static __device__ __forceinline__ void get(raw r, int (&q)[4])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = (int)(r << (24 - 8 * i)) >> 24;
    }
    static __device__ __forceinline__ raw put(const int (&q)[4])
    {
        uint32_t r = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) r |= (uint32_t)(q[i] & 255) << (8 * i);
        return r;
    }
};
template <> struct Kept<1> {
    typedef int8_t raw;
    static __device__ __forceinline__ raw none() { return 0; }
    static __device__ __forceinline__ void get(raw r, int (&q)[1]) { q[0] = r; }
    static __device__ __forceinline__ raw put(const int (&q)[1]) { return (int8_t)q[0]; }
};

}  // namespace gs
