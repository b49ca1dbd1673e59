// Shared pieces of the attention kernels: the argument block that the launchers take and the
// visibility rule.  Mathematics (per sequence b, query head h, key/value head g = h / group):
//   s_ij = scale q_i.k_j      lse_i = log sum_j exp s_ij      o_i = sum_j exp(s_ij - lse_i) v_j
// over the visible keys of row i, which are one interval [lo(i), hi(i)): with n_q, n_k the lengths
// of the sequence and off = n_k - n_q,
//   lo(i) = max(0, i + off - left), hi(i) = min(n_k, i + off + right + 1), nothing if i >= n_q;
// a negative left or right lifts that bound.  Seen from key j the visible queries are again an
// interval, [j - off - right, j - off + left].
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>
#include <mutex>

#include "gs_common.cuh"

namespace gs {

static constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;

struct AttnTensor {
    void *p;
    int64_t sb, sl, sh;               // strides in elements: sequence, position, head
};

struct AttnArgs {
    AttnTensor q, k, v, out, dout, dq, dk, dv;
    float *lse, *delta;               // [batch][q_heads][q_len]; delta heads the caller's scratch
    const int32_t *q_lens, *k_lens;   // may be null
    int64_t batch;
    int32_t q_len, k_len, q_heads, kv_heads, group, dim;
    int32_t left, right;              // < 0: unbounded; otherwise at most q_len + k_len
    float scale;
    int32_t dtype;
};

struct AttnSeq {                      // one sequence's lengths
    int nq, nk, off;
};

__device__ __forceinline__ AttnSeq attn_seq(const AttnArgs &a, int64_t b)
{
    AttnSeq s;
    // a length outside [0, padded length] is clamped: the library never follows it out of range
    s.nq = a.q_lens ? min(max(__ldg(a.q_lens + b), 0), a.q_len) : a.q_len;
    s.nk = a.k_lens ? min(max(__ldg(a.k_lens + b), 0), a.k_len) : a.k_len;
    s.off = s.nk - s.nq;
    return s;
}

__device__ __forceinline__ int attn_lo(const AttnArgs &a, const AttnSeq &s, int i)
{
    return a.left < 0 ? 0 : max(0, i + s.off - a.left);
}
// 0 for a row past the sequence's end, so that [lo, hi) is empty there
__device__ __forceinline__ int attn_hi(const AttnArgs &a, const AttnSeq &s, int i)
{
    if (i >= s.nq) return 0;
    return a.right < 0 ? s.nk : min(s.nk, i + s.off + a.right + 1);
}
// queries that see a key of [j0, j1): the range [first, last)
__device__ __forceinline__ int attn_q_first(const AttnArgs &a, const AttnSeq &s, int j0)
{
    return a.right < 0 ? 0 : max(0, j0 - s.off - a.right);
}
__device__ __forceinline__ int attn_q_last(const AttnArgs &a, const AttnSeq &s, int j1)
{
    return a.left < 0 ? s.nq : min(s.nq, j1 - s.off + a.left);
}

template <typename T> __device__ __forceinline__ float to_f(T x);
template <> __device__ __forceinline__ float to_f<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_f<__half>(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ float from_f<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_f<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// Lets `kernel` use up to `bytes` of dynamic shared memory on the current device; `done` is the kernel's own record of
// what each device allows already (the attribute costs about a microsecond to set).  Setting and recording are one step
// under a lock: of two threads that ask for different sizes, the smaller one must not undo the larger.
struct SharedRecord {
    std::atomic<int> bytes[64];
    std::mutex lock;
};
template <typename K>
static inline gs_status allow_shared(K kernel, int bytes, SharedRecord &done)
{
    int dev = 0;
    GS_CUDA_TRY(cudaGetDevice(&dev));
    const bool known = dev >= 0 && dev < 64;
    if (known && done.bytes[dev].load(std::memory_order_acquire) >= bytes) return GS_OK;
    std::lock_guard<std::mutex> hold(done.lock);
    if (known && done.bytes[dev].load(std::memory_order_relaxed) >= bytes) return GS_OK;
    GS_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
    if (known) done.bytes[dev].store(bytes, std::memory_order_release);
    return GS_OK;
}

// Accesses of four elements (of `es` bytes) need every row of every tensor aligned to them
static inline bool rows_of_four(const AttnArgs &a, size_t es, bool backward)
{
    auto ok = [&](const AttnTensor &t) {
        return ((uintptr_t)t.p % (4 * es)) == 0 && (t.sb | t.sl | t.sh) % 4 == 0;
    };
    bool v = a.dim % 4 == 0 && ok(a.q) && ok(a.k) && ok(a.v) && ok(a.out);
    if (backward) v = v && ok(a.dout) && ok(a.dq) && ok(a.dk) && ok(a.dv);
    return v;
}
static inline gs_status blocks_ok(int64_t blocks)
{
    if (blocks <= 0x7FFFFFFF) return GS_OK;
    set_error("attention of %lld row tiles exceeds one launch", (long long)blocks);
    return GS_ERR_UNSUPPORTED;
}

// gs_attn_simt.cu
gs_status attn_simt_forward(const AttnArgs &a, cudaStream_t st);
gs_status attn_simt_backward(const AttnArgs &a, cudaStream_t st);

// gs_attn_f32.cu
gs_status attn_f32_forward(const AttnArgs &a, cudaStream_t st);
gs_status attn_f32_backward(const AttnArgs &a, cudaStream_t st);
// gs_attn_walk.cu
bool attn_walk_ok(const AttnArgs &a, bool backward);
gs_status attn_walk_forward(const AttnArgs &a, cudaStream_t st);
gs_status attn_walk_backward(const AttnArgs &a, cudaStream_t st);
// gs_attn_tc.cu
bool attn_tc_forward_ok(const AttnArgs &a);
gs_status attn_tc_forward(const AttnArgs &a, cudaStream_t st);
gs_status attn_stall_drill(cudaStream_t st);
// gs_attn_tc_bwd.cu
bool attn_tc_backward_ok(const AttnArgs &a);
int64_t attn_tc_backward_work(int64_t batch, int32_t q_len, int32_t k_len, int32_t q_heads, int32_t kv_heads);   // floats
gs_status attn_tc_backward(const AttnArgs &a, cudaStream_t st);

}  // namespace gs
