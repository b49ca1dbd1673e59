// Argument checks and kernel choice of gs_attention_forward / gs_attention_backward.
#include <math.h>
#include <string.h>

#include "gs_attn.cuh"

namespace gs {

static gs_status bad(const char *what)
{
    set_error("invalid argument: %s", what);
    return GS_ERR_INVALID_ARG;
}

static AttnTensor tensor(const void *p, const int64_t (&stride)[3])
{
    AttnTensor t;
    t.p = const_cast<void *>(p);
    t.sb = stride[0];
    t.sl = stride[1];
    t.sh = stride[2];
    return t;
}

// rows that are written must not share elements: an extent above one needs a non-zero stride
static bool writable(const AttnTensor &t, int64_t batch, int64_t len, int64_t heads)
{
    return (batch <= 1 || t.sb != 0) && (len <= 1 || t.sl != 0) && (heads <= 1 || t.sh != 0);
}

static gs_status fill(const gs_attention_config *c, AttnArgs *a)
{
    if (!c) return bad("config is NULL");
    if (c->dtype != GS_TABLE_F32 && c->dtype != GS_TABLE_F16 && c->dtype != GS_TABLE_BF16)
        return bad("dtype must be GS_TABLE_F32, GS_TABLE_F16 or GS_TABLE_BF16");
    if (c->batch < 0 || c->q_len < 0 || c->k_len < 0) return bad("negative batch or length");
    if (c->q_heads <= 0 || c->kv_heads <= 0 || c->q_heads % c->kv_heads != 0)
        return bad("q_heads must be a positive multiple of kv_heads");
    if (c->head_dim <= 0) return bad("head_dim must be positive");
    if (!(c->scale > 0.0f) || !isfinite(c->scale)) return bad("scale must be positive and finite");
    if (c->head_dim > 128) {
        set_error("head_dim %d is not supported (1..128)", c->head_dim);
        return GS_ERR_UNSUPPORTED;
    }
    if (c->q_len > (1 << 29) || c->k_len > (1 << 29) || c->q_heads > (1 << 20) || c->batch > ((int64_t)1 << 31)) {
        set_error("lengths up to 2^29, 2^20 heads and 2^31 sequences are supported");
        return GS_ERR_UNSUPPORTED;
    }
    // rows of all heads, which launches and scratch are counted in, fit 64 bits with room to spare
    const int64_t longest = c->q_len > c->k_len ? c->q_len : c->k_len;
    if (longest > 0 && c->batch * c->q_heads > ((int64_t)1 << 56) / longest) {
        set_error("attention of more than 2^56 rows is not supported");
        return GS_ERR_UNSUPPORTED;
    }
    memset(a, 0, sizeof(*a));
    a->batch = c->batch;
    a->q_len = c->q_len;
    a->k_len = c->k_len;
    a->q_heads = c->q_heads;
    a->kv_heads = c->kv_heads;
    a->group = c->q_heads / c->kv_heads;
    a->dim = c->head_dim;
    // a bound past both lengths hides nothing
    const int64_t reach = (int64_t)c->q_len + c->k_len;
    a->left = c->window_left < 0 || c->window_left >= reach ? -1 : c->window_left;
    a->right = c->window_right < 0 || c->window_right >= reach ? -1 : c->window_right;
    a->scale = c->scale;
    a->dtype = c->dtype;
    a->q_lens = c->d_q_lens;
    a->k_lens = c->d_k_lens;
    return GS_OK;
}

static gs_status pointers_ok(const AttnTensor *t, int n, int32_t dtype)
{
    const uintptr_t es = dtype == GS_TABLE_F32 ? 4 : 2;
    for (int i = 0; i < n; ++i) {
        if (!t[i].p) return bad("null pointer");
        if ((uintptr_t)t[i].p % es) return bad("tensor not aligned to its element size");
    }
    return GS_OK;
}

// Whether fp32 tensors that attn_walk_ok accepts go there (products as three of tf32 each, whole heads in
// shared memory) or to the CUDA cores.  Measured, whole heads | CUDA cores, us:
//  forward : 8192 heads of 30 x 32 36 | 90, 4096 of 60 x 64 121 | 169, 2048 of 30 x 128 61 | 62, 1024 of 90 x 128 168 | 288
//  backward: 2048 heads of 100 x 64 807 | 1058, 1024 of 90 x 128 746 | 1086, 32 of 100 x 64 49 | 27; up to 64 positions, where
//            a block of the CUDA cores has all of a head, 4096 of 60 x 64 675 | 422, 16384 of 16 x 32 110 | 82, but
//            16384 of 40 x 32 with a window of 10 on each side 427 | 731
static bool f32_whole(const AttnArgs &a, bool backward)
{
    const int n = a.q_len > a.k_len ? a.q_len : a.k_len;
    if (!backward) return a.dim <= 64 || n > 64;
    if (n > 64) return a.batch * a.kv_heads >= sm_count();
    return n > 32 && a.dim <= 32 && a.left >= 0 && a.right >= 0 && a.left + a.right <= 32;
}

// Whether the fp32 tensors that are left go to 64-row tiles on the tensor cores or to the CUDA cores.  Measured,
// tensor | CUDA cores, us (causal unless said):
//  forward : 8 x 4 heads of 333 x 64 33 | 33, 16 x 8 heads of 333 x 64 69 | 98, 16 heads of 2048 x 64 230 | 294, 16 of
//            2048 x 128 413 | 532, 16 of 4096 x 64, all visible, 1381 | 2111, 64 x 4 heads of 200 x 32, window 10, 24 | 57
//  backward: 16 x 8 heads of 333 x 64 229 | 326, 16 heads of 2048 x 64 799 | 964, 16 of 4096 x 64 5048 | 7263, 200 x 32
//            82 | 170; but 8 x 4 heads of 333 x 64 114 | 83, where the blocks do not fill the device one and a half
//            times and the CUDA cores' 32-row tiles are twice as many, and 16 heads of 2048 x 128 4031 | 2415 (the
//            accumulators of 128 columns do not fit a thread's registers).
static bool f32_tiles(const AttnArgs &a, bool backward)
{
    if (a.dtype != GS_TABLE_F32 || a.q_len <= 0 || a.k_len <= 0) return false;
    const int n = a.q_len > a.k_len ? a.q_len : a.k_len;
    if (n <= 64 || !backward) return n > 64;
    const int64_t blocks = (n + 63) / 64 * a.batch * (a.q_heads + a.kv_heads);
    return a.dim <= 64 && blocks >= 3 * (int64_t)sm_count();
}

}  // namespace gs

using namespace gs;

extern "C" {

gs_status gs_attention_forward(const gs_attention_config *cfg, const void *d_q, const void *d_k, const void *d_v,
                               void *d_out, float *d_lse, void *stream)
{
    AttnArgs a;
    gs_status s = fill(cfg, &a);
    if (s != GS_OK) return s;
    if (a.batch == 0 || a.q_len == 0) return GS_OK;
    a.q = tensor(d_q, cfg->q_stride);
    a.k = tensor(d_k, cfg->k_stride);
    a.v = tensor(d_v, cfg->v_stride);
    a.out = tensor(d_out, cfg->out_stride);
    a.lse = d_lse;
    const AttnTensor need[4] = {a.q, a.out, a.k, a.v};
    if ((s = pointers_ok(need, a.k_len ? 4 : 2, a.dtype)) != GS_OK) return s;
    if (!d_lse) return bad("d_lse is NULL");
    if (!writable(a.out, a.batch, a.q_len, a.q_heads)) return bad("out has a zero stride");
    if ((s = stalled_before()) != GS_OK) return s;
    // 16-bit tensors: up to 128 positions by whole heads, longer ones on 128 x 128 tiles, which need TMA.  Between 65
    // and 128 positions the wide heads go to the tiles as well: 4096 heads of 100 x 128 take 127 us there and
    // 146 us whole, 8192 heads of 100 x 64 196 and 141 us.
    const bool tiles = a.k_len > 0 && attn_tc_forward_ok(a);
    const bool whole = a.dtype == GS_TABLE_F32 ? f32_whole(a, false) : !(tiles && a.q_len > 64 && a.dim > 64);
    if (whole && attn_walk_ok(a, false)) return attn_walk_forward(a, (cudaStream_t)stream);
    if (tiles) return attn_tc_forward(a, (cudaStream_t)stream);
    if (f32_tiles(a, false)) return attn_f32_forward(a, (cudaStream_t)stream);
    return attn_simt_forward(a, (cudaStream_t)stream);
}

gs_status gs_attention_backward(const gs_attention_config *cfg, const void *d_dout, const void *d_q, const void *d_k,
                                const void *d_v, const void *d_out, const float *d_lse, float *d_work, void *d_dq,
                                void *d_dk, void *d_dv, void *stream)
{
    AttnArgs a;
    gs_status s = fill(cfg, &a);
    if (s != GS_OK) return s;
    if (a.batch == 0 || (a.q_len == 0 && a.k_len == 0)) return GS_OK;
    a.q = tensor(d_q, cfg->q_stride);
    a.k = tensor(d_k, cfg->k_stride);
    a.v = tensor(d_v, cfg->v_stride);
    a.out = tensor(d_out, cfg->out_stride);
    a.dout = tensor(d_dout, cfg->dout_stride);
    a.dq = tensor(d_dq, cfg->dq_stride);
    a.dk = tensor(d_dk, cfg->dk_stride);
    a.dv = tensor(d_dv, cfg->dv_stride);
    a.lse = const_cast<float *>(d_lse);
    a.delta = d_work;
    const AttnTensor on_q[4] = {a.q, a.out, a.dout, a.dq}, on_k[4] = {a.k, a.v, a.dk, a.dv};
    if (a.q_len) {
        if ((s = pointers_ok(on_q, 4, a.dtype)) != GS_OK) return s;
        if (!d_lse || !d_work) return bad("null pointer");
    }
    if (a.k_len && (s = pointers_ok(on_k, 4, a.dtype)) != GS_OK) return s;
    if (!writable(a.dq, a.batch, a.q_len, a.q_heads) || !writable(a.dk, a.batch, a.k_len, a.kv_heads) ||
        !writable(a.dv, a.batch, a.k_len, a.kv_heads))
        return bad("a gradient has a zero stride");
    if ((s = stalled_before()) != GS_OK) return s;
    // As above; backward, 4096 heads of 100 x 128 321 us on tiles and 523 us whole, 8192 heads of 100 x 64 424 and
    // 490 us, but 272 us with a window of 10 on each side, which the whole heads make use of.
    const bool tiles = a.q_len > 0 && a.k_len > 0 && attn_tc_backward_ok(a);
    const bool narrow = a.left >= 0 && a.right >= 0 && a.left + a.right < 64;
    const bool wide = (a.q_len > 64 || a.k_len > 64) && (a.dim > 64 || (a.dim > 32 && !narrow));
    const bool whole = a.dtype == GS_TABLE_F32 ? f32_whole(a, true) : !(tiles && wide);
    if (whole && attn_walk_ok(a, true)) return attn_walk_backward(a, (cudaStream_t)stream);
    if (tiles) return attn_tc_backward(a, (cudaStream_t)stream);
    if (f32_tiles(a, true)) return attn_f32_backward(a, (cudaStream_t)stream);
    return attn_simt_backward(a, (cudaStream_t)stream);
}

gs_status gs_stall_drill(void *stream) { return attn_stall_drill((cudaStream_t)stream); }

int64_t gs_attention_backward_work(const gs_attention_config *cfg)
{
    AttnArgs a;
    if (fill(cfg, &a) != GS_OK) return -1;
    return a.batch * a.q_heads * a.q_len + attn_tc_backward_work(a.batch, a.q_len, a.k_len, a.q_heads, a.kv_heads);
}

}  // extern "C"
