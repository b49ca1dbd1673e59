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
// shared memory) or to the CUDA cores.  Measured, whole heads | CUDA cores, us (all visible unless said):
//  forward : 8192 heads of 30 x 32 41 | 88, 4096 of 60 x 64 126 | 159, with a window of 5 on each side 93 | 160, 2048 of
//            30 x 128 57 | 63, 1024 of 90 x 128 159 | 284
//  backward, beyond 64 positions: 2048 heads of 100 x 64 822 | 1057, 1024 of 90 x 128 769 | 1082, 150 of 100 x 64, window 10,
//            57 | 85, 140 of 100 x 64 61 | 75, 32 of 100 x 64 60 | 27
//  backward, up to 64 positions, where a block of the CUDA cores has all of a head: 4096 heads of 60 x 64 711 | 316, window 5
//            547 | 310, 4096 of 40 x 64, window 10, 349 | 303, 16384 of 16 x 32 110 | 86, 4096 of 60 x 32 252 | 201, window
//            20 253 | 200, window 10 204 | 197; but 16384 of 40 x 32, window 10, 433 | 741.  A causal bound alone, 4096 of
//            48 x 32 110 | 193, is on the wrong side of the rule.
static bool f32_whole(const AttnArgs &a, bool backward)
{
    const int n = a.q_len > a.k_len ? a.q_len : a.k_len;
    if (!backward) return a.dim <= 64 || n > 64;
    if (n > 64) return a.batch * a.kv_heads >= sm_count();
    return n > 32 && a.dim <= 32 && a.left >= 0 && a.right >= 0 && a.left + a.right <= 32;
}

// Whether the fp32 tensors that are left go to 64-row tiles on the tensor cores or to the CUDA cores.  Measured,
// tensor | CUDA cores, us (causal unless said):
//  forward : 8 x 4 heads of 333 x 64 34 | 33, 12 x 4 36 | 40, 16 x 8 67 | 94, 16 heads of 2048 x 64 230 | 294, 16 of
//            2048 x 128 413 | 532, 16 of 4096 x 64, all visible, 1381 | 2111, 64 x 4 heads of 200 x 32, window 10, 24 | 57
//  backward, by the number of 64-row blocks (n): 4 x 4 heads of 700 x 64 (352) 225 | 149, 8 x 4 of 333 x 64 (384) 115 | 81,
//            10 x 4 (480) 117 | 112, 12 x 4 (576) 112 | 126, 8 x 4 of 700 x 64 (704) 261 | 252, 16 x 4 of 333 x 64 (768)
//            142 | 168, 20 x 4 (960) 156 | 210, 16 x 8 (1536) 244 | 327, 40 x 4 of 150 x 64 (960) 84 | 123, 4 x 4 of 1024 x 32, all
//            visible, (512) 194 | 295, 16 heads of 4096 x 64 5048 | 7263: where the blocks do not fill the device one and a
//            half times (444), the CUDA cores' 32-row tiles, twice as many, are ahead.  16 heads of 2048 x 128 4031 |
//            2415: the accumulators of 128 columns do not fit a thread's registers.
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
    // 16-bit tensors: up to 128 positions by whole heads, longer ones on 128 x 128 tiles, which need TMA (without it
    // the CUDA cores take 61 us instead of 13 for 4 x 4 heads of 500 x 64, causal, and 117 instead of 17 backward).  Between 65
    // and 128 positions the wide heads go to the tiles as well.  Tiles | whole, us: 4096 heads of 100 x 128 136 | 141, 300 of
    // them 16 | 18, 4096 of 70 x 128 131 | 112; 8192 of 100 x 64 226 | 136, 4096 of 60 x 128 130 | 57.  With a window of 10 on
    // each side, which only whole heads make use of, 4096 of 100 x 128 take 140 | 84: the rule does not look at windows.
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
    // As above.  Backward, tiles | whole, us: 4096 heads of 100 x 128 345 | 525, with a window of 10 on each side 346 | 308 (the
    // rule takes tiles for both), 8192 heads of 100 x 64 469 | 490, window 10 468 | 273, causal 4096 of 128 x 64 259 | 232, 4096
    // of 100 x 32 216 | 201, 300 heads of 100 x 64 27 | 31.
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
