// Argument checks of gs_layer_norm_forward / gs_layer_norm_backward.
#include <math.h>

#include "gs_norm.cuh"

namespace gs {

static gs_status fill(const gs_layer_norm_config *c, NormArgs *a)
{
    if (!c) return bad("config is NULL");
    if (!known_type(c->dtype)) return bad("dtype must be GS_TABLE_F32, GS_TABLE_F16 or GS_TABLE_BF16");
    if (c->weight_dtype != GS_TABLE_F32 && c->weight_dtype != c->dtype) return bad("weight_dtype must be GS_TABLE_F32 or dtype");
    if (c->batch < 0 || c->length < 0 || c->columns <= 0) return bad("negative batch or length, or no columns");
    if (!(c->eps >= 0.0f) || !isfinite(c->eps)) return bad("eps must be finite and >= 0");
    if (c->columns > NORM_MOST_COLUMNS) {
        set_error("layer norm of %d columns is not supported (1..%d)", c->columns, NORM_MOST_COLUMNS);
        return GS_ERR_UNSUPPORTED;
    }
    const int64_t most = (int64_t)1 << 40;
    if (c->batch > most || c->length > most || (c->length > 0 && c->batch > most / c->length)) {
        set_error("layer norm of more than 2^40 rows is not supported");
        return GS_ERR_UNSUPPORTED;
    }
    *a = NormArgs{};
    a->rows = c->batch * c->length;
    a->length = c->length > 0 ? c->length : 1;
    a->columns = c->columns;
    a->kept_blocks = (c->columns + KEPT_BLOCK - 1) / KEPT_BLOCK;
    a->weight_f32 = c->weight_dtype == GS_TABLE_F32;
    a->eps = c->eps;
    a->lens = c->d_lens;
    return GS_OK;
}

static NormRows rows(const void *p, const int64_t (&stride)[2]) { return {const_cast<void *>(p), stride[0], stride[1], 0, 0}; }

// Checks the tensors, the first `outputs` of which are written; tells whether 16-byte accesses fit all of them, and takes
// the batch for one long sequence where that is the same.
static gs_status tensors(const gs_layer_norm_config *c, NormArgs *a, NormRows **t, int n, int outputs, bool *aligned)
{
    const int64_t es = (int64_t)size_of(c->dtype);
    const uintptr_t vector = size_of(c->weight_dtype);
    if ((uintptr_t)a->weight % vector || (uintptr_t)a->bias % vector) return bad("weight or bias not aligned to its element size");
    if ((uintptr_t)a->stats % 8) return bad("d_stats must be aligned to 8 bytes");
    if ((uintptr_t)a->partial % 4 || (uintptr_t)a->scales % 4) return bad("d_work or d_scales not aligned to its element size");
    bool wide = c->columns * es % 16 == 0, one = !c->d_lens;
    for (int i = 0; i < n; ++i) {
        if (!t[i]->p) return bad("null pointer");
        if ((uintptr_t)t[i]->p % es) return bad("tensor not aligned to its element size");
        if (i < outputs && ((c->batch > 1 && t[i]->sb == 0) || (c->length > 1 && t[i]->st == 0))) return bad("an output has a zero stride");
        wide = wide && (uintptr_t)t[i]->p % 16 == 0 && (t[i]->sb * es | t[i]->st * es) % 16 == 0;
        one = one && (c->batch == 1 || t[i]->sb == t[i]->st * c->length);
    }
    if (one) a->length = a->rows;
    a->by_length = Divider(a->length);
    a->vectors_wide = (uintptr_t)a->weight % 16 == 0 && (uintptr_t)a->bias % 16 == 0;
    *aligned = wide;
    return GS_OK;
}

}  // namespace gs

using namespace gs;

extern "C" {

gs_status gs_layer_norm_forward(const gs_layer_norm_config *cfg, const void *d_x, const void *d_weight, const void *d_bias,
                                void *d_y, float *d_stats, int8_t *d_packed, float *d_scales, void *stream)
{
    NormArgs a;
    gs_status s = fill(cfg, &a);
    if (s != GS_OK || a.rows == 0) return s;
    if (!d_packed != !d_scales) return bad("d_packed and d_scales belong together");
    a.x = rows(d_x, cfg->x_stride);
    a.y = rows(d_y, cfg->y_stride);
    a.weight = d_weight;
    a.bias = d_bias;
    a.stats = d_stats;
    a.scales = d_scales;
    NormRows *all[2] = {&a.y, &a.x};
    bool aligned;
    if ((s = tensors(cfg, &a, all, 2, 1, &aligned)) != GS_OK) return s;
    cudaStream_t st = (cudaStream_t)stream;
    if (d_packed && aligned && (uintptr_t)d_packed % 8 == 0) {
        a.packed = d_packed;
    } else if (d_packed) {
        s = checkpoint_pack(cfg->dtype, a.x, cfg->d_lens, cfg->batch, cfg->length, cfg->columns, d_packed, d_scales, st);
        if (s != GS_OK) return s;
    }
    return norm_forward(a, cfg->dtype, aligned, st);
}

int64_t gs_layer_norm_backward_work(const gs_layer_norm_config *cfg)
{
    NormArgs a;
    if (fill(cfg, &a) != GS_OK) return -1;
    return norm_backward_partials(a.rows, a.columns, cfg->dtype) * 2 * a.columns;
}

gs_status gs_layer_norm_backward(const gs_layer_norm_config *cfg, const void *d_dy, const void *d_x, const int8_t *d_packed,
                                 const float *d_scales, const void *d_weight, const float *d_stats, float *d_work, void *d_dx,
                                 void *d_dweight, void *d_dbias, void *stream)
{
    NormArgs a;
    gs_status s = fill(cfg, &a);
    if (s != GS_OK) return s;
    const bool sums = d_dweight || d_dbias;
    cudaStream_t st = (cudaStream_t)stream;
    if (a.rows == 0) {                                 // nothing to add up
        const size_t bytes = a.columns * size_of(cfg->weight_dtype);
        if (d_dweight) GS_CUDA_TRY(cudaMemsetAsync(d_dweight, 0, bytes, st));
        if (d_dbias) GS_CUDA_TRY(cudaMemsetAsync(d_dbias, 0, bytes, st));
        return GS_OK;
    }
    if (!d_x == !d_packed || !d_packed != !d_scales) return bad("x is taken either from d_x or from d_packed and d_scales");
    if (!d_stats || (sums && !d_work)) return bad("null pointer");
    a.dx = rows(d_dx, cfg->dx_stride);
    a.dy = rows(d_dy, cfg->dy_stride);
    a.x = rows(d_x, cfg->x_stride);
    a.packed = const_cast<int8_t *>(d_packed);
    a.scales = const_cast<float *>(d_scales);
    a.weight = d_weight;
    a.stats = const_cast<float *>(d_stats);
    a.partial = d_work;
    NormRows *all[3] = {&a.dx, &a.dy, &a.x};
    bool aligned;
    if ((s = tensors(cfg, &a, all, d_x ? 3 : 2, 1, &aligned)) != GS_OK) return s;
    return norm_backward(a, cfg->dtype, aligned && (uintptr_t)d_packed % 8 == 0, d_dweight, d_dbias, st);
}

}  // extern "C"
