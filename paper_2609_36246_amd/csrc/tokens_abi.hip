// Host side of include/olive_tokens.h: argument validation and the launch of each operator.
#include <hip/hip_runtime.h>

#include <cmath>

#include "tokens_internal.hpp"

using namespace olive;

namespace {

constexpr int64_t kMaxInt = 0x7fffffff;

olive_status check_hip(hipError_t e) { return e == hipSuccess ? OLIVE_OK : OLIVE_E_HIP; }
bool known(int32_t dtype) { return dtype == OLIVE_F32 || dtype == OLIVE_BF16; }
int esize(int32_t dtype) { return dtype == OLIVE_BF16 ? 2 : 4; }
bool misplaced(const void *p, int32_t dtype) { return (uintptr_t)p % esize(dtype) != 0; }

// Whether a matrix's rows lie apart as they must: an output's do not overlap, an input's may be one
// row again, and no row's address passes 63 bits.
bool apart(int64_t rows, int64_t width, int64_t stride, bool output) {
    if (rows <= 1) return true;
    return stride >= (output ? width : 0) && stride <= ((int64_t)1 << 60) / rows;
}

// Whether an output that begins where an input does is the same matrix, whose rows are read before they are
// written; with other strides it would write rows that are still to be read.
bool same_or_apart(int64_t rows, const void *in, int64_t in_stride, const void *out, int64_t out_stride) {
    return !in || in != out || rows <= 1 || in_stride == out_stride;
}

olive_status check_workspace(const void *w, int64_t have, int64_t need) {
    if (need <= 0) return OLIVE_OK;
    if (!w) return OLIVE_E_NULL;
    if ((uintptr_t)w & 15) return OLIVE_E_UNSUPPORTED;
    return have < need ? OLIVE_E_SHAPE : OLIVE_OK;
}

olive_status check_embed(const olive_embed_desc *d) {
    if (!d) return OLIVE_E_NULL;
    if (d->size != (int32_t)sizeof(*d)) return OLIVE_E_RANGE;
    if (!known(d->dtype)) return OLIVE_E_DTYPE;
    if (d->tokens < 0 || d->vocab < 1 || d->vocab > kMaxInt || d->width < 1) return OLIVE_E_SHAPE;
    if (d->tokens > ((int64_t)1 << 26) || d->width > 65536) return OLIVE_E_UNSUPPORTED;
    if (!std::isfinite(d->scale)) return OLIVE_E_RANGE;
    return d->tokens > 0 && !d->ids ? OLIVE_E_NULL : OLIVE_OK;
}

EmbedArgs embed_args(const olive_embed_desc *d) {
    EmbedArgs a{};
    a.ids = d->ids;
    a.tokens = (int32_t)d->tokens;
    a.vocab = (int32_t)d->vocab;
    a.width = d->width;
    a.scale = d->scale;
    return a;
}

olive_status check_norm(const olive_norm_desc *d) {
    if (!d) return OLIVE_E_NULL;
    if (d->size != (int32_t)sizeof(*d)) return OLIVE_E_RANGE;
    if (!known(d->dtype)) return OLIVE_E_DTYPE;
    if (d->rows < 0 || d->rows > kMaxInt || d->width < 1) return OLIVE_E_SHAPE;
    if (d->width > 16384) return OLIVE_E_UNSUPPORTED;
    if (d->kind != OLIVE_NORM_RMS && d->kind != OLIVE_NORM_LAYER) return OLIVE_E_RANGE;
    if (!std::isfinite(d->eps) || d->eps < 0.f) return OLIVE_E_RANGE;
    return misplaced(d->weight, d->dtype) || misplaced(d->bias, d->dtype) ? OLIVE_E_UNSUPPORTED : OLIVE_OK;
}

NormArgs norm_args(const olive_norm_desc *d) {
    NormArgs a{};
    a.rows = (int32_t)d->rows;
    a.width = d->width;
    a.layer = d->kind == OLIVE_NORM_LAYER;
    a.eps = d->eps;
    a.inv_width = 1.0 / (double)d->width;
    a.weight = d->weight;
    a.bias = d->bias;
    return a;
}

olive_status check_sample(const olive_sample_desc *d) {
    if (!d) return OLIVE_E_NULL;
    if (d->size != (int32_t)sizeof(*d)) return OLIVE_E_RANGE;
    if (!known(d->dtype)) return OLIVE_E_DTYPE;
    if (d->rows < 0 || d->vocab < 1) return OLIVE_E_SHAPE;
    if (d->rows > (1 << 20) || d->vocab > (1 << 24)) return OLIVE_E_UNSUPPORTED;
    return d->rows > 0 && !d->uniform ? OLIVE_E_NULL : OLIVE_OK;
}

SampleArgs sample_args(const olive_sample_desc *d) {
    SampleArgs a{};
    a.rows = (int32_t)d->rows;
    a.vocab = (int32_t)d->vocab;
    a.uniform = d->uniform;
    a.temperature = d->temperature;
    a.top_k = d->top_k;
    a.top_p = d->top_p;
    a.min_p = d->min_p;
    return a;
}

}  // namespace

extern "C" {

olive_status olive_embed(const olive_embed_desc *desc, const void *table, int64_t table_stride,
                         void *out, int64_t out_stride, void *hip_stream) {
    const olive_status s = check_embed(desc);
    if (s != OLIVE_OK) return s;
    if (desc->tokens == 0) return OLIVE_OK;
    if (!table || !out) return OLIVE_E_NULL;
    if (!apart(desc->vocab, desc->width, table_stride, false) || !apart(desc->tokens, desc->width, out_stride, true))
        return OLIVE_E_SHAPE;
    if (misplaced(table, desc->dtype) || misplaced(out, desc->dtype)) return OLIVE_E_UNSUPPORTED;
    // (wavefronts of a launch, four to a workgroup)
    if (desc->tokens * ((desc->width + 255) / 256) / 4 >= kMostBlocks) return OLIVE_E_SHAPE;
    EmbedArgs a = embed_args(desc);
    a.table = {(char *)table, table_stride};
    a.out = {(char *)out, out_stride};
    a.stream = streamed(desc->tokens, desc->width, esize(desc->dtype));
    return check_hip(launch_embed(a, desc->dtype == OLIVE_BF16, (hipStream_t)hip_stream));
}

olive_status olive_embed_workspace(const olive_embed_desc *desc, int64_t *bytes) {
    if (!bytes) return OLIVE_E_NULL;
    const olive_status s = check_embed(desc);
    if (s != OLIVE_OK) return s;
    *bytes = embed_backward_bytes(embed_args(desc));
    return OLIVE_OK;
}

olive_status olive_embed_backward(const olive_embed_desc *desc, const void *grad_out,
                                  int64_t grad_out_stride, void *grad_table,
                                  int64_t grad_table_stride, int32_t grad_dtype,
                                  int32_t accumulate, void *workspace, int64_t workspace_bytes,
                                  void *hip_stream) {
    olive_status s = check_embed(desc);
    if (s != OLIVE_OK) return s;
    if (!known(grad_dtype)) return OLIVE_E_DTYPE;
    if (accumulate != 0 && accumulate != 1) return OLIVE_E_RANGE;
    if (!grad_table || (desc->tokens > 0 && !grad_out)) return OLIVE_E_NULL;
    if (!apart(desc->tokens, desc->width, grad_out_stride, false) ||
        !apart(desc->vocab, desc->width, grad_table_stride, true))
        return OLIVE_E_SHAPE;
    if (misplaced(grad_out, desc->dtype) || misplaced(grad_table, grad_dtype)) return OLIVE_E_UNSUPPORTED;
    EmbedArgs a = embed_args(desc);
    s = check_workspace(workspace, workspace_bytes, embed_backward_bytes(a));
    if (s != OLIVE_OK) return s;
    if (desc->tokens == 0 && accumulate) return OLIVE_OK;
    a.table = {(char *)grad_table, grad_table_stride};
    a.out = {(char *)grad_out, grad_out_stride};
    a.accumulate = accumulate == 1;
    a.work = (char *)workspace;
    return check_hip(launch_embed_backward(a, desc->dtype == OLIVE_BF16, grad_dtype == OLIVE_BF16,
                                           (hipStream_t)hip_stream));
}

olive_status olive_row_norm(const olive_norm_desc *desc, const void *x, int64_t x_stride,
                            const void *residual, int64_t residual_stride, void *out,
                            int64_t out_stride, void *sum, int64_t sum_stride, void *hip_stream) {
    const olive_status s = check_norm(desc);
    if (s != OLIVE_OK) return s;
    if (desc->rows == 0) return OLIVE_OK;
    if (!x || !out) return OLIVE_E_NULL;
    const int64_t n = desc->rows, w = desc->width;
    if (!apart(n, w, x_stride, false) || (residual && !apart(n, w, residual_stride, false)) ||
        !apart(n, w, out_stride, true) || (sum && !apart(n, w, sum_stride, true)))
        return OLIVE_E_SHAPE;
    if (out == sum || !same_or_apart(n, x, x_stride, out, out_stride) || !same_or_apart(n, x, x_stride, sum, sum_stride) ||
        !same_or_apart(n, residual, residual_stride, out, out_stride) ||
        !same_or_apart(n, residual, residual_stride, sum, sum_stride))
        return OLIVE_E_SHAPE;
    for (const void *p : {x, residual, (const void *)out, (const void *)sum})
        if (misplaced(p, desc->dtype)) return OLIVE_E_UNSUPPORTED;
    NormArgs a = norm_args(desc);
    a.x = {(char *)x, x_stride};
    if (residual) a.res = {(char *)residual, residual_stride};
    a.out = {(char *)out, out_stride};
    if (sum) a.sum = {(char *)sum, sum_stride};
    a.stream = streamed(n, w, esize(desc->dtype));
    return check_hip(launch_norm(a, desc->dtype == OLIVE_BF16, (hipStream_t)hip_stream));
}

olive_status olive_row_norm_workspace(const olive_norm_desc *desc, int64_t *bytes) {
    if (!bytes) return OLIVE_E_NULL;
    const olive_status s = check_norm(desc);
    if (s != OLIVE_OK) return s;
    *bytes = norm_backward_bytes(norm_args(desc));
    return OLIVE_OK;
}

olive_status olive_row_norm_backward(const olive_norm_desc *desc, const void *h, int64_t h_stride,
                                     const void *grad_out, int64_t grad_out_stride,
                                     const void *grad_sum, int64_t grad_sum_stride, void *grad_h,
                                     int64_t grad_h_stride, float *grad_weight, float *grad_bias,
                                     void *workspace, int64_t workspace_bytes, void *hip_stream) {
    olive_status s = check_norm(desc);
    if (s != OLIVE_OK) return s;
    const int64_t n = desc->rows, w = desc->width;
    if (n > 0 && (!h || !grad_out || !grad_h)) return OLIVE_E_NULL;
    if (!apart(n, w, h_stride, false) || !apart(n, w, grad_out_stride, false) ||
        (grad_sum && !apart(n, w, grad_sum_stride, false)) || !apart(n, w, grad_h_stride, true))
        return OLIVE_E_SHAPE;
    if (!same_or_apart(n, grad_out, grad_out_stride, grad_h, grad_h_stride) ||
        !same_or_apart(n, grad_sum, grad_sum_stride, grad_h, grad_h_stride))
        return OLIVE_E_SHAPE;
    for (const void *p : {h, grad_out, grad_sum, (const void *)grad_h})
        if (misplaced(p, desc->dtype)) return OLIVE_E_UNSUPPORTED;
    if ((uintptr_t)grad_weight % 4 || (uintptr_t)grad_bias % 4) return OLIVE_E_UNSUPPORTED;
    const bool sums = grad_weight || grad_bias;
    int64_t need = 0;
    olive_row_norm_workspace(desc, &need);
    s = check_workspace(workspace, workspace_bytes, sums ? need : 0);
    if (s != OLIVE_OK) return s;
    if (n == 0 && !sums) return OLIVE_OK;
    NormArgs a = norm_args(desc);
    a.x = {(char *)h, h_stride};
    if (grad_sum) a.res = {(char *)grad_sum, grad_sum_stride};
    a.out = {(char *)grad_h, grad_h_stride};
    a.sum = {(char *)grad_out, grad_out_stride};
    a.stream = streamed(n, w, esize(desc->dtype));
    a.gw = grad_weight;
    a.gb = grad_bias;
    a.part = (float *)workspace;
    return check_hip(launch_norm_backward(a, desc->dtype == OLIVE_BF16, (hipStream_t)hip_stream));
}

olive_status olive_sample_workspace(const olive_sample_desc *desc, int64_t *bytes) {
    if (!bytes) return OLIVE_E_NULL;
    const olive_status s = check_sample(desc);
    if (s != OLIVE_OK) return s;
    *bytes = sample_bytes(sample_args(desc), desc->dtype == OLIVE_BF16);
    return OLIVE_OK;
}

olive_status olive_sample(const olive_sample_desc *desc, const void *logits, int64_t logits_stride,
                          int32_t *token, float *logp, int32_t *kept, void *workspace,
                          int64_t workspace_bytes, void *hip_stream) {
    olive_status s = check_sample(desc);
    if (s != OLIVE_OK) return s;
    if (desc->rows == 0) return OLIVE_OK;
    if (!logits || !token) return OLIVE_E_NULL;
    if (!apart(desc->rows, desc->vocab, logits_stride, false)) return OLIVE_E_SHAPE;
    if (misplaced(logits, desc->dtype)) return OLIVE_E_UNSUPPORTED;
    SampleArgs a = sample_args(desc);
    const bool bf16 = desc->dtype == OLIVE_BF16;
    s = check_workspace(workspace, workspace_bytes, sample_bytes(a, bf16));
    if (s != OLIVE_OK) return s;
    a.logits = {(char *)logits, logits_stride};
    a.token = token;
    a.logp = logp;
    a.kept = kept;
    a.work = (char *)workspace;
    return check_hip(launch_sample(a, bf16, (hipStream_t)hip_stream));
}

}  // extern "C"
