// Host side of include/olive_layers.h: argument validation and the launch of each operator.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <new>

#include "layers_internal.hpp"

using namespace olive;

struct olive_clip_ctx {
    ClipTensor *tensors = nullptr;
    ClipChunk *chunks = nullptr;
    double *part = nullptr;
    int64_t n_chunks = 0;
};

namespace {

constexpr int64_t kMaxInt = 0x7fffffff;

olive_status check_hip(hipError_t e) { return e == hipSuccess ? OLIVE_OK : OLIVE_E_HIP; }

HeadsArg heads(const olive_heads *h) {
    return h ? HeadsArg{(char *)h->data, h->stride_token, h->stride_head} : HeadsArg{nullptr, 0, 0};
}
bool missing(const olive_heads *h) { return !h || !h->data; }
bool misplaced(const olive_heads *h, int esz) { return h && (uintptr_t)h->data % esz != 0; }

olive_status check_qk(const olive_qk_desc *d) {
    if (!d) return OLIVE_E_NULL;
    if (d->size != (int32_t)sizeof(*d)) return OLIVE_E_RANGE;
    if (d->dtype != OLIVE_F32 && d->dtype != OLIVE_BF16) return OLIVE_E_DTYPE;
    if (d->tokens < 0 || d->tokens > kMaxInt || d->heads_q < 0 || d->heads_k < 0 || d->head_dim < 1)
        return OLIVE_E_SHAPE;
    if ((int64_t)d->heads_q + d->heads_k < 1) return OLIVE_E_SHAPE;
    if (d->head_dim > 256 || (int64_t)d->heads_q + d->heads_k > 4096) return OLIVE_E_UNSUPPORTED;
    if (d->rot_dim < 0 || d->rot_dim > d->head_dim || (d->rot_dim & 1)) return OLIVE_E_RANGE;
    if (d->layout != OLIVE_ROPE_HALF && d->layout != OLIVE_ROPE_PAIRS) return OLIVE_E_RANGE;
    if (!std::isfinite(d->eps) || d->eps < 0.f) return OLIVE_E_RANGE;
    if (d->rot_dim > 0 && d->tokens > 0) {
        if (!d->positions || !d->cos || !d->sin) return OLIVE_E_NULL;
        if (d->num_positions < 1) return OLIVE_E_SHAPE;
    }
    if (d->slots && d->slot_rows < 0) return OLIVE_E_SHAPE;
    return OLIVE_OK;
}

QkArgs qk_args(const olive_qk_desc *d) {
    QkArgs a{};
    a.tokens = (int32_t)d->tokens;
    a.hq = d->heads_q;
    a.hk = d->heads_k;
    a.d = d->head_dim;
    a.rot = d->rot_dim;
    a.layout = d->layout;
    a.eps = d->eps;
    a.positions = d->positions;
    a.num_positions = d->num_positions;
    a.cos = d->cos;
    a.sin = d->sin;
    a.wq = d->weight_q;
    a.wk = d->weight_k;
    a.slots = d->slots;
    a.slot_rows = d->slot_rows;
    return a;
}

int64_t tiles(int64_t n, int64_t t) { return (n + t - 1) / t; }

olive_status check_attn(const olive_attn_desc *d) {
    if (!d) return OLIVE_E_NULL;
    if (d->size != (int32_t)sizeof(*d)) return OLIVE_E_RANGE;
    if (d->dtype != OLIVE_F32 && d->dtype != OLIVE_BF16) return OLIVE_E_DTYPE;
    if (d->num_groups < 1 || d->num_seqs < d->num_groups || d->num_seqs >= (1 << 20) ||
        d->heads_kv < 1 || d->heads_q < d->heads_kv || d->heads_q > 4096 ||
        d->heads_q % d->heads_kv || d->head_dim < 1 || d->max_q < 1 || d->total_q < 0 ||
        d->total_q > kMaxInt / d->heads_q || d->max_prefix < 0 || d->max_prefix > kMaxInt || d->max_suffix < 0 ||
        d->max_suffix > kMaxInt - d->max_prefix || d->prefix_rows < 0 || d->suffix_rows < 0)
        return OLIVE_E_SHAPE;
    if (d->head_dim > 256) return OLIVE_E_UNSUPPORTED;
    if (!std::isfinite(d->scale)) return OLIVE_E_RANGE;
    if (!d->group_seqs || !d->cu_q || !d->prefix_start || !d->prefix_len || !d->suffix_len)
        return OLIVE_E_NULL;
    if (d->max_suffix > 0) {
        if (!d->suffix_start == !d->page_table) return OLIVE_E_NULL;
        if (d->page_table) {
            if (d->page_size < 1 || d->table_stride < 0 || d->table_stride > kMaxInt ||
                d->table_stride * d->page_size < d->max_suffix)
                return OLIVE_E_SHAPE;
        }
    }
    // workgroups of a launch (16 rows or keys each in the kernels with the smallest tiles): of the
    // sequences' and the groups' rows, of the keys
    const int64_t g = d->heads_q / d->heads_kv;
    const int64_t rows = tiles((int64_t)d->max_q * g, 16) * d->num_seqs;
    const int64_t keys = tiles(d->max_prefix, 16) * d->num_groups + tiles(d->max_suffix, 16) * d->num_seqs;
    const int64_t shared = tiles(d->total_q * g, 16) + d->num_groups;
    if (rows + shared > kMostBlocks / d->heads_kv || keys > kMostBlocks / d->heads_kv) return OLIVE_E_SHAPE;
    return OLIVE_OK;
}

AttnArgs attn_args(const olive_attn_desc *d) {
    AttnArgs a{};
    a.groups = d->num_groups;
    a.seqs = d->num_seqs;
    a.hq = d->heads_q;
    a.hk = d->heads_kv;
    a.d = d->head_dim;
    a.max_q = (int32_t)(d->max_q < d->total_q ? d->max_q : d->total_q);
    a.total_q = (int32_t)d->total_q;
    a.max_prefix = d->max_prefix;
    a.max_suffix = d->max_suffix;
    a.prefix_rows = d->prefix_rows;
    a.suffix_rows = d->suffix_rows;
    a.group_seqs = d->group_seqs;
    a.cu_q = d->cu_q;
    a.prefix_start = d->prefix_start;
    a.prefix_len = d->prefix_len;
    a.suffix_len = d->suffix_len;
    a.suffix_start = d->suffix_start;
    a.pages = d->max_suffix > 0 ? d->page_table : nullptr;
    a.table_stride = d->table_stride;
    a.page_size = d->page_size;
    a.scale = d->scale;
    return a;
}

olive_status check_workspace(const void *w, int64_t have, int64_t need) {
    if (need <= 0) return OLIVE_OK;
    if (!w) return OLIVE_E_NULL;
    if ((uintptr_t)w & 15) return OLIVE_E_UNSUPPORTED;
    return have < need ? OLIVE_E_SHAPE : OLIVE_OK;
}

}  // namespace

extern "C" {

olive_status olive_qk_norm_rope(const olive_qk_desc *desc, const olive_heads *q,
                                const olive_heads *k, const olive_heads *v,
                                const olive_heads *q_out, const olive_heads *k_out,
                                const olive_heads *v_out, void *hip_stream) {
    const olive_status s = check_qk(desc);
    if (s != OLIVE_OK) return s;
    if (desc->tokens == 0) return OLIVE_OK;
    if (desc->heads_q && (missing(q) || missing(q_out))) return OLIVE_E_NULL;
    if (desc->heads_k && (missing(k) || missing(k_out))) return OLIVE_E_NULL;
    if (missing(v) != missing(v_out)) return OLIVE_E_NULL;
    const int esz = desc->dtype == OLIVE_BF16 ? 2 : 4;
    for (const olive_heads *h : {q, k, v, q_out, k_out, v_out})
        if (misplaced(h, esz)) return OLIVE_E_UNSUPPORTED;
    QkArgs a = qk_args(desc);
    if (a.hq) a.q = heads(q), a.qo = heads(q_out);
    if (a.hk) a.k = heads(k), a.ko = heads(k_out);
    if (a.hk && !missing(v)) {
        a.v = heads(v);
        a.vo = heads(v_out);
        a.hv = a.hk;
    }
    return check_hip(launch_qk_forward(a, desc->dtype == OLIVE_BF16, (hipStream_t)hip_stream));
}

olive_status olive_qk_norm_rope_workspace(const olive_qk_desc *desc, int64_t *bytes) {
    if (!bytes) return OLIVE_E_NULL;
    const olive_status s = check_qk(desc);
    if (s != OLIVE_OK) return s;
    *bytes = (int64_t)kQkBwdBlocks * 2 * desc->head_dim * (int64_t)sizeof(float);
    return OLIVE_OK;
}

olive_status olive_qk_norm_rope_backward(const olive_qk_desc *desc, const olive_heads *q,
                                         const olive_heads *k, const olive_heads *grad_q_out,
                                         const olive_heads *grad_k_out,
                                         const olive_heads *grad_q, const olive_heads *grad_k,
                                         float *grad_weight_q, float *grad_weight_k,
                                         void *workspace, int64_t workspace_bytes,
                                         void *hip_stream) {
    olive_status s = check_qk(desc);
    if (s != OLIVE_OK) return s;
    if ((grad_weight_q && !desc->weight_q) || (grad_weight_k && !desc->weight_k)) return OLIVE_E_NULL;
    if (desc->tokens > 0) {
        if (desc->heads_q && (missing(q) || missing(grad_q_out) || missing(grad_q))) return OLIVE_E_NULL;
        if (desc->heads_k && (missing(k) || missing(grad_k_out) || missing(grad_k))) return OLIVE_E_NULL;
    }
    const int esz = desc->dtype == OLIVE_BF16 ? 2 : 4;
    for (const olive_heads *h : {q, k, grad_q_out, grad_k_out, grad_q, grad_k})
        if (misplaced(h, esz)) return OLIVE_E_UNSUPPORTED;
    const bool weights = grad_weight_q || grad_weight_k;
    int64_t need = 0;
    olive_qk_norm_rope_workspace(desc, &need);
    s = check_workspace(workspace, workspace_bytes, weights ? need : 0);
    if (s != OLIVE_OK) return s;
    if (desc->tokens == 0 && !weights) return OLIVE_OK;
    QkArgs a = qk_args(desc);
    if (a.hq) a.q = heads(q), a.qo = heads(grad_q_out), a.gq = heads(grad_q);
    if (a.hk) a.k = heads(k), a.ko = heads(grad_k_out), a.gk = heads(grad_k);
    a.gwq = grad_weight_q;
    a.gwk = grad_weight_k;
    a.part = (float *)workspace;
    return check_hip(launch_qk_backward(a, desc->dtype == OLIVE_BF16, (hipStream_t)hip_stream));
}

olive_status olive_prefix_attention_workspace(const olive_attn_desc *desc, int32_t backward,
                                              int64_t *bytes) {
    if (!bytes) return OLIVE_E_NULL;
    const olive_status s = check_attn(desc);
    if (s != OLIVE_OK) return s;
    const AttnArgs a = attn_args(desc);
    const bool bf16 = desc->dtype == OLIVE_BF16;
    *bytes = backward ? attn_backward_bytes(a, bf16) : attn_forward_bytes(a, bf16);
    return OLIVE_OK;
}

olive_status olive_prefix_attention(const olive_attn_desc *desc, const olive_heads *q,
                                    const olive_heads *k_prefix, const olive_heads *v_prefix,
                                    const olive_heads *k_suffix, const olive_heads *v_suffix,
                                    const olive_heads *out, float *lse, void *workspace,
                                    int64_t workspace_bytes, void *hip_stream) {
    olive_status s = check_attn(desc);
    if (s != OLIVE_OK) return s;
    if (desc->total_q == 0) return OLIVE_OK;
    if (missing(q) || missing(out)) return OLIVE_E_NULL;
    if (desc->max_prefix > 0 && (missing(k_prefix) || missing(v_prefix))) return OLIVE_E_NULL;
    if (desc->max_suffix > 0 && (missing(k_suffix) || missing(v_suffix))) return OLIVE_E_NULL;
    const int esz = desc->dtype == OLIVE_BF16 ? 2 : 4;
    for (const olive_heads *h : {q, k_prefix, v_prefix, k_suffix, v_suffix, out})
        if (misplaced(h, esz)) return OLIVE_E_UNSUPPORTED;
    AttnArgs a = attn_args(desc);
    const bool bf16 = desc->dtype == OLIVE_BF16;
    s = check_workspace(workspace, workspace_bytes, attn_forward_bytes(a, bf16));
    if (s != OLIVE_OK) return s;
    a.q = heads(q);
    a.kp = heads(k_prefix);
    a.vp = heads(v_prefix);
    a.ks = heads(k_suffix);
    a.vs = heads(v_suffix);
    a.o = heads(out);
    a.lse = lse;
    a.work = (char *)workspace;
    return check_hip(launch_attn_forward(a, bf16, (hipStream_t)hip_stream));
}

olive_status olive_prefix_attention_backward(
    const olive_attn_desc *desc, const olive_heads *q, const olive_heads *k_prefix,
    const olive_heads *v_prefix, const olive_heads *k_suffix, const olive_heads *v_suffix,
    const olive_heads *out, const float *lse, const olive_heads *grad_out,
    const olive_heads *grad_q, const olive_heads *grad_k_prefix,
    const olive_heads *grad_v_prefix, const olive_heads *grad_k_suffix,
    const olive_heads *grad_v_suffix, void *workspace, int64_t workspace_bytes,
    void *hip_stream) {
    olive_status s = check_attn(desc);
    if (s != OLIVE_OK) return s;
    if (desc->max_suffix > 0 && desc->page_table) return OLIVE_E_UNSUPPORTED;
    if (desc->total_q > 0 && (missing(q) || missing(out) || missing(grad_out) || missing(grad_q) || !lse))
        return OLIVE_E_NULL;
    if (desc->max_prefix > 0 && (missing(k_prefix) || missing(v_prefix) || missing(grad_k_prefix) ||
                                 missing(grad_v_prefix)))
        return OLIVE_E_NULL;
    if (desc->max_suffix > 0 && (missing(k_suffix) || missing(v_suffix) || missing(grad_k_suffix) ||
                                 missing(grad_v_suffix)))
        return OLIVE_E_NULL;
    const int esz = desc->dtype == OLIVE_BF16 ? 2 : 4;
    for (const olive_heads *h : {q, k_prefix, v_prefix, k_suffix, v_suffix, out, grad_out, grad_q,
                                 grad_k_prefix, grad_v_prefix, grad_k_suffix, grad_v_suffix})
        if (misplaced(h, esz)) return OLIVE_E_UNSUPPORTED;
    AttnArgs a = attn_args(desc);
    const bool bf16 = desc->dtype == OLIVE_BF16;
    s = check_workspace(workspace, workspace_bytes, attn_backward_bytes(a, bf16));
    if (s != OLIVE_OK) return s;
    a.q = heads(q);
    a.kp = heads(k_prefix);
    a.vp = heads(v_prefix);
    a.ks = heads(k_suffix);
    a.vs = heads(v_suffix);
    a.o = heads(out);
    a.lse = const_cast<float *>(lse);
    a.go = heads(grad_out);
    a.gq = heads(grad_q);
    a.gkp = heads(grad_k_prefix);
    a.gvp = heads(grad_v_prefix);
    a.gks = heads(grad_k_suffix);
    a.gvs = heads(grad_v_suffix);
    a.work = (char *)workspace;
    return check_hip(launch_attn_backward(a, bf16, (hipStream_t)hip_stream));
}

olive_status olive_grad_clip_init(olive_clip_ctx **out, const olive_grad_tensor *list,
                                  int32_t count, void *hip_stream) {
    if (!out) return OLIVE_E_NULL;
    *out = nullptr;
    if (count < 0) return OLIVE_E_SHAPE;
    if (count > 0 && !list) return OLIVE_E_NULL;
    int64_t n_chunks = 0;
    for (int32_t i = 0; i < count; ++i) {
        const olive_grad_tensor &t = list[i];
        if (t.n < 0) return OLIVE_E_SHAPE;
        if ((t.dtype != OLIVE_F32 && t.dtype != OLIVE_BF16) ||
            (t.out && t.dtype_out != OLIVE_F32 && t.dtype_out != OLIVE_BF16))
            return OLIVE_E_DTYPE;
        if (t.n > 0 && !t.grad) return OLIVE_E_NULL;
        if (t.out && t.out == t.grad && t.dtype_out != t.dtype) return OLIVE_E_RANGE;
        if ((uintptr_t)t.grad % (t.dtype == OLIVE_BF16 ? 2 : 4) ||
            (t.out && (uintptr_t)t.out % (t.dtype_out == OLIVE_BF16 ? 2 : 4)))
            return OLIVE_E_UNSUPPORTED;
        const int64_t c = t.n / kClipChunk + (t.n % kClipChunk > 0);
        if (c > kMaxInt - n_chunks) return OLIVE_E_SHAPE;
        n_chunks += c;
    }
    olive_clip_ctx *ctx = new (std::nothrow) olive_clip_ctx;
    ClipTensor *ht = new (std::nothrow) ClipTensor[(size_t)count + 1];
    ClipChunk *hc = new (std::nothrow) ClipChunk[n_chunks + 1];
    olive_status s = ctx && ht && hc ? OLIVE_OK : OLIVE_E_NOMEM;
    if (s == OLIVE_OK) {
        int64_t at = 0;
        for (int32_t i = 0; i < count; ++i) {
            const olive_grad_tensor &t = list[i];
            ht[i] = ClipTensor{t.grad, t.out, t.n, t.dtype == OLIVE_BF16, t.dtype_out == OLIVE_BF16};
            for (int64_t j = 0; j < t.n; j += kClipChunk)
                hc[at++] = ClipChunk{j, i, (int32_t)(t.n - j < kClipChunk ? t.n - j : kClipChunk)};
        }
        ctx->n_chunks = n_chunks;
        hipStream_t st = (hipStream_t)hip_stream;
        if (hipMalloc((void **)&ctx->tensors, sizeof(ClipTensor) * ((size_t)count + 1)) != hipSuccess ||
            hipMalloc((void **)&ctx->chunks, sizeof(ClipChunk) * (n_chunks + 1)) != hipSuccess ||
            hipMalloc((void **)&ctx->part, sizeof(double) * kClipBlocks) != hipSuccess)
            s = OLIVE_E_NOMEM;
        else if ((count && hipMemcpyAsync(ctx->tensors, ht, sizeof(ClipTensor) * count,
                                          hipMemcpyHostToDevice, st) != hipSuccess) ||
                 (n_chunks && hipMemcpyAsync(ctx->chunks, hc, sizeof(ClipChunk) * n_chunks,
                                             hipMemcpyHostToDevice, st) != hipSuccess) ||
                 hipStreamSynchronize(st) != hipSuccess)
            s = OLIVE_E_HIP;
    }
    delete[] ht;
    delete[] hc;
    if (s != OLIVE_OK) {
        if (ctx) {
            (void)hipFree(ctx->tensors);
            (void)hipFree(ctx->chunks);
            (void)hipFree(ctx->part);
        }
        delete ctx;
        return s;
    }
    *out = ctx;
    return OLIVE_OK;
}

olive_status olive_grad_clip(olive_clip_ctx *ctx, float max_norm, float *norm, void *hip_stream) {
    if (!ctx) return OLIVE_E_NULL;
    if (!(max_norm >= 0.f)) return OLIVE_E_RANGE;
    return check_hip(launch_clip(ctx->tensors, ctx->chunks, ctx->n_chunks, ctx->part, max_norm, norm,
                                 (hipStream_t)hip_stream));
}

olive_status olive_grad_clip_free(olive_clip_ctx *ctx) {
    if (!ctx) return OLIVE_OK;
    const hipError_t e = hipDeviceSynchronize();
    (void)hipFree(ctx->tensors);
    (void)hipFree(ctx->chunks);
    (void)hipFree(ctx->part);
    delete ctx;
    return check_hip(e);
}

}  // extern "C"
