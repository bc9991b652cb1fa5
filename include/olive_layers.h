/*
 * olive_layers.h -- C ABI of the layer operators that stand on either side of the scoring
 * (olive_score.h): a student continues prefixes that several rollouts share (Sec. 3.1: the
 * prefix is rolled in once and continued several times), and is updated on them.
 *
 *   olive_qk_norm_rope       an RMS norm of every query and key head and the position
 *                            rotation, in one pass; optionally the keys and values go to
 *                            their rows of a cache in the same pass. With its backward.
 *   olive_prefix_attention   attention of sequences that share a prefix by groups, each
 *                            with a causal suffix of its own (packed rows or cache pages):
 *                            single tokens, short runs, whole continuations, prompts. With
 *                            its backward for packed suffixes.
 *   olive_grad_clip          the global norm over many gradients, and the gradients scaled
 *                            so that it does not exceed a limit.
 *
 * The conventions of olive_score.h hold: device pointers on the current device, calls that
 * take a stream only validate host-visible arguments and enqueue kernels on it (no
 * allocation, memset or synchronisation: they may be captured into a HIP graph), no call
 * throws or aborts. Results do not depend on the order in which workgroups run: the same
 * call on the same inputs gives the same bits.
 *
 * Sums, softmax statistics and norms are held in 32 bits or more whatever the dtype, and
 * an output is rounded to its dtype once. With bf16 the attention's weights, and in its
 * backward their gradients, are rounded to bf16 too, as operands of the next product.
 * Workspaces are the caller's: a call leaves
 * nothing in them that a later call reads, and calls that may overlap need one each.
 */
#ifndef OLIVE_LAYERS_H
#define OLIVE_LAYERS_H

#include "olive_score.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A [tokens][heads][head_dim] view: the elements of a head are contiguous, tokens and
 * heads lie at any distance (in elements), so the parts of one projection's rows can be
 * passed as they are. data is aligned to its element type. */
typedef struct {
    void *data;                  /* device */
    int64_t stride_token;
    int64_t stride_head;
} olive_heads;

/* ------------------------------------------------- norms of heads with the rotation -- */

#define OLIVE_ROPE_HALF 0  /* element i pairs with i + rot_dim / 2 */
#define OLIVE_ROPE_PAIRS 1 /* element 2 i pairs with 2 i + 1 */

/*
 *   n = x * (mean(x^2) + eps)^-1/2 * weight       (x itself where the weight is NULL)
 *   y = (n_a cos - n_b sin, n_b cos + n_a sin)    for each pair (a, b) of the first rot_dim
 *                                                 elements; the others are n
 * with cos and sin from the rows that the tokens' positions select: tables of the caller's,
 * so that any frequencies, scaled for long contexts or not, are expressed by them.
 */
typedef struct {
    int32_t size;                /* sizeof(olive_qk_desc) (checked) */
    int32_t dtype;               /* olive_dtype of the heads and the weights */
    int64_t tokens;              /* >= 0 (0: the call does nothing), < 2^31 */
    int32_t heads_q;             /* >= 0; the heads of q and k together in [1, 4096] */
    int32_t heads_k;             /* >= 0 */
    int32_t head_dim;            /* in [1, 256] */
    int32_t rot_dim;             /* even, in [0, head_dim] */
    int32_t layout;              /* OLIVE_ROPE_* */
    float eps;                   /* finite, >= 0 */
    const int32_t *positions;    /* device [tokens] in [0, num_positions); NULL if rot_dim = 0 */
    int64_t num_positions;       /* rows of cos and sin */
    const float *cos, *sin;      /* device [num_positions][rot_dim / 2]; NULL if rot_dim = 0 */
    const void *weight_q;        /* device [head_dim] or NULL (q is only rotated) */
    const void *weight_k;        /* device [head_dim] or NULL (k is only rotated) */
    const int32_t *slots;        /* device [tokens] or NULL: the row of k_out and v_out that a
                                    token's key and value go to (distinct; a row that is
                                    negative or >= slot_rows is not written) */
    int64_t slot_rows;           /* rows of k_out and v_out when slots is set */
} olive_qk_desc;

/*
 * q_out and k_out get the normed and rotated heads; they may be q and k themselves (in
 * place), else they do not overlap them. v and v_out: NULL, or the values of heads_k heads
 * and where they are copied to (the rows of k_out). q / q_out may be NULL when heads_q = 0,
 * k / k_out when heads_k = 0. A token whose position is out of range gets NaN (its value is
 * copied as it is).
 * Errors: E_NULL, E_SHAPE, E_DTYPE, E_RANGE (size, layout, rot_dim, eps), E_UNSUPPORTED
 * (more than 256 elements or 4096 heads; a view that is not aligned to its type), E_HIP.
 */
olive_status olive_qk_norm_rope(const olive_qk_desc *desc, const olive_heads *q,
                                const olive_heads *k, const olive_heads *v,
                                const olive_heads *q_out, const olive_heads *k_out,
                                const olive_heads *v_out, void *hip_stream);

/* Bytes of olive_qk_norm_rope_backward's workspace (host; no device needed). */
olive_status olive_qk_norm_rope_workspace(const olive_qk_desc *desc, int64_t *bytes);

/*
 * The gradients of q, k and of the norms' weights from those of q_out and k_out
 * (desc->slots is not read: the gradients lie in the tokens' order):
 *   g = rotation transposed of grad_out,   grad_weight = sum over tokens and heads of g x r
 *   grad_x = r (g w - x r mean(g w x r)),  r = (mean(x^2) + eps)^-1/2
 * grad_q and grad_k may be grad_q_out and grad_k_out themselves. grad_weight_q and
 * grad_weight_k: fp32 [head_dim] or NULL; NULL where the weight is. workspace: device,
 * 16-byte aligned, needed where a weight gradient is asked for.
 * Errors: as olive_qk_norm_rope, plus E_SHAPE for a workspace that is too small and
 * E_UNSUPPORTED for one that is not aligned.
 */
olive_status olive_qk_norm_rope_backward(const olive_qk_desc *desc, const olive_heads *q,
                                         const olive_heads *k, const olive_heads *grad_q_out,
                                         const olive_heads *grad_k_out,
                                         const olive_heads *grad_q, const olive_heads *grad_k,
                                         float *grad_weight_q, float *grad_weight_k,
                                         void *workspace, int64_t workspace_bytes,
                                         void *hip_stream);

/* ------------------------------------------------------- attention on shared prefixes -- */

/*
 * Sequences [group_seqs[g], group_seqs[g + 1]) share prefix g: rows prefix_start[g] +
 * [0, prefix_len[g]) of the prefix keys and values. Sequence b has suffix_len[b] tokens of
 * its own, and its queries, rows [cu_q[b], cu_q[b + 1]) of q, are the last n_b of them:
 * query i sees the whole prefix and the suffix tokens j <= suffix_len[b] - n_b + i. A
 * query that sees nothing gets zeros and the log-normaliser -inf. Query head h reads key
 * head h / (heads_q / heads_kv).
 *   out = sum_j p_j v_j,   p = exp(scale q k_j - lse),   lse = log sum_j exp(scale q k_j)
 * The suffix rows are packed, suffix_start[b] + j, or pages: token j of sequence b is row
 * page_table[b * table_stride + j / page_size] * page_size + j % page_size.
 * max_q, max_prefix and max_suffix bound what the device arrays hold and choose how the
 * work is split; a sequence beyond them, or with rows outside the buffers, gets NaN (with
 * pages: at least the queries that see a token of such a page). One whose cu_q entries are
 * not in order within [0, total_q] is left out; others of a call with such entries, or with
 * group_seqs out of order, may get NaN where their rows do not lie between the first and the
 * last entry of their group. Rows that two sequences or groups have get no defined value.
 * Rows of keys and values that no sequence has are never read into a result.
 */
typedef struct {
    int32_t size;                /* sizeof(olive_attn_desc) (checked) */
    int32_t dtype;               /* olive_dtype of every view */
    int32_t num_groups;          /* G >= 1, G <= num_seqs */
    int32_t num_seqs;            /* B >= 1, < 2^20 */
    int32_t heads_q;             /* a multiple of heads_kv, <= 4096 */
    int32_t heads_kv;            /* >= 1 */
    int32_t head_dim;            /* in [1, 256] */
    int32_t max_q;               /* >= 1: most queries of a sequence */
    int64_t total_q;             /* cu_q[B] (host copy of it), >= 0 (0: nothing is done);
                                    total_q * heads_q < 2^31 */
    int64_t max_prefix;          /* >= 0, < 2^31: longest prefix */
    int64_t max_suffix;          /* >= 0, < 2^31: longest suffix */
    int64_t prefix_rows;         /* rows of the prefix keys and values */
    int64_t suffix_rows;         /* rows of the suffix keys and values */
    const int32_t *group_seqs;   /* device [G + 1]: 0 first, not decreasing, B last */
    const int32_t *cu_q;         /* device [B + 1]: 0 first, not decreasing, total_q last */
    const int64_t *prefix_start; /* device [G] */
    const int32_t *prefix_len;   /* device [G] */
    const int32_t *suffix_len;   /* device [B] */
    const int64_t *suffix_start; /* device [B], or NULL with a page table */
    const int32_t *page_table;   /* device [B][table_stride], or NULL with suffix_start */
    int64_t table_stride;        /* entries a sequence, * page_size >= max_suffix */
    int32_t page_size;           /* >= 1 with a page table */
    float scale;                 /* finite */
} olive_attn_desc;

/* Bytes of the forward's workspace (backward: 0) or of the backward's (1). Host only. They
 * grow with total_q, heads_q and head_dim alone (two times min(64 r, 65536 + r) (head_dim + 2)
 * values for r = total_q heads_q rows; 8 r bytes and 1024 tiles of 128 keys for the backward):
 * the workspace of the largest call of a dtype serves the others. */
olive_status olive_prefix_attention_workspace(const olive_attn_desc *desc, int32_t backward,
                                              int64_t *bytes);

/*
 * out: [total_q][heads_q] heads. lse: device fp32 [total_q][heads_q] or NULL. The prefix
 * views may be NULL when max_prefix = 0, the suffix views when max_suffix = 0. workspace:
 * device, 16-byte aligned, NULL if 0 bytes are needed.
 * Errors: E_NULL, E_SHAPE (sizes; a workspace that is too small), E_DTYPE, E_RANGE (size,
 * scale), E_UNSUPPORTED (head_dim > 256; a view that is not aligned to its type, a workspace
 * that is not aligned), E_HIP.
 */
olive_status olive_prefix_attention(const olive_attn_desc *desc, const olive_heads *q,
                                    const olive_heads *k_prefix, const olive_heads *v_prefix,
                                    const olive_heads *k_suffix, const olive_heads *v_suffix,
                                    const olive_heads *out, float *lse, void *workspace,
                                    int64_t workspace_bytes, void *hip_stream);

/*
 * The gradients of q and of the keys and values from out's, with out and lse of the
 * forward. The gradient of a prefix row is the sum over its group's sequences; rows that
 * belong to no prefix or suffix are not written, and no two prefixes or suffixes overlap.
 * Packed suffixes only (E_UNSUPPORTED with a page table). A sequence that is out of range
 * or left out makes NaN of the gradients of its suffix and of its group's prefix; where
 * these rows themselves are out of range they are not written. A value that is not finite may reach
 * the gradients of other rows and keys of its sequence and group, also of queries that do not
 * see it (the forward keeps it from them).
 */
olive_status olive_prefix_attention_backward(
    const olive_attn_desc *desc, const olive_heads *q, const olive_heads *k_prefix,
    const olive_heads *v_prefix, const olive_heads *k_suffix, const olive_heads *v_suffix,
    const olive_heads *out, const float *lse, const olive_heads *grad_out,
    const olive_heads *grad_q, const olive_heads *grad_k_prefix,
    const olive_heads *grad_v_prefix, const olive_heads *grad_k_suffix,
    const olive_heads *grad_v_suffix, void *workspace, int64_t workspace_bytes,
    void *hip_stream);

/* --------------------------------------------------------------- gradient clipping -- */

typedef struct olive_clip_ctx olive_clip_ctx; /* opaque */

/* One gradient: n contiguous values (0 allowed), and where the scaled ones go. */
typedef struct {
    const void *grad;            /* device, aligned to its type; may be NULL if n = 0 */
    void *out;                   /* device: grad itself (in place), a buffer that overlaps no
                                    gradient, or NULL (the gradient counts for the norm and
                                    is not scaled) */
    int64_t n;
    int32_t dtype;               /* olive_dtype of grad */
    int32_t dtype_out;           /* olive_dtype of out; dtype when out is grad */
} olive_grad_tensor;

/*
 * A list of count >= 0 gradients (host array, copied). The context holds the list and the
 * partial sums on the device; init synchronises the stream. It borrows the gradients: a
 * program whose gradients stay where they are keeps the context (making one costs more than a
 * call on small gradients).
 * Errors: E_NULL, E_SHAPE (a negative count or n, more values than the chunks' count holds),
 * E_DTYPE, E_RANGE (in place with another dtype_out), E_UNSUPPORTED (a gradient or output that
 * is not aligned to its type), E_NOMEM, E_HIP.
 */
olive_status olive_grad_clip_init(olive_clip_ctx **out, const olive_grad_tensor *list,
                                  int32_t count, void *hip_stream);

/*
 *   norm = (sum over all gradients of their squares)^1/2      (summed in 64 bits)
 *   out  = grad * min(1, max_norm / (norm + 1e-6))
 * norm: device fp32 [1] or NULL. max_norm >= 0; +inf: out gets the gradients unscaled
 * (nothing is written in place). A norm that is not finite in fp32 leaves the gradients
 * unscaled too, and the caller skips the step by it. A context takes one call at a time.
 * Errors: E_NULL, E_RANGE (max_norm negative or NaN), E_HIP.
 */
olive_status olive_grad_clip(olive_clip_ctx *ctx, float max_norm, float *norm,
                             void *hip_stream);

/* Release a context (NULL is accepted). Synchronises the device. */
olive_status olive_grad_clip_free(olive_clip_ctx *ctx);

#ifdef __cplusplus
}
#endif

#endif /* OLIVE_LAYERS_H */
