/*
 * olive_tokens.h -- C ABI of the operators between tokens and rows, beside the scoring
 * (olive_score.h) and the layers (olive_layers.h): what a student's rollouts and its update
 * need at both ends of the model (Sec. 3.1: the student samples its own prefix, and is
 * updated on what follows).
 *
 *   olive_embed       rows of an embedding table, scaled. With the table's gradient by sorted
 *                     tokens, written whole or added to one that is there (the gradient of
 *                     the vocabulary projection, where both share one weight).
 *   olive_row_norm    the residual added, then a layer norm or an RMS norm of every row, in
 *                     one pass. With its backward and the gradients of weight and bias.
 *   olive_sample      the next token of every row of logits: temperature, top-k, top-p and
 *                     min-p of each row, from given uniform numbers, with its log-prob.
 *
 * The conventions of olive_score.h hold: device pointers on the current device, calls that
 * take a stream only validate host-visible arguments and enqueue kernels on it (no
 * allocation, memset or synchronisation: they may be captured into a HIP graph), no call
 * throws or aborts. Results do not depend on the order in which workgroups run: the same
 * call on the same inputs gives the same bits.
 *
 * Sums, statistics and norms are held in 32 bits or more whatever the dtype, the masses that
 * a token is drawn by in 64, and an output is rounded to its dtype once. Matrices are
 * [rows][width] with contiguous rows that lie `stride` elements apart: an output's are at
 * least width apart, an input's may be the same row again (stride 0). Workspaces are the
 * caller's: a call leaves nothing in them that a later call reads, and calls that may
 * overlap need one each.
 */
#ifndef OLIVE_TOKENS_H
#define OLIVE_TOKENS_H

#include "olive_score.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ----------------------------------------------------------------------- embedding -- */

/*
 *   out[t] = scale * table[ids[t]]            (a row of zeros where ids[t] is negative: the
 *                                              padding that the scoring's argmax marks by -1)
 * A token >= vocab gets a row of NaN.
 */
typedef struct {
    int32_t size;                /* sizeof(olive_embed_desc) (checked) */
    int32_t dtype;               /* olive_dtype of the table and out (backward: of grad_out) */
    int64_t tokens;              /* >= 0, <= 2^26 */
    int64_t vocab;               /* rows of the table, >= 1, < 2^31 */
    int32_t width;               /* in [1, 65536] */
    float scale;                 /* finite */
    const int32_t *ids;          /* device [tokens] (NULL if tokens = 0) */
} olive_embed_desc;

/*
 * table: [vocab][width], out: [tokens][width]; they do not overlap.
 * Errors: E_NULL, E_SHAPE (sizes, strides), E_DTYPE, E_RANGE (size, scale), E_UNSUPPORTED
 * (more than 2^26 tokens or 65536 elements; a matrix that is not aligned to its type), E_HIP.
 */
olive_status olive_embed(const olive_embed_desc *desc, const void *table, int64_t table_stride,
                         void *out, int64_t out_stride, void *hip_stream);

/* Bytes of olive_embed_backward's workspace (host; no device needed). */
olive_status olive_embed_workspace(const olive_embed_desc *desc, int64_t *bytes);

/*
 *   grad_table[v] (+)= scale * sum over t with ids[t] = v of grad_out[t]
 * summed in 32 bits, in an order that the tokens alone decide. accumulate 0: the whole table is
 * written, zeros for tokens that do not occur; accumulate 1: only the rows of tokens that occur
 * are read and written. grad_dtype: olive_dtype of grad_table. Negative tokens and tokens >=
 * vocab have no part in it. grad_out and grad_table do not overlap. workspace: device, 16-byte
 * aligned, of olive_embed_workspace's bytes; NULL if 0 are needed (up to 1024 tokens; else 16
 * bytes a token, and for every 16 to 64 tokens two rows in fp32, each of the width rounded up to
 * a multiple of 512).
 * Errors: as olive_embed, plus E_SHAPE for a workspace that is too small.
 */
olive_status olive_embed_backward(const olive_embed_desc *desc, const void *grad_out,
                                  int64_t grad_out_stride, void *grad_table,
                                  int64_t grad_table_stride, int32_t grad_dtype,
                                  int32_t accumulate, void *workspace, int64_t workspace_bytes,
                                  void *hip_stream);

/* ----------------------------------------------------------------------- row norms -- */

#define OLIVE_NORM_RMS 0   /* n = h (mean(h^2) + eps)^-1/2 */
#define OLIVE_NORM_LAYER 1 /* n = (h - mean(h)) (mean((h - mean(h))^2) + eps)^-1/2 */

/*
 *   h = x + residual, rounded to the dtype (x itself without a residual)
 *   y = n * weight + bias           (a NULL weight is 1, a NULL bias 0)
 * for values of any size: squares need not be numbers of fp32, and the mean is summed in 64 bits.
 */
typedef struct {
    int32_t size;                /* sizeof(olive_norm_desc) (checked) */
    int32_t dtype;               /* olive_dtype of the rows, weight and bias */
    int64_t rows;                /* >= 0 (0: nothing is normed), < 2^31 */
    int32_t width;               /* in [1, 16384] */
    int32_t kind;                /* OLIVE_NORM_* */
    float eps;                   /* finite, >= 0 */
    const void *weight;          /* device [width] or NULL */
    const void *bias;            /* device [width] or NULL */
} olive_norm_desc;

/*
 * x, residual, out, sum: [rows][width]; residual NULL: none; sum: where h goes, or NULL.
 * out or sum may be x or residual themselves (with their strides), and each other's buffers
 * are distinct; other overlaps are not allowed. The rows are normed as the sum that is stored.
 * Errors: E_NULL, E_SHAPE (sizes, strides, out where sum is, or an output where an input of
 * other strides is), E_DTYPE, E_RANGE (size, kind, eps),
 * E_UNSUPPORTED (more than 16384 elements; a matrix that is not aligned to its type), E_HIP.
 */
olive_status olive_row_norm(const olive_norm_desc *desc, const void *x, int64_t x_stride,
                            const void *residual, int64_t residual_stride, void *out,
                            int64_t out_stride, void *sum, int64_t sum_stride, void *hip_stream);

/* Bytes of olive_row_norm_backward's workspace (host; no device needed). */
olive_status olive_row_norm_workspace(const olive_norm_desc *desc, int64_t *bytes);

/*
 * From the normed rows h (the forward's sum, or x without a residual) and the gradient of y:
 *   g = grad_out * weight,  r = (mean(..) + eps)^-1/2 as in the forward
 *   grad_h = r (g - n mean(g n) [- mean(g) for the layer norm]) + grad_sum
 *   grad_weight = sum over rows of grad_out n,  grad_bias = sum over rows of grad_out
 * grad_sum: the gradient that reaches the stored sum from elsewhere (the residual stream),
 * or NULL; grad_h is the gradient of x and of the residual alike. grad_h may be grad_out or
 * grad_sum themselves. grad_weight, grad_bias: fp32 [width], written whole (zeros without
 * rows), or NULL; they need no weight or bias in the descriptor. workspace: device, 16-byte
 * aligned, needed where one of them is asked for.
 * Errors: as olive_row_norm, plus E_SHAPE for a workspace that is too small.
 */
olive_status olive_row_norm_backward(const olive_norm_desc *desc, const void *h, int64_t h_stride,
                                     const void *grad_out, int64_t grad_out_stride,
                                     const void *grad_sum, int64_t grad_sum_stride, void *grad_h,
                                     int64_t grad_h_stride, float *grad_weight, float *grad_bias,
                                     void *workspace, int64_t workspace_bytes, void *hip_stream);

/* ------------------------------------------------------------------------ sampling -- */

/*
 * Of a row of logits z, with w_v = exp((z_v - max z) / temperature), and its tokens v in
 * order (the larger logit first, the lower index first among equal ones, -inf left out), the
 * first n are kept:
 *   n = max(1, min(n_k, n_p, n_m)),   n_k = min(top_k, tokens)         (top_k <= 0: all)
 *   n_p = the least n' with  w_1 + .. + w_n' >= top_p (w_1 + .. + w_n_k)   (top_p >= 1: all)
 *   n_m = the number of tokens with  w >= min_p                         (min_p <= 0: all)
 * and the token drawn is the first kept one in the order of the vocabulary where the sum of
 * the kept w up to it exceeds u times the sum of all of them (u = 0: the first kept one, u =
 * 1: the last). temperature 0 is greedy: the first token in order, alone.
 */
typedef struct {
    int32_t size;                /* sizeof(olive_sample_desc) (checked) */
    int32_t dtype;               /* olive_dtype of the logits */
    int64_t rows;                /* >= 0 (0: the call does nothing), <= 2^20 */
    int64_t vocab;               /* in [1, 2^24] */
    const float *uniform;        /* device [rows]: u in [0, 1] */
    const float *temperature;    /* device [rows], finite, >= 0; or NULL: 1 */
    const int32_t *top_k;        /* device [rows] or NULL: all */
    const float *top_p;          /* device [rows] or NULL: all */
    const float *min_p;          /* device [rows] or NULL: all */
} olive_sample_desc;

/* Bytes of olive_sample's workspace (host; no device needed). */
olive_status olive_sample_workspace(const olive_sample_desc *desc, int64_t *bytes);

/*
 * logits: [rows][vocab]. token: int32 [rows]. logp: fp32 [rows] or NULL, the log of the
 * token's share of the kept sum. kept: int32 [rows] or NULL, n. A row with a NaN or +inf, one
 * that is -inf throughout, and one whose settings are NaN or out of range gets token -1,
 * logp NaN and kept 0. workspace: device, 16-byte aligned, NULL if 0 bytes are needed.
 * Errors: E_NULL, E_SHAPE (sizes, a workspace that is too small), E_DTYPE, E_RANGE (size),
 * E_UNSUPPORTED (more than 2^20 rows or 2^24 tokens; logits that are not aligned to their
 * type, a workspace that is not aligned), E_HIP.
 */
olive_status olive_sample(const olive_sample_desc *desc, const void *logits, int64_t logits_stride,
                          int32_t *token, float *logp, int32_t *kept, void *workspace,
                          int64_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* OLIVE_TOKENS_H */
