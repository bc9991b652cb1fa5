/* Host rejection paths of include/olive_layers.h; no call here reaches a device. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "olive_layers.h"

static int failures;
#define EXPECT(call, want)                                                        \
    do {                                                                          \
        const olive_status got_ = (call);                                         \
        if (got_ != (want)) {                                                     \
            printf("line %d: %s = %d, expected %d\n", __LINE__, #call, got_, want); \
            ++failures;                                                           \
        }                                                                         \
    } while (0)

static int words[64];        /* addresses that are never followed on a device */

int main(void) {
    int64_t n = 0;
    const olive_heads h = {words, 64, 16}, none = {NULL, 0, 0}, odd = {(char *)words + 1, 64, 16};

    olive_qk_desc q;
    memset(&q, 0, sizeof q);
    EXPECT(olive_qk_norm_rope(NULL, &h, &h, NULL, &h, &h, NULL, NULL), OLIVE_E_NULL);
    EXPECT(olive_qk_norm_rope(&q, &h, &h, NULL, &h, &h, NULL, NULL), OLIVE_E_RANGE);
    q.size = sizeof q;
    q.dtype = OLIVE_BF16;
    q.tokens = 4;
    q.heads_q = 2;
    q.heads_k = 1;
    q.head_dim = 16;
    q.rot_dim = 16;
    EXPECT(olive_qk_norm_rope(&q, &h, &h, NULL, &h, &h, NULL, NULL), OLIVE_E_NULL);
    q.positions = words;
    q.cos = q.sin = (const float *)words;
    EXPECT(olive_qk_norm_rope(&q, &h, &h, NULL, &h, &h, NULL, NULL), OLIVE_E_SHAPE);
    q.num_positions = 8;
    EXPECT(olive_qk_norm_rope(&q, NULL, &h, NULL, &h, &h, NULL, NULL), OLIVE_E_NULL);
    EXPECT(olive_qk_norm_rope(&q, &h, &none, NULL, &h, &h, NULL, NULL), OLIVE_E_NULL);
    EXPECT(olive_qk_norm_rope(&q, &h, &h, &h, &h, &h, NULL, NULL), OLIVE_E_NULL);
    EXPECT(olive_qk_norm_rope(&q, &odd, &h, NULL, &h, &h, NULL, NULL), OLIVE_E_UNSUPPORTED);
    q.eps = NAN;
    EXPECT(olive_qk_norm_rope(&q, &h, &h, NULL, &h, &h, NULL, NULL), OLIVE_E_RANGE);
    q.eps = 0.f;
    EXPECT(olive_qk_norm_rope_workspace(&q, NULL), OLIVE_E_NULL);
    EXPECT(olive_qk_norm_rope_workspace(&q, &n), OLIVE_OK);
    q.weight_q = words;
    EXPECT(olive_qk_norm_rope_backward(&q, &h, &h, &h, &h, &h, &h, (float *)words, NULL, NULL, n, NULL),
           OLIVE_E_NULL);
    EXPECT(olive_qk_norm_rope_backward(&q, &h, &h, &h, &h, &h, &h, (float *)words, NULL, words, n - 1, NULL),
           n ? OLIVE_E_SHAPE : OLIVE_OK);
    EXPECT(olive_qk_norm_rope_backward(&q, &h, &h, &h, &h, &h, &h, NULL, (float *)words, words, n, NULL),
           OLIVE_E_NULL);

    olive_attn_desc a;
    memset(&a, 0, sizeof a);
    EXPECT(olive_prefix_attention(NULL, &h, &h, &h, &h, &h, &h, NULL, NULL, 0, NULL), OLIVE_E_NULL);
    EXPECT(olive_prefix_attention_workspace(NULL, 0, &n), OLIVE_E_NULL);
    a.size = sizeof a;
    a.dtype = OLIVE_BF16;
    a.num_groups = 1;
    a.num_seqs = 3;
    a.heads_q = 4;
    a.heads_kv = 2;
    a.head_dim = 64;
    a.max_q = 1;
    a.total_q = 3;
    a.max_prefix = 1000000;
    a.max_suffix = 70;
    a.prefix_rows = 1000000;
    a.suffix_rows = 210;
    a.scale = 0.125f;
    a.group_seqs = a.cu_q = a.prefix_len = a.suffix_len = words;
    a.prefix_start = (const int64_t *)words;
    EXPECT(olive_prefix_attention_workspace(&a, 0, &n), OLIVE_E_NULL);      /* no suffix rows */
    a.suffix_start = (const int64_t *)words;
    EXPECT(olive_prefix_attention_workspace(&a, 0, NULL), OLIVE_E_NULL);
    EXPECT(olive_prefix_attention_workspace(&a, 0, &n), OLIVE_OK);
    EXPECT(olive_prefix_attention(&a, &h, &h, &h, &h, &h, &h, NULL, NULL, 0, NULL), n ? OLIVE_E_NULL : OLIVE_OK);
    EXPECT(olive_prefix_attention(&a, &h, NULL, &h, &h, &h, &h, NULL, words, n, NULL), OLIVE_E_NULL);
    EXPECT(olive_prefix_attention(&a, &h, &h, &h, &h, &h, &odd, NULL, words, n, NULL), OLIVE_E_UNSUPPORTED);
    EXPECT(olive_prefix_attention_workspace(&a, 1, &n), OLIVE_OK);
    EXPECT(olive_prefix_attention_backward(&a, &h, &h, &h, &h, &h, &h, NULL, &h, &h, &h, &h, &h, &h, words, n, NULL),
           OLIVE_E_NULL);
    EXPECT(olive_prefix_attention_backward(&a, &h, &h, &h, &h, &h, &h, (float *)words, &h, &h, &h, &h, &h, &h,
                                           words, n - 1, NULL), OLIVE_E_SHAPE);
    /* sizes at the edges of the host's arithmetic */
    a.max_suffix = 0;
    a.max_prefix = 0;
    EXPECT(olive_prefix_attention_workspace(&a, 0, &n), OLIVE_OK);
    a.max_prefix = 0x7fffffff;
    EXPECT(olive_prefix_attention_workspace(&a, 0, &n), OLIVE_OK);
    a.total_q = 0x7fffffff / 4;
    a.max_q = 0x7fffffff;         /* 3 sequences x 2^28 tiles of 16 rows x 2 heads */
    EXPECT(olive_prefix_attention_workspace(&a, 0, &n), OLIVE_OK);
    a.num_seqs = 5;               /* 5 x 2^28 x 2 workgroups are more than a launch holds */
    EXPECT(olive_prefix_attention_workspace(&a, 0, &n), OLIVE_E_SHAPE);
    a.num_seqs = 3;
    a.max_q = 1 << 20;
    EXPECT(olive_prefix_attention_workspace(&a, 1, &n), OLIVE_OK);
    a.total_q += 1;
    EXPECT(olive_prefix_attention_workspace(&a, 0, &n), OLIVE_E_SHAPE);
    a.total_q = 3;
    a.num_groups = 0;
    EXPECT(olive_prefix_attention_workspace(&a, 0, &n), OLIVE_E_SHAPE);
    a.num_groups = 1;
    a.heads_kv = 0;
    EXPECT(olive_prefix_attention_workspace(&a, 0, &n), OLIVE_E_SHAPE);

    olive_clip_ctx *c = (olive_clip_ctx *)words;
    const olive_grad_tensor t = {words, words, -1, OLIVE_F32, OLIVE_F32};
    EXPECT(olive_grad_clip_init(NULL, &t, 1, NULL), OLIVE_E_NULL);
    EXPECT(olive_grad_clip_init(&c, &t, 1, NULL), OLIVE_E_SHAPE);
    if (c) {
        printf("a failed init left a context\n");
        ++failures;
    }
    EXPECT(olive_grad_clip_init(&c, NULL, 1, NULL), OLIVE_E_NULL);
    EXPECT(olive_grad_clip(NULL, 1.f, NULL, NULL), OLIVE_E_NULL);
    EXPECT(olive_grad_clip_free(NULL), OLIVE_OK);
    return failures ? 1 : 0;
}
