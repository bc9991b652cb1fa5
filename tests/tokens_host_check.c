/* Host rejection paths of include/olive_tokens.h; no call here reaches a device. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "olive_tokens.h"

static int failures;
#define EXPECT(call, want)                                                        \
    do {                                                                          \
        const olive_status got_ = (call);                                         \
        if (got_ != (want)) {                                                     \
            printf("line %d: %s = %d, expected %d\n", __LINE__, #call, got_, want); \
            ++failures;                                                           \
        }                                                                         \
    } while (0)

static int words[64] __attribute__((aligned(16))); /* addresses that are never followed on a device */

int main(void) {
    int64_t n = 0;
    olive_embed_desc e;
    memset(&e, 0, sizeof e);
    EXPECT(olive_embed(NULL, words, 8, words, 8, NULL), OLIVE_E_NULL);
    EXPECT(olive_embed(&e, words, 8, words, 8, NULL), OLIVE_E_RANGE);
    e.size = sizeof e;
    e.dtype = OLIVE_BF16;
    e.tokens = 4;
    e.vocab = 10;
    e.width = 8;
    EXPECT(olive_embed(&e, words, 8, words, 8, NULL), OLIVE_E_NULL);
    e.ids = words;
    EXPECT(olive_embed(&e, words, 8, words, 7, NULL), OLIVE_E_SHAPE);
    EXPECT(olive_embed(&e, words, INT64_MAX, words, 8, NULL), OLIVE_E_SHAPE);
    EXPECT(olive_embed(&e, words, INT64_MIN, words, 8, NULL), OLIVE_E_SHAPE);
    EXPECT(olive_embed(&e, (char *)words + 1, 8, words, 8, NULL), OLIVE_E_UNSUPPORTED);
    EXPECT(olive_embed_workspace(&e, NULL), OLIVE_E_NULL);
    EXPECT(olive_embed_workspace(NULL, &n), OLIVE_E_NULL);
    /* sizes at the edges of the host's arithmetic */
    e.tokens = (int64_t)1 << 26;
    e.vocab = 0x7fffffff;
    e.width = 65536;
    EXPECT(olive_embed_workspace(&e, &n), OLIVE_OK);
    if (n) EXPECT(olive_embed_backward(&e, words, 65536, words, 65536, OLIVE_F32, 1, words, n - 1, NULL), OLIVE_E_SHAPE);
    e.tokens = 0;
    EXPECT(olive_embed_workspace(&e, &n), OLIVE_OK);
    e.tokens = INT64_MAX;
    EXPECT(olive_embed_workspace(&e, &n), OLIVE_E_UNSUPPORTED);
    e.tokens = 4;
    EXPECT(olive_embed_backward(&e, words, 65536, words, 65536, 7, 1, words, 1 << 30, NULL), OLIVE_E_DTYPE);
    EXPECT(olive_embed_backward(&e, words, 65536, words, 65536, OLIVE_F32, 3, words, 1 << 30, NULL), OLIVE_E_RANGE);

    olive_norm_desc m;
    memset(&m, 0, sizeof m);
    EXPECT(olive_row_norm(NULL, words, 8, NULL, 0, words, 8, NULL, 0, NULL), OLIVE_E_NULL);
    EXPECT(olive_row_norm(&m, words, 8, NULL, 0, words, 8, NULL, 0, NULL), OLIVE_E_RANGE);
    m.size = sizeof m;
    m.dtype = OLIVE_F32;
    m.rows = 0x7fffffff;
    m.width = 16384;
    m.eps = NAN;
    EXPECT(olive_row_norm(&m, words, 8, NULL, 0, words, 8, NULL, 0, NULL), OLIVE_E_RANGE);
    m.eps = 0.f;
    EXPECT(olive_row_norm(&m, words, 16384, NULL, 0, words, 16383, NULL, 0, NULL), OLIVE_E_SHAPE);
    EXPECT(olive_row_norm(&m, words, (int64_t)1 << 40, NULL, 0, words, 16384, NULL, 0, NULL), OLIVE_E_SHAPE);
    EXPECT(olive_row_norm_workspace(&m, &n), OLIVE_OK);
    EXPECT(olive_row_norm_backward(&m, words, 16384, words, 16384, NULL, 0, words, 16384, (float *)words, NULL, words,
                                   n - 1, NULL), OLIVE_E_SHAPE);
    EXPECT(olive_row_norm_backward(&m, words, 16384, words, 16384, NULL, 0, words, 16384, (float *)words, NULL, NULL, n,
                                   NULL), OLIVE_E_NULL);

    olive_sample_desc s;
    memset(&s, 0, sizeof s);
    EXPECT(olive_sample(NULL, words, 8, words, NULL, NULL, words, 0, NULL), OLIVE_E_NULL);
    EXPECT(olive_sample(&s, words, 8, words, NULL, NULL, words, 0, NULL), OLIVE_E_RANGE);
    s.size = sizeof s;
    s.dtype = OLIVE_BF16;
    s.rows = 1 << 20;
    s.vocab = 1 << 24;
    EXPECT(olive_sample_workspace(&s, &n), OLIVE_E_NULL);
    s.uniform = (const float *)words;
    EXPECT(olive_sample_workspace(&s, &n), OLIVE_OK);
    if (n) EXPECT(olive_sample(&s, words, 1 << 24, words, NULL, NULL, words, n - 1, NULL), OLIVE_E_SHAPE);
    EXPECT(olive_sample(&s, words, (int64_t)1 << 41, words, NULL, NULL, words, n, NULL), OLIVE_E_SHAPE);
    s.rows = INT64_MAX;
    EXPECT(olive_sample_workspace(&s, &n), OLIVE_E_UNSUPPORTED);
    s.rows = 1;
    s.vocab = INT64_MAX;
    EXPECT(olive_sample_workspace(&s, &n), OLIVE_E_UNSUPPORTED);
    return failures ? 1 : 0;
}
