// Launchers of the token operators (include/olive_tokens.h) and their argument structs.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "layers_internal.hpp"
#include "olive_tokens.h"

namespace olive {

struct RowsArg {                     // a [rows][width] matrix
    char *p;
    int64_t st;                      // elements between rows
};

// Whether an output is written past the caches: where the next kernel finds little of it there anyway (of widths
// that are multiples of 16 bytes; the others' vectors are written a part at a time). Rows of
// tokens and then their norm, 134 MB each: 88 us for 94 (the rows alone 30 for 45, norms of 268 MB 222
// for 230); of 34 MB 27 for 25, of 17 MB 18 for 17.
inline bool streamed(int64_t rows, int64_t width, int esz) { return rows * width * esz >= (int64_t)96 << 20; }

// ---- embedding -----------------------------------------------------------------------------
struct EmbedArgs {
    const int32_t *ids;
    int32_t tokens, vocab, width;
    float scale;
    RowsArg table, out;              // backward: the table's gradient, and that of the rows
    bool accumulate, stream;         // stream: out is written past the caches
    char *work;
};

int64_t embed_backward_bytes(const EmbedArgs &a);
hipError_t launch_embed(const EmbedArgs &a, bool bf16, hipStream_t st);
hipError_t launch_embed_backward(const EmbedArgs &a, bool bf16, bool table_bf16, hipStream_t st);

// ---- row norms -----------------------------------------------------------------------------
struct NormArgs {
    RowsArg x, res, out, sum;        // backward: h, grad_sum, grad_h, grad_out
    const void *weight, *bias;
    float *gw, *gb;                  // backward: or NULL
    float *part;                     // backward: [workgroups][2][width] partial sums
    int32_t rows, width, layer;
    float eps;
    double inv_width;
    bool stream;                     // what is written goes past the caches
};

int64_t norm_backward_bytes(const NormArgs &a);
hipError_t launch_norm(const NormArgs &a, bool bf16, hipStream_t st);
hipError_t launch_norm_backward(const NormArgs &a, bool bf16, hipStream_t st);

// ---- sampling ------------------------------------------------------------------------------
struct SampleArgs {
    RowsArg logits;
    int32_t rows, vocab;
    const float *uniform, *temperature;
    const int32_t *top_k;
    const float *top_p, *min_p;
    int32_t *token, *kept;
    float *logp;
    char *work;
};

int64_t sample_bytes(const SampleArgs &a, bool bf16);
hipError_t launch_sample(const SampleArgs &a, bool bf16, hipStream_t st);

}  // namespace olive
