// Launchers of the layer operators (include/olive_layers.h): their argument structs and the
// size rules that the host and the kernels share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "olive_layers.h"

namespace olive {

constexpr int kChipUnits = 256;      // compute units of an MI355X

// A grid has fewer than 2^32 threads along a dimension (of a launch with more, some workgroups
// never run, without an error), so workgroups of 256 threads past the first 2^23 go to further
// rows of it. The last row is a whole one: a kernel finds nothing to do at an index past its work.
constexpr int64_t kGridRow = 1 << 23;
constexpr int64_t kMostBlocks = 0x7fffffff - 2 * kGridRow;   // (with whole rows indexes fit an int)
inline dim3 grid_of(int64_t blocks) {
    if (blocks <= kGridRow) return dim3((uint32_t)blocks);
    return dim3((uint32_t)kGridRow, (uint32_t)((blocks + kGridRow - 1) / kGridRow));
}
#ifdef __HIPCC__
__device__ __forceinline__ int block_index() { return (int)(blockIdx.y * (uint32_t)kGridRow + blockIdx.x); }
#endif

// Division of 0 <= n < 2^31 by a d that is known on the host: with k = 31 + ceil(log2 d) and
// m = ceil(2^k / d), n m / 2^k is off by less than n / 2^k < 1 / d, so its floor is the quotient.
struct Div {
    uint32_t d, mul, shift;
    static Div of(int64_t d) {
        Div r{(uint32_t)d, 0, 0};
        uint32_t bits = 0;
        while (((int64_t)1 << bits) < d) ++bits;
        if (d > 1) {
            r.mul = (uint32_t)((((unsigned __int128)1 << (31 + bits)) + d - 1) / d);
            r.shift = bits - 1;
        }
        return r;
    }
    __host__ __device__ int quot(int n) const {
        return d == 1 ? n : (int)((uint32_t)((uint64_t)(uint32_t)n * mul >> 32) >> shift);
    }
    __host__ __device__ int rem(int n, int q) const { return n - q * (int)d; }
};

// at + n, no further than end (rows, tokens and keys go up to 2^31 - 1, where the sum passes 32 bits).
__host__ __device__ inline int upto(int at, int n, int end) { return n < (int64_t)end - at ? at + n : end; }

struct HeadsArg {                    // olive_heads with a typed use in the kernels
    char *p;
    int64_t st, sh;                  // elements between tokens and heads
};

// ---- norms of heads with the rotation ----------------------------------------------------
struct QkArgs {
    HeadsArg q, k, v, qo, ko, vo;    // backward: qo / ko hold the gradients of the outputs
    HeadsArg gq, gk;                 // backward: gradients of q and k
    int32_t tokens, hq, hk, hv, d, rot, layout;
    float eps;
    const int32_t *positions;
    int64_t num_positions;
    const float *cos, *sin;
    const void *wq, *wk;
    const int32_t *slots;
    int64_t slot_rows;
    float *gwq, *gwk;                // backward: weight gradients or NULL
    float *part;                     // backward: [blocks][2][d] partial weight gradients
};

constexpr int kQkBwdBlocks = 1024;   // workgroups of the backward at most (its partial rows)

hipError_t launch_qk_forward(const QkArgs &a, bool bf16, hipStream_t st);
hipError_t launch_qk_backward(const QkArgs &a, bool bf16, hipStream_t st);

// ---- gradient clipping -------------------------------------------------------------------
struct ClipTensor {
    const void *in;
    void *out;
    int64_t n;
    int32_t bf16_in, bf16_out;
};
struct ClipChunk {
    int64_t start;                   // first value of the chunk in its tensor
    int32_t tensor;
    int32_t n;                       // its values
};
constexpr int kClipChunk = 16384;    // values of a chunk
constexpr int kClipBlocks = 2048;    // workgroups of the norm pass at most (its partial sums)

hipError_t launch_clip(const ClipTensor *tensors, const ClipChunk *chunks, int64_t n_chunks,
                       double *part, float max_norm, float *norm, hipStream_t st);

// ---- attention on shared prefixes --------------------------------------------------------
struct AttnArgs {
    HeadsArg q, kp, vp, ks, vs, o;
    float *lse;                      // [total_q][hq], forward: or NULL
    HeadsArg go, gq, gkp, gvp, gks, gvs;   // backward
    int32_t groups, seqs, hq, hk, d, max_q;
    int32_t total_q;                 // total_q * hq < 2^31
    int64_t max_prefix, max_suffix, prefix_rows, suffix_rows;
    const int32_t *group_seqs, *cu_q;
    const int64_t *prefix_start;
    const int32_t *prefix_len, *suffix_len;
    const int64_t *suffix_start;
    const int32_t *pages;
    int64_t table_stride;
    int32_t page_size;
    float scale;
    char *work;                      // workspace
};

int64_t attn_forward_bytes(const AttnArgs &a, bool bf16);
int64_t attn_backward_bytes(const AttnArgs &a, bool bf16);
// Whether the matrix-instruction kernels run a call: by its sizes, and with its views.
bool attn_mfma_sizes(const AttnArgs &a, bool bf16);
bool attn_mfma_applies(const AttnArgs &a, bool bf16);
hipError_t launch_attn_generic(const AttnArgs &a, bool bf16, hipStream_t st);
hipError_t launch_attn_generic_backward(const AttnArgs &a, bool bf16, hipStream_t st);
hipError_t launch_attn_forward(const AttnArgs &a, bool bf16, hipStream_t st);
hipError_t launch_attn_backward(const AttnArgs &a, bool bf16, hipStream_t st);

}  // namespace olive
