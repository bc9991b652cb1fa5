// Rows of an embedding table by tokens, and the table's gradient.
#include "rows.hpp"
#include "tokens_internal.hpp"

namespace olive {
namespace {

// Wavefront w: token w / chunks, vectors (w % chunks) * per ... of its row.
template <typename T, int VEC>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a, int chunks, int per) {
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)block_index() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t = w / chunks;
    if (t >= a.tokens) return;
    const int nvec = a.width / VEC, v0 = (int)(w % chunks) * per, v1 = min(v0 + per, nvec);
    const int id = a.ids[t];
    const bool there = id >= 0 && id < a.vocab;
    const T *src = (const T *)a.table.p + (there ? id : 0) * a.table.st;
    T *dst = (T *)a.out.p + t * a.out.st;
    for (int v = v0 + lane; v < v1; v += 64) {
        float x[VEC];
        if (there) {
            get_vec<T, VEC>(src + v * VEC, x);
#pragma unroll
            for (int j = 0; j < VEC; ++j) x[j] *= a.scale;
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) x[j] = id < 0 ? 0.f : __builtin_nanf("");
        }
        put_vec<T, VEC>(dst + v * VEC, x);
    }
}

template <typename TT, int VEC>
__global__ __launch_bounds__(256) void embed_zero_kernel(EmbedArgs a) {
    const int nvec = a.width / VEC;
    const float zero[VEC] = {};
    for (int64_t r = block_index(); r < a.vocab; r += (int64_t)gridDim.x * gridDim.y)
        for (int v = threadIdx.x; v < nvec; v += 256) put_vec<TT, VEC>((TT *)a.table.p + r * a.table.st + v * VEC, zero);
}

// The wavefront of a token's first occurrence finds the others and adds their rows in order.
template <typename T, typename TT, int VEC>
__global__ __launch_bounds__(256) void embed_grad_kernel(EmbedArgs a, int chunks) {
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)block_index() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t = w / chunks;
    if (t >= a.tokens) return;
    const int id = a.ids[t];
    if (id < 0 || id >= a.vocab) return;
    for (int64_t s = 0; s < t; s += 64)
        if (__ballot(s + lane < t && a.ids[s + lane] == id)) return;
    const int nvec = a.width / VEC, v = (int)(w % chunks) * 64 + lane;
    float sum[VEC] = {};
    for (int64_t s = t; s < a.tokens; s += 64) {
        uint64_t m = __ballot(s + lane < a.tokens && a.ids[s + lane] == id);
        for (; m; m &= m - 1) {
            const int64_t r = s + __builtin_ctzll(m);
            if (v < nvec) {
                float x[VEC];
                get_vec<T, VEC>((const T *)a.out.p + r * a.out.st + v * VEC, x);
#pragma unroll
                for (int j = 0; j < VEC; ++j) sum[j] += x[j];
            }
        }
    }
    if (v >= nvec) return;
    TT *dst = (TT *)a.table.p + id * a.table.st + v * VEC;
    float old[VEC] = {};
    if (a.accumulate) get_vec<TT, VEC>(dst, old);
#pragma unroll
    for (int j = 0; j < VEC; ++j) sum[j] = fmaf(sum[j], a.scale, old[j]);
    put_vec<TT, VEC>(dst, sum);
}

template <typename T, int VEC>
hipError_t forward(const EmbedArgs &a, hipStream_t st) {
    const int nvec = a.width / VEC;
    const int per = 64, chunks = (nvec + per - 1) / per;
    embed_kernel<T, VEC><<<grid_of(((int64_t)a.tokens * chunks + 3) / 4), 256, 0, st>>>(a, chunks, per);
    return hipGetLastError();
}

template <typename T, typename TT, int VEC>
hipError_t backward(const EmbedArgs &a, hipStream_t st) {
    if (!a.accumulate) {
        embed_zero_kernel<TT, VEC><<<a.vocab < 4096 ? a.vocab : 4096, 256, 0, st>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || a.tokens == 0) return e;
    }
    const int chunks = (a.width / VEC + 63) / 64;
    embed_grad_kernel<T, TT, VEC><<<grid_of(((int64_t)a.tokens * chunks + 3) / 4), 256, 0, st>>>(a, chunks);
    return hipGetLastError();
}

template <typename T, typename TT>
hipError_t backward(const EmbedArgs &a, hipStream_t st) {
    constexpr int WIDE = 4;
    if (a.width % WIDE == 0 && rows_aligned({a.out}, WIDE * sizeof(T), sizeof(T)) &&
        rows_aligned({a.table}, WIDE * sizeof(TT), sizeof(TT)))
        return backward<T, TT, WIDE>(a, st);
    return backward<T, TT, 1>(a, st);
}

template <typename T>
hipError_t forward(const EmbedArgs &a, hipStream_t st) {
    constexpr int WIDE = 16 / sizeof(T);
    if (a.width % WIDE == 0 && rows_aligned({a.table, a.out}, 16, sizeof(T))) return forward<T, WIDE>(a, st);
    return forward<T, 1>(a, st);
}

}  // namespace

int64_t embed_backward_bytes(const EmbedArgs &) { return 0; }

hipError_t launch_embed(const EmbedArgs &a, bool bf16, hipStream_t st) {
    return bf16 ? forward<uint16_t>(a, st) : forward<float>(a, st);
}
hipError_t launch_embed_backward(const EmbedArgs &a, bool bf16, bool table_bf16, hipStream_t st) {
    if (bf16) return table_bf16 ? backward<uint16_t, uint16_t>(a, st) : backward<uint16_t, float>(a, st);
    return table_bf16 ? backward<float, uint16_t>(a, st) : backward<float, float>(a, st);
}

}  // namespace olive
