// Layer norm and RMS norm of rows, with the residual added before, and their backward.
//
// A row lies in the registers of WAVES wavefronts, VEC * NV elements a lane, so that it is read
// once: mean and mean square of what is left are two sums over the registers.
#include "rows.hpp"
#include "tokens_internal.hpp"

namespace olive {
namespace {

// The sum over a row's lanes, the same in all of them. `join`: LDS of the row, WAVES values.
template <int WAVES>
__device__ __forceinline__ float row_total(float v, float *join) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    if constexpr (WAVES > 1) {
        __syncthreads();                     // (the values of the sum before are read)
        if ((threadIdx.x & 63) == 0) join[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) v += join[i];
    }
    return v;
}

// 1 / root (v_rsq_f32 is off by one unit at most, and takes a subnormal number for 0: small ones
// are scaled).
__device__ __forceinline__ float inverse_root(float m) {
    const bool small = m < 0x1p-100f;
    return __builtin_amdgcn_rsqf(small ? m * 0x1p100f : m) * (small ? 0x1p50f : 1.f);
}

constexpr int threads_of(int waves) { return waves > 4 ? 64 * waves : 256; }

template <typename T, int VEC, int NV, int WAVES>
struct Rows {
    static constexpr int kThreads = threads_of(WAVES);
    static constexpr int kRows = kThreads / (64 * WAVES);      // rows of a workgroup at a time
    static __device__ __forceinline__ int lane() { return threadIdx.x % (64 * WAVES); }
    static __device__ __forceinline__ int sub() { return threadIdx.x / (64 * WAVES); }

    // elements of a row that this lane holds (0 past its end)
    static __device__ __forceinline__ void load(const char *p, int64_t at, int nvec, float (&x)[NV][VEC]) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = lane() + 64 * WAVES * i;
            if (v < nvec) {
                get_vec<T, VEC>((const T *)p + at + v * VEC, x[i]);
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j) x[i][j] = 0.f;
            }
        }
    }
    static __device__ __forceinline__ void store(char *p, int64_t at, int nvec, const float (&x)[NV][VEC]) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = lane() + 64 * WAVES * i;
            if (v < nvec) put_vec<T, VEC>((T *)p + at + v * VEC, x[i]);
        }
    }
    // h - mean (layer norm) in place; the inverse root of its mean square
    static __device__ __forceinline__ float normed(const NormArgs &a, int nvec, float (&h)[NV][VEC], float *join) {
        if (a.layer) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) s += h[i][j];
            const float mean = row_total<WAVES>(s, join) / (float)a.width;   // (exact where all are equal)
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) h[i][j] = lane() + 64 * WAVES * i < nvec ? h[i][j] - mean : 0.f;
        }
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) s = fmaf(h[i][j], h[i][j], s);
        return inverse_root(row_total<WAVES>(s, join) / (float)a.width + a.eps);
    }
};

template <typename T, int VEC, int NV, int WAVES>
__global__ __launch_bounds__(threads_of(WAVES)) void norm_kernel(NormArgs a) {
    using R = Rows<T, VEC, NV, WAVES>;
    __shared__ float join[WAVES];
    const int nvec = a.width / VEC;
    for (int64_t r = (int64_t)blockIdx.x * R::kRows + R::sub(); r < a.rows; r += (int64_t)gridDim.x * R::kRows) {
        float h[NV][VEC], w[NV][VEC];
        R::load(a.x.p, r * a.x.st, nvec, h);
        if (a.res.p) {
            R::load(a.res.p, r * a.res.st, nvec, w);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) h[i][j] = RowElem<T>::get(RowElem<T>::put(h[i][j] + w[i][j]));
        }
        if (a.sum.p) R::store(a.sum.p, r * a.sum.st, nvec, h);
        const float rr = R::normed(a, nvec, h, join);
        if (a.weight) R::load((const char *)a.weight, 0, nvec, w);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) h[i][j] = h[i][j] * rr * (a.weight ? w[i][j] : 1.f);
        if (a.bias) {
            R::load((const char *)a.bias, 0, nvec, w);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) h[i][j] += w[i][j];
        }
        R::store(a.out.p, r * a.out.st, nvec, h);
    }
}

// Persistent workgroups over rows; a lane sums its columns' weight and bias gradients over its
// rows, and each group of WAVES wavefronts writes one partial row of both.
template <typename T, int VEC, int NV, int WAVES>
__global__ __launch_bounds__(threads_of(WAVES)) void norm_backward_kernel(NormArgs a) {
    using R = Rows<T, VEC, NV, WAVES>;
    __shared__ float join[WAVES];
    const int nvec = a.width / VEC;
    const float inv = 1.f / (float)a.width;
    float gw[NV][VEC] = {}, gb[NV][VEC] = {};
    for (int64_t r = (int64_t)blockIdx.x * R::kRows + R::sub(); r < a.rows; r += (int64_t)gridDim.x * R::kRows) {
        float h[NV][VEC], g[NV][VEC], w[NV][VEC];
        R::load(a.x.p, r * a.x.st, nvec, h);
        R::load(a.sum.p, r * a.sum.st, nvec, g);
        if (a.weight) R::load((const char *)a.weight, 0, nvec, w);
        const float rr = R::normed(a, nvec, h, join);
        float sg = 0.f, sn = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                h[i][j] *= rr;
                if (R::lane() + 64 * WAVES * i < nvec) {
                    gw[i][j] = fmaf(g[i][j], h[i][j], gw[i][j]);
                    gb[i][j] += g[i][j];
                }
                if (a.weight) g[i][j] *= w[i][j];
                sg += g[i][j];
                sn = fmaf(g[i][j], h[i][j], sn);
            }
        sn = row_total<WAVES>(sn, join) * inv;
        sg = a.layer ? row_total<WAVES>(sg, join) * inv : 0.f;
        if (a.res.p) R::load(a.res.p, r * a.res.st, nvec, w);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                g[i][j] = rr * (g[i][j] - h[i][j] * sn - sg);
                if (a.res.p) g[i][j] += w[i][j];
            }
        R::store(a.out.p, r * a.out.st, nvec, g);
    }
    if (!a.gw && !a.gb) return;
    float *part = a.part + ((int64_t)blockIdx.x * R::kRows + R::sub()) * 2 * a.width;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = R::lane() + 64 * WAVES * i;
        if (v < nvec) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                part[v * VEC + j] = gw[i][j];
                part[a.width + v * VEC + j] = gb[i][j];
            }
        }
    }
}

__global__ __launch_bounds__(256) void norm_weight_kernel(NormArgs a, int parts) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= 2 * a.width) return;
    float s = 0.f;
    for (int i = 0; i < parts; ++i) s += a.part[(int64_t)i * 2 * a.width + c];
    float *out = c < a.width ? a.gw : a.gb;
    if (out) out[c < a.width ? c : c - a.width] = s;
}

template <typename T, int VEC, int NV, int WAVES>
hipError_t go(const NormArgs &a, bool backward, hipStream_t st) {
    using R = Rows<T, VEC, NV, WAVES>;
    const int64_t groups = ((int64_t)a.rows + R::kRows - 1) / R::kRows;
    if (!backward) {
        norm_kernel<T, VEC, NV, WAVES><<<(int)(groups < 2048 ? groups : 2048), R::kThreads, 0, st>>>(a);
        return hipGetLastError();
    }
    const int most = kNormBlocks / R::kRows, blocks = (int)(groups < most ? (groups > 0 ? groups : 1) : most);
    norm_backward_kernel<T, VEC, NV, WAVES><<<blocks, R::kThreads, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || (!a.gw && !a.gb)) return e;
    norm_weight_kernel<<<(2 * a.width + 255) / 256, 256, 0, st>>>(a, blocks * R::kRows);
    return hipGetLastError();
}

template <typename T>
hipError_t pick(const NormArgs &a, bool backward, hipStream_t st) {
    constexpr int WIDE = 16 / sizeof(T);
    const bool wide = a.width % WIDE == 0 && rows_aligned({a.x, a.res, a.out, a.sum}, 16, sizeof(T)) &&
                      (((uintptr_t)a.weight | (uintptr_t)a.bias) & 15) == 0;
    if (wide && a.width <= 64 * WIDE * 4) return go<T, WIDE, 4, 1>(a, backward, st);
    if (wide) return go<T, WIDE, 16 / WIDE, 16>(a, backward, st);
    if (a.width <= 64 * 4 * 4) return go<T, 1, 4, 4>(a, backward, st);
    return go<T, 1, 16, 16>(a, backward, st);
}

}  // namespace

hipError_t launch_norm(const NormArgs &a, bool bf16, hipStream_t st) {
    return bf16 ? pick<uint16_t>(a, false, st) : pick<float>(a, false, st);
}
hipError_t launch_norm_backward(const NormArgs &a, bool bf16, hipStream_t st) {
    return bf16 ? pick<uint16_t>(a, true, st) : pick<float>(a, true, st);
}

}  // namespace olive
