// Layer norm and RMS norm of rows, with the residual added before, and their backward.
//
// A row lies in the registers of WAVES wavefronts, NV vectors of 16 bytes a lane, so that it is read
// once: mean and mean square of what is left are sums over the registers. One wavefront holds up to
// 4096 bf16 elements (backward 2048, with the sums of the weight's gradients beside them), so that most
// rows need no barrier; what is read of a row is asked for at once. Bound by memory: 32768 rows with the
// residual, 4096 wide, 212 us (5.1 TB/s; with 16 wavefronts a row, half of them idle, 346), the backward
// 2048 wide 102 us (5.2 TB/s), of which the weight gradient's second pass 5. Layer norms have kernels of their
// own, for the registers (256 and 107 us; of 4096 rows of 16384, 224 us for 362 in the RMS norm's kernel).
#include "rows.hpp"
#include "tokens_internal.hpp"
#include "wave_ops.hpp"

namespace olive {
namespace {

// LDS of a row: a value of each of its wavefronts.
template <int WAVES>
struct Join { double wide[WAVES]; float narrow[WAVES]; };

// The sum over a row's lanes, the same in all of them.
template <int WAVES, typename V>
__device__ __forceinline__ V row_total(V v, V *join) {
    v = wave_sum(v);
    if constexpr (WAVES > 1) {
        __syncthreads();                     // (the values of the sum before are read)
        if ((threadIdx.x & 63) == 0) join[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) v += join[i];
        v = wave_read(v, 0);                 // (to scalar registers)
    }
    return v;
}

// Rows of one wavefront share a workgroup of four; else a workgroup has one row.
constexpr int threads_of(int waves) { return waves == 1 ? 256 : 64 * waves; }

// TAIL: the width is no multiple of a vector (any alignment is read the same).
template <typename T, bool LAYER, int NV, int WAVES, bool TAIL>
struct Rows {
    static constexpr int VEC = 16 / (int)sizeof(T);
    static constexpr int kRows = threads_of(WAVES) / (64 * WAVES);   // rows of a workgroup at a time
    using Vec = Lot;
    static __device__ __forceinline__ int lane() { return threadIdx.x % (64 * WAVES); }
    static __device__ __forceinline__ int sub() {
        return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / WAVES;
    }
    static __device__ __forceinline__ int vec(int i) { return lane() + 64 * WAVES * i; }

    static __device__ __forceinline__ void load(const char *p, int64_t at, int width, Vec (&x)[NV]) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if constexpr (TAIL) {
                x[i] = load_lot((const T *)p + at, vec(i) * VEC, width, 0);
            } else {
                x[i] = Lot{{0, 0, 0, 0}};
                if (vec(i) * VEC < width) x[i] = read_lot((const T *)p + at + vec(i) * VEC);
            }
        }
    }
    static __device__ __forceinline__ void store(char *p, int64_t at, int width, const float (&x)[NV][VEC], bool stream) {
#pragma unroll
        for (int i = 0; i < NV; ++i) store(p, at, width, i, pack_lot<T>(x[i]), stream);
    }
    static __device__ __forceinline__ void store(char *p, int64_t at, int width, int i, const Lot &x, bool stream) {
        if constexpr (TAIL) store_lot((T *)p + at, vec(i) * VEC, width, x);
        else if (vec(i) * VEC < width) write_lot((T *)p + at + vec(i) * VEC, x, stream);
    }
    static __device__ __forceinline__ void multiply(float (&h)[NV][VEC], float by) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) h[i][j] *= by;
    }
    static __device__ __forceinline__ float mean_square(const NormArgs &a, const float (&h)[NV][VEC], Join<WAVES> &join) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) s = fmaf(h[i][j], h[i][j], s);
        return row_total<WAVES>(s, join.narrow) / (float)a.width;
    }
    // h - mean (layer norm) in place, 0 past the row's end, times `scale` (1, or a power of two where fp32 does not
    // hold the squares); the inverse root of its mean square with eps.
    static __device__ __forceinline__ float normed(const NormArgs &a, float (&h)[NV][VEC], Join<WAVES> &join, float &scale) {
        scale = 1.f;
        if constexpr (LAYER) {
            // The mean in 64 bits, exact for equal values: a sum in 32 is off by some 2^-24 of the values, which
            // is no small share of their distance from the mean where they are nearly alike (2 to 4 %
            // of a layer norm's time).
            double s = 0.0;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) s += (double)h[i][j];
            s = row_total<WAVES>(s, join.wide);
            // (the quotient with its remainder's, in fewer registers than a division)
            double mean = s * a.inv_width;
            mean = fma(fma(-mean, (double)a.width, s), a.inv_width, mean);
            // (else no distance from it passes fp32's largest number)
            if (__builtin_expect(fabs(mean) >= 0x1p103, 0)) {
                scale = 0x1p-100f;
                mean *= 0x1p-100;
                multiply(h, scale);
            }
            const float high = (float)mean, low = (float)(mean - (double)high);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) h[i][j] = vec(i) * VEC + j < a.width ? h[i][j] - high - low : 0.f;
        }
        float m = mean_square(a, h, join) + a.eps * scale * scale;
        // Infinite, or so small that what fp32 does not hold of the squares counts (2^-126 of their mean at most): by
        // values a power of two smaller or larger, whose squares add up to 2^70 and 2^114 at most and whose mean
        // square is 2^-86 and 2^-112 at least. (After the scale above it is so small where every distance is 0,
        // whatever eps.)
        if (__builtin_expect(!(m >= 0x1p-100f && m < __builtin_inff()), 0)) {
            const float by = m < 0x1p-100f ? 0x1p100f : 0x1p-100f;
            scale = wave_read(by > 1.f && a.eps >= 0x1p-100f ? 1.f : by, 0);
            multiply(h, by);
            m = mean_square(a, h, join) + a.eps * scale * scale;
        }
        return __builtin_amdgcn_rsqf(m);                     // (off by one unit at most)
    }
};

// Wavefronts a SIMD that the kernels ask for: what they have registers for but for one to five, which go to scratch
// (fp32 rows of 4096, backward: 106 us, with one wavefront 112; bf16 rows of 2048 with bias: 107, 147). 1: as it comes.
constexpr int forward_waves(int values, int waves, bool tail) { return values == 32 && waves <= 4 && !tail ? 3 : 1; }
constexpr int backward_waves(int nv, int waves, bool tail, bool bias) {
    if (nv == 1) return tail ? 5 : 1;
    if (nv == 2) return bias ? 3 : 4;
    return !bias || (nv == 4 && waves == 1 && !tail) ? 2 : 1;
}

template <typename T, bool LAYER, int NV, int WAVES, bool TAIL>
__global__ __launch_bounds__(threads_of(WAVES), forward_waves(NV * kLot<T>, WAVES, TAIL)) void norm_kernel(NormArgs a) {
    using R = Rows<T, LAYER, NV, WAVES, TAIL>;
    constexpr int VEC = R::VEC;
    __shared__ Join<WAVES> join;
    const int width = a.width;
    for (int64_t r = (int64_t)blockIdx.x * R::kRows + R::sub(); r < a.rows; r += (int64_t)gridDim.x * R::kRows) {
        float h[NV][VEC], scale;
        typename R::Vec x[NV], y[NV], w[NV];
        R::load(a.x.p, r * a.x.st, width, x);
        if (a.res.p) R::load(a.res.p, r * a.res.st, width, y);
        if (a.weight) R::load((const char *)a.weight, 0, width, w);
#pragma unroll
        for (int i = 0; i < NV; ++i) unpack_lot<T>(x[i], h[i]);
        if (a.res.p) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float t[VEC];
                unpack_lot<T>(y[i], t);
#pragma unroll
                for (int j = 0; j < VEC; ++j) t[j] += h[i][j];
                x[i] = pack_lot<T>(t);
                unpack_lot<T>(x[i], h[i]);
            }
        }
        if (a.sum.p) {
#pragma unroll
            for (int i = 0; i < NV; ++i) R::store(a.sum.p, r * a.sum.st, width, i, x[i], a.stream);
        }
        const float rr = R::normed(a, h, join, scale);
        if (a.bias) R::load((const char *)a.bias, 0, width, y);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float u[VEC], v[VEC];
            if (a.weight) unpack_lot<T>(w[i], u);
            if (a.bias) unpack_lot<T>(y[i], v);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                h[i][j] = h[i][j] * rr * (a.weight ? u[j] : 1.f);
                if (a.bias) h[i][j] += v[j];
            }
        }
        R::store(a.out.p, r * a.out.st, width, h, a.stream);
    }
}

// Persistent workgroups over rows; a lane sums its columns' weight and bias gradients over its
// rows, the workgroup joins them in a fixed order and writes one partial row of both.
template <typename T, bool LAYER, int NV, int WAVES, bool TAIL, bool BIAS>
__global__ __launch_bounds__(threads_of(WAVES), backward_waves(NV, WAVES, TAIL, BIAS)) void norm_backward_kernel(NormArgs a) {
    using R = Rows<T, LAYER, NV, WAVES, TAIL>;
    constexpr int VEC = R::VEC;
    __shared__ Join<WAVES> join;
    const int width = a.width;
    const float inv = 1.f / (float)width;
    float gw[NV][VEC] = {}, gb[BIAS ? NV : 1][VEC] = {};
    for (int64_t r = (int64_t)blockIdx.x * R::kRows + R::sub(); r < a.rows; r += (int64_t)gridDim.x * R::kRows) {
        float h[NV][VEC], g[NV][VEC], scale;
        typename R::Vec x[NV], y[NV], z[NV], w[NV];
        R::load(a.x.p, r * a.x.st, width, x);
        R::load(a.sum.p, r * a.sum.st, width, y);
        if (a.res.p) R::load(a.res.p, r * a.res.st, width, z);
        if (a.weight) R::load((const char *)a.weight, 0, width, w);
#pragma unroll
        for (int i = 0; i < NV; ++i) unpack_lot<T>(x[i], h[i]);
        const float rr = R::normed(a, h, join, scale);
        float sg = 0.f, sn = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float u[VEC];
            unpack_lot<T>(y[i], g[i]);
            if (a.weight) unpack_lot<T>(w[i], u);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                h[i][j] *= rr;
                // (past the row's end x = y = 0, and eps may be 0)
                if (R::vec(i) * VEC + j < width) gw[i][j] = fmaf(g[i][j], h[i][j], gw[i][j]);
                if constexpr (BIAS) gb[i][j] += g[i][j];
                if (a.weight) g[i][j] *= u[j];
                sg += g[i][j];
                sn = fmaf(g[i][j], h[i][j], sn);
            }
        }
        sn = row_total<WAVES>(sn, join.narrow) * inv;
        sg = LAYER ? row_total<WAVES>(sg, join.narrow) * inv : 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float u[VEC];
            if (a.res.p) unpack_lot<T>(z[i], u);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                g[i][j] = rr * (g[i][j] - h[i][j] * sn - sg) * scale;
                if (a.res.p) g[i][j] += u[j];
            }
        }
        R::store(a.out.p, r * a.out.st, width, g, a.stream);
    }
    if (!a.gw && !a.gb) return;
    float *part = a.part + (int64_t)blockIdx.x * 2 * width;
    const auto put = [&](const float (&s)[VEC], int i, float *to) {
        float v[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] = s[j];
        if constexpr (R::kRows > 1) {
            __shared__ float rows[R::kRows][64 * VEC];
            __syncthreads();
#pragma unroll
            for (int j = 0; j < VEC; ++j) rows[R::sub()][j * 64 + R::lane()] = v[j];
            __syncthreads();
            if (R::sub()) return;
#pragma unroll
            for (int j = 0; j < VEC; ++j)
#pragma unroll
                for (int k = 1; k < R::kRows; ++k) v[j] += rows[k][j * 64 + R::lane()];
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            if (R::vec(i) * VEC + j < width) to[R::vec(i) * VEC + j] = v[j];
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        put(gw[i], i, part);
        if constexpr (BIAS) put(gb[i], i, part + width);
    }
}

// Sums the partial rows: 64 columns a workgroup, every 16th row a wavefront.
constexpr int kJoinWaves = 16;

__global__ __launch_bounds__(64 * kJoinWaves) void norm_weight_kernel(NormArgs a, int parts) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    float *out = blockIdx.y ? a.gb : a.gw;
    if (!out) return;
    const float *from = a.part + (int64_t)blockIdx.y * a.width + c;
    float s = 0.f;
    if (c < a.width)
#pragma unroll 8
        for (int i = wave; i < parts; i += kJoinWaves) s += from[(int64_t)i * 2 * a.width];
    __shared__ float join[kJoinWaves][64];
    join[wave][lane] = s;
    __syncthreads();
    if (wave || c >= a.width) return;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < kJoinWaves; ++i) s += join[i][lane];
    out[c] = s;
}

template <typename T, bool LAYER, int NV, int WAVES>
hipError_t forward(const NormArgs &a, hipStream_t st) {
    using R = Rows<T, LAYER, NV, WAVES, false>;
    const int64_t groups = ((int64_t)a.rows + R::kRows - 1) / R::kRows;
    const int blocks = (int)(groups < (1 << 20) ? groups : 1 << 20);
    if (a.width % R::VEC) norm_kernel<T, LAYER, NV, WAVES, true><<<blocks, threads_of(WAVES), 0, st>>>(a);
    else norm_kernel<T, LAYER, NV, WAVES, false><<<blocks, threads_of(WAVES), 0, st>>>(a);
    return hipGetLastError();
}

// Wavefronts of a row in the backward, and its workgroups at most: 8 wavefronts a compute unit.
int waves_of(int width) {
    int w = 1;
    while (w * 2048 < width) w *= 2;             // (32 values of each kind a lane)
    return w;
}
int blocks_of(int width) { return width <= 2048 ? 512 : 2048 / waves_of(width); }

template <typename T, bool LAYER, int NV, int WAVES>
hipError_t backward(const NormArgs &a, hipStream_t st) {
    using R = Rows<T, LAYER, NV, WAVES, false>;
    const int64_t groups = ((int64_t)a.rows + R::kRows - 1) / R::kRows, most = blocks_of(a.width);
    const int blocks = (int)(groups < most ? (groups > 0 ? groups : 1) : most);
    const auto run = [&](auto kernel) { kernel<<<blocks, threads_of(WAVES), 0, st>>>(a); };
    if (a.width % R::VEC) run(norm_backward_kernel<T, LAYER, NV, WAVES, true, true>);       // (bias or not)
    else if (a.gb) run(norm_backward_kernel<T, LAYER, NV, WAVES, false, true>);
    else run(norm_backward_kernel<T, LAYER, NV, WAVES, false, false>);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || (!a.gw && !a.gb)) return e;
    norm_weight_kernel<<<dim3((a.width + 63) / 64, a.gb ? 2 : 1), 64 * kJoinWaves, 0, st>>>(a, blocks);
    return hipGetLastError();
}

template <typename T, bool LAYER>
hipError_t pick_forward(const NormArgs &a, hipStream_t st) {
    constexpr int one = 64 * 16 / (int)sizeof(T);                // elements of a vector a lane
    if (a.width <= one) return forward<T, LAYER, 1, 1>(a, st);
    if (a.width <= 2 * one) return forward<T, LAYER, 2, 1>(a, st);
    if (a.width <= 4 * one) return forward<T, LAYER, 4, 1>(a, st);
    if (a.width <= 8 * one) return forward<T, LAYER, 8, 1>(a, st);
    if (a.width <= 16 * one) return forward<T, LAYER, 4, 4>(a, st);
    return forward<T, LAYER, 4, 16>(a, st);
}

template <typename T, bool LAYER>
hipError_t pick_backward(const NormArgs &a, hipStream_t st) {
    constexpr int one = 64 * 16 / (int)sizeof(T), full = 2048 / one;
    if (a.width <= one) return backward<T, LAYER, 1, 1>(a, st);
    if (a.width <= 2 * one) return backward<T, LAYER, 2, 1>(a, st);
    switch (waves_of(a.width)) {
        case 1: return backward<T, LAYER, full, 1>(a, st);
        case 2: return backward<T, LAYER, full, 2>(a, st);
        case 4: return backward<T, LAYER, full, 4>(a, st);
        default: return backward<T, LAYER, full, 8>(a, st);
    }
}

}  // namespace

int64_t norm_backward_bytes(const NormArgs &a) {
    return (int64_t)blocks_of(a.width) * 2 * a.width * (int64_t)sizeof(float);
}

hipError_t launch_norm(const NormArgs &a, bool bf16, hipStream_t st) {
    if (a.layer) return bf16 ? pick_forward<uint16_t, true>(a, st) : pick_forward<float, true>(a, st);
    return bf16 ? pick_forward<uint16_t, false>(a, st) : pick_forward<float, false>(a, st);
}
hipError_t launch_norm_backward(const NormArgs &a, bool bf16, hipStream_t st) {
    if (a.layer) return bf16 ? pick_backward<uint16_t, true>(a, st) : pick_backward<float, true>(a, st);
    return bf16 ? pick_backward<uint16_t, false>(a, st) : pick_backward<float, false>(a, st);
}

}  // namespace olive
