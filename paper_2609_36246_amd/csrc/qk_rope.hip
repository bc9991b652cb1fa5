// RMS norm of query and key heads with the position rotation, and its backward.
//
// A row (one head of one token) lies in LPR consecutive lanes of a wavefront, VEC elements
// each, so the sums over a head are a few lane exchanges and the partner elements of the
// rotation come from another lane or the same vector. A wavefront keeps to one token while
// it walks over heads: the angles and weights of its elements stay in registers.
//
// Bound by memory: 7 (backward 14) operations an element for 4 (6) bytes in bf16.
#include "layers_internal.hpp"
#include "olive_device.hpp"

namespace olive {
namespace {

template <typename T> struct Elem;
template <> struct Elem<float> {
    static __device__ __forceinline__ float get(float v) { return v; }
    static __device__ __forceinline__ float put(float v) { return v; }
};
template <> struct Elem<uint16_t> {
    static __device__ __forceinline__ float get(uint16_t v) { return bf16_bits_to_f32(v); }
    static __device__ __forceinline__ uint16_t put(float v) {
        return (uint16_t)(pack_bf16x2(v, v) & 0xffffu);
    }
};

template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Pack { T v[VEC]; };

template <typename T, int VEC>
__device__ __forceinline__ void load_vec(const T *p, float (&x)[VEC]) {
    const Pack<T, VEC> u = *(const Pack<T, VEC> *)p;
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[j] = Elem<T>::get(u.v[j]);
}
template <typename T, int VEC>
__device__ __forceinline__ void store_vec(T *p, const float (&x)[VEC]) {
    Pack<T, VEC> u;
#pragma unroll
    for (int j = 0; j < VEC; ++j) u.v[j] = Elem<T>::put(x[j]);
    *(Pack<T, VEC> *)p = u;
}

__device__ __forceinline__ float row_sum(float v, int lpr) {
    for (int o = lpr >> 1; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// What a lane keeps of a token: for each of its elements the cosine and the signed sine of
// y = x cos + partner * sin (forward), 1 and 0 past the rotated part, and NaN where the
// position is out of range.
template <int VEC, int NV>
struct Angles {
    float c[NV][VEC], s[NV][VEC];
    int partner[NV];                  // vector whose elements are this one's partners
};

template <int VEC, int NV>
__device__ __forceinline__ void load_angles(const QkArgs &a, int t, int li, int nvec,
                                            Angles<VEC, NV> &g) {
    const int half = a.rot >> 1;
    const int64_t pos = a.rot ? (int64_t)a.positions[t] : 0;
    const bool ok = !a.rot || (pos >= 0 && pos < a.num_positions);
    const int64_t row = ok ? pos * half : 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int e0 = (li + 64 * v) * VEC;
        g.partner[v] = li + 64 * v;
        if (a.layout == OLIVE_ROPE_HALF) {
            if (e0 < half) g.partner[v] += half / VEC;
            else if (e0 < a.rot) g.partner[v] -= half / VEC;
        } else if (VEC == 1 && e0 < a.rot) {
            g.partner[v] ^= 1;
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const int e = e0 + j;
            float c = 1.f, s = 0.f;
            if (e < a.rot) {
                const bool first = a.layout == OLIVE_ROPE_HALF ? e < half : !(e & 1);
                const int p = a.layout == OLIVE_ROPE_HALF ? (e < half ? e : e - half) : e >> 1;
                c = a.cos[row + p];
                s = first ? -a.sin[row + p] : a.sin[row + p];
            }
            g.c[v][j] = ok ? c : __builtin_nanf("");
            g.s[v][j] = ok ? s : __builtin_nanf("");
        }
    }
}

// x cos + partner * sin of a row; SIGN -1 is the transposed rotation.
template <int VEC, int NV, int SIGN>
__device__ __forceinline__ void rotate(const Angles<VEC, NV> &g, int rot, int layout, int li,
                                       int lpr, float (&x)[NV][VEC]) {
    float p[NV][VEC];
    if (VEC > 1 && layout == OLIVE_ROPE_PAIRS) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < VEC; ++j) p[v][j] = x[v][VEC > 1 ? j ^ 1 : j];
    } else {
        const int base = (threadIdx.x & 63) & ~(lpr - 1);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int src = base + (g.partner[v] & (lpr - 1)), pv = g.partner[v] >> 6;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                p[v][j] = 0.f;
#pragma unroll
                for (int w = 0; w < NV; ++w) {
                    const float y = __shfl(x[w][j], src);
                    if (NV == 1 || w == pv) p[v][j] = y;
                }
            }
        }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const bool turned = (li + 64 * v) * VEC + j < rot;
            x[v][j] = x[v][j] * g.c[v][j] + (turned ? p[v][j] : 0.f) * (SIGN * g.s[v][j]);
        }
}

template <typename T, int VEC, int NV>
__device__ __forceinline__ void load_weight(const void *w, int li, int nvec,
                                            float (&x)[NV][VEC]) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int i = li + 64 * v;
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            x[v][j] = w && i < nvec ? Elem<T>::get(((const T *)w)[i * VEC + j]) : 1.f;
    }
}

// Wavefront w of the grid: token w / chunks, rows (w % chunks) * per ... of its q, k and v.
template <typename T, int VEC, int NV>
__global__ __launch_bounds__(256) void qk_forward_kernel(QkArgs a, int lpr, int chunks, int per) {
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int t = (int)(w / chunks);
    if (t >= a.tokens) return;
    const int li = lane & (lpr - 1), sub = lane / lpr, rpw = 64 / lpr;
    const int nvec = a.d / VEC;
    const int rows = a.hq + a.hk + a.hv;
    const int h0 = (int)(w % chunks) * per, h1 = min(rows, h0 + per);

    Angles<VEC, NV> g;
    load_angles<VEC, NV>(a, t, li, nvec, g);
    float wq[NV][VEC], wk[NV][VEC];
    load_weight<T, VEC, NV>(a.wq, li, nvec, wq);
    load_weight<T, VEC, NV>(a.wk, li, nvec, wk);
    const int64_t slot = a.slots ? (int64_t)a.slots[t] : t;
    const bool put = !a.slots || (slot >= 0 && slot < a.slot_rows);

    for (int h = h0; h < h1; h += rpw) {
        const int r = h + sub;
        const bool live = r < h1;
        const bool is_q = r < a.hq, is_v = r >= a.hq + a.hk;
        const T *src;
        T *dst;
        if (is_q) {
            src = (const T *)a.q.p + t * a.q.st + r * a.q.sh;
            dst = (T *)a.qo.p + t * a.qo.st + r * a.qo.sh;
        } else if (!is_v) {
            src = (const T *)a.k.p + t * a.k.st + (r - a.hq) * a.k.sh;
            dst = (T *)a.ko.p + slot * a.ko.st + (r - a.hq) * a.ko.sh;
        } else {
            src = (const T *)a.v.p + t * a.v.st + (r - a.hq - a.hk) * a.v.sh;
            dst = (T *)a.vo.p + slot * a.vo.st + (r - a.hq - a.hk) * a.vo.sh;
        }
        float x[NV][VEC];
        float ss = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int i = li + 64 * v;
            if (live && i < nvec) {
                load_vec<T, VEC>(src + i * VEC, x[v]);
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j) x[v][j] = 0.f;
            }
#pragma unroll
            for (int j = 0; j < VEC; ++j) ss = fmaf(x[v][j], x[v][j], ss);
        }
        ss = row_sum(ss, lpr);
        if (!is_v) {
            const float r_ = (is_q ? a.wq : a.wk) ? 1.f / sqrtf(ss / (float)a.d + a.eps) : 1.f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < VEC; ++j) x[v][j] *= r_ * (is_q ? wq[v][j] : wk[v][j]);
        }
        float y[NV][VEC];
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < VEC; ++j) y[v][j] = x[v][j];
        rotate<VEC, NV, 1>(g, a.rot, a.layout, li, lpr, y);
        if (live && (is_q || put)) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int i = li + 64 * v;
                if (i < nvec) store_vec<T, VEC>(dst + i * VEC, is_v ? x[v] : y[v]);
            }
        }
    }
}

// Persistent wavefronts over tokens; a lane sums its elements' weight gradients over all its
// rows, the workgroup joins them in a fixed order and writes one partial row.
template <typename T, int VEC, int NV>
__global__ __launch_bounds__(256) void qk_backward_kernel(QkArgs a, int lpr) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int li = lane & (lpr - 1), sub = lane / lpr, rpw = 64 / lpr;
    const int nvec = a.d / VEC;
    const int rows = a.hq + a.hk;
    const int stride = gridDim.x * 4;
    float wq[NV][VEC], wk[NV][VEC], sq[NV][VEC] = {}, sk[NV][VEC] = {};
    load_weight<T, VEC, NV>(a.wq, li, nvec, wq);
    load_weight<T, VEC, NV>(a.wk, li, nvec, wk);

    for (int t = blockIdx.x * 4 + wave; t < a.tokens; t += stride) {
        Angles<VEC, NV> g;
        load_angles<VEC, NV>(a, t, li, nvec, g);
        for (int h = 0; h < rows; h += rpw) {
            const int r = h + sub;
            const bool live = r < rows, is_q = r < a.hq;
            const T *src, *grd;
            T *dst;
            if (is_q) {
                src = (const T *)a.q.p + t * a.q.st + r * a.q.sh;
                grd = (const T *)a.qo.p + t * a.qo.st + r * a.qo.sh;
                dst = (T *)a.gq.p + t * a.gq.st + r * a.gq.sh;
            } else {
                src = (const T *)a.k.p + t * a.k.st + (r - a.hq) * a.k.sh;
                grd = (const T *)a.ko.p + t * a.ko.st + (r - a.hq) * a.ko.sh;
                dst = (T *)a.gk.p + t * a.gk.st + (r - a.hq) * a.gk.sh;
            }
            float x[NV][VEC], y[NV][VEC];
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int i = li + 64 * v;
                if (live && i < nvec) {
                    load_vec<T, VEC>(src + i * VEC, x[v]);
                    load_vec<T, VEC>(grd + i * VEC, y[v]);
                } else {
#pragma unroll
                    for (int j = 0; j < VEC; ++j) x[v][j] = y[v][j] = 0.f;
                }
            }
            rotate<VEC, NV, -1>(g, a.rot, a.layout, li, lpr, y);
            if ((is_q ? a.wq : a.wk)) {
                float ss = 0.f, sh = 0.f;
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        ss = fmaf(x[v][j], x[v][j], ss);
                        sh = fmaf(y[v][j] * (is_q ? wq[v][j] : wk[v][j]), x[v][j], sh);
                    }
                ss = row_sum(ss, lpr);
                sh = row_sum(sh, lpr);
                const float r_ = 1.f / sqrtf(ss / (float)a.d + a.eps);
                const float m = r_ * r_ * (sh / (float)a.d);
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        // (rows that are not there have x = y = 0)
                        const float gw = live && (li + 64 * v) < nvec ? y[v][j] * (x[v][j] * r_) : 0.f;
                        if (is_q) sq[v][j] += gw; else sk[v][j] += gw;
                        y[v][j] = r_ * (y[v][j] * (is_q ? wq[v][j] : wk[v][j]) - x[v][j] * m);
                    }
            }
            if (live) {
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const int i = li + 64 * v;
                    if (i < nvec) store_vec<T, VEC>(dst + i * VEC, y[v]);
                }
            }
        }
    }
    if (!a.gwq && !a.gwk) return;
    __shared__ float join[4][2][256];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            float u = sq[v][j], w = sk[v][j];
            for (int o = lpr; o < 64; o <<= 1) {
                u += __shfl_xor(u, o);
                w += __shfl_xor(w, o);
            }
            const int i = li + 64 * v;
            if (sub == 0 && i < nvec) {
                join[wave][0][i * VEC + j] = u;
                join[wave][1][i * VEC + j] = w;
            }
        }
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * a.d; e += 256) {
        const int f = e >= a.d, i = e - f * a.d;
        a.part[(int64_t)blockIdx.x * 2 * a.d + e] =
            (join[0][f][i] + join[1][f][i]) + (join[2][f][i] + join[3][f][i]);
    }
}

// Sums the partial rows: 16 columns a workgroup, 16 threads a column.
__global__ __launch_bounds__(256) void qk_weight_grad_kernel(QkArgs a, int blocks) {
    const int col = blockIdx.x * 16 + (threadIdx.x & 15), part = threadIdx.x >> 4;
    float s = 0.f;
    if (col < 2 * a.d)
        for (int b = part; b < blocks; b += 16) s += a.part[(int64_t)b * 2 * a.d + col];
    __shared__ float join[16][17];
    join[part][threadIdx.x & 15] = s;
    __syncthreads();
    if (part == 0 && col < 2 * a.d) {
        float u = 0.f;
        for (int i = 0; i < 16; ++i) u += join[i][threadIdx.x & 15];
        float *out = col < a.d ? a.gwq : a.gwk;
        if (out) out[col < a.d ? col : col - a.d] = u;
    }
}

template <typename T, int VEC, int NV>
hipError_t go(const QkArgs &a, bool backward, hipStream_t st) {
    const int nvec = a.d / VEC;
    int lpr = 1;
    while (lpr < nvec && lpr < 64) lpr <<= 1;
    if (!backward) {
        const int rpw = 64 / lpr, rows = a.hq + a.hk + a.hv;
        // a wavefront walks over all heads of its token where there are tokens enough to
        // fill the chip, else over a share of them
        int per = rows;
        while (per > rpw && (int64_t)a.tokens * ((rows + per - 1) / per) < kChipUnits * 16)
            per = (per + 1) / 2;
        per = (per + rpw - 1) / rpw * rpw;
        const int chunks = (rows + per - 1) / per;
        const int64_t waves = (int64_t)a.tokens * chunks;
        qk_forward_kernel<T, VEC, NV><<<(unsigned)((waves + 3) / 4), 256, 0, st>>>(a, lpr, chunks,
                                                                                   per);
        return hipGetLastError();
    }
    const int blocks = max(1, min(kQkBwdBlocks, (a.tokens + 3) / 4));
    qk_backward_kernel<T, VEC, NV><<<blocks, 256, 0, st>>>(a, lpr);
    if (a.gwq || a.gwk) qk_weight_grad_kernel<<<(2 * a.d + 15) / 16, 256, 0, st>>>(a, blocks);
    return hipGetLastError();
}

bool aligned(const HeadsArg &h, int bytes, int esz) {
    return !h.p || (((uintptr_t)h.p | (uint64_t)(h.st * esz) | (uint64_t)(h.sh * esz)) % bytes) == 0;
}

// The widest vector that divides the heads and their halves, and that every view is aligned
// to; one element a lane and step for the rest (odd halves, odd strides).
template <typename T>
hipError_t pick(const QkArgs &a, bool backward, hipStream_t st) {
    constexpr int WIDE = 16 / sizeof(T);
    const int unit = a.layout == OLIVE_ROPE_HALF ? a.rot / 2 : a.rot;
    const auto fits = [&](int vec) {
        if (a.d % vec || unit % vec) return false;
        const int b = vec * (int)sizeof(T);
        for (const HeadsArg *h : {&a.q, &a.k, &a.v, &a.qo, &a.ko, &a.vo, &a.gq, &a.gk})
            if (!aligned(*h, b, sizeof(T))) return false;
        return true;
    };
    if (fits(WIDE)) return go<T, WIDE, 1>(a, backward, st);
    if (fits(2) && a.d <= 128) return go<T, 2, 1>(a, backward, st);
    if (a.d <= 64) return go<T, 1, 1>(a, backward, st);
    if (a.d <= 128) return go<T, 1, 2>(a, backward, st);
    return go<T, 1, 4>(a, backward, st);
}

}  // namespace

hipError_t launch_qk_forward(const QkArgs &a, bool bf16, hipStream_t st) {
    return bf16 ? pick<uint16_t>(a, false, st) : pick<float>(a, false, st);
}
hipError_t launch_qk_backward(const QkArgs &a, bool bf16, hipStream_t st) {
    return bf16 ? pick<uint16_t>(a, true, st) : pick<float>(a, true, st);
}

}  // namespace olive
