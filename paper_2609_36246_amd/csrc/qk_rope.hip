// RMS norm of query and key heads with the position rotation, and its backward.
//
// A row (one head of one token) lies in LPR consecutive lanes of a wavefront, VEC elements
// each, so the sums over a head are a few lane exchanges and the partner elements of the
// rotation come from another lane or the same vector. A wavefront keeps to one token while
// it walks over heads: the angles and weights of its elements stay in registers.
//
// Bound by memory: 7 (backward 14) operations an element for 4 (6) bytes in bf16. 32768 tokens
// of 40 heads of 128: 160 us, 4.2 TB/s (a large copy: 4.75); the backward of 24 heads 139 us,
// 4.4 TB/s, of which 6 us the weight gradients' second pass; 8 tokens into a cache 5 us.
#include <type_traits>

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

// A value from another lane of the same 16, without LDS: CTRL is the DPP pattern.
template <int CTRL, int BANKS = 0xf>
__device__ __forceinline__ float dpp(float old, float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(old), __float_as_int(v), CTRL, 0xf, BANKS, false));
}
constexpr int kRor = 0x120, kShl = 0x100, kShr = 0x110, kHalfMirror = 0x141;
constexpr int quad(int a, int b, int c, int d) { return a | b << 2 | c << 4 | d << 6; }

// Sum over the LPR lanes of a row (LPR 0: `lpr` of them).
template <int LPR>
__device__ __forceinline__ float row_sum(float v, int lpr) {
    if constexpr (LPR == 16) {
        v += dpp<kRor + 8>(v, v);
        v += dpp<kRor + 4>(v, v);
        v += dpp<kRor + 2>(v, v);
        v += dpp<kRor + 1>(v, v);
    } else if constexpr (LPR == 8) {
        v += dpp<kHalfMirror>(v, v);
        v += dpp<quad(2, 3, 0, 1)>(v, v);
        v += dpp<quad(1, 0, 3, 2)>(v, v);
    } else {
        for (int o = lpr >> 1; o > 0; o >>= 1) v += __shfl_xor(v, o);
    }
    return v;
}
// The value of the lane LPR / 2 away in the same row.
template <int LPR>
__device__ __forceinline__ float across(float v) {
    if constexpr (LPR == 16) return dpp<kRor + 8>(v, v);
    const float lo = dpp<kShl + 4, 0x5>(v, v);       // lanes 0..3 of 8 take 4..7
    return dpp<kShr + 4, 0xa>(lo, v);                // and the other way round
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

// x cos + partner * sin of a row; SIGN -1 is the transposed rotation. LPR: the whole head turns
// by halves that lie LPR / 2 lanes apart (0: any rotation).
template <int VEC, int NV, int LPR, int SIGN>
__device__ __forceinline__ void rotate(const Angles<VEC, NV> &g, int rot, int layout, int li, int lpr,
                                       float (&x)[NV][VEC]) {
    if constexpr (LPR > 0) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) x[0][j] = fmaf(across<LPR>(x[0][j]), SIGN * g.s[0][j], x[0][j] * g.c[0][j]);
        return;
    }
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
            x[v][j] = fmaf(turned ? p[v][j] : 0.f, SIGN * g.s[v][j], x[v][j] * g.c[v][j]);
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

// 1 / root of the mean square (v_rsq_f32 is off by one unit at most, and takes a subnormal number
// for 0: small ones are scaled).
__device__ __forceinline__ float inv_root(float ss, float inv_d, float eps) {
    const float m = fmaf(ss, inv_d, eps);
    const bool small = m < 0x1p-100f;
    return __builtin_amdgcn_rsqf(small ? m * 0x1p100f : m) * (small ? 0x1p50f : 1.f);
}

// Wavefront w of the grid: token w / chunks, rows (w % chunks) * per ... of its q, k and v.
template <typename T, int VEC, int NV, int LPR>
__global__ __launch_bounds__(256) void qk_forward_kernel(QkArgs a, int lpr_, int chunks, int per) {
    const int lpr = LPR ? LPR : lpr_;
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)block_index() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t t = (uint32_t)(w / chunks);
    if (t >= (uint32_t)a.tokens) return;
    const int li = lane & (lpr - 1), sub = lane / lpr, rpw = 64 / lpr;
    const int nvec = a.d / VEC;
    const int h0 = (int)(w % chunks) * per, h1 = h0 + per;
    const float inv_d = 1.f / (float)a.d;

    Angles<VEC, NV> g;
    load_angles<VEC, NV>(a, t, li, nvec, g);
    const int64_t slot = a.slots ? (int64_t)a.slots[t] : t;
    const bool put = !a.slots || (slot >= 0 && slot < a.slot_rows);

    // heads [first, first + n) of this wavefront's rows are those of one view
    const auto heads = [&](auto kind, int first, int n, const HeadsArg &from, const HeadsArg &to, const void *weight,
                           int64_t row, bool keep) {
        constexpr bool COPY = decltype(kind)::value;
        const T *src = (const T *)from.p + t * from.st;
        T *dst = (T *)to.p + row * to.st;
        float wt[NV][VEC];
        load_weight<T, VEC, NV>(weight, li, nvec, wt);
        for (int h = max(h0 - first, 0); h < min(h1 - first, n); h += rpw) {
            const int r = h + sub;
            const bool live = r < min(h1 - first, n);
            if constexpr (COPY) {                    // (bits, so that a NaN keeps its own)
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const int i = li + 64 * v;
                    if (live && keep && i < nvec)
                        *(Pack<T, VEC> *)(dst + r * to.sh + i * VEC) = *(const Pack<T, VEC> *)(src + r * from.sh + i * VEC);
                }
                continue;
            }
            float x[NV][VEC], ss = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int i = li + 64 * v;
                if (live && i < nvec) {
                    load_vec<T, VEC>(src + r * from.sh + i * VEC, x[v]);
                } else {
#pragma unroll
                    for (int j = 0; j < VEC; ++j) x[v][j] = 0.f;
                }
            }
            if (weight) {
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) ss = fmaf(x[v][j], x[v][j], ss);
                const float rr = inv_root(row_sum<LPR>(ss, lpr), inv_d, a.eps);
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) x[v][j] = x[v][j] * rr * wt[v][j];
            }
            rotate<VEC, NV, LPR, 1>(g, a.rot, a.layout, li, lpr, x);
            if (live && keep) {
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const int i = li + 64 * v;
                    if (i < nvec) store_vec<T, VEC>(dst + r * to.sh + i * VEC, x[v]);
                }
            }
        }
    };
    heads(std::false_type{}, 0, a.hq, a.q, a.qo, a.wq, t, true);
    heads(std::false_type{}, a.hq, a.hk, a.k, a.ko, a.wk, slot, put);
    if (a.hv) heads(std::true_type{}, a.hq + a.hk, a.hv, a.v, a.vo, nullptr, slot, put);
}

// Persistent wavefronts over tokens; a lane sums its elements' weight gradients over all its
// rows, the workgroup joins them in a fixed order and writes one partial row.
template <typename T, int VEC, int NV, int LPR>
__global__ __launch_bounds__(256) void qk_backward_kernel(QkArgs a, int lpr_) {
    const int lpr = LPR ? LPR : lpr_;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & (lpr - 1), sub = lane / lpr, rpw = 64 / lpr;
    const int nvec = a.d / VEC;
    const uint32_t stride = gridDim.x * 4;
    const float inv_d = 1.f / (float)a.d;
    float wq[NV][VEC], wk[NV][VEC], sq[NV][VEC] = {}, sk[NV][VEC] = {};
    load_weight<T, VEC, NV>(a.wq, li, nvec, wq);
    load_weight<T, VEC, NV>(a.wk, li, nvec, wk);

    for (uint32_t t = blockIdx.x * 4 + wave; t < (uint32_t)a.tokens; t += stride) {
        Angles<VEC, NV> g;
        load_angles<VEC, NV>(a, t, li, nvec, g);
        const auto heads = [&](int n, const HeadsArg &from, const HeadsArg &grad, const HeadsArg &to, bool normed,
                               const float (&wt)[NV][VEC], float (&sum)[NV][VEC]) {
            const T *src = (const T *)from.p + t * from.st, *grd = (const T *)grad.p + t * grad.st;
            T *dst = (T *)to.p + t * to.st;
            for (int h = 0; h < n; h += rpw) {
                const int r = h + sub;
                const bool live = r < n;
                float x[NV][VEC], y[NV][VEC];
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const int i = li + 64 * v;
                    if (live && i < nvec) {
                        load_vec<T, VEC>(src + r * from.sh + i * VEC, x[v]);
                        load_vec<T, VEC>(grd + r * grad.sh + i * VEC, y[v]);
                    } else {
#pragma unroll
                        for (int j = 0; j < VEC; ++j) x[v][j] = y[v][j] = 0.f;
                    }
                }
                rotate<VEC, NV, LPR, -1>(g, a.rot, a.layout, li, lpr, y);
                if (normed) {
                    float ss = 0.f, sh = 0.f;
#pragma unroll
                    for (int v = 0; v < NV; ++v)
#pragma unroll
                        for (int j = 0; j < VEC; ++j) {
                            ss = fmaf(x[v][j], x[v][j], ss);
                            sh = fmaf(y[v][j] * wt[v][j], x[v][j], sh);
                        }
                    ss = row_sum<LPR>(ss, lpr);
                    sh = row_sum<LPR>(sh, lpr);
                    const float rr = inv_root(ss, inv_d, a.eps), m = rr * (sh * inv_d);
#pragma unroll
                    for (int v = 0; v < NV; ++v)
#pragma unroll
                        for (int j = 0; j < VEC; ++j) {
                            // (a row that is not there has x = y = 0, and eps may be 0)
                            const float n = x[v][j] * rr;
                            if (live && li + 64 * v < nvec) sum[v][j] = fmaf(y[v][j], n, sum[v][j]);
                            y[v][j] = rr * (y[v][j] * wt[v][j] - n * m);
                        }
                }
                if (live) {
#pragma unroll
                    for (int v = 0; v < NV; ++v) {
                        const int i = li + 64 * v;
                        if (i < nvec) store_vec<T, VEC>(dst + r * to.sh + i * VEC, y[v]);
                    }
                }
            }
        };
        heads(a.hq, a.q, a.qo, a.gq, a.wq != nullptr, wq, sq);
        heads(a.hk, a.k, a.ko, a.gk, a.wk != nullptr, wk, sk);
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

// Sums the partial rows: 4 columns a workgroup, every 256th row a thread (at most 4 of them, all
// loads in flight together: the pass is a chain of waits, and few rows a thread keep it short).
__global__ __launch_bounds__(256) void qk_weight_grad_kernel(QkArgs a, int blocks) {
    const int cols = 2 * a.d, c0 = blockIdx.x * 4;
    float s[4] = {};
#pragma unroll
    for (int k = 0; k < kQkBwdBlocks / 256; ++k) {
        const int b = threadIdx.x + 256 * k;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (b < blocks && c0 + i < cols) s[i] += a.part[(int64_t)b * cols + c0 + i];
    }
    __shared__ float join[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        for (int o = 32; o > 0; o >>= 1) s[i] += __shfl_xor(s[i], o);
        if ((threadIdx.x & 63) == 0) join[threadIdx.x >> 6][i] = s[i];
    }
    __syncthreads();
    const int i = threadIdx.x, c = c0 + i;
    if (i >= 4 || c >= cols) return;
    float *out = c < a.d ? a.gwq : a.gwk;
    if (out) out[c < a.d ? c : c - a.d] = (join[0][i] + join[1][i]) + (join[2][i] + join[3][i]);
}

template <typename T, int VEC, int NV, int LPR>
hipError_t launch(const QkArgs &a, int lpr, bool backward, hipStream_t st) {
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
        qk_forward_kernel<T, VEC, NV, LPR><<<grid_of((waves + 3) / 4), 256, 0, st>>>(a, lpr, chunks, per);
        return hipGetLastError();
    }
    const int blocks = min(kQkBwdBlocks, (a.tokens - 1) / 4 + 1);   // (one without tokens)
    qk_backward_kernel<T, VEC, NV, LPR><<<blocks, 256, 0, st>>>(a, lpr);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.gwq || a.gwk) qk_weight_grad_kernel<<<(2 * a.d + 3) / 4, 256, 0, st>>>(a, blocks);
    return hipGetLastError();
}

template <typename T, int VEC, int NV>
hipError_t go(const QkArgs &a, bool backward, hipStream_t st) {
    const int nvec = a.d / VEC;
    int lpr = 1;
    while (lpr < nvec && lpr < 64) lpr <<= 1;
    // whole heads that turn by halves, on 16 or 8 lanes: sums and partners without LDS
    if constexpr (NV == 1 && VEC * sizeof(T) == 16) {
        const bool halves = a.layout == OLIVE_ROPE_HALF && a.rot == a.d && nvec == lpr;
        if (halves && lpr == 16) return launch<T, VEC, NV, 16>(a, lpr, backward, st);
        if (halves && lpr == 8) return launch<T, VEC, NV, 8>(a, lpr, backward, st);
    }
    return launch<T, VEC, NV, 0>(a, lpr, backward, st);
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
