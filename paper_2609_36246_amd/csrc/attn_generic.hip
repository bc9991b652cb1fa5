// Attention on shared prefixes and its backward for every type, head size and stride: 32-bit
// products on the vector units. 16 query rows (a row is one query head of one token) against
// tiles of 16 keys, a thread for each pair; the running maximum and sum of the softmax and
// the output stay in registers over the one pass along the keys.
#include "attn_seq.hpp"
#include "olive_device.hpp"

namespace olive {
namespace {

constexpr int R = 16, KT = 16, THREADS = 256, MAXC = 16;   // MAXC * 16 >= head_dim

template <typename T>
__device__ __forceinline__ const T *row_ptr(const HeadsArg &h, int64_t t, int64_t head) {
    return (const T *)h.p + t * h.st + head * h.sh;
}
template <typename T>
__device__ __forceinline__ void put(const HeadsArg &h, int64_t t, int64_t head, int e, float v) {
    T *p = (T *)h.p + t * h.st + head * h.sh + e;
    if constexpr (sizeof(T) == 2) *p = (T)(pack_bf16x2(v, v) & 0xffffu);
    else *p = v;
}

__device__ __forceinline__ float max16(float v) {
    for (int o = 8; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}
__device__ __forceinline__ float sum16(float v) {
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// Rows r0 .. r0 + 15 of a token range into LDS (zeros past its end): row r is token r / g.
template <typename T>
__device__ __forceinline__ void load_rows(const HeadsArg &h, int64_t q0, int64_t r0, int64_t rows,
                                          int g, int kvh, int d, int ld, float *dst) {
    for (int i = threadIdx.x; i < R * d; i += THREADS) {
        const int r = i / d, e = i - r * d;
        float v = 0.f;
        if (r0 + r < rows) {
            const int64_t tok = (r0 + r) / g;
            v = load_elem<T>(row_ptr<T>(h, q0 + tok, kvh * g + (r0 + r - tok * g)), e);
        }
        dst[r * ld + e] = v;
    }
}

// Keys j0 .. j0 + 15 of a sequence's prefix and suffix (zeros past `end`).
template <typename T>
__device__ __forceinline__ void load_keys(const AttnArgs &a, const SeqView &s, const HeadsArg &p,
                                          const HeadsArg &u, int j0, int end, int kvh, int ld,
                                          float *dst, bool &bad) {
    for (int i = threadIdx.x; i < KT * a.d; i += THREADS) {
        const int r = i / a.d, e = i - r * a.d, j = j0 + r;
        float v = 0.f;
        if (j < end)
            v = load_elem<T>(j < s.plen ? row_ptr<T>(p, s.pstart + j, kvh)
                                        : row_ptr<T>(u, suffix_row(a, s, j - s.plen, bad), kvh), e);
        dst[r * ld + e] = v;
    }
}

__device__ __forceinline__ float dot(const float *x, const float *y, int d) {
    float s = 0.f;
    for (int e = 0; e < d; ++e) s = fmaf(x[e], y[e], s);
    return s;
}

struct Unit { int b, kvh; int64_t r0; };
__device__ __forceinline__ Unit unit_of(const AttnArgs &a, int tiles) {
    Unit u;
    u.kvh = blockIdx.x % a.hk;
    const int v = blockIdx.x / a.hk;
    u.r0 = (int64_t)(v % tiles) * R;
    u.b = v / tiles;
    return u;
}

template <typename T>
__global__ __launch_bounds__(THREADS) void attn_generic_kernel(AttnArgs a, int tiles) {
    extern __shared__ float lds[];
    const int ld = a.d + 1, g = a.hq / a.hk;
    float *qs = lds, *ks = qs + R * ld, *vs = ks + KT * ld, *ps = vs + KT * ld;
    const Unit u = unit_of(a, tiles);
    const SeqView s = load_seq(a, u.b);
    const int64_t rows = (int64_t)s.n * g;
    const int r = threadIdx.x >> 4, c = threadIdx.x & 15;
    if (s.skip || u.r0 >= rows) return;
    if (s.bad) {
        if (u.r0) return;
        for (int64_t i = threadIdx.x; i < rows * a.d; i += THREADS) {
            const int64_t row = i / a.d, tok = row / g;
            put<T>(a.o, s.q0 + tok, u.kvh * g + (row - tok * g), (int)(i - row * a.d), __builtin_nanf(""));
        }
        if (a.lse)
            for (int64_t row = threadIdx.x; row < rows; row += THREADS)
                a.lse[(s.q0 + row / g) * a.hq + u.kvh * g + row % g] = __builtin_nanf("");
        return;
    }
    load_rows<T>(a.q, s.q0, u.r0, rows, g, u.kvh, a.d, ld, qs);
    const int64_t row = u.r0 + r;
    const int tok = (int)(row / g);
    const int seen = row < rows ? s.plen + suffix_seen(s, tok) : 0;
    const int last = (int)(min(rows, u.r0 + R) - 1) / g;
    const int end = s.plen + suffix_seen(s, last);
    float m = kNegInf, l = 0.f, acc[MAXC] = {};
    bool bad = false;
    for (int j0 = 0; j0 < end; j0 += KT) {
        __syncthreads();
        load_keys<T>(a, s, a.kp, a.ks, j0, end, u.kvh, ld, ks, bad);
        load_keys<T>(a, s, a.vp, a.vs, j0, end, u.kvh, ld, vs, bad);
        __syncthreads();
        float z = j0 + c < seen ? dot(qs + r * ld, ks + c * ld, a.d) * a.scale : kNegInf;
        const float m2 = fmaxf(m, max16(z));
        const float p = m2 == kNegInf && z == kNegInf ? 0.f : expf(z - m2);
        const float f = m == m2 ? 1.f : expf(m - m2);
        m = m2;
        l = l * f + sum16(p);
        ps[r * KT + c] = p;
        __syncthreads();
        // a key that a row does not see adds nothing to it, whatever its value holds
        const int keys = min(KT, seen - j0);
#pragma unroll
        for (int i = 0; i < MAXC; ++i) {
            const int e = c + 16 * i;
            if (e >= a.d) continue;
            float v = acc[i] * f;
            for (int k = 0; k < keys; ++k) v = fmaf(ps[r * KT + k], vs[k * ld + e], v);
            acc[i] = v;
        }
    }
    if (__syncthreads_or(bad)) l = __builtin_nanf("");
    if (row >= rows) return;
    const int64_t t = s.q0 + tok;
    const int head = u.kvh * g + (int)(row - (int64_t)tok * g);
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
        const int e = c + 16 * i;
        if (e >= a.d) continue;
        put<T>(a.o, t, head, e, acc[i] * inv);
    }
    if (a.lse && c == 0) a.lse[t * a.hq + head] = l == 0.f ? kNegInf : m + logf(l);
}

// delta = sum of grad_out * out of a row: 64 lanes a row.
template <typename T>
__global__ __launch_bounds__(THREADS) void attn_delta_kernel(AttnArgs a, float *delta) {
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (w >= a.total_q * a.hq) return;
    const int64_t t = w / a.hq;
    const int head = (int)(w - t * a.hq);
    const T *x = row_ptr<T>(a.o, t, head), *y = row_ptr<T>(a.go, t, head);
    float s = 0.f;
    for (int e = threadIdx.x & 63; e < a.d; e += 64) s = fmaf(load_elem<T>(x, e), load_elem<T>(y, e), s);
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if ((threadIdx.x & 63) == 0) delta[w] = s;
}

// p and dz of a pair from its two products; lse and delta are the row's.
__device__ __forceinline__ float pair_p(float z, float lse) {
    return lse == kNegInf ? 0.f : expf(z - lse);
}

template <typename T>
__global__ __launch_bounds__(THREADS) void attn_generic_dq_kernel(AttnArgs a, int tiles,
                                                                  const float *delta) {
    extern __shared__ float lds[];
    const int ld = a.d + 1, g = a.hq / a.hk;
    float *qs = lds, *gs = qs + R * ld, *ks = gs + R * ld, *vs = ks + KT * ld, *ps = vs + KT * ld;
    const Unit u = unit_of(a, tiles);
    const SeqView s = load_seq(a, u.b);
    const int64_t rows = (int64_t)s.n * g;
    const int r = threadIdx.x >> 4, c = threadIdx.x & 15;
    if (s.skip || u.r0 >= rows) return;
    if (s.bad) {
        if (u.r0) return;
        for (int64_t i = threadIdx.x; i < rows * a.d; i += THREADS) {
            const int64_t row = i / a.d, tok = row / g;
            put<T>(a.gq, s.q0 + tok, u.kvh * g + (row - tok * g), (int)(i - row * a.d), __builtin_nanf(""));
        }
        return;
    }
    load_rows<T>(a.q, s.q0, u.r0, rows, g, u.kvh, a.d, ld, qs);
    load_rows<T>(a.go, s.q0, u.r0, rows, g, u.kvh, a.d, ld, gs);
    const int64_t row = u.r0 + r;
    const int tok = (int)(row / g);
    const int64_t t = s.q0 + tok;
    const int head = u.kvh * g + (int)(row - (int64_t)tok * g);
    const bool live = row < rows;
    const float lse = live ? a.lse[t * a.hq + head] : kNegInf;
    const float del = live ? delta[t * a.hq + head] : 0.f;
    const int seen = live ? s.plen + suffix_seen(s, tok) : 0;
    const int end = s.plen + suffix_seen(s, (int)(min(rows, u.r0 + R) - 1) / g);
    float acc[MAXC] = {};
    bool bad = false;
    for (int j0 = 0; j0 < end; j0 += KT) {
        __syncthreads();
        load_keys<T>(a, s, a.kp, a.ks, j0, end, u.kvh, ld, ks, bad);
        load_keys<T>(a, s, a.vp, a.vs, j0, end, u.kvh, ld, vs, bad);
        __syncthreads();
        float dz = 0.f;
        if (j0 + c < seen) {
            const float p = pair_p(dot(qs + r * ld, ks + c * ld, a.d) * a.scale, lse);
            dz = p * (dot(gs + r * ld, vs + c * ld, a.d) - del) * a.scale;
        }
        ps[r * KT + c] = dz;
        __syncthreads();
        const int keys = min(KT, seen - j0);
#pragma unroll
        for (int i = 0; i < MAXC; ++i) {
            const int e = c + 16 * i;
            if (e >= a.d) continue;
            float v = acc[i];
            for (int k = 0; k < keys; ++k) v = fmaf(ps[r * KT + k], ks[k * ld + e], v);
            acc[i] = v;
        }
    }
    if (!live) return;
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
        const int e = c + 16 * i;
        if (e >= a.d) continue;
        put<T>(a.gq, t, head, e, acc[i]);
    }
}

// 16 keys of a prefix (seen by every row of its group) or of a suffix against all the rows
// that see them.
template <typename T, bool PREFIX>
__global__ __launch_bounds__(THREADS) void attn_generic_dkv_kernel(AttnArgs a, int tiles,
                                                                   const float *delta) {
    extern __shared__ float lds[];
    const int ld = a.d + 1, g = a.hq / a.hk;
    float *qs = lds, *gs = qs + R * ld, *ks = gs + R * ld, *vs = ks + KT * ld, *ps = vs + KT * ld,
          *ds = ps + R * KT;
    const int kvh = blockIdx.x % a.hk;
    const int v = blockIdx.x / a.hk, own = v / tiles, j0 = (v - own * tiles) * KT;
    const HeadsArg &kh = PREFIX ? a.kp : a.ks, &vh = PREFIX ? a.vp : a.vs;
    const HeadsArg &gk = PREFIX ? a.gkp : a.gks, &gv = PREFIX ? a.gvp : a.gvs;
    int64_t q0, toks, krow;
    int keys, first = 0;            // first: suffix keys that query 0 sees, less one
    if (PREFIX) {
        const int b0 = a.group_seqs[own], b1 = a.group_seqs[own + 1];
        if (b0 < 0 || b1 < b0 || b1 > a.seqs || !prefix_ok(a, own)) return;
        keys = a.prefix_len[own];
        krow = a.prefix_start[own];
        q0 = a.cu_q[b0];
        toks = a.cu_q[b1] - q0;
    } else {
        const SeqView s = load_seq(a, own);
        if (s.skip || s.bad) return;
        keys = s.slen;
        krow = s.sstart;
        q0 = s.q0;
        toks = s.n;
        first = s.slen - s.n;
    }
    if (j0 >= keys || q0 < 0 || toks < 0 || q0 + toks > a.total_q) return;
    for (int i = threadIdx.x; i < KT * a.d; i += THREADS) {
        const int k = i / a.d, e = i - k * a.d;
        const bool in = j0 + k < keys;
        ks[k * ld + e] = in ? load_elem<T>(row_ptr<T>(kh, krow + j0 + k, kvh), e) : 0.f;
        vs[k * ld + e] = in ? load_elem<T>(row_ptr<T>(vh, krow + j0 + k, kvh), e) : 0.f;
    }
    const int r = threadIdx.x >> 4, c = threadIdx.x & 15;
    float dk[MAXC] = {}, dv[MAXC] = {};
    const int64_t rows = toks * g;
    // the first row that sees the tile's first key
    const int64_t from = PREFIX ? 0 : (int64_t)max(0, j0 - first) * g / R * R;
    for (int64_t r0 = from; r0 < rows; r0 += R) {
        __syncthreads();
        load_rows<T>(a.q, q0, r0, rows, g, kvh, a.d, ld, qs);
        load_rows<T>(a.go, q0, r0, rows, g, kvh, a.d, ld, gs);
        __syncthreads();
        const int64_t row = r0 + r, tok = row / g;
        float p = 0.f, dz = 0.f;
        if (row < rows && j0 + c < keys && (PREFIX || j0 + c <= first + tok)) {
            const int64_t at = (q0 + tok) * a.hq + kvh * g + (row - tok * g);
            p = pair_p(dot(qs + r * ld, ks + c * ld, a.d) * a.scale, a.lse[at]);
            dz = p * (dot(gs + r * ld, vs + c * ld, a.d) - delta[at]) * a.scale;
        }
        ps[c * R + r] = p;
        ds[c * R + r] = dz;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < MAXC; ++i) {
            const int e = c + 16 * i;
            if (e >= a.d) continue;
            float x = dk[i], y = dv[i];
            for (int k = 0; k < R; ++k) {
                x = fmaf(ds[r * R + k], qs[k * ld + e], x);
                y = fmaf(ps[r * R + k], gs[k * ld + e], y);
            }
            dk[i] = x;
            dv[i] = y;
        }
    }
    if (j0 + r >= keys) return;
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
        const int e = c + 16 * i;
        if (e >= a.d) continue;
        put<T>(gk, krow + j0 + r, kvh, e, dk[i]);
        put<T>(gv, krow + j0 + r, kvh, e, dv[i]);
    }
}

int64_t tiles_of(int64_t n, int tile) { return (n + tile - 1) / tile; }

template <typename T>
hipError_t forward(const AttnArgs &a, hipStream_t st) {
    const int tiles = (int)tiles_of((int64_t)a.max_q * (a.hq / a.hk), R);
    const size_t bytes = sizeof(float) * ((R + 2 * KT) * (a.d + 1) + R * KT);
    attn_generic_kernel<T><<<(unsigned)((int64_t)a.seqs * tiles * a.hk), THREADS, bytes, st>>>(a, tiles);
    return hipGetLastError();
}

template <typename T>
hipError_t backward(const AttnArgs &a, hipStream_t st) {
    float *delta = (float *)a.work;
    const int g = a.hq / a.hk;
    const int tiles = (int)tiles_of((int64_t)a.max_q * g, R);
    const size_t bytes = sizeof(float) * ((2 * R + 2 * KT) * (a.d + 1) + 2 * R * KT);
    if (a.total_q > 0) {
        attn_delta_kernel<T><<<(unsigned)tiles_of(a.total_q * a.hq, 4), THREADS, 0, st>>>(a, delta);
        attn_generic_dq_kernel<T><<<(unsigned)((int64_t)a.seqs * tiles * a.hk), THREADS, bytes, st>>>(
            a, tiles, delta);
    }
    const int pt = (int)tiles_of(a.max_prefix, KT), sl = (int)tiles_of(a.max_suffix, KT);
    if (pt)
        attn_generic_dkv_kernel<T, true><<<(unsigned)((int64_t)a.groups * pt * a.hk), THREADS, bytes, st>>>(
            a, pt, delta);
    if (sl)
        attn_generic_dkv_kernel<T, false><<<(unsigned)((int64_t)a.seqs * sl * a.hk), THREADS, bytes, st>>>(
            a, sl, delta);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_generic(const AttnArgs &a, bool bf16, hipStream_t st) {
    return bf16 ? forward<uint16_t>(a, st) : forward<float>(a, st);
}
hipError_t launch_attn_generic_backward(const AttnArgs &a, bool bf16, hipStream_t st) {
    return bf16 ? backward<uint16_t>(a, st) : backward<float>(a, st);
}

}  // namespace olive
