// Attention on shared prefixes and its backward for every type, head size and stride: 32-bit
// products on the matrix units (v_mfma_f32_16x16x4_f32), operands straight from memory.
//
// A workgroup takes 16 query rows (a row is one query head of one token), or 16 keys in the
// pass for the keys' gradients; its 4 wavefronts take different tiles of 16 along the other
// axis and join their sums through LDS at the end. The first product is formed so that its
// result is the second one's operand where it lies: a lane holds 4 values of one column, and
// product i of the next sum takes the i-th of them from every lane, with rows of the other
// operand to match.
//
// Bound by the waits for the operands: forward and backward of 3 runs of 30 to 90 tokens on a
// prefix of 150, fp32, 4 / 2 heads of 64: 39 us (12 forward, 3 delta, 24 gradients).
#include "attn_seq.hpp"
#include "olive_device.hpp"

namespace olive {
namespace {

constexpr int R = 16, THREADS = 256;
constexpr int kSideBySide = 4 * kChipUnits;   // workgroups of the backward's passes that one launch takes
typedef float floatx4 __attribute__((ext_vector_type(4)));

struct GenArgs {
    AttnArgs a;
    Div g, tiles, ptiles, stiles;    // (tiles: of a sequence's rows; of a prefix's and a suffix's keys)
    int dq_blocks, prefix_blocks;    // backward: workgroups of the pass for dq, of the prefixes' keys
    bool quads;                      // 4 elements of a row can be read at once
    float *delta;                    // backward: [total_q][hq] sums of grad_out * out
};

__device__ __forceinline__ floatx4 mfma4(float x, float y, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(x, y, c, 0, 0, 0);
}

template <typename T>
__device__ __forceinline__ const T *row_ptr(const HeadsArg &h, int64_t t, int64_t head) {
    return (const T *)h.p + t * h.st + head * h.sh;
}
template <typename T>
__device__ __forceinline__ void put(T *p, float v) {
    if constexpr (sizeof(T) == 2) *p = (T)(pack_bf16x2(v, v) & 0xffffu);
    else *p = v;
}

// NT 16-element blocks cover the head. Block n of a row as a first or second operand: elements
// 16 n + 4 q + 0..3 (q = lane / 16), zeros past d.
template <typename T, int NT>
__device__ __forceinline__ void load_row(const T *p, int d, bool quads, floatx4 (&x)[NT]) {
    const int q = (threadIdx.x & 63) >> 4;
    if (quads) {
        struct alignas(4 * sizeof(T)) Quad { T v[4]; };
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int i = 16 * n + 4 * q;
            Quad u{};
            if (i < d) u = *(const Quad *)(p + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[n][e] = load_elem<T>(u.v, e);
        }
        return;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = 16 * n + 4 * q + e;
            x[n][e] = i < d ? load_elem<T>(p, i) : 0.f;
        }
}
// Rows 4 q + 0..3 (their pointers) as a transposed first operand: element 16 n + lane % 16.
template <typename T, int NT>
__device__ __forceinline__ void load_cols(const T *const (&p)[4], int d, floatx4 (&x)[NT]) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int i = 16 * n + (threadIdx.x & 15);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[n][e] = i < d ? load_elem<T>(p[e], i) : 0.f;
    }
}
// Sum over the head of two rows' products: 16 x 16 results.
template <int NT>
__device__ __forceinline__ floatx4 product(const floatx4 (&x)[NT], const floatx4 (&y)[NT]) {
    floatx4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) c = mfma4(x[n][e], y[n][e], c);
    return c;
}
template <int NT>
__device__ __forceinline__ void add_outer(const floatx4 (&x)[NT], floatx4 p, floatx4 (&acc)[NT]) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[n] = mfma4(x[n][e], p[e], acc[n]);
}
__device__ __forceinline__ float max_of_quarters(float v) {
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float sum_of_quarters(float v) {
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// 16 query rows of a sequence; this lane's is row lane % 16 (a copy of the last one past the end).
struct Rows {
    SeqView s;
    int kvh, r0, rows;
    int tok, t, head;                // of this lane's row
    bool live, any;
};
__device__ __forceinline__ Rows find_rows(const GenArgs &f, int block) {
    const AttnArgs &a = f.a;
    Rows w;
    const int v = (uint32_t)block / (uint32_t)a.hk, b = f.tiles.quot(v);
    w.kvh = block - v * a.hk;
    w.r0 = f.tiles.rem(v, b) * R;
    w.s = load_seq(a, min(b, a.seqs - 1));
    w.rows = w.s.n * (int)f.g.d;
    w.any = b < a.seqs && !w.s.skip && w.r0 < w.rows;
    const int r = w.r0 + (threadIdx.x & 15), c = max(0, min(r, w.rows - 1));
    w.live = r < w.rows;
    w.tok = f.g.quot(c);
    w.head = w.kvh * (int)f.g.d + f.g.rem(c, w.tok);
    w.t = w.s.q0 + w.tok;
    return w;
}
// Every row of a sequence that is out of range.
template <typename T>
__device__ __forceinline__ void put_nan(const GenArgs &f, const Rows &w, const HeadsArg &o, float *lse) {
    if (w.r0) return;
    for (int r = threadIdx.x; r < w.rows; r += THREADS) {
        const int k = f.g.quot(r), t = w.s.q0 + k, head = w.kvh * (int)f.g.d + f.g.rem(r, k);
        T *p = (T *)row_ptr<T>(o, t, head);
        for (int e = 0; e < f.a.d; ++e) put<T>(p + e, __builtin_nanf(""));
        if (lse) lse[(int64_t)t * f.a.hq + head] = __builtin_nanf("");
    }
}

// Key j of the prefix and suffix together (a copy of key `end` - 1 from there on).
template <typename T>
__device__ __forceinline__ void key_ptrs(const AttnArgs &a, const SeqView &s, int kvh, int j, int end, bool &bad,
                                         const T *&k, const T *&v) {
    j = min(j, end - 1);
    if (j < s.plen) {
        k = row_ptr<T>(a.kp, s.pstart + j, kvh);
        v = row_ptr<T>(a.vp, s.pstart + j, kvh);
    } else {
        const int64_t row = suffix_row(a, s, j - s.plen, bad);
        k = row_ptr<T>(a.ks, row, kvh);
        v = row_ptr<T>(a.vs, row, kvh);
    }
}

template <typename T, int NT>
__global__ __launch_bounds__(THREADS, NT > 8 ? 1 : 2) void attn_generic_kernel(GenArgs f) {
    extern __shared__ float lds[];
    const AttnArgs &a = f.a;
    const Rows w = find_rows(f, block_index());
    if (!w.any) return;
    if (w.s.bad) {
        put_nan<T>(f, w, a.o, a.lse);
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, quarter = lane >> 4;
    floatx4 q[NT], acc[NT];
    load_row<T, NT>(row_ptr<T>(a.q, w.t, w.head), a.d, f.quads, q);
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n] = (floatx4)(0.f);
    const int seen = w.live ? w.s.plen + suffix_seen(w.s, w.tok) : 0;
    const int least = w.s.plen + suffix_seen(w.s, f.g.quot(w.r0));
    const int end = w.s.plen + suffix_seen(w.s, f.g.quot(upto(w.r0, R, w.rows) - 1));
    float m = kNegInf, l = 0.f;
    bool bad = false;
    for (int j0 = wave * R; j0 < end; j0 = upto(j0, 4 * R, end)) {
        const T *kp, *vp, *col[4], *unused;
        key_ptrs<T>(a, w.s, w.kvh, j0 + (lane & 15), end, bad, kp, vp);
#pragma unroll
        for (int e = 0; e < 4; ++e) key_ptrs<T>(a, w.s, w.kvh, j0 + 4 * quarter + e, end, bad, unused, col[e]);
        floatx4 x[NT];
        load_row<T, NT>(kp, a.d, f.quads, x);
        floatx4 z = product<NT>(x, q), p;
        float top = kNegInf;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            z[e] = j0 + 4 * quarter + e < seen ? z[e] * a.scale : kNegInf;
            top = fmaxf(top, z[e]);
        }
        const float m2 = fmaxf(m, max_of_quarters(top));
        const float r = m == m2 ? 1.f : expf(m - m2), m0 = m2 == kNegInf ? 0.f : m2;
        m = m2;
        l *= r;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            p[e] = expf(z[e] - m0);
            l += p[e];
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[n] *= r;
        load_cols<T, NT>(col, a.d, x);
        bool special = false;
        if (j0 > least - R) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) special |= !(fabsf(x[n][e]) < __builtin_inff());
        }
        if (!__any(special)) {
            add_outer<NT>(x, p, acc);
            continue;
        }
        // A value that is not finite, and rows that do not see its key: key by key, without the
        // rows that do not see it.
        for (int k = 0; k < R; ++k) {
            const T *v;
            key_ptrs<T>(a, w.s, w.kvh, j0 + k, end, bad, unused, v);
            const int e = k & 3;
            const float pk = __shfl(e == 0 ? p[0] : e == 1 ? p[1] : e == 2 ? p[2] : p[3],
                                    (k >> 2) * 16 + (lane & 15));
            if (j0 + k >= seen) continue;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = 16 * n + 4 * quarter + i;
                    if (at < a.d) acc[n][i] = fmaf(pk, load_elem<T>(v, at), acc[n][i]);
                }
        }
    }
    l = sum_of_quarters(l);
    bad = __syncthreads_or(bad);
    // [wave][row]: maximum, sum; [wave][row][element]
    float2 *ml = (float2 *)lds;
    float *o = lds + 2 * 4 * R;
    const int ld = a.d + 1, row = lane & 15;
    if (quarter == 0) ml[wave * R + row] = make_float2(m, l);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = 16 * n + 4 * quarter + i;
            if (at < a.d) o[(wave * R + row) * ld + at] = acc[n][i];
        }
    __syncthreads();
    // 16 threads a row, whose row is the one of their lane % 16 found above
    float wt[4], top = kNegInf, sum = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) top = fmaxf(top, ml[k * R + row].x);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 x = ml[k * R + row];
        wt[k] = x.x == top ? 1.f : expf(x.x - top);
        sum += x.y * wt[k];
    }
    if (bad) sum = __builtin_nanf("");
    if (!w.live) return;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    T *out = (T *)row_ptr<T>(a.o, w.t, w.head);
    for (int e = threadIdx.x >> 4; e < a.d; e += 16) {
        float x = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) x = fmaf(o[(k * R + row) * ld + e], wt[k], x);
        put<T>(out + e, x * inv);
    }
    if (a.lse && threadIdx.x < R) a.lse[(int64_t)w.t * a.hq + w.head] = sum == 0.f ? kNegInf : top + logf(sum);
}

// delta = sum of grad_out * out of a row: 64 lanes a row.
template <typename T>
__global__ __launch_bounds__(THREADS) void attn_delta_kernel(GenArgs f) {
    const AttnArgs &a = f.a;
    const int64_t w = (int64_t)block_index() * 4 + (threadIdx.x >> 6);
    if (w >= (int64_t)a.total_q * a.hq) return;
    const int t = (int)w / a.hq, head = (int)w - t * a.hq;
    const T *x = row_ptr<T>(a.o, t, head), *y = row_ptr<T>(a.go, t, head);
    float s = 0.f;
    for (int e = threadIdx.x & 63; e < a.d; e += 64) s = fmaf(load_elem<T>(x, e), load_elem<T>(y, e), s);
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if ((threadIdx.x & 63) == 0) f.delta[w] = s;
}

// p of a pair from its scaled score and the row's log-normaliser.
__device__ __forceinline__ float pair_p(float z, float lse) { return lse == kNegInf ? 0.f : expf(z - lse); }

// Adds the four wavefronts' sums of 16 columns (lane % 16) and writes them, scaled: column c of
// the first `cols` to out(c).
template <typename T, int NT, typename F>
__device__ __forceinline__ void join_and_put(float *o, const floatx4 (&acc)[NT], int d, int cols, float scale, F out) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, ld = d + 1;
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = 16 * n + 4 * (lane >> 4) + i;
            if (at < d) o[(wave * R + c) * ld + at] = acc[n][i];
        }
    __syncthreads();
    if (c >= cols) return;
    T *p = out(c);
    for (int e = threadIdx.x >> 4; e < d; e += 16)
        put<T>(p + e, ((o[c * ld + e] + o[(R + c) * ld + e]) + (o[(2 * R + c) * ld + e] + o[(3 * R + c) * ld + e])) * scale);
}

template <typename T, int NT>
__device__ __forceinline__ void dq_tile(const GenArgs &f, int block, float *lds) {
    const AttnArgs &a = f.a;
    const Rows w = find_rows(f, block);
    if (!w.any) return;
    if (w.s.bad) {
        put_nan<T>(f, w, a.gq, nullptr);
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, quarter = lane >> 4;
    floatx4 q[NT], go[NT], acc[NT];
    load_row<T, NT>(row_ptr<T>(a.q, w.t, w.head), a.d, f.quads, q);
    load_row<T, NT>(row_ptr<T>(a.go, w.t, w.head), a.d, f.quads, go);
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n] = (floatx4)(0.f);
    const int64_t at = (int64_t)w.t * a.hq + w.head;
    const float lse = a.lse[at], delta = f.delta[at];
    const int seen = w.live ? w.s.plen + suffix_seen(w.s, w.tok) : 0;
    const int end = w.s.plen + suffix_seen(w.s, f.g.quot(upto(w.r0, R, w.rows) - 1));
    bool bad = false;
    for (int j0 = wave * R; j0 < end; j0 = upto(j0, 4 * R, end)) {
        const T *kp, *vp, *col[4], *unused;
        key_ptrs<T>(a, w.s, w.kvh, j0 + (lane & 15), end, bad, kp, vp);
#pragma unroll
        for (int e = 0; e < 4; ++e) key_ptrs<T>(a, w.s, w.kvh, j0 + 4 * quarter + e, end, bad, col[e], unused);
        floatx4 x[NT];
        load_row<T, NT>(kp, a.d, f.quads, x);
        floatx4 z = product<NT>(x, q);
        load_row<T, NT>(vp, a.d, f.quads, x);
        const floatx4 y = product<NT>(x, go);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            z[e] = j0 + 4 * quarter + e < seen ? pair_p(z[e] * a.scale, lse) * (y[e] - delta) : 0.f;
        load_cols<T, NT>(col, a.d, x);
        add_outer<NT>(x, z, acc);
    }
    const int g = f.g.d;
    join_and_put<T, NT>(lds, acc, a.d, min(R, w.rows - w.r0), a.scale, [&](int c) {
        const int k = f.g.quot(w.r0 + c);
        return (T *)row_ptr<T>(a.gq, w.s.q0 + k, w.kvh * g + f.g.rem(w.r0 + c, k));
    });
}

// 16 keys of a prefix (seen by every row of its group) or of a suffix against all the rows
// that see them.
template <typename T, int NT, bool PREFIX>
__device__ __forceinline__ void dkv_tile(const GenArgs &f, int block, float *lds) {
    const AttnArgs &a = f.a;
    const Div &tiles = PREFIX ? f.ptiles : f.stiles;
    const int u = (uint32_t)block / (uint32_t)a.hk, kvh = block - u * a.hk, g = f.g.d;
    const int own = tiles.quot(u), j0 = tiles.rem(u, own) * R;
    if (own >= (PREFIX ? a.groups : a.seqs)) return;
    const HeadsArg &kh = PREFIX ? a.kp : a.ks, &vh = PREFIX ? a.vp : a.vs;
    const HeadsArg &gk = PREFIX ? a.gkp : a.gks, &gv = PREFIX ? a.gvp : a.gvs;
    int q0, toks, keys, first = 0;  // first: suffix keys that query 0 sees, less one
    int64_t krow;
    bool nan;                        // a sequence that has these keys is out of range: the sums are NaN
    if (PREFIX) {
        int q1;
        nan = !group_in_order(a, a.group_seqs[own], a.group_seqs[own + 1], q0, q1);
        if (!prefix_ok(a, own)) return;
        keys = a.prefix_len[own];
        krow = a.prefix_start[own];
        toks = q1 - q0;
    } else {
        const SeqView s = load_seq(a, own);
        nan = s.skip || s.bad;
        keys = s.keys;
        krow = s.sstart;
        q0 = s.q0;
        toks = s.n;
        first = s.slen - s.n;
    }
    if (j0 >= keys) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, quarter = lane >> 4;
    const int key = j0 + (lane & 15), rows = nan ? 0 : toks * g;
    floatx4 k[NT], v[NT], dk[NT], dv[NT];
    load_row<T, NT>(row_ptr<T>(kh, krow + min(key, keys - 1), kvh), a.d, f.quads, k);
    load_row<T, NT>(row_ptr<T>(vh, krow + min(key, keys - 1), kvh), a.d, f.quads, v);
#pragma unroll
    for (int n = 0; n < NT; ++n) dk[n] = dv[n] = (floatx4)(nan ? __builtin_nanf("") : 0.f);
    // the first row that sees this lane's key, and the tile's first one
    const auto row_of = [&](int j) { return PREFIX ? 0 : (int)min((int64_t)rows, (int64_t)max(0, j - first) * g); };
    const int from = row_of(key);
    for (int r0 = upto(row_of(j0) / R * R, wave * R, rows); r0 < rows; r0 = upto(r0, 4 * R, rows)) {
        const T *qc[4], *gc[4];
        float lse[4], delta[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = min(r0 + 4 * quarter + e, rows - 1), tok = f.g.quot(r);
            const int t = q0 + tok, head = kvh * g + f.g.rem(r, tok);
            qc[e] = row_ptr<T>(a.q, t, head);
            gc[e] = row_ptr<T>(a.go, t, head);
            lse[e] = a.lse[(int64_t)t * a.hq + head];
            delta[e] = f.delta[(int64_t)t * a.hq + head];
        }
        const int r = min(r0 + (lane & 15), rows - 1), tok = f.g.quot(r);
        const int t = q0 + tok, head = kvh * g + f.g.rem(r, tok);
        floatx4 x[NT], p, z;
        load_row<T, NT>(row_ptr<T>(a.q, t, head), a.d, f.quads, x);
        z = product<NT>(x, k);
        load_row<T, NT>(row_ptr<T>(a.go, t, head), a.d, f.quads, x);
        const floatx4 y = product<NT>(x, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int row = r0 + 4 * quarter + e;
            p[e] = row >= from && row < rows ? pair_p(z[e] * a.scale, lse[e]) : 0.f;
            z[e] = p[e] == 0.f ? 0.f : p[e] * (y[e] - delta[e]);
        }
        load_cols<T, NT>(gc, a.d, x);
        add_outer<NT>(x, p, dv);
        load_cols<T, NT>(qc, a.d, x);
        add_outer<NT>(x, z, dk);
    }
    const int cols = min(R, keys - j0);
    join_and_put<T, NT>(lds, dk, a.d, cols, a.scale, [&](int c) { return (T *)row_ptr<T>(gk, krow + j0 + c, kvh); });
    join_and_put<T, NT>(lds, dv, a.d, cols, 1.f, [&](int c) { return (T *)row_ptr<T>(gv, krow + j0 + c, kvh); });
}

// The passes for dq and for the keys' gradients need nothing of each other. Up to four workgroups
// a compute unit of both together they run side by side in one launch: few workgroups that wait
// for loads. More of them get two launches, in each of which all take about as long. Backward with
// its delta in fp32, one launch against two (us): heads of 64, 128 workgroups 35 : 48, 680 86 : 100,
// 848 64 : 74, 1328 138 : 122, 1360 106 : 118, 1744 179 : 159; heads of 128, 128 workgroups
// 56 : 76, 848 119 : 124, 2632 552 : 497.
template <typename T, int NT, bool DQ, bool DKV>
__global__ __launch_bounds__(THREADS, NT > (DKV ? 4 : 8) ? 1 : 2) void attn_generic_backward_kernel(GenArgs f) {
    extern __shared__ float lds[];
    int block = block_index();
    if constexpr (DQ) {
        if (!DKV || block < f.dq_blocks) {
            dq_tile<T, NT>(f, block, lds);
            return;
        }
        block -= f.dq_blocks;
    }
    if constexpr (DKV) {
        if (block < f.prefix_blocks) dkv_tile<T, NT, true>(f, block, lds);
        else dkv_tile<T, NT, false>(f, block - f.prefix_blocks, lds);
    }
}

int64_t tiles_of(int64_t n) { return (n + R - 1) / R; }

// Whether rows of every operand lie on 4 elements.
bool in_quads(const AttnArgs &a, int esz) {
    if (a.d % 4) return false;
    for (const HeadsArg *h : {&a.q, &a.kp, &a.vp, &a.ks, &a.vs, &a.go})
        if (h->p && (((uintptr_t)h->p | (uint64_t)(h->st * esz) | (uint64_t)(h->sh * esz)) & (4 * esz - 1))) return false;
    return true;
}

template <typename T, int NT>
hipError_t forward(const AttnArgs &a, hipStream_t st) {
    const int64_t tiles = tiles_of((int64_t)a.max_q * (a.hq / a.hk));
    GenArgs f{};
    f.a = a;
    f.g = Div::of(a.hq / a.hk);
    f.tiles = Div::of(tiles);
    f.quads = in_quads(a, sizeof(T));
    attn_generic_kernel<T, NT><<<grid_of(a.seqs * tiles * a.hk), THREADS,
                                 sizeof(float) * (2 * 4 * R + 4 * R * (a.d + 1)), st>>>(f);
    return hipGetLastError();
}

template <typename T, int NT>
hipError_t backward(const AttnArgs &a, hipStream_t st) {
    const int64_t g = a.hq / a.hk, tiles = tiles_of(a.max_q * g);
    const size_t bytes = sizeof(float) * 4 * R * (a.d + 1);
    const int64_t pt = tiles_of(a.max_prefix), sl = tiles_of(a.max_suffix);
    const auto div = [](int64_t d) { return Div::of(d > 0 ? d : 1); };
    GenArgs f{};
    f.a = a;
    f.g = Div::of(g);
    f.tiles = div(tiles);
    f.ptiles = div(pt);
    f.stiles = div(sl);
    f.quads = in_quads(a, sizeof(T));
    f.delta = (float *)a.work;
    const int64_t rows = a.total_q > 0 ? a.seqs * tiles * a.hk : 0;
    const int64_t prefix = a.groups * pt * a.hk, keys = prefix + a.seqs * sl * a.hk;
    f.prefix_blocks = (int)prefix;
    hipError_t e = hipSuccess;
    if (rows) {
        attn_delta_kernel<T><<<grid_of(((int64_t)a.total_q * a.hq + 3) / 4), THREADS, 0, st>>>(f);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if constexpr (NT <= 8) {
        if (rows + keys <= kSideBySide) {
            f.dq_blocks = (int)rows;
            if (rows + keys)
                attn_generic_backward_kernel<T, NT, true, true><<<(unsigned)(rows + keys), THREADS, bytes, st>>>(f);
            return hipGetLastError();
        }
    }
    if (rows) attn_generic_backward_kernel<T, NT, true, false><<<grid_of(rows), THREADS, bytes, st>>>(f);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (keys) attn_generic_backward_kernel<T, NT, false, true><<<grid_of(keys), THREADS, bytes, st>>>(f);
    return hipGetLastError();
}

template <typename T>
hipError_t by_size(const AttnArgs &a, bool back, hipStream_t st) {
    if (a.d <= 64) return back ? backward<T, 4>(a, st) : forward<T, 4>(a, st);
    if (a.d <= 128) return back ? backward<T, 8>(a, st) : forward<T, 8>(a, st);
    return back ? backward<T, 16>(a, st) : forward<T, 16>(a, st);
}

}  // namespace

hipError_t launch_attn_generic(const AttnArgs &a, bool bf16, hipStream_t st) {
    return bf16 ? by_size<uint16_t>(a, false, st) : by_size<float>(a, false, st);
}
hipError_t launch_attn_generic_backward(const AttnArgs &a, bool bf16, hipStream_t st) {
    return bf16 ? by_size<uint16_t>(a, true, st) : by_size<float>(a, true, st);
}

}  // namespace olive
