// Backward of the attention on shared prefixes, bf16 on matrix instructions (head_dim a
// multiple of 8 up to 128, rows on 16 bytes).
//
//   p = exp(scale q k - lse),   dp = do v^T,   ds = p (dp - delta),   delta = sum of do * out
//   dq = scale ds K,   dk = scale ds^T q,   dv = p^T do
//
// Two passes that each form p and ds again, so that every gradient is summed by one workgroup
// in a fixed order (7 products for the 5 of a single pass with atomic additions):
//   dq   32 query rows a wavefront; the keys and values pass through LDS. The products lie as
//        keys x rows, so a lane holds one row and ds^T is the next product's operand as it is.
//   dkv  32 keys a wavefront, held with their values in registers; the query rows and their
//        output gradients pass through LDS. The products lie as rows x keys, a lane holds one
//        key, and p and ds are the operands of dv^T = do^T p and dk^T = q^T ds as they are.
// The transposed operands come out of LDS through the transposing read. p and ds are rounded
// to bf16 as operands (fp32 products run at an eighth of the rate); all sums are fp32. delta is
// formed of the stored outputs, so where few keys are seen, and dp - delta cancels, their rounding
// counts: dq and dk are 0.0044 (2-norm) from the exact ones where queries see up to 2 keys, 0.0034
// up to 8, 0.0029 up to 32, 0.0026 up to 200, 0.0024 to 0.0025 beyond (rounded alone: 0.0017).
// A prefix's keys meet the rows of all its sequences; where there are too few key tiles to fill
// the chip the rows are cut into parts, whose fp32 sums a last kernel adds in order.
//
// Bound by the products: 8 runs of 1024 tokens on 2 prefixes of 4096, 16 / 8 heads of 128: dq
// 428 us and dkv 596 us (matrix units 54 and 48 % busy at 1.8 to 1.9 GHz), lse and delta 15 us.
#include "attn_tile.hpp"

namespace olive {
namespace {

constexpr int DQ_KEYS = 64;          // keys of a tile of the dq pass
constexpr int KEYS = 128;            // keys of a workgroup of the dkv pass
constexpr int ROWS = 32;             // query rows of a tile of the dkv pass

struct BwdPlan {
    RowOrder order;                  // of a sequence's tiles of 128 rows
    int ptiles, stiles;              // tiles of KEYS keys of a prefix, of a suffix
    int np, ns;                      // parts of the rows
    RowOrder porder, sorder;         // of the key tiles of a prefix, of a suffix
    int64_t q_units, p_units, s_units;   // workgroups of the dq pass, of the dkv pass
};

BwdPlan make_plan(const AttnArgs &a) {
    BwdPlan p{};
    const int64_t g = a.hq / a.hk, seq_rows = a.max_q * g;
    p.order = RowOrder::of(ceil_div(seq_rows, 128));
    p.q_units = a.seqs * p.order.units() * a.hk;
    p.ptiles = (int)ceil_div(a.max_prefix, KEYS);
    p.stiles = (int)ceil_div(a.max_suffix, KEYS);
    const int64_t pu = (int64_t)a.groups * p.ptiles * a.hk, su = (int64_t)a.seqs * p.stiles * a.hk;
    // two workgroups a compute unit; a part of at least four row tiles
    const auto split = [&](int64_t units, int64_t rows) {
        const int64_t most = ceil_div(rows, 4 * ROWS);
        int64_t n = units > 0 ? 2 * kChipUnits / units : 1;
        n = n < most ? n : most;
        return (int)(n < 1 ? 1 : n);
    };
    p.np = split(pu, ceil_div(a.total_q * g, a.groups));
    p.ns = split(pu * p.np + su, seq_rows);
    p.porder = RowOrder::of(p.ptiles);
    p.sorder = RowOrder::of(p.stiles);
    p.p_units = pu * p.np;
    p.s_units = su * p.ns;
    return p;
}

struct BwdArgs {
    AttnArgs a;
    BwdPlan p;
    DieOrder qd, pd, sd;
    Div g, hk, seqs, groups, ptiles, stiles, pall, sall, np, ns;   // (pall, sall: tiles of a part)
    // [hk][total_q][g] each: what the products of a row begin at, so that z is scale^-1 (scale q
    // k - lse) and y is dp - delta
    float *nlse;                     // -lse / scale, -inf for a row that sees nothing
    float *ndelta;                   // -delta
    float *part;                     // fp32 parts: prefix tiles, then suffix tiles
};

// lse and delta of a row: DP / 8 lanes a row.
template <int DP>
__global__ __launch_bounds__(256) void attn_stats_kernel(BwdArgs f) {
    const AttnArgs &a = f.a;
    constexpr int LPR = DP / 8;
    const int64_t r = ((int64_t)block_index() * 256 + threadIdx.x) / LPR;
    const int c = threadIdx.x % LPR, nch = a.d / 8, g = a.hq / a.hk;
    if (r >= (int64_t)a.total_q * a.hq) return;
    const int t = (int)r / a.hq, head = (int)r - t * a.hq;
    const uintx4 x = __builtin_bit_cast(uintx4, load_chunk(head_row(a.o, t, head), c, nch));
    const uintx4 y = __builtin_bit_cast(uintx4, load_chunk(head_row(a.go, t, head), c, nch));
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s = fmaf(__uint_as_float(x[i] << 16), __uint_as_float(y[i] << 16), s);
        s = fmaf(__uint_as_float(x[i] & 0xffff0000u), __uint_as_float(y[i] & 0xffff0000u), s);
    }
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if (c == 0) {
        const float lse = a.lse[r];
        const int64_t at = ((int64_t)(head / g) * a.total_q + t) * g + head % g;
        f.nlse[at] = lse == kNegInf ? kNegInf : -lse / a.scale;
        f.ndelta[at] = -s;
    }
}

// DB 32-element blocks of the padded head are formed.
template <int DP, int DB>
__global__ __launch_bounds__(256, 2) void attn_dq_kernel(BwdArgs f) {
    constexpr int KT = DQ_KEYS, KS = 2 * DB;
    using L = Loader<DP, KT>;
    extern __shared__ __attribute__((aligned(1024))) char lds_mem[];
    const uint32_t lds = (uint32_t)(uintptr_t)(lds_void *)lds_mem;
    const AttnArgs &a = f.a;
    int u = f.qd.unit(block_index());
    if (u >= f.qd.units) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane >> 5, g = f.g.d, nch = a.d >> 3;
    // chunk of row tiles x sequence x key head x tile of the chunk
    int v = f.p.order.chunk.quot(u);
    const int in = f.p.order.chunk.rem(u, v);
    u = v;
    v = f.hk.quot(u);
    Work w;
    w.kvh = f.hk.rem(u, v);
    u = v;
    v = f.seqs.quot(u);
    const int b = f.seqs.rem(u, v);
    const int rt = f.p.order.tile(v, in);
    if (rt < 0) return;
    w.s = load_seq(a, b);
    w.part = 0;
    w.rows = w.s.n * g;
    w.r0 = rt * 128;
    if (w.s.skip || w.r0 >= w.rows) return;
    if (w.s.bad) {
        for (int r = threadIdx.x; rt == 0 && r < w.rows; r += 256) {
            const int k = f.g.quot(r);
            for (int e = 0; e < a.d; ++e)
                ((uint16_t *)head_row(a.gq, w.s.q0 + k, w.kvh * g + f.g.rem(r, k)))[e] = 0x7fc0;
        }
        return;
    }
    w.pt = tiles_of<KT>(w.s.plen);
    w.t0 = 0;
    w.t1 = w.pt + tiles_of<KT>(suffix_seen(w.s, f.g.quot(upto(w.r0, 128, w.rows) - 1)));
    make_uniform(w);
    if (nch < DP / 8) {
        for (int i = threadIdx.x; i < 2 * 2 * KT * DP / 8; i += 256)
            ((uint4 *)lds_mem)[i] = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
    }
    const int row = w.r0 + 32 * wave + (lane & 31), crow = min(row, w.rows - 1);
    const int tok = f.g.quot(crow), head = w.kvh * g + f.g.rem(crow, tok);
    const int t = w.s.q0 + tok;
    bf16x8 q[KS], go[KS];
    {
        const uint16_t *p = head_row(a.q, t, head), *o = head_row(a.go, t, head);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            q[s] = load_chunk(p, 2 * s + h, nch);
            go[s] = load_chunk(o, 2 * s + h, nch);
        }
    }
    const int64_t at = ((int64_t)w.kvh * a.total_q + w.s.q0) * g + crow;
    const float ndelta = f.ndelta[at];
    const int seen = suffix_seen(w.s, tok);
    const int least = suffix_seen(w.s, f.g.quot(min(w.r0 + 32 * wave, w.rows - 1)));
    const float c = a.scale * kLog2e;
    floatx16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = zero16();

    const float nl = f.nlse[at] * c;
    constexpr int RB = TileRow<DP>::BYTES, NB = KT / 32, FN = 2 * KS + 2 * DB;   // operands of a block
    RowReader<DP> kr;
    ColReader<DP> kc;
    kr.open(lds, lane);
    kc.open(lds, lane);
    L load;
    if (w.t0 < w.t1) {
        load.open(a, w, w.t0 < w.pt);
        load.template issue<0>(a, w, w.t0, lds);
    }
    const auto step = [&](auto stage, int kt) {
        constexpr int AT = decltype(stage)::value * 2 * L::BYTES, NEXT = 2 * L::BYTES - AT;
        tile_barrier();
        if (kt + 1 < w.t1) load.template issue<NEXT>(a, w, kt + 1, lds);
        scalar_loads_done();
        const bool pre = kt < w.pt;
        const int limit = pre ? w.s.plen : seen, lowest = pre ? w.s.plen : least;
        // operands of block b: KS of its keys, KS of its values, 2 DB of its keys transposed
        const auto at = [&](int x) {
            const int b = x / FN, i = x % FN;
            return i < KS       ? kr.read(i, AT + b * 32 * RB)
                   : i < 2 * KS ? kr.read(i - KS, AT + L::BYTES + b * 32 * RB)
                                : kc.read((i - 2 * KS) % DB, AT + (2 * b + (i - 2 * KS) / DB) * 16 * RB);
        };
        bf16x8 f[2][4], p;
        floatx16 z, y;
#pragma unroll
        for (int i = 0; i < 4; ++i) f[0][i] = at(i);
#pragma unroll
        for (int n = 0; n < NB * FN / 4; ++n) {
            if (n + 1 < NB * FN / 4) {
#pragma unroll
                for (int i = 0; i < 4; ++i) f[(n + 1) & 1][i] = at(4 * (n + 1) + i);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int b = (4 * n + i) / FN, x = (4 * n + i) % FN;
                if (x < KS) {
                    z = mfma(f[n & 1][i], q[x], x == 0 ? zero16() : z);
                } else if (x < 2 * KS) {
                    y = mfma(f[n & 1][i], go[x - KS], x == KS ? zero16() : y);
                } else {
                    const int mm = (x - 2 * KS) / DB, d = (x - 2 * KS) % DB;
                    if (x == 2 * KS) {
                        const int j0 = (pre ? kt : kt - w.pt) * KT + 32 * b;
                        if (j0 > lowest - 32) {
#pragma unroll
                            for (int e = 0; e < 16; ++e) z[e] = j0 + acc_row(e, lane) < limit ? z[e] : kNegInf;
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e) z[e] = fast_exp2(fmaf(z[e], c, nl)) * (y[e] + ndelta);
                    }
                    if (d == 0) p = pack8(z, mm);
                    acc[d] = mfma(f[n & 1][i], p, acc[d]);
                }
            }
        }
    };
    for (int kt = w.t0; kt < w.t1; kt += 2) {
        step(Const<0>{}, kt);
        if (kt + 1 < w.t1) step(Const<1>{}, kt + 1);
    }
    if (row >= w.rows) return;
    uint16_t *o = (uint16_t *)head_row(a.gq, t, head);
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = 32 * d + 8 * i + 4 * h;
            if (e < a.d) {
                uint2 v;
                v.x = pack_bf16x2(acc[d][4 * i] * a.scale, acc[d][4 * i + 1] * a.scale);
                v.y = pack_bf16x2(acc[d][4 * i + 2] * a.scale, acc[d][4 * i + 3] * a.scale);
                *(uint2 *)(o + e) = v;
            }
        }
}

// The keys of one workgroup of the dkv pass and the query rows that they meet.
struct KeyWork {
    bool prefix;
    int keys, j0;                    // keys of the prefix or suffix, the first of this tile
    int64_t krow;                    // row of its first key
    int q0, rows;                    // the rows begin at token q0
    int first;                       // suffix keys that query 0 sees, less one
    int kvh, part, parts;
    int tile;                        // index of the tile among all of its kind (fp32 parts)
    bool nan;                        // a sequence that has these keys is out of range: no rows, the sums are NaN
};

// v: tile x owner x key head x part (tiles of one owner and head first: they read the same rows)
__device__ __forceinline__ bool find_keys(const BwdArgs &f, bool prefix, int v, KeyWork &w) {
    const AttnArgs &a = f.a;
    w.prefix = prefix;
    const Div &tiles = prefix ? f.ptiles : f.stiles, &owners = prefix ? f.groups : f.seqs;
    w.parts = prefix ? f.p.np : f.p.ns;
    w.part = (prefix ? f.pall : f.sall).quot(v);
    w.tile = (prefix ? f.pall : f.sall).rem(v, w.part);
    const int x = tiles.quot(w.tile);
    w.j0 = tiles.rem(w.tile, x) * KEYS;
    w.kvh = owners.quot(x);
    const int own = owners.rem(x, w.kvh), g = f.g.d;
    w.first = 0;
    if (w.prefix) {
        int q0, q1;
        w.nan = !group_in_order(a, a.group_seqs[own], a.group_seqs[own + 1], q0, q1);
        if (!prefix_ok(a, own)) return false;
        w.keys = a.prefix_len[own];
        w.krow = a.prefix_start[own];
        w.q0 = q0;
        w.rows = w.nan ? 0 : (q1 - q0) * g;
    } else {
        const SeqView s = load_seq(a, own);
        w.nan = s.skip || s.bad;
        w.keys = s.keys;
        w.krow = s.sstart;
        w.q0 = s.q0;
        w.rows = w.nan ? 0 : s.n * g;
        w.first = s.slen - s.n;
    }
    w.keys = uniform32(w.keys);
    w.j0 = uniform32(w.j0);
    w.krow = uniform64(w.krow);
    w.q0 = uniform32(w.q0);
    w.rows = uniform32(w.rows);
    w.first = uniform32(w.first);
    return w.j0 < w.keys;
}

// The v of find_keys that is the u-th to run: chunk of tiles x part x owner x key head x tile of
// the chunk. The first keys meet the most rows under a causal mask; -1: there is none.
__device__ __forceinline__ int key_unit(const BwdArgs &f, const RowOrder &order, const Div &owners, const Div &parts,
                                        const Div &all, int u) {
    int v = order.chunk.quot(u);
    const int in = order.chunk.rem(u, v);
    u = v;
    v = f.hk.quot(u);
    const int kvh = f.hk.rem(u, v);
    u = v;
    v = owners.quot(u);
    const int own = owners.rem(u, v);
    u = v;
    v = parts.quot(u);
    const int part = parts.rem(u, v), t = v * (int)order.chunk.d + in;
    if (t >= order.tiles) return -1;
    return part * (int)all.d + (kvh * (int)owners.d + own) * order.tiles + t;
}

// Tiles of ROWS query rows and their output gradients on their way into LDS, with the rows'
// statistics: rows past the end are copies of the last one.
template <int DP>
struct RowLoader {
    using R = TileRow<DP>;
    static constexpr int N = ROWS / 4 / R::PER_DMA;
    static constexpr int BYTES = ROWS * R::BYTES;
    static constexpr int STAGE = 2 * BYTES + 1024;
    int g, step_t, step_r;           // heads of a group; ROWS / g and ROWS % g
    float inv_g;
    int tok, rem;                    // token of the tile's first row, and its head in the group
    int left;                        // rows from the tile's first to the end

    __device__ __forceinline__ void open(const BwdArgs &f, const KeyWork &w, int r0) {
        g = f.g.d;
        step_t = f.g.quot(ROWS);
        step_r = f.g.rem(ROWS, step_t);
        inv_g = 1.f / (float)g;
        const int k = f.g.quot(r0);
        tok = w.q0 + k;
        rem = f.g.rem(r0, k);
        left = w.rows - r0;
    }
    // (each call takes the next tile)
    __device__ __forceinline__ void issue(const BwdArgs &f, const KeyWork &w, uint32_t lds) {
        const AttnArgs &a = f.a;
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int nch = a.d / 8;
        const int last = min(left, ROWS) - 1;
        const char *qb = a.q.p + (tok * a.q.st + (int64_t)w.kvh * g * a.q.sh) * 2;
        const char *gb = a.go.p + (tok * a.go.st + (int64_t)w.kvh * g * a.go.sh) * 2;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int r = wave * (ROWS / 4) + n * R::PER_DMA + lane / R::CHUNKS;
            const int x = rem + min(r, last);
            // x / g: at most 4096 + 32, where this product is exact below the half
            const int t = (int)(((float)x + 0.5f) * inv_g), j = x - t * g;
            const int ch = (lane & (R::CHUNKS - 1)) ^ R::swz(r);
            const uint32_t to = lds + (wave * (ROWS / 4) + n * R::PER_DMA) * R::BYTES;
            // the launcher takes strides for which these offsets fit 32 bits
            if (ch < nch) {
                dma16_from<0>(qb, (t * (uint32_t)a.q.st + j * (uint32_t)a.q.sh) * 2 + ch * 16, to);
                dma16_from<BYTES>(gb, (t * (uint32_t)a.go.st + j * (uint32_t)a.go.sh) * 2 + ch * 16, to);
            }
        }
        if (wave == 0) {
            const int64_t at = ((int64_t)w.kvh * a.total_q + tok) * g + rem + min(lane & 31, last);
            dma4((const char *)((lane < 32 ? f.nlse : f.ndelta) + at), lds + 2 * BYTES);
        }
        tok += step_t;
        rem += step_r;
        if (rem >= g) {
            rem -= g;
            ++tok;
        }
        left -= ROWS;
    }
};

template <int DP, int DB>
__global__ __launch_bounds__(256, 2) void attn_dkv_kernel(BwdArgs f) {
    constexpr int KS = 2 * DB;
    using L = RowLoader<DP>;
    extern __shared__ __attribute__((aligned(1024))) char lds_mem[];
    const uint32_t lds = (uint32_t)(uintptr_t)(lds_void *)lds_mem;
    const AttnArgs &a = f.a;
    KeyWork w;
    const int block = block_index();
    const bool pre = block < f.pd.blocks;
    int u = pre ? f.pd.unit(block) : f.sd.unit(block - f.pd.blocks);
    if (u >= (pre ? f.pd.units : f.sd.units)) return;
    u = pre ? key_unit(f, f.p.porder, f.groups, f.np, f.pall, u) : key_unit(f, f.p.sorder, f.seqs, f.ns, f.sall, u);
    if (u < 0 || !find_keys(f, pre, u, w)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane >> 5, g = f.g.d, nch = a.d >> 3;
    if (nch < DP / 8) {
        for (int i = threadIdx.x; i < 2 * L::STAGE / 16; i += 256)
            ((uint4 *)lds_mem)[i] = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
    }
    const int key = w.j0 + 32 * wave + (lane & 31);
    const int64_t krow = w.krow + min(key, w.keys - 1);
    constexpr int RB = TileRow<DP>::BYTES;
    RowReader<DP> rr;
    ColReader<DP> rc;
    rr.open(lds, lane);
    rc.open(lds, lane);
    // the wavefront's keys in LDS, their values in registers
    const int kl = 2 * L::STAGE + wave * 32 * RB;
    bf16x8 v[KS];
    {
        const uint16_t *kp = head_row(pick(w.prefix, a.kp, a.ks), krow, w.kvh);
        const uint16_t *vp = head_row(pick(w.prefix, a.vp, a.vs), krow, w.kvh);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            rr.write(s, kl, load_chunk(kp, 2 * s + h, nch));
            v[s] = load_chunk(vp, 2 * s + h, nch);
        }
    }
    const float c = a.scale * kLog2e;
    floatx16 dk[DB], dv[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) dk[d] = dv[d] = w.nan ? (floatx16)(__builtin_nanf("")) : zero16();
    // this part's tiles of the rows from the first that sees the tile's first key
    // (64 bits: max_suffix keys by g rows)
    const auto row_of = [&](int j) { return w.prefix ? 0 : (int)min((int64_t)w.rows, (int64_t)max(0, j - w.first) * g); };
    int r0 = row_of(w.j0) / ROWS * ROWS, i0, i1;
    part_range(tiles_of<ROWS>(w.rows - r0), w.prefix ? f.np : f.ns, w.part, i0, i1);
    r0 += i0 * ROWS;
    // the first rows that see this lane's key, and this wavefront's last and first one
    // (of the keys that are there: past them the difference may pass 32 bits)
    const int from = row_of(key), from_hi = row_of(min(w.j0 + 32 * wave + 31, w.keys - 1)), from_lo = row_of(w.j0 + 32 * wave);
    L load;
    if (i0 < i1) {
        load.open(f, w, r0);
        load.issue(f, w, lds);
    }
    const auto step = [&](auto stage, int i) {
        constexpr int AT = decltype(stage)::value * L::STAGE, NEXT = L::STAGE - AT;
        tile_barrier();
        if (i + 1 < i1) load.issue(f, w, lds + NEXT);
        const int row0 = r0;
        r0 = (int)((uint32_t)r0 + ROWS);
        scalar_loads_done();
        if (row0 <= from_lo - ROWS) return;                   // no row of the tile sees this wavefront's keys
        floatx16 p, y;
        // lane's registers are rows 8 j + 4 h + 0..3 of the tile
        const uint32_t sb = lds + AT + 2 * L::BYTES + 16 * h;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const floatx4 x = OLIVE_LDS(floatx4, sb + 32 * j);
            p[4 * j] = x[0], p[4 * j + 1] = x[1], p[4 * j + 2] = x[2], p[4 * j + 3] = x[3];
        }
        bf16x8 fa[2][2], fb[2][2], fr[2][2];
#pragma unroll
        for (int x = 0; x < 2; ++x) fa[0][x] = rr.read(x, AT), fb[0][x] = rr.read(x, kl);
#pragma unroll
        for (int n = 0; n < KS / 2; ++n) {
            if (n + 1 < KS / 2) {
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    fa[(n + 1) & 1][x] = rr.read(2 * n + 2 + x, AT), fb[(n + 1) & 1][x] = rr.read(2 * n + 2 + x, kl);
            } else {
#pragma unroll
                for (int x = 0; x < 2; ++x) fr[0][x] = rr.read(x, AT + L::BYTES);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const floatx4 x = OLIVE_LDS(floatx4, sb + 128 + 32 * j);
                    y[4 * j] = x[0], y[4 * j + 1] = x[1], y[4 * j + 2] = x[2], y[4 * j + 3] = x[3];
                }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) p = mfma(fa[n & 1][x], fb[n & 1][x], p);
        }
        if (row0 > w.rows - ROWS || row0 < from_hi) {
            const int lo = max(0, from - row0), hi = w.rows - row0;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int r = acc_row(e, lane);
                p[e] = r >= lo && r < hi ? p[e] : kNegInf;
            }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) p[e] = fast_exp2(p[e] * c);
        // KS output gradients, 2 DB of them transposed, 2 DB query rows transposed
        constexpr int FN = KS + 4 * DB;
        const auto at = [&](int x) {
            const int i = x - KS;
            return x < KS        ? rr.read(x, AT + L::BYTES)
                   : i < 2 * DB ? rc.read(i % DB, AT + L::BYTES + i / DB * 16 * RB)
                                : rc.read(i % DB, AT + (i / DB - 2) * 16 * RB);
        };
        bf16x8 o;
#pragma unroll
        for (int n = 0; n < FN / 2; ++n) {
            if (n + 1 < FN / 2) {
#pragma unroll
                for (int x = 0; x < 2; ++x) fr[(n + 1) & 1][x] = at(2 * n + 2 + x);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int x = 2 * n + j, d = (x - KS) % DB, mm = (x - KS) / DB;
                if (x < KS) {
                    y = mfma(fr[n & 1][j], v[x < KS ? x : 0], y);
                } else if (mm < 2) {
                    if (d == 0) o = pack8(p, mm);
                    dv[d] = mfma(fr[n & 1][j], o, dv[d]);
                } else {
                    if (x == KS + 2 * DB) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) y[e] *= p[e];
                    }
                    if (d == 0) o = pack8(y, mm - 2);
                    dk[d] = mfma(fr[n & 1][j], o, dk[d]);
                }
            }
        }
    };
    for (int i = i0; i < i1; i += 2) {
        step(Const<0>{}, i);
        if (i + 1 < i1) step(Const<1>{}, i + 1);
    }
    if (key >= w.keys) return;
    if (w.parts == 1) {
        uint16_t *ko = (uint16_t *)head_row(pick(w.prefix, a.gkp, a.gks), krow, w.kvh);
        uint16_t *vo = (uint16_t *)head_row(pick(w.prefix, a.gvp, a.gvs), krow, w.kvh);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = 32 * d + 8 * i + 4 * h;
                if (e >= a.d) continue;
                uint2 x;
                x.x = pack_bf16x2(dk[d][4 * i] * a.scale, dk[d][4 * i + 1] * a.scale);
                x.y = pack_bf16x2(dk[d][4 * i + 2] * a.scale, dk[d][4 * i + 3] * a.scale);
                *(uint2 *)(ko + e) = x;
                x.x = pack_bf16x2(dv[d][4 * i], dv[d][4 * i + 1]);
                x.y = pack_bf16x2(dv[d][4 * i + 2], dv[d][4 * i + 3]);
                *(uint2 *)(vo + e) = x;
            }
        return;
    }
    // [part][tile][key][dk, dv][d], after the prefix's where both have parts
    const int64_t tiles = w.prefix ? f.pall.d : f.sall.d;
    const int64_t before = w.prefix || f.p.np == 1 ? 0 : f.p.p_units * KEYS * 2 * a.d;
    float *o = f.part + before + (((int64_t)w.part * tiles + w.tile) * KEYS + (key - w.j0)) * 2 * a.d;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = 32 * d + 8 * i + 4 * h;
            if (e >= a.d) continue;
            *(float4 *)(o + e) = make_float4(dk[d][4 * i] * a.scale, dk[d][4 * i + 1] * a.scale,
                                             dk[d][4 * i + 2] * a.scale, dk[d][4 * i + 3] * a.scale);
            *(float4 *)(o + a.d + e) = make_float4(dv[d][4 * i], dv[d][4 * i + 1], dv[d][4 * i + 2], dv[d][4 * i + 3]);
        }
}

// Adds the parts of a tile's gradients: a workgroup a tile.
__global__ __launch_bounds__(256) void attn_dkv_join_kernel(BwdArgs f, int first) {
    const AttnArgs &a = f.a;
    const int pt = (int)(f.p.p_units ? f.pall.d : 0);
    const int i = first + blockIdx.x;              // tiles of the prefixes, then of the suffixes
    KeyWork w;
    if (!find_keys(f, i < pt, i < pt ? i : i - pt, w) || w.parts == 1) return;
    const int64_t tiles = w.prefix ? f.pall.d : f.sall.d;
    const int64_t before = w.prefix || f.p.np == 1 ? 0 : f.p.p_units * KEYS * 2 * a.d;
    const int quads = a.d / 4;
    const int n = min(KEYS, w.keys - w.j0) * 2 * quads;
    for (int x = threadIdx.x; x < n; x += 256) {
        const int e = 4 * (x % quads), kv = x / quads & 1, key = x / (2 * quads);
        const float *p = f.part + before + ((int64_t)w.tile * KEYS + key) * 2 * a.d + kv * a.d + e;
        float4 s = *(const float4 *)p;
        for (int k = 1; k < w.parts; ++k) {
            const float4 y = *(const float4 *)(p + (int64_t)k * tiles * KEYS * 2 * a.d);
            s.x += y.x, s.y += y.y, s.z += y.z, s.w += y.w;
        }
        const HeadsArg o = pick(kv, pick(w.prefix, a.gvp, a.gvs), pick(w.prefix, a.gkp, a.gks));
        uint2 v;
        v.x = pack_bf16x2(s.x, s.y);
        v.y = pack_bf16x2(s.z, s.w);
        *(uint2 *)((uint16_t *)head_row(o, w.krow + w.j0 + key, w.kvh) + e) = v;
    }
}

template <int DP, int DB>
hipError_t go(const BwdArgs &f, hipStream_t st) {
    const AttnArgs &a = f.a;
    const BwdPlan &p = f.p;
    hipError_t e = hipSuccess;
    if (a.total_q > 0) {
        attn_stats_kernel<DP><<<grid_of(ceil_div((int64_t)a.total_q * a.hq, 256 / (DP / 8))), 256, 0, st>>>(f);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        attn_dq_kernel<DP, DB><<<grid_of(f.qd.blocks), 256, 2 * 2 * DQ_KEYS * DP * 2, st>>>(f);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (p.p_units + p.s_units == 0) return e;
    attn_dkv_kernel<DP, DB><<<grid_of((int64_t)f.pd.blocks + f.sd.blocks), 256,
                              2 * RowLoader<DP>::STAGE + KEYS * DP * 2, st>>>(f);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    // (of a kind that has parts there are at most two tiles a compute unit)
    const int64_t pt = p.p_units / p.np, stl = p.s_units / p.ns;
    const int64_t first = p.np > 1 ? 0 : pt, end = p.ns > 1 ? pt + stl : pt;
    if (end > first) attn_dkv_join_kernel<<<(unsigned)(end - first), 256, 0, st>>>(f, (int)first);
    return hipGetLastError();
}

}  // namespace

// A bound that grows with total_q, the heads and their size alone: parts of the rows are made
// where the key tiles times the parts are at most two a compute unit.
int64_t attn_backward_bytes(const AttnArgs &a, bool bf16) {
    const int64_t rows = (int64_t)a.total_q * a.hq;
    if (!attn_mfma_sizes(a, bf16) || a.d > 128) return rows * (int64_t)sizeof(float);   // (the generic kernels' delta)
    return (rows * 2 * (int64_t)sizeof(float) + 15) / 16 * 16 +
           (int64_t)2 * 2 * kChipUnits * KEYS * 2 * a.d * (int64_t)sizeof(float);
}

hipError_t launch_attn_backward(const AttnArgs &a, bool bf16, hipStream_t st) {
    if (a.d > 128 || !attn_mfma_applies(a, bf16)) return launch_attn_generic_backward(a, bf16, st);
    BwdArgs f{};
    f.a = a;
    f.p = make_plan(a);
    f.qd = DieOrder::of(f.p.q_units);
    f.pd = DieOrder::of(a.groups * f.p.porder.units() * a.hk * f.p.np);
    f.sd = DieOrder::of(a.seqs * f.p.sorder.units() * a.hk * f.p.ns);
    const auto div = [](int64_t d) { return Div::of(d > 0 ? d : 1); };
    f.g = div(a.hq / a.hk);
    f.seqs = div(a.seqs);
    f.groups = div(a.groups);
    f.hk = div(a.hk);
    f.ptiles = div(f.p.ptiles);
    f.stiles = div(f.p.stiles);
    f.np = div(f.p.np);
    f.ns = div(f.p.ns);
    f.pall = div(f.p.p_units / f.p.np);
    f.sall = div(f.p.s_units / f.p.ns);
    f.nlse = (float *)a.work;
    f.ndelta = f.nlse + (int64_t)a.total_q * a.hq;
    f.part = (float *)(a.work + ((int64_t)a.total_q * a.hq * 2 * (int64_t)sizeof(float) + 15) / 16 * 16);
    if (a.d <= 32) return go<64, 1>(f, st);
    if (a.d <= 64) return go<64, 2>(f, st);
    return a.d <= 96 ? go<128, 3>(f, st) : go<128, 4>(f, st);
}

}  // namespace olive
