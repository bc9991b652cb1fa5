// Attention on shared prefixes, bf16 on matrix instructions (head_dim a multiple of 8, rows on
// 16 bytes).
//
// A workgroup of 4 wavefronts takes 32 WR query rows of one key head (a row is one query head
// of one token) and a range of key tiles. The product is formed as z^T = K q^T, so that a lane
// holds one query row's scores: the running maximum and sum are the lane's own, and the
// exponentials, rounded to bf16, are the second operand of out^T = V^T p^T as they lie. V^T
// comes out of LDS through the transposing read. With WR = 4 the wavefronts share every key;
// with WR = 2 or 1 they take different keys of a tile (WK = 4 / WR of them a row) and join
// their maxima, sums and outputs at the end: few rows are bound by the loads of the keys, and
// all four wavefronts have to have loads in flight.
//
// Two ways to cut a call:
//   own     rows of one sequence, its prefix and then its suffix in one pass; split along the
//           keys where there are too few row tiles to fill the chip
//   shared  (single tokens, short runs) the rows of all sequences of a group against the
//           prefix, so that it is read once for 32 WR of them, and each sequence's rows
//           against its suffix
// Parts of a row meet in a second kernel through fp32 partial outputs.
//
// The weights are rounded to bf16 as operands because fp32 products run at an eighth of the rate
// (153 against 1200 TFLOP/s in large ones); their sum is formed of the unrounded ones. With it an
// output is 0.0020 to 0.0024 (2-norm) from the exact one, with its own rounding alone 0.0017.
//
// Single tokens are bound by the reading of the keys and values (64 sequences on 4 prefixes of
// 16000 to 32768 tokens, 32 / 8 heads of 128: 125 us and 6 us for the join, 4.3 TB/s; 4 sequences on one of
// 4096, 16 heads: 13 us and 5 us for the join, chains of waits). Long runs are bound by the
// products and the exponentials beside them (8 runs of 1024 tokens on 2 prefixes of 4096, 16 / 8
// heads of 128: 337 us, 920 TFLOP/s; prompts of 1200 to 6000 tokens with heads of 64, where a
// score has half the products: 250 us, 770 TFLOP/s). Kernel times of a trace, clocks settled.
#include "attn_tile.hpp"

namespace olive {
namespace {

constexpr float kRescale = 8.f;      // the running maximum may lag by 2^8 (see below)

// How a call is cut: a function of the descriptor alone (the workspace goes by it).
struct FwdPlan {
    bool shared;
    int wr;                          // 32-row blocks of a workgroup
    int np, ns;                      // parts along the prefix and the suffix (own: np = 0, and
                                     // ns along both)
    int ptiles, stiles;              // row tiles: over all groups (a bound), of a sequence
    RowOrder order;                  // of a sequence's row tiles
    int64_t p_units, s_units;        // workgroups
    __host__ __device__ int parts() const { return np + ns; }
    __host__ __device__ bool direct() const { return !shared && ns == 1; }
};

__host__ __device__ constexpr int tile_keys(int dp, int wr) {
    return wr == 4 ? (dp == 256 ? 32 : 64) : wr == 2 ? 64 : 128;
}

// Rows of partial outputs that the workspace holds for the parts along one axis. They grow with
// the rows alone, so that the workspace of the largest call serves the others: along an axis
// there are at most 64 parts, and at most places / (row tiles) + 1 of them, whose rows together
// are at most places row tiles and the rows once more.
int64_t kept_rows(const AttnArgs &a) {
    const int64_t rows = (int64_t)a.total_q * a.hq, some = 64 * rows, many = 2 * kChipUnits * 128 + rows;
    return some < many ? some : many;
}

FwdPlan make_plan(const AttnArgs &a) {
    FwdPlan p{};
    const int64_t g = a.hq / a.hk, dp = padded(a.d);
    const int64_t seq_rows = a.max_q * g;
    // rows of a group, if the groups are alike
    const int64_t group_rows = ceil_div(a.total_q * g, a.groups);
    // Up to two tiles of rows a sequence, the group's rows fill the tiles better than each
    // sequence's own: runs of up to 97 tokens of 3 heads 34 us for 43, of up to 128 tokens of 4
    // heads 82 us for 105.
    p.shared = a.max_prefix > 0 && a.seqs > a.groups && a.total_q * g <= 256 * (int64_t)a.seqs;
    const auto pick = [&](int64_t rows) { return rows <= 32 && dp < 256 ? 1 : rows <= 64 ? 2 : 4; };
    // (with a block of rows a sequence or less, four blocks would leave the suffixes to one
    // wavefront of each workgroup: 64 single tokens on one prefix of 8192 80 us, with two 74)
    p.wr = pick(!p.shared ? seq_rows : seq_rows <= 32 && group_rows > 64 ? 64 : group_rows);
    const int64_t kt = tile_keys((int)dp, p.wr), bm = 32 * p.wr;
    const int64_t pk = ceil_div(a.max_prefix, kt), sk = ceil_div(a.max_suffix, kt);
    p.stiles = (int)ceil_div(seq_rows, bm);
    // What the workspace holds (attn_forward_bytes) also where more queries come than max_q says.
    const int64_t most = kept_rows(a) / ((int64_t)a.total_q * a.hq);
    // Parts of as many key tiles each as fill the places on the chip (one workgroup a compute
    // unit where it takes over half of the LDS, else two).
    const int64_t places = kChipUnits * ((dp >= 128 && p.wr == 1) || dp == 256 ? 1 : 2);
    const auto parts = [&](int64_t tiles, int64_t len) {
        const int64_t n = len > 0 ? ceil_div(tiles, len) : 1;
        return (int)(n < 1 ? 1 : n < most ? n : most);
    };
    const int64_t s_tiles = (int64_t)a.seqs * p.stiles * a.hk;
    p.order = RowOrder::of(p.stiles);
    const int64_t s_all = a.seqs * p.order.units() * a.hk;
    if (p.shared) {
        const int64_t likely = a.groups * ceil_div(group_rows, bm) * a.hk;
        const int64_t len = ceil_div(likely * pk + s_tiles * sk, places);
        p.ptiles = (int)(ceil_div(a.total_q * g, bm) + a.groups - 1);
        p.np = parts(pk, len);
        p.ns = parts(sk, len);
        p.p_units = (int64_t)p.ptiles * a.hk * p.np;
        p.s_units = s_all * p.ns;
    } else {
        const int64_t len = ceil_div(s_tiles * (pk + sk), places);
        p.ns = s_tiles >= places ? 1 : parts(pk + sk, len < 2 ? 2 : len);
        p.s_units = s_all * p.ns;
    }
    return p;
}

struct FwdArgs {
    AttnArgs a;
    FwdPlan p;
    DieOrder pd, sd;
    Div g, hk, seqs, ptiles, np, ns;
    float *po;                       // [part][total_q hq][d]
    float2 *pml;                     // [part][total_q hq]: maximum (log2 units), sum
};

// The row tile of flat index i over the groups: groups of 64 a step, by prefix sums. A group's
// first token, rows, and prefix go into w; false: no such tile. Where cu_q is not in order, a group
// has the rows that no earlier one has: the tiles of all are then no more than the plan's.
template <int BM>
__device__ __forceinline__ bool find_group(const AttnArgs &a, int g_heads, int i, Work &w) {
    const int lane = threadIdx.x & 63;
    int end = 0;                                     // of the groups before these 64
    bool broken = false;
    for (int g0 = 0; g0 < a.groups; g0 += 64) {
        const int g = g0 + lane;
        int q0 = end, q1 = end, plen = 0;
        int64_t pstart = 0;
        bool ordered = true;
        if (g < a.groups) {
            const bool ok = prefix_ok(a, g);
            plen = ok ? a.prefix_len[g] : 0;
            pstart = a.prefix_start[g];
            ordered = group_tokens(a, a.group_seqs[g], a.group_seqs[g + 1], q0, q1);
        }
        // (a group begins at the entry that the one before it ends at)
        broken |= __any(!ordered);
        if (broken) {
            int most = ordered ? q1 : 0;
            for (int o = 1; o < 64; o <<= 1) {
                const int v = __shfl_up(most, o);
                if (lane >= o) most = max(most, v);
            }
            const int m = __shfl_up(most, 1);
            q0 = max(q0, max(end, lane ? m : 0));
            q1 = ordered ? max(q0, q1) : q0;
            most = max(end, most);
            end = __builtin_amdgcn_readlane(most, 63);
        } else {
            end = __builtin_amdgcn_readlane(q1, 63);
        }
        const int rows = (q1 - q0) * g_heads, n = tiles_of<BM>(rows);
        int sum = n;
        for (int o = 1; a.groups > 1 && o < 64; o <<= 1) {
            const int v = __shfl_up(sum, o);
            if (lane >= o) sum += v;
        }
        const uint64_t hit = __ballot(i < sum);
        if (hit) {
            const int l = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)hit) - 1);
            w.s.q0 = __builtin_amdgcn_readlane(q0, l);
            w.rows = __builtin_amdgcn_readlane(rows, l);
            w.s.plen = __builtin_amdgcn_readlane(plen, l);
            w.s.pstart = (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(pstart >> 32), l) << 32) |
                                   (uint32_t)__builtin_amdgcn_readlane((int)pstart, l));
            w.r0 = (i - __builtin_amdgcn_readlane(sum - n, l)) * BM;
            return true;
        }
        i -= __builtin_amdgcn_readlane(sum, 63);
    }
    return false;
}

// A part without tiles is written too: the second kernel reads every part of a row.
template <int DP, int WR>
__device__ __forceinline__ bool find_work(const FwdArgs &f, int block, Work &w) {
    const AttnArgs &a = f.a;
    constexpr int BM = 32 * WR, KT = tile_keys(DP, WR);
    if (block < f.pd.blocks) {
        const int u = f.pd.unit(block);
        if (u >= f.pd.units) return false;
        const int v = f.ptiles.quot(u), i = f.ptiles.rem(u, v);
        w.part = f.hk.quot(v);
        w.kvh = f.hk.rem(v, w.part);
        w.s = SeqView{};
        if (!find_group<BM>(a, f.g.d, i, w)) return false;
        w.pt = tiles_of<KT>(w.s.plen);
        part_range(w.pt, f.np, w.part, w.t0, w.t1);
        return true;
    }
    int u = f.sd.unit(block - f.pd.blocks);
    if (u >= f.sd.units) return false;
    // chunk of row tiles x part x sequence x key head x tile of the chunk (the heads inside, so
    // that what lies side by side on the dies takes equally long)
    int v = f.p.order.chunk.quot(u);
    const int in = f.p.order.chunk.rem(u, v);
    u = v;
    v = f.hk.quot(u);
    w.kvh = f.hk.rem(u, v);
    u = v;
    v = f.seqs.quot(u);
    const int b = f.seqs.rem(u, v);
    u = v;
    v = f.ns.quot(u);
    w.part = f.ns.rem(u, v);
    const int rt = f.p.order.tile(v, in);
    if (rt < 0) return false;
    w.r0 = rt * BM;
    w.s = load_seq(a, b);
    w.rows = w.s.n * (int)f.g.d;
    if (w.s.skip || w.r0 >= w.rows) return false;
    // (a sequence that is out of range has no keys: its rows get NaN from the first row tile,
    // which may have rows past max_q to mark)
    if (w.s.bad && w.r0) return false;
    const int st = tiles_of<KT>(suffix_seen(w.s, f.g.quot(upto(w.r0, BM, w.rows) - 1)));
    w.pt = f.p.shared ? 0 : tiles_of<KT>(w.s.plen);
    part_range(w.pt + st, f.ns, w.part, w.t0, w.t1);
    w.part += f.p.np;
    return true;
}

// One pass along the key tiles [w.t0, w.t1): out^T (unscaled), the maximum in log2 units and
// this half's share of the sum, of the query row `lane % 32` of a wavefront. Returns whether a
// page lay outside the cache.
template <int DP, int DB, int WR>
__device__ __forceinline__ bool key_loop(const AttnArgs &a, const Work &w, uint32_t lds, int wk, bool idle, int seen,
                                         int least, const bf16x8 (&q)[2 * DB], floatx16 (&acc)[DB],
                                         float &m, float &l) {
    constexpr int WK = 4 / WR, KT = tile_keys(DP, WR), NB = KT / 32 / WK, KS = 2 * DB;
    using L = Loader<DP, KT>;
    const int lane = threadIdx.x & 63;
    const float c = a.scale * kLog2e;
    constexpr int RB = TileRow<DP>::BYTES, KN = NB * KS, VN = NB * 2 * DB;
    constexpr int GS = KN % 4 ? 2 : 4;               // operands that are read ahead together
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = zero16();
    m = kNegInf;
    l = 0.f;
    RowReader<DP> kr;
    ColReader<DP> vr;
    kr.open(lds + wk * NB * 32 * RB, lane);
    vr.open(lds + L::BYTES + wk * NB * 32 * RB, lane);
    L load;
    if (w.t0 < w.t1) {
        load.open(a, w, w.t0 < w.pt);
        load.look_up(a, w, w.t0);
        load.template issue<0>(a, w, w.t0, lds);
        load.look_up(a, w, w.t0 + 1);
    }
    const auto step = [&](auto stage, int kt) {
        constexpr int AT = decltype(stage)::value * 2 * L::BYTES, NEXT = 2 * L::BYTES - AT;
        tile_barrier();
        if (kt + 1 < w.t1) {
            load.template issue<NEXT>(a, w, kt + 1, lds);
            load.look_up(a, w, kt + 2);
        }
        scalar_loads_done();
        if (idle) return;                            // (it has loaded its share of the tile)
        // operand i of the scores (block i / KS, step i % KS), then of the outputs (16 keys
        // i / DB, elements i % DB)
        bf16x8 f[2][GS];
        const auto k_at = [&](int i) { return kr.read(i % KS, AT + i / KS * 32 * RB); };
        const auto v_at = [&](int i) { return vr.read(i % DB, AT + i / DB * 16 * RB); };
        floatx16 z[NB];
#pragma unroll
        for (int i = 0; i < GS; ++i) f[0][i] = k_at(i);
#pragma unroll
        for (int n = 0; n < KN / GS; ++n) {
#pragma unroll
            for (int i = 0; i < GS; ++i)
                f[(n + 1) & 1][i] = GS * (n + 1) < KN ? k_at(GS * (n + 1) + i) : v_at(i);
#pragma unroll
            for (int i = 0; i < GS; ++i) {
                const int x = GS * n + i, b = x / KS, s = x % KS;
                z[b] = mfma(f[n & 1][i], q[s], s == 0 ? zero16() : z[b]);
            }
        }
        // masks: the end of the prefix, and the suffix keys that a row does not see
        const bool pre = kt < w.pt;
        const int j0 = (pre ? kt : kt - w.pt) * KT + wk * NB * 32;
        const int limit = pre ? w.s.plen : seen;
        const bool masked = j0 > (pre ? w.s.plen : least) - NB * 32;
        if (masked) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    z[b][i] = j0 + 32 * b + acc_row(i, lane) < limit ? z[b][i] : kNegInf;
        }
        float top = kNegInf;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, z[b][i]);
        top = max_of_halves(top) * c;
        // The maximum that the weights refer to follows the running one only when it falls
        // more than 2^8 behind: fp32 sums have the room, and the outputs are seldom rescaled.
        if (__any(top > m + kRescale)) {
            const float m2 = fmaxf(m, top);
            const float r = m2 == m ? 1.f : fast_exp2(m - m2);
            m = m2;
            l *= r;
#pragma unroll
            for (int d = 0; d < DB; ++d) acc[d] *= r;
        }
        const float m0 = m == kNegInf ? 0.f : m;
        bf16x8 p;
#pragma unroll
        for (int n = 0; n < VN / GS; ++n) {
            constexpr int V0 = KN / GS;               // where the values' first group lies in f
            if (n + 1 < VN / GS) {
#pragma unroll
                for (int i = 0; i < GS; ++i) f[(V0 + n + 1) & 1][i] = v_at(GS * (n + 1) + i);
            }
#pragma unroll
            for (int i = 0; i < GS; ++i) {
                const int x = GS * n + i, d = x % DB, b = x / DB / 2, mm = x / DB % 2;
                if (d == 0) {
                    // the weights of the next 16 keys
                    float sum = 0.f;
#pragma unroll
                    for (int e = 8 * mm; e < 8 * mm + 8; ++e) {
                        z[b][e] = fast_exp2(fmaf(z[b][e], c, -m0));
                        sum += z[b][e];
                    }
                    l += sum;
                    p = pack8(z[b], mm);
                }
                acc[d] = mfma(f[(V0 + n) & 1][i], p, acc[d]);
            }
        }
    };
    for (int kt = w.t0; kt < w.t1; kt += 2) {
        step(Const<0>{}, kt);
        if (kt + 1 < w.t1) step(Const<1>{}, kt + 1);
    }
    return load.bad;
}

// A value that is not finite makes a NaN of the product also in rows that do not see its key
// (their weight of it is 0). Where a unit's result is not finite and such a value lies among
// the keys that not all its rows see, its rows are formed again one by one, each over the keys
// that it sees. False: there is none.
template <int KT>
__device__ __forceinline__ bool row_by_row(const FwdArgs &f, const Work &w, int bm, bool alone) {
    const AttnArgs &a = f.a;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (w.t0 >= w.t1) return false;
    bool off_table = false;
    const auto key_row = [&](bool pre, int j) { return pre ? w.s.pstart + j : suffix_row(a, w.s, j, off_table); };
    {
        bool found = false;
        const auto look = [&](bool pre, int j) {
            const uint16_t *v = head_row(pick(pre, a.vp, a.vs), key_row(pre, j), w.kvh);
            for (int e = lane; e < a.d; e += 64) found |= (v[e] & 0x7f80) == 0x7f80;
        };
        const int s0 = suffix_seen(w.s, f.g.quot(w.r0));
        const int j0 = max(0, min(s0, w.s.slen - 1));
        for (int i = wave; i < w.s.slen - j0; i += 4) look(false, j0 + i);
        if (w.s.plen > 0) look(true, w.s.plen - 1);   // (copies of it stand for keys past the end)
        if (!__syncthreads_or(found)) return false;
    }
    for (int i = wave; i < min(bm, w.rows - w.r0); i += 4) {
        const int row = w.r0 + i, tok = f.g.quot(row), head = w.kvh * (int)f.g.d + f.g.rem(row, tok);
        const int t = w.s.q0 + tok;
        const int seen = suffix_seen(w.s, tok);
        const uint16_t *q = head_row(a.q, t, head);
        float x[4], o[4] = {}, m = kNegInf, l = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = lane + 64 * i < a.d ? load_elem<uint16_t>(q, lane + 64 * i) : 0.f;
        for (int kt = w.t0; kt < w.t1; ++kt) {
            const bool pre = kt < w.pt;
            const int j0 = (pre ? kt : kt - w.pt) * KT, end = upto(j0, KT, pre ? w.s.plen : seen);
            for (int j = j0; j < end; ++j) {
                const int64_t at = key_row(pre, j);
                const uint16_t *k = head_row(pick(pre, a.kp, a.ks), at, w.kvh), *v = head_row(pick(pre, a.vp, a.vs), at, w.kvh);
                float z = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (lane + 64 * i < a.d) z = fmaf(x[i], load_elem<uint16_t>(k, lane + 64 * i), z);
                for (int s = 32; s > 0; s >>= 1) z += __shfl_xor(z, s);
                z *= a.scale * kLog2e;
                const float m2 = fmaxf(m, z), r = m2 == m ? 1.f : fast_exp2(m - m2);
                const float p = z == kNegInf ? 0.f : fast_exp2(z - m2);
                m = m2;
                l = l * r + p;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (lane + 64 * i < a.d) o[i] = fmaf(p, load_elem<uint16_t>(v, lane + 64 * i), o[i] * r);
            }
        }
        if (__any(off_table) || alone) l = __builtin_nanf("");
        const int64_t orow = (int64_t)t * a.hq + head, slot = (int64_t)w.part * a.total_q * a.hq + orow;
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = lane + 64 * i;
            if (e >= a.d) continue;
            if (f.p.direct()) ((uint16_t *)head_row(a.o, t, head))[e] = (uint16_t)pack_bf16x2(o[i] * inv, 0.f);
            else f.po[slot * a.d + e] = o[i];
        }
        if (lane == 0) {
            if (!f.p.direct()) f.pml[slot] = make_float2(m, l);
            else if (a.lse) a.lse[orow] = l == 0.f ? kNegInf : (m + fast_log2(l)) * kLn2;
        }
    }
    return true;
}

// DB 32-element blocks of the padded head are formed.
template <int DP, int DB, int WR>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void attn_fwd_kernel(FwdArgs f) {
    constexpr int WK = 4 / WR, KT = tile_keys(DP, WR), KS = 2 * DB;
    extern __shared__ __attribute__((aligned(1024))) char lds_mem[];
    const uint32_t lds = (uint32_t)(uintptr_t)(lds_void *)lds_mem;
    const AttnArgs &a = f.a;
    Work w;
    const int block = block_index();
    if (!find_work<DP, WR>(f, block, w)) return;
    make_uniform(w);
    // (asked for here, looked at after the keys)
    const bool suffix_rows = f.p.shared && block >= f.pd.blocks;
    const int32_t entry = suffix_rows && !w.s.bad ? group_entry(a, w.s) : 0;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wr = wave / WK, wk = wave % WK, h = lane >> 5;
    const int g = f.g.d, nch = a.d >> 3;
    if (nch < DP / 8) {
        for (int i = threadIdx.x; i < 2 * 2 * KT * DP / 8; i += 256)
            ((uint4 *)lds_mem)[i] = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
    }

    // this lane's query row
    const int row = w.r0 + 32 * wr + (lane & 31), crow = min(row, w.rows - 1);
    const bool live = row < w.rows;
    const int tok = f.g.quot(crow), head = w.kvh * g + f.g.rem(crow, tok);
    const int t = w.s.q0 + tok;
    bf16x8 q[KS];
    {
        const uint16_t *p = head_row(a.q, t, head);
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = load_chunk(p, 2 * s + h, nch);
    }
    // suffix keys it sees, and the fewest that a row of this wavefront sees
    const int seen = suffix_seen(w.s, tok);
    const int least = suffix_seen(w.s, f.g.quot(min(w.r0 + 32 * wr, w.rows - 1)));
    floatx16 acc[DB];
    float m, l;
    const bool off_table = key_loop<DP, DB, WR>(a, w, lds, wk, w.r0 + 32 * wr >= w.rows, seen, least, q, acc, m, l);
    // a sequence whose rows do not lie among its group's: they against the prefix are nobody's work
    const bool alone = suffix_rows && !w.s.bad && __any(!entry_holds(a, w.s, entry));
    {
        float s = 0.f;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) s = fmaf(acc[d][i], 0.f, s);
        if (__syncthreads_or(!(s == 0.f)) && row_by_row<KT>(f, w, 32 * WR, alone)) return;
    }
    l += __shfl_xor(l, 32);

    const int orow = t * a.hq + head;
    const bool bad = __syncthreads_or(off_table) || w.s.bad || alone;
    // the registers (4 consecutive elements of the head each) that this wavefront writes
    int g0 = 0;
    if (WK > 1) {
        // the row's wavefronts leave their parts in LDS and take a share of the elements each
        float2 *ml = (float2 *)(lds_mem + 4 * DB * 4096);
        float4 *po = (float4 *)lds_mem;
        if (h == 0) ml[wave * 32 + lane] = make_float2(m, l);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                po[(wave * DB * 4 + d * 4 + j) * 64 + lane] =
                    make_float4(acc[d][4 * j], acc[d][4 * j + 1], acc[d][4 * j + 2], acc[d][4 * j + 3]);
        __syncthreads();
        float pm[WK], pl[WK], top = kNegInf;
#pragma unroll
        for (int k = 0; k < WK; ++k) {
            const float2 v = ml[(wr * WK + k) * 32 + (lane & 31)];
            pm[k] = v.x;
            pl[k] = v.y;
            top = fmaxf(top, v.x);
        }
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < WK; ++k) {
            pm[k] = pm[k] == top ? 1.f : fast_exp2(pm[k] - top);
            sum += pl[k] * pm[k];
        }
        m = top;
        l = sum;
        g0 = wk * (DB * 4 / WK);
#pragma unroll
        for (int i = 0; i < DB * 4 / WK; ++i) {
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < WK; ++k) {
                const float4 v = po[((wr * WK + k) * DB * 4 + g0 + i) * 64 + lane];
                o.x = fmaf(v.x, pm[k], o.x);
                o.y = fmaf(v.y, pm[k], o.y);
                o.z = fmaf(v.z, pm[k], o.z);
                o.w = fmaf(v.w, pm[k], o.w);
            }
            acc[i / 4][4 * (i % 4)] = o.x;
            acc[i / 4][4 * (i % 4) + 1] = o.y;
            acc[i / 4][4 * (i % 4) + 2] = o.z;
            acc[i / 4][4 * (i % 4) + 3] = o.w;
        }
    }
    if (bad) l = __builtin_nanf("");
    if (w.s.bad) {
        // every row of the sequence, also those past max_q: the outputs, or sums for the second
        // kernel to make them of
        const int64_t part = (int64_t)w.part * a.total_q * a.hq;
        for (int r = threadIdx.x; r < w.rows; r += 256) {
            const int k = f.g.quot(r), tk = w.s.q0 + k, hd = w.kvh * g + f.g.rem(r, k);
            if (!f.p.direct()) {
                f.pml[part + (int64_t)tk * a.hq + hd] = make_float2(0.f, __builtin_nanf(""));
                continue;
            }
            for (int e = 0; e < a.d; ++e) ((uint16_t *)head_row(a.o, tk, hd))[e] = 0x7fc0;
            if (a.lse) a.lse[tk * a.hq + hd] = __builtin_nanf("");
        }
        return;
    }
    if (!live) return;
    const bool first = wk == 0 && h == 0;
    if (f.p.direct()) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        uint16_t *o = (uint16_t *)head_row(a.o, t, head);
#pragma unroll
        for (int i = 0; i < DB * 4 / WK; ++i) {
            const int e = 8 * (g0 + i) + 4 * h;
            if (e < a.d) {
                uint2 v;
                v.x = pack_bf16x2(acc[i / 4][4 * (i % 4)] * inv, acc[i / 4][4 * (i % 4) + 1] * inv);
                v.y = pack_bf16x2(acc[i / 4][4 * (i % 4) + 2] * inv, acc[i / 4][4 * (i % 4) + 3] * inv);
                *(uint2 *)(o + e) = v;
            }
        }
        if (a.lse && first) a.lse[orow] = l == 0.f ? kNegInf : (m + fast_log2(l)) * kLn2;
        return;
    }
    const int64_t slot = (int64_t)w.part * a.total_q * a.hq + orow;
    if (first) f.pml[slot] = make_float2(m, l);
    if (w.t0 == w.t1) return;
#pragma unroll
    for (int i = 0; i < DB * 4 / WK; ++i) {
        const int e = 8 * (g0 + i) + 4 * h;
        if (e < a.d)
            *(float4 *)(f.po + slot * a.d + e) =
                make_float4(acc[i / 4][4 * (i % 4)], acc[i / 4][4 * (i % 4) + 1], acc[i / 4][4 * (i % 4) + 2],
                            acc[i / 4][4 * (i % 4) + 3]);
    }
}

// Joins the parts of each row: a wavefront a row, 4 elements a lane; the lanes left over take
// other parts of the same elements.
__global__ __launch_bounds__(256) void attn_join_kernel(FwdArgs f) {
    const AttnArgs &a = f.a;
    const uint32_t row = (uint32_t)block_index() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= (uint32_t)(a.total_q * a.hq)) return;
    const int r = (int)row, parts = f.p.parts();
    const int lane = threadIdx.x & 63;
    const int64_t step = (int64_t)a.total_q * a.hq;
    // (at most 128 parts)
    float2 x = make_float2(kNegInf, 0.f), y = x;
    if (lane < parts) x = f.pml[lane * step + r];
    if (lane + 64 < parts) y = f.pml[(lane + 64) * step + r];
    const int t = r / a.hq, head = r - t * a.hq;
    if (!any_has_token(a, t)) return;
    float top = fmaxf(x.x, y.x);
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float wx = x.x == top ? 1.f : fast_exp2(x.x - top), wy = y.x == top ? 1.f : fast_exp2(y.x - top);
    float sum = x.y * wx + y.y * wy;
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    const int lpr = a.d <= 64 ? 16 : a.d <= 128 ? 32 : 64, e = 4 * (lane & (lpr - 1)), first = lane / lpr;
    const int every = 64 / lpr;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = first; i < parts + first; i += 4 * every) {
        float4 v[4];
        float w[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const int k = i + n * every;
            // a part that has nothing of the row holds no outputs
            const float l = __shfl(k < 64 ? x.y : y.y, k & 63);
            w[n] = __shfl(k < 64 ? wx : wy, k & 63);
            const bool in = k < parts && e < a.d && !(l == 0.f);
            v[n] = in ? *(const float4 *)(f.po + (k * step + r) * a.d + e) : make_float4(0.f, 0.f, 0.f, 0.f);
            w[n] = in ? w[n] : 0.f;
        }
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            o.x = fmaf(v[n].x, w[n], o.x);
            o.y = fmaf(v[n].y, w[n], o.y);
            o.z = fmaf(v[n].z, w[n], o.z);
            o.w = fmaf(v[n].w, w[n], o.w);
        }
    }
    for (int s = lpr; s < 64; s <<= 1) {
        o.x += __shfl_xor(o.x, s);
        o.y += __shfl_xor(o.y, s);
        o.z += __shfl_xor(o.z, s);
        o.w += __shfl_xor(o.w, s);
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    if (lane < lpr && e < a.d) {
        uint2 v;
        v.x = pack_bf16x2(o.x * inv, o.y * inv);
        v.y = pack_bf16x2(o.z * inv, o.w * inv);
        *(uint2 *)((uint16_t *)head_row(a.o, t, head) + e) = v;
    }
    if (a.lse && lane == 0) a.lse[r] = sum == 0.f ? kNegInf : (top + fast_log2(sum)) * kLn2;
}

template <int DP, int DB, int WR>
hipError_t go(const FwdArgs &f, hipStream_t st) {
    constexpr int KT = tile_keys(DP, WR);
    constexpr int stages = 2 * 2 * KT * DP * 2, join = WR < 4 ? 4 * (DP / 32) * 4096 + 1024 : 0;
    const dim3 grid = grid_of((int64_t)f.pd.blocks + f.sd.blocks);
    attn_fwd_kernel<DP, DB, WR><<<grid, 256, stages > join ? stages : join, st>>>(f);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || f.p.direct()) return e;
    attn_join_kernel<<<grid_of(ceil_div((int64_t)f.a.total_q * f.a.hq, 4)), 256, 0, st>>>(f);
    return hipGetLastError();
}

// Rows on 16 bytes, and the offsets of 128 of them, or of a group's heads, in 32 bits.
bool rows_on_16(const HeadsArg &h, int g) {
    return !h.p || ((((uintptr_t)h.p | (uint64_t)(h.st * 2) | (uint64_t)(h.sh * 2)) & 15) == 0 &&
                    h.st >= 0 && h.st < (1 << 23) && h.sh >= 0 && h.sh < (1 << 29) / g);
}

}  // namespace

bool attn_mfma_sizes(const AttnArgs &a, bool bf16) {
    return bf16 && a.d % 8 == 0 && a.scale > 0.f;
}
bool attn_mfma_applies(const AttnArgs &a, bool bf16) {
    if (!attn_mfma_sizes(a, bf16)) return false;
    for (const HeadsArg *h : {&a.q, &a.kp, &a.vp, &a.ks, &a.vs, &a.o, &a.go, &a.gq, &a.gkp, &a.gvp, &a.gks,
                              &a.gvs})
        if (!rows_on_16(*h, a.hq / a.hk)) return false;
    return true;
}

int64_t attn_forward_bytes(const AttnArgs &a, bool bf16) {
    if (!attn_mfma_sizes(a, bf16)) return 0;
    return 2 * kept_rows(a) * (a.d + 2) * (int64_t)sizeof(float);
}

hipError_t launch_attn_forward(const AttnArgs &a, bool bf16, hipStream_t st) {
    if (!attn_mfma_applies(a, bf16)) return launch_attn_generic(a, bf16, st);
    FwdArgs f{};
    f.a = a;
    f.p = make_plan(a);
    f.pd = DieOrder::of(f.p.p_units);
    f.sd = DieOrder::of(f.p.s_units);
    f.g = Div::of(a.hq / a.hk);
    f.hk = Div::of(a.hk);
    f.seqs = Div::of(a.seqs);
    f.ptiles = Div::of(f.p.ptiles > 0 ? f.p.ptiles : 1);
    f.np = Div::of(f.p.np > 0 ? f.p.np : 1);
    f.ns = Div::of(f.p.ns);
    const int64_t rows = (int64_t)f.p.parts() * a.total_q * a.hq;
    f.po = (float *)a.work;
    f.pml = (float2 *)(f.po + rows * a.d);
    const auto by_rows = [&](auto dp, auto db) {
        constexpr int DP = decltype(dp)::value, DB = decltype(db)::value;
        if (f.p.wr == 4) return go<DP, DB, 4>(f, st);
        if constexpr (DP < 256)
            if (f.p.wr == 1) return go<DP, DB, 1>(f, st);
        return go<DP, DB, 2>(f, st);
    };
    if (a.d <= 32) return by_rows(Const<64>{}, Const<1>{});
    if (a.d <= 64) return by_rows(Const<64>{}, Const<2>{});
    if (a.d <= 96) return by_rows(Const<128>{}, Const<3>{});
    if (a.d <= 128) return by_rows(Const<128>{}, Const<4>{});
    return by_rows(Const<256>{}, Const<8>{});
}

}  // namespace olive
