// The next token of rows of logits: temperature, top-k, top-p, min-p, from given numbers.
//
// What is kept is a run of the tokens in order (value, then index). The order is never formed:
// tokens are counted in bins by value, the bin where the run ends is found from the cumulative
// counts and masses, and only that bin is looked into. The token is then found in the order of
// the vocabulary by halving ranges (128 at a time) by their kept masses.
//
//  - bf16 (`Coarse`): a bin is one value, so a bin's mass is its count times one weight, and no
//    token's own exponential is formed. Long rows are counted in parts by a first kernel (28 KB
//    of 16-bit counts each), a workgroup a row adds them up and does the rest.
//  - fp32, and rows whose values no table of bins holds (`Fine`): bins are 1/32 of a unit of
//    (max - z) / T wide; a token's mass is added to its bin in fixed point, relative to the bin's
//    edge, so that the sum does not depend on its order. Inside the last bin the run's end is
//    found digit by digit of (value, index).
//
// A call of few rows is a chain of waits and of steps that all threads join. Code is kept short where a
// workgroup runs it once (loops over a lane's tokens are rolled): instructions come from the L2 cache
// a line at a time (8 fp32 rows of 32000 with top-k 50: 52 us unrolled, 25 rolled, with the kept ones put in
// order). Of bf16 rows of 151936: 4 without cuts 13 us, 64 with settings of their own 40, 512 with a nucleus
// 90, of which half is the counting (3.6 tokens a clock and compute unit: 21 vector instructions a token, by which
// the SIMDs are busy 95 % of the time; LDS, with its atomics, is 37 %).
//
// Masses are 64-bit: a token changes where the error of the sums passes u times their total over a
// border, and a row has as many borders as tokens.
#include <type_traits>

#include "rows.hpp"
#include "tokens_internal.hpp"
#include "wave_ops.hpp"

namespace olive {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;

// ---------------------------------------------------------------------- bins of bf16 values
// Magnitudes in [2^-40, 2^15) have a bin of their own each, in blocks of 128 (one power of two):
// 55 blocks of positive values, the largest first, a block for zero, 55 of negative ones, and a
// block for what lies below -2^15 (masks of the lowest values), whose bin is counted only.
constexpr int kLow = 87 << 7, kHigh = 142 << 7, kSide = kHigh - kLow;
constexpr int kZeroBin = kSide, kNegative = kZeroBin + 128, kBelow = kNegative + kSide;
constexpr int kBlocks = (kBelow >> 7) + 1, kBins = kBlocks * 128;
static_assert(kBlocks == 112 && kSide % 128 == 0, "");
constexpr int kSlots = 48;                       // blocks of a row that may be in use

enum : int { kSkip = -1, kBad = -2, kOdd = -3 };  // -inf; NaN or +inf; a value without a bin

__device__ __forceinline__ int bin_of(uint32_t bits) {
    const int m = (int)(bits & 0x7fffu), r = m - kLow;
    const bool neg = bits & 0x8000u;
    if ((uint32_t)r < (uint32_t)kSide) return neg ? kNegative + r : kSide - 1 - r;
    if (m == 0) return kZeroBin;
    if (m > 0x7f80 || (m == 0x7f80 && !neg)) return kBad;
    if (m == 0x7f80) return kSkip;
    return neg && m >= kHigh ? kBelow : kOdd;
}
__device__ __forceinline__ float value_of(int bin) {
    const uint32_t bits = bin < kSide ? kLow + kSide - 1 - bin : bin == kZeroBin ? 0u : 0x8000u + kLow + (bin - kNegative);
    return bf16_bits_to_f32(bits);
}

// ------------------------------------------------------------------------------------ parts
// A part of a row: its counts, or of a row that keeps every token its mass alone.
struct PartHead {
    uint64_t blocks[2];                          // blocks that hold counts
    double mass;                                 // relative to the largest value
    float top;
    int32_t n;                                   // tokens that are not -inf
    int32_t flags;                               // bit 0: a bad value, bit 1: one without a bin
    int32_t pad[7];
};
static_assert(sizeof(PartHead) == 64, "");
constexpr int kPartThreads = 512;
constexpr int kMostParts = 64, kMostPart = 65024;            // (16-bit counts)
template <typename T> constexpr int kWhole = kPartThreads * kLot<T> * 4;     // tokens of a part whose mass is formed at once

struct Parts {
    int32_t count, len;
    int32_t bytes;                               // of a part in the workspace
};

// Rows of up to 16384 bf16 tokens are counted by the workgroup that does the rest, in one launch. So are cut ones
// of up to 65024 (what counts of 16 bits hold) in calls of more than 1024 rows, which need no workspace
// then (1100 rows of 65024: 183 us; with two parts 132, and 57 KB a row). Else a call has 2048 parts over its rows
// (16 a row at most, of 4096 tokens at least, and as many as 65024 tokens a part ask for: a part costs the second
// launch its counts, 64 rows of 151936 take the same with 8 and with 16); where every token is kept 1024 parts
// (64 a row at most, of 2048 tokens at least and of kWhole at most). Rows of fp32 that are cut are not
// split (count 0).
Parts parts_of(const SampleArgs &a, bool bf16) {
    const int whole = bf16 ? kWhole<uint16_t> : kWhole<float>;
    // (every row keeps every token, or the first alone)
    const bool plain = !a.top_k && !a.top_p && !a.min_p && a.vocab <= kMostParts * whole;
    if (!bf16 && (!plain || a.vocab <= 4096)) return Parts{0, 0, 0};
    int64_t s = (plain ? 1024 : 2048) / a.rows, least = (a.vocab + kMostPart - 1) / kMostPart;
    if (plain) least = (a.vocab + whole - 1) / whole;
    const int64_t most = plain ? (a.vocab + 2047) / 2048 : (a.vocab + 4095) / 4096;
    if (bf16 && a.vocab <= 16384) s = least = 1;
    if (s > most) s = most;
    if (s > (plain ? kMostParts : 16)) s = plain ? kMostParts : 16;
    if (s < least) s = least;
    const int64_t len = ((a.vocab + s - 1) / s + 511) / 512 * 512;
    return Parts{(int32_t)((a.vocab + len - 1) / len), (int32_t)len, plain ? 64 : kBins * 2 + 64};
}

// A lane's tokens from i on, -inf past `end`.
template <typename T>
__device__ __forceinline__ Lot load_tokens(const T *z, int i, int end) {
    return load_lot(z, i, end, sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u);
}
// The same of WORDS words: 4, or 1 (two bf16 tokens or one of fp32), the first.
template <typename T, int WORDS>
__device__ __forceinline__ Lot load_some(const T *z, int i, int end) {
    if constexpr (WORDS == 4) {
        return load_tokens(z, i, end);
    } else {
        static_assert(WORDS == 1, "");
        Lot x{{sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u}};
        if constexpr (sizeof(T) == 2) {
            struct __attribute__((packed, aligned(2))) Loose { uint32_t w; };
            if (i + 2 <= end) x.w[0] = ((const Loose *)(z + i))->w;
            else if (i < end) x.w[0] = 0xff800000u | z[i];
        } else {
            if (i < end) x.w[0] = __float_as_uint(z[i]);
        }
        return x;
    }
}
// fn(j, bits) for each token j of a lot.
template <typename T, int UNROLL = 1, int WORDS = 4, typename F>
__device__ __forceinline__ void each_token(Lot x, F fn) {
#pragma unroll UNROLL
    for (int k = 0; k < WORDS; ++k) {
        if constexpr (sizeof(T) == 2) {
            fn(2 * k, x.w[0] & 0xffffu);
            fn(2 * k + 1, x.w[0] >> 16);
        } else {
            fn(k, x.w[0]);
        }
        x.w[0] = x.w[1], x.w[1] = x.w[2], x.w[2] = x.w[3];
    }
}
template <typename T>
__device__ __forceinline__ float token_value(uint32_t bits) {
    return sizeof(T) == 2 ? bf16_bits_to_f32(bits) : __uint_as_float(bits);
}

// Counts of [begin, end) of a row into 16-bit bins (two to a word); the flags of its odd values.
// Four lots a thread are on their way together, the first ones while `clear` makes the bins empty.
template <int THREADS, typename Clear>
__device__ __forceinline__ int count_bins(const uint16_t *z, int begin, int end, uint32_t *hist, Clear clear) {
    constexpr int kAhead = 4;
    int flags = 0;
    Lot x[kAhead];
    const int first = begin + (int)threadIdx.x * 8;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) x[k] = load_tokens(z, first + k * THREADS * 8, end);
    clear();
#pragma unroll 1
    for (int i0 = first; i0 < end; i0 += kAhead * THREADS * 8) {
        if (i0 != first) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) x[k] = load_tokens(z, i0 + k * THREADS * 8, end);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (i0 + k * THREADS * 8 >= end) break;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int b = bin_of(j & 1 ? x[k].w[j >> 1] >> 16 : x[k].w[j >> 1] & 0xffffu);
                if (b >= 0) atomicAdd(hist + (b >> 1), 1u << ((b & 1) * 16));
                else flags |= b == kBad ? 1 : b == kOdd ? 2 : 0;
            }
        }
    }
    return flags;
}

// e^x for x <= 0: 2^n e^r with n the nearest whole number to x / ln 2, by the series of e^r (|r| <= ln 2 / 2:
// r^13 / 13! is 2^-52), its even and odd terms side by side. n ln 2 is taken off in two parts, as Cody and Waite
// give it: ln 2 to a multiple of 2^-32, so that its product with n (11 bits) is exact, and what is left of it.
__device__ __forceinline__ double exp_below(double x) {
    x = fmax(x, -1100.0);
    const double n = rint(x * 1.4426950408889634);
    const double r = fma(n, -1.9082149292705877e-10, fma(n, -0.6931471803691238, x)), q = r * r;
    double even = fma(q, 1.0 / 479001600, 1.0 / 3628800), odd = fma(q, 1.0 / 39916800, 1.0 / 362880);
    even = fma(q, even, 1.0 / 40320);
    odd = fma(q, odd, 1.0 / 5040);
    even = fma(q, even, 1.0 / 720);
    odd = fma(q, odd, 1.0 / 120);
    even = fma(q, even, 1.0 / 24);
    odd = fma(q, odd, 1.0 / 6);
    even = fma(q, even, 0.5);
    odd = fma(q, odd, 1.0);
    even = fma(q, even, 1.0);
    return ldexp(fma(r, odd, even), (int)n);
}

struct Settings {
    float u, temp, p, mp;
    int k;
    bool ok, greedy;                             // greedy: the first token alone
};

__device__ __forceinline__ Settings settings_of(const SampleArgs &a, int row) {
    Settings s;
    s.u = a.uniform[row];
    s.temp = a.temperature ? a.temperature[row] : 1.f;
    s.p = a.top_p ? a.top_p[row] : 1.f;
    s.mp = a.min_p ? a.min_p[row] : 0.f;
    s.k = a.top_k ? a.top_k[row] : 0;
    s.ok = s.u >= 0.f && s.u <= 1.f && s.temp >= 0.f && s.temp < __builtin_inff() && s.p == s.p && s.mp == s.mp;
    s.greedy = s.temp == 0.f || s.mp > 1.f || s.k == 1;
    if (s.greedy) s.k = 1, s.p = 1.f, s.mp = 0.f;
    if (s.temp == 0.f) s.temp = 1.f;
    return s;
}

// Of calls without cuts: a part's largest value, and its mass relative to that.
template <typename T>
__global__ __launch_bounds__(kPartThreads) void sample_masses_kernel(SampleArgs a, Parts p) {
    constexpr int kPartWaves = kPartThreads / 64;
    const int64_t row = blockIdx.x;
    const int part = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int begin = part * p.len, end = min(a.vocab, begin + p.len);
    const T *z = (const T *)a.logits.p + row * a.logits.st;
    PartHead *head = (PartHead *)(a.work + (row * p.count + part) * p.bytes);
    const Settings s = settings_of(a, row);
    if (!s.ok) return;
    __shared__ Lot lots[kWhole<T> / kLot<T>];    // (a thread's own)
    const int mine = (end - begin + kPartThreads * kLot<T> - 1) / (kPartThreads * kLot<T>);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < mine) lots[i * kPartThreads + tid] = load_tokens(z, begin + (tid + i * kPartThreads) * kLot<T>, end);
    uint32_t top = 0, bad = 0;
    int n = 0;
#pragma unroll 1
    for (int i = 0; i < mine; ++i)
        each_token<T>(lots[i * kPartThreads + tid], [&](int, uint32_t bits) {
            const float v = token_value<T>(bits);
            bad |= !(v < __builtin_inff());
            n += v > kNegInf;
            top = max(top, f2ord(v));
        });
    __shared__ uint32_t tops[kPartWaves], bads[kPartWaves];
    __shared__ int ns[kPartWaves];
    __shared__ double masses[kPartWaves];
    top = wave_max(top);
    n = wave_sum(n);
    if (lane == 0) tops[wave] = top, ns[wave] = n, bads[wave] = 0;
    if (__ballot(bad) && lane == 0) bads[wave] = 1;
    __syncthreads();
    for (int i = 0; i < kPartWaves; ++i) top = max(top, tops[i]);
    const double first = (double)ord2f(top), inv = 1.0 / (double)s.temp;
    double mass = 0.0;
#pragma unroll 1
    for (int i = 0; i < mine; ++i)
        each_token<T>(lots[i * kPartThreads + tid], [&](int, uint32_t bits) {
            const float v = token_value<T>(bits);
            mass += v > kNegInf ? exp_below(((double)v - first) * inv) : 0.0;
        });
    mass = wave_sum(mass);
    if (lane == 0) masses[wave] = mass;
    __syncthreads();
    if (tid == 0) {
        PartHead h{};
        h.top = (float)first;
        for (int i = 0; i < kPartWaves; ++i) h.mass += masses[i], h.n += ns[i], h.flags |= (int)bads[i];
        *head = h;
    }
}

// Of the others: the counts of a part's bins, and which blocks of them hold any.
__global__ __launch_bounds__(kPartThreads) void sample_counts_kernel(SampleArgs a, Parts p) {
    __shared__ uint32_t hist[kBins / 2];
    __shared__ uint32_t used[4], flags;
    constexpr int kPartWaves = kPartThreads / 64;
    const int64_t row = blockIdx.x;
    const int part = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int begin = part * p.len, end = min(a.vocab, begin + p.len);
    const uint16_t *z = (const uint16_t *)a.logits.p + row * a.logits.st;
    char *to = a.work + (row * p.count + part) * p.bytes;
    PartHead *head = (PartHead *)to;
    const int f = count_bins<kPartThreads>(z, begin, end, hist, [&]() {
        for (int i = tid; i < kBins / 8; i += kPartThreads) ((uint4 *)hist)[i] = make_uint4(0, 0, 0, 0);
        if (tid < 4) used[tid] = 0;
        if (tid == 4) flags = 0;
        __syncthreads();
    });
    if (f) atomicOr(&flags, (uint32_t)f);
    __syncthreads();
    for (int b = wave; b < kBlocks; b += kPartWaves) {
        const uint32_t c = hist[b * 64 + lane];
        if (!__ballot(c != 0)) continue;
        ((uint32_t *)(to + 64))[b * 64 + lane] = c;
        if (lane == 0) atomicOr(used + (b >> 5), 1u << (b & 31));
    }
    __syncthreads();
    if (tid == 0) {
        head->blocks[0] = used[0] | (uint64_t)used[1] << 32;
        head->blocks[1] = used[2] | (uint64_t)used[3] << 32;
        head->flags = (int32_t)flags;
    }
}

// ------------------------------------------------------------------------- block-wide steps
// The sums over the threads before this one, and over all, of a count and a mass.
__device__ __forceinline__ void block_scan(int c, double m, int &cb, double &mb, int &call, double &mall) {
    __shared__ int jc[kWaves];
    __shared__ double jm[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int cs = wave_scan(c);
    const double ms = wave_scan(m);
    __syncthreads();
    if (lane == 63) jc[wave] = cs, jm[wave] = ms;
    __syncthreads();
    cb = cs - c, call = 0;
    double before = 0.0;
    mall = 0.0;
    for (int i = 0; i < kWaves; ++i) {
        if (i < wave) cb += jc[i], before += jm[i];
        call += jc[i], mall += jm[i];
    }
    mb = before + wave_before(ms);
}

__device__ __forceinline__ void no_answer(const SampleArgs &a, int row) {
    if (threadIdx.x != 0) return;
    a.token[row] = -1;
    if (a.logp) a.logp[row] = __builtin_nanf("");
    if (a.kept) a.kept[row] = 0;
}

// Where the token lies: ranges of [begin, end) by their kept masses, at most 128 at a time, then
// the lots of one. `item(i, bits, fn)` calls fn(kept, tie, weight) for a token; of the ties the
// first `ties` in order are kept, with `tie_weight`.
struct Range { double mass; int kept, ties; };
constexpr int kRanges = 128;

struct Drawn {                                   // what is looked for, in the range at hand
    double want;
    float u;
    int ties;
};

// Of the ranges in order, two a lane: the one that holds the token (-1: none has any kept), and what
// is looked for in it.
__device__ __forceinline__ int pick_range(const Range *r, int n, double w, Drawn &d) {
    const int lane = threadIdx.x & 63;
    Range x[2];
    int ties[2], kept[2];
    double mass[2];
    int t = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        x[i] = 2 * lane + i < n ? r[2 * lane + i] : Range{0.0, 0, 0};
        t += x[i].ties;
    }
    int before = wave_scan(t) - t;
    double own = 0.0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        ties[i] = min(max(d.ties - before, 0), x[i].ties);
        before += x[i].ties;
        kept[i] = x[i].kept + ties[i];
        mass[i] = x[i].mass + ties[i] * w;
        own += mass[i];
    }
    double at = wave_before(wave_scan(own));
    int found = 1 << 30, last = -1;
    double left = 0.0, left_last = 0.0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (kept[i] > 0) {
            last = 2 * lane + i;
            left_last = d.want - at;
            if (found == 1 << 30 && (d.u == 0.f || (d.u < 1.f && at + mass[i] > d.want))) {
                found = 2 * lane + i;
                left = d.want - at;
            }
        }
        at += mass[i];
    }
    uint64_t hit = __ballot(found != 1 << 30);
    int src = hit ? __builtin_ctzll(hit) : 0;
    if (!hit) {
        hit = __ballot(last >= 0);
        if (!hit) return -1;
        src = 63 - __builtin_clzll(hit);
        found = last;
        left = left_last;
    }
    found = wave_read(found, src);
    d.want = wave_read(left, src);
    d.ties = wave_read(found & 1 ? ties[1] : ties[0], src);
    return found;
}

template <typename T, int UNROLL = 1, int WORDS = 4, typename Item>
__device__ __forceinline__ int locate(const T *z, const Item &item, int begin, int end, double tie_weight, Drawn d,
                                      Range *ranges) {
    constexpr int kL = WORDS * 4 / (int)sizeof(T), kC = 64 * kL;     // tokens of a lane and of a cell
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll 1
    while (end - begin > kC) {
        const int step = max(kC, ((end - begin + kRanges - 1) / kRanges + kC - 1) / kC * kC);
        const int n = (end - begin + step - 1) / step, cells = step / kC;
        __syncthreads();                         // (the ranges before are read)
        // this wavefront's cells, those of the ranges wave, wave + 16, ..: three are on their way
        Lot ahead[3];
        int at = begin + wave * step, left = cells, r = wave;
        int next = at, next_left = cells;
        const auto load_next = [&]() {
            const Lot x = load_some<T, WORDS>(z, next + lane * kL, end);
            next += kC;
            if (--next_left == 0) next += (kWaves - 1) * step, next_left = cells;
            next = min(next, end);
            return x;
        };
#pragma unroll
        for (int j = 0; j < 3; ++j) ahead[j] = load_next();
        Range x{0.0, 0, 0};
#pragma unroll 1
        while (r < n) {
            const Lot y = ahead[0];
            ahead[0] = ahead[1], ahead[1] = ahead[2];
            ahead[2] = load_next();
            each_token<T, UNROLL, WORDS>(y, [&](int j, uint32_t bits) {
                item(at + lane * kL + j, bits, [&](bool kept, bool tie, double w) {
                    x.mass += w;
                    x.kept += kept;
                    x.ties += tie;
                });
            });
            at += kC;
            if (--left > 0) continue;
            x.mass = wave_sum(x.mass);
            x.kept = wave_sum(x.kept);
            x.ties = wave_sum(x.ties);
            if (lane == 0) ranges[r] = x;
            x = Range{0.0, 0, 0};
            r += kWaves, at += (kWaves - 1) * step, left = cells;
        }
        __syncthreads();
        r = max(0, pick_range(ranges, n, tie_weight, d));
        begin += r * step;
        end = min(end, begin + step);
    }
    // a lot a lane, every wavefront for itself: its mass, then its tokens one by one
    const Lot y = load_some<T, WORDS>(z, begin + lane * kL, end);
    int before = 0, found = -1, last = -1;
    double at = 0.0;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
        each_token<T, UNROLL, WORDS>(y, [&](int j, uint32_t bits) {
            const int i = begin + lane * kL + j;
            item(i, bits, [&](bool kept, bool tie, double w) {
                const bool keep = i < end && (kept || (tie && before < d.ties));
                before += tie;
                if (!keep) return;
                at += tie ? tie_weight : w;
                last = i;
                if (found < 0 && (d.u == 0.f || (d.u < 1.f && at > d.want))) found = i;
            });
        });
        if (pass) break;
        // (of the lane's ties in the first pass as many were added as it has before the limit)
        const int ties = before, first = wave_scan(ties) - ties;
        at += (min(max(d.ties - first, 0), ties) - min(ties, d.ties)) * tie_weight;
        at = wave_before(wave_scan(at));
        before = first;
        found = last = -1;
    }
    uint64_t hit = __ballot(found >= 0);
    if (hit) return wave_read(found, __builtin_ctzll(hit));
    hit = __ballot(last >= 0);
    return wave_read(last, hit ? 63 - __builtin_clzll(hit) : 0);
}

// ------------------------------------------------------------------------------ fine bins
constexpr int kFineBins = 2048, kFineList = 4096;
constexpr int kFew = 256, kFewList = 1024;       // top_k of which the kept tokens are put in order

__device__ __forceinline__ double exp_small(double x) {      // e^-x for 0 <= x <= 1/32, to 2^-53
    double r = -1.0 / 5040;
    r = fma(r, x, 1.0 / 720);
    r = fma(r, x, -1.0 / 120);
    r = fma(r, x, 1.0 / 24);
    r = fma(r, x, -1.0 / 6);
    r = fma(r, x, 0.5);
    r = fma(r, x, -1.0);
    return fma(r, x, 1.0);
}

struct FinePool {
    uint32_t count[kFineBins];
    alignas(16) uint64_t mass[kFineBins];        // in fixed point, relative to the bin's edge
    double edge[kFineBins];                      // e^(-b / 32)
    uint32_t key[kFineList], index[kFineList];
    uint32_t dcount[256];
    uint64_t dmass[256];
    Range ranges[kRanges];
    uint32_t top, n, bad, listed, least;
    int bin, above, first, last;
    double before;                               // mass above a bin
};

// An end of the run: tokens of the bins before `bin`, and those of it at or above `comp`.
struct Edge {
    int bin;
    uint64_t comp;                               // value, then the index from the last to the first
    int kept;
    double mass;
};

// Counts a token of mass x into bin b; together where a wavefront's tokens are all alike, which would
// wait for each other (an fp32 row of 151936 with a nucleus: 606 us for 1699 where all are equal, 148 for
// 345 at T = 0.01, whose tokens nearly all lie in the last bin, and 181 for 168 at T = 1).
__device__ __forceinline__ void add_to(uint32_t *count, uint64_t *mass, int b, uint64_t x) {
    const int b0 = __builtin_amdgcn_readfirstlane(b);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)x), hi = __builtin_amdgcn_readfirstlane((int)(x >> 32));
    const uint64_t here = __ballot(true);
    uint32_t n = 1;
    if (__ballot(b == b0 && x == ((uint64_t)hi << 32 | lo)) == here) {
        if ((int)(threadIdx.x & 63) != __builtin_ctzll(here)) return;
        n = (uint32_t)__popcll(here);
    }
    atomicAdd(count + b, n);
    atomicAdd((unsigned long long *)mass + b, (unsigned long long)n * x);
}

__device__ __forceinline__ double b_mass(const FinePool &f, int b, double back) { return (double)f.mass[b] * back * f.edge[b]; }
__device__ __forceinline__ uint64_t comp_of(uint32_t key, int i) {
    return (uint64_t)key << 24 | (0xffffff - (uint32_t)i);
}

// The run's end among `n` tokens at least `k` of which are known to be the first of the row: they are put
// in order by counting for each the ones before it, k <= 256 are kept.
template <typename T, typename Scaled>
__device__ __forceinline__ void sample_few(const SampleArgs &a, int row, const Settings &s, FinePool &f, int n,
                                           const Scaled &scaled) {
    const int tid = threadIdx.x, k = s.k;
    uint64_t *comp = f.mass, *sorted = f.mass + kFewList;
    double *weight = f.edge;
    static_assert(2 * kFewList <= kFineBins, "");
    const uint64_t mine = tid < n ? comp_of(f.key[tid], (int)f.index[tid]) : 0;
    if (tid < (n + 7 & ~7)) comp[tid] = mine;                // (0 behind the last, to a multiple of 8)
    if (tid == 0) f.first = 0x7fffffff, f.last = -1;
    __syncthreads();
    if (tid < n) {
        int rank = 0;
#pragma unroll 2
        for (int i = 0; i < n; i += 4) {
            const ulonglong2 x = *(const ulonglong2 *)(comp + i), y = *(const ulonglong2 *)(comp + i + 2);
            rank += (x.x > mine) + (x.y > mine) + (y.x > mine) + (y.y > mine);
        }
        sorted[rank] = mine;
    }
    __syncthreads();
    const uint64_t own = tid < k ? sorted[tid] : 0;
    const int index = 0xffffff - (int)(own & 0xffffff);
    const double w = tid < k ? exp_below(-scaled(ord2f((uint32_t)(own >> 24)))) : 0.0;
    if (tid < k) weight[tid] = w;
    int cb, call;
    double mb, all;
    block_scan(0, w, cb, mb, call, all);
    // (the run's tokens are counted: what lies above either limit is the first part of the order)
    const bool in_p = tid < k && (tid == 0 || !(s.p < 1.f) || mb < (double)s.p * all);
    const bool in_m = tid < k && (tid == 0 || !(s.mp > 0.f) || w >= (double)s.mp);
    const bool in = in_p && in_m;
    double total;
    int kept;
    block_scan(in, in ? w : 0.0, cb, mb, kept, total);
    const double want = (double)s.u * total;
    if (in) {
        double at = 0.0;
#pragma unroll 4
        for (int i = 0; i < kept; ++i) at += 0xffffff - (int)(sorted[i] & 0xffffff) <= index ? weight[i] : 0.0;
        atomicMax(&f.last, index);
        if (s.u == 0.f || (s.u < 1.f && at > want)) atomicMin(&f.first, index);
    }
    __syncthreads();
    if (tid == 0) {
        const int token = f.first == 0x7fffffff ? f.last : f.first;
        a.token[row] = token;
        const float v = RowElem<T>::get(((const T *)a.logits.p + row * a.logits.st)[token]);
        if (a.logp) a.logp[row] = (float)(-scaled(v) - log(total));
        if (a.kept) a.kept[row] = kept;
    }
}

template <typename T>
__device__ __forceinline__ void sample_fine(const SampleArgs &a, int row, const Settings &s, FinePool &f) {
    const T *z = (const T *)a.logits.p + row * a.logits.st;
    const int tid = threadIdx.x, V = a.vocab;
    // every token that is not -inf: fn(value, index). `light`: all of them, for a few instructions each that
    // are worth their unrolling
    const auto each = [&](auto fn, auto light) {
        constexpr int kStep = kThreads * kLot<T>, kAhead = 4;
        const int first = tid * kLot<T>;
        Lot ahead[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) ahead[j] = load_tokens(z, min(first + j * kStep, V), V);
#pragma unroll 1
        for (int i = first; i < V; i += kStep) {
            const Lot x = ahead[0];
#pragma unroll
            for (int j = 0; j + 1 < kAhead; ++j) ahead[j] = ahead[j + 1];
            ahead[kAhead - 1] = load_tokens(z, min(i + kAhead * kStep, V), V);
            each_token<T, decltype(light)::value ? 4 : 1>(x, [&](int j, uint32_t bits) {
                const float v = token_value<T>(bits) + 0.f;        // (-0 and 0 are the same value)
                if (decltype(light)::value || !(v == kNegInf)) fn(v, i + j);
            });
        }
    };
    if (tid == 0) f.top = 0, f.n = 0, f.bad = 0, f.listed = 0, f.least = 0xffffffffu;
    __syncthreads();
    uint32_t n = 0, bad = 0;
    float most = kNegInf;
    each([&](float v, int) {
        bad |= !(v < __builtin_inff());
        most = fmaxf(most, v);
        n += v > kNegInf;
    }, std::true_type{});
    uint32_t top = f2ord(most);
    if (s.k > 0 && s.k <= kFew) {
        // the least of the largest values of k groups of threads or more: k tokens at least reach it
        uint32_t group = top;
        for (int o = 1; o * 2 <= (s.k <= 64 ? 16 : s.k <= 128 ? 8 : 4); o <<= 1)
            group = max(group, (uint32_t)__shfl_xor((int)group, o));
        const uint32_t least = ~wave_max(~group);
        if ((tid & 63) == 0) atomicMin(&f.least, least);
    }
    top = wave_max(top);
    n = wave_sum(n);
    if ((tid & 63) == 0) {
        atomicMax(&f.top, top);
        atomicAdd(&f.n, n);
    }
    if (bad) atomicOr(&f.bad, 1u);
    __syncthreads();
    if (f.bad || f.n == 0 || !s.ok) return no_answer(a, row);
    const double zmax = (double)ord2f(f.top), inv = 1.0 / (double)s.temp;
    const auto scaled = [&](float v) { return (zmax - (double)v) * inv; };
    const int total = (int)f.n;
    if (s.k > 0 && s.k <= kFew && s.k < total && f.least > f2ord(kNegInf)) {
        const float least = ord2f(f.least);
        each([&](float v, int i) {
            if (!(v >= least)) return;
            const uint32_t at = atomicAdd(&f.listed, 1u);
            if (at < (uint32_t)kFewList) f.key[at] = f2ord(v), f.index[at] = i;
        }, std::true_type{});
        __syncthreads();
        if (f.listed <= (uint32_t)kFewList) return sample_few<T>(a, row, s, f, (int)f.listed, scaled);
    }

    for (int i = tid; i < kFineBins; i += kThreads) f.count[i] = 0, f.mass[i] = 0, f.edge[i] = exp_below(i * -0.03125);
    __syncthreads();
    int bits = 0;
    while ((V >> bits) > 0) ++bits;
    const double unit = ldexp(1.0, 62 - bits), back = ldexp(1.0, bits - 62);
    const auto bin_at = [&](double t) { return t < 63.96875 ? (int)(t * 32.0) : kFineBins - 1; };
    // a weight relative to its bin's edge, in fixed point (of the last bin, whose mass is less than the sums'
    // roundings, none)
    const auto rel = [&](double t, int b) { return b < kFineBins - 1 ? exp_small(t - b * 0.03125) : 0.0; };
    const auto fixed = [&](double t, int b) { return (unsigned long long)(rel(t, b) * unit + 0.5); };
    each([&](float v, int) {
        const double t = scaled(v);
        const int b = bin_at(t);
        add_to(f.count, f.mass, b, fixed(t, b));
    }, std::false_type{});
    __syncthreads();
    int c[2], cb, call;
    double m[2], mb, mall;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        c[i] = (int)f.count[2 * tid + i];
        m[i] = b_mass(f, 2 * tid + i, back);
    }
    block_scan(c[0] + c[1], m[0] + m[1], cb, mb, call, mall);

    // Where the run ends: by the count of top_k, then by the mass of top_p. The bin is the first that
    // reaches it; inside, the digits of value and index are found one after the other.
    Edge end{kFineBins, 0, total, mall};
#pragma unroll 1
    for (int by_mass = 0; by_mass < 2; ++by_mass) {
        if (by_mass ? !(s.p < 1.f) : !(s.k > 0 && s.k < total)) continue;
        const double share = (double)s.p * end.mass;
        __syncthreads();
        if (tid == 0) f.bin = kFineBins, f.listed = 0;
        __syncthreads();
        const bool in0 = c[0] && (by_mass ? mb + m[0] >= share : cb + c[0] >= s.k);
        const bool in1 = c[1] && (by_mass ? mb + m[0] + m[1] >= share : cb + c[0] + c[1] >= s.k);
        if (in0 || in1) atomicMin(&f.bin, 2 * tid + !in0);
        __syncthreads();
        const int b = f.bin;
        if (by_mass && (b >= kFineBins - 1 || b > end.bin)) continue;
        if (tid == b >> 1) {
            f.above = cb + (b & 1 ? c[0] : 0);
            f.before = mb + (b & 1 ? m[0] : 0.0);
        }
        const bool list = f.count[b] <= (uint32_t)kFineList;
        if (list) {
            each([&](float v, int i) {
                if (bin_at(scaled(v)) != b) return;
                const uint32_t at = atomicAdd(&f.listed, 1u);
                f.key[at] = f2ord(v);
                f.index[at] = i;
            }, std::false_type{});
        }
        __syncthreads();
        const int above = f.above, count = s.k - above;
        const double before = f.before, want = (share - before) / f.edge[b] * unit;
        uint64_t prefix = 0, most = 0;
        Edge e{b, 0, 0, 0.0};
#pragma unroll 1
        for (int shift = 48; shift >= 0; shift -= 8) {
            if (tid < 256) f.dcount[tid] = 0, f.dmass[tid] = 0;
            __syncthreads();
            const auto add = [&](float v, int i) {
                const uint64_t comp = comp_of(f2ord(v), i);
                if ((comp >> shift >> 8) != prefix) return;
                const int d = 255 - (int)(comp >> shift & 255);
                add_to(f.dcount, f.dmass, d, fixed(scaled(v), b));
            };
            if (list) for (int i = tid; i < (int)f.listed; i += kThreads) add(ord2f(f.key[i]), (int)f.index[i]);
            else each([&](float v, int i) { if (bin_at(scaled(v)) == b) add(v, i); }, std::false_type{});
            __syncthreads();
            // every wavefront for itself: 4 digits a lane
            const int lane = tid & 63;
            int dc[4], cs = 0;
            uint64_t dm[4], ms = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                cs += dc[i] = (int)f.dcount[4 * lane + i];
                ms += dm[i] = f.dmass[4 * lane + i];
            }
            int cr = wave_scan(cs) - cs;
            uint64_t mr = wave_scan(ms) - ms;
            bool ends = false;
            int digit = -1, c_at = 0, n_at = 0;  // where it ends, or the lane's last digit that has any
            uint64_t m_at = 0, w_at = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (dc[i] > 0 && !ends) {
                    ends = by_mass ? (double)(most + mr + dm[i]) >= want : e.kept + cr + dc[i] >= count;
                    digit = 4 * lane + i, c_at = cr, m_at = mr, n_at = dc[i], w_at = dm[i];
                }
                cr += dc[i], mr += dm[i];
            }
            const uint64_t hit = __ballot(ends), any = __ballot(digit >= 0);
            const int src = hit ? __builtin_ctzll(hit) : any ? 63 - __builtin_clzll(any) : 0;
            prefix = prefix << 8 | (uint64_t)(255 - wave_read(digit, src));
            e.kept += wave_read(c_at, src);
            most += wave_read(m_at, src);
            n_at = wave_read(n_at, src);
            w_at = wave_read(w_at, src);
            __syncthreads();
            if (n_at == 1 || (!by_mass && e.kept + n_at == count)) {     // all of this digit
                e.comp = prefix << shift;
                e.kept += n_at;
                most += w_at;
                break;
            }
        }
        e.mass = (double)most * back * f.edge[b] + before;
        e.kept += above;
        if (e.bin < end.bin || e.comp > end.comp) end = e;
    }
    if (s.mp > 0.f) {
        const int b = bin_at(-log((double)s.mp));
        __syncthreads();
        if (tid == 0) f.least = 0xffffffffu, f.listed = 0, f.dmass[0] = 0;
        if (tid == b >> 1) {
            f.above = cb + (b & 1 ? c[0] : 0);
            f.before = mb + (b & 1 ? m[0] : 0.0);
        }
        __syncthreads();
        each([&](float v, int) {
            const double t = scaled(v);
            if (bin_at(t) != b || !(exp_below(-t) >= (double)s.mp)) return;
            atomicMin(&f.least, f2ord(v));
            atomicAdd(&f.listed, 1u);
            atomicAdd((unsigned long long *)f.dmass, fixed(t, b));
        }, std::false_type{});
        __syncthreads();
        // (a comp that no token reaches where the bin has none)
        const Edge e{b, f.listed ? (uint64_t)f.least << 24 : ~0ull, f.above + (int)f.listed,
                     f.before + (double)f.dmass[0] * back * f.edge[b]};
        if (e.bin < end.bin || (e.bin == end.bin && e.comp > end.comp)) end = e;
    }
    const auto item = [&](int i, uint32_t bits, auto fn) {
        const float v = token_value<T>(bits) + 0.f;
        const double t = scaled(v);
        const int b = v > kNegInf ? bin_at(t) : kFineBins;
        const bool kept = b < end.bin || (b == end.bin && b < kFineBins && comp_of(f2ord(v), i) >= end.comp);
        fn(kept, false, kept ? f.edge[b] * rel(t, b) : 0.0);
    };
    const int token = locate(z, item, 0, V, 0.0, Drawn{(double)s.u * end.mass, s.u, 0}, f.ranges);
    if (tid == 0) {
        a.token[row] = token;
        if (a.logp) a.logp[row] = (float)(-scaled(RowElem<T>::get(z[token])) - log(end.mass));
        if (a.kept) a.kept[row] = end.kept;
    }
}

// LEFT: of the rows only those that the coarse bins have left (their token is kLeft).
constexpr int kLeft = -2;

template <typename T, bool LEFT>
__global__ __launch_bounds__(kThreads) void sample_fine_kernel(SampleArgs a) {
    __shared__ FinePool f;
    if (LEFT && a.token[blockIdx.x] != kLeft) return;
    sample_fine<T>(a, blockIdx.x, settings_of(a, blockIdx.x), f);
}

// ---------------------------------------------------------------------------- coarse bins
struct CoarsePool {
    double weight[kSlots * 128 + 256];           // 0 past the bins in use, and after the cut past the run
    uint32_t count[kSlots * 128];
    uint64_t blocks[kMostParts][2];
    Range ranges[kRanges];
    uint32_t used[4], flags;
    int16_t place[512];                          // of a value's sign and exponent: its block's first bin here
    uint8_t block[kSlots];
    int first, bin_k, ties_k, bin_p, bin_m, above;
    double mass;
};
struct CoarseRow : CoarsePool { uint32_t hist[kBins / 2]; };   // of a row that is counted here

// A row that keeps every token, from its parts' masses: the part, then the token by its own weights.
// A greedy row: the first of its largest.
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_all_kernel(SampleArgs a, Parts parts) {
    __shared__ Range ranges[kRanges];
    const int row = blockIdx.x, lane = threadIdx.x & 63, S = parts.count;
    const T *z = (const T *)a.logits.p + row * a.logits.st;
    const Settings s = settings_of(a, row);
    if (!s.ok) return no_answer(a, row);
    float top = kNegInf;
    double mass = 0.0;
    int n = 0, flags = 0;
    if (lane < S) {
        const PartHead *h = (const PartHead *)(a.work + ((int64_t)row * S + lane) * parts.bytes);
        top = h->top;
        mass = h->mass;
        n = h->n;
        flags = h->flags;
    }
    if (__ballot(flags != 0)) return no_answer(a, row);
    const int there = wave_sum(n);
    if (there == 0) return no_answer(a, row);
    const double zmax = (double)ord2f(wave_max(f2ord(n > 0 ? top : kNegInf))), inv = 1.0 / (double)s.temp;
    mass = n > 0 ? mass * exp_below(((double)top - zmax) * inv) : 0.0;
    const double all = wave_sum(mass);
    if (threadIdx.x < S) ranges[lane] = Range{mass, s.greedy ? n > 0 && (double)top == zmax : n, 0};
    __syncthreads();
    Drawn d{(double)s.u * all, s.greedy ? 0.f : s.u, 0};
    const int q = max(0, pick_range(ranges, S, 0.0, d)), begin = q * parts.len;
    const auto item = [&](int, uint32_t bits, auto fn) {
        const float v = token_value<T>(bits);
        const bool in = s.greedy ? (double)v == zmax : v > kNegInf;
        fn(in, false, in ? exp_below(((double)v - zmax) * inv) : 0.0);
    };
    const int token = locate<T, 1, 1>(z, item, begin, min(a.vocab, begin + parts.len), 0.0, d, ranges);
    if (threadIdx.x == 0) {
        a.token[row] = token;
        if (a.logp) a.logp[row] = (float)(((double)RowElem<T>::get(z[token]) - zmax) * inv - (s.greedy ? 0.0 : log(all)));
        if (a.kept) a.kept[row] = s.greedy ? 1 : there;
    }
}

// MANY: 64 registers, so that two workgroups share a compute unit, and the rows that these bins do
// not hold are left to a launch of their own (4.5 us); else they are answered here.
template <bool SPLIT, bool MANY>
__global__ __launch_bounds__(kThreads, MANY ? 8 : 4) void sample_coarse_kernel(SampleArgs a, Parts parts) {
    using Coarse = std::conditional_t<SPLIT, CoarsePool, CoarseRow>;
    __shared__ union Pool {
        Coarse c;
        std::conditional_t<MANY, char, FinePool> f;
        __device__ Pool() {}
    } pool;
    Coarse &f = pool.c;
    constexpr int kPer = kSlots * 128 / kThreads;
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int V = a.vocab, S = parts.count;
    const uint16_t *z = (const uint16_t *)a.logits.p + row * a.logits.st;
    const char *part = a.work + (int64_t)row * S * parts.bytes;
    const Settings s = settings_of(a, row);
    PartHead own{};
    if constexpr (SPLIT)
        if (tid < S) own = *(const PartHead *)(part + tid * parts.bytes);
    if (!s.ok) return no_answer(a, row);

    // ---- the blocks in use, and the counts of their bins
    if (tid < 4) f.used[tid] = 0;
    if (tid == 4) f.flags = 0, f.first = kSlots * 128, f.bin_k = f.bin_p = kSlots * 128, f.bin_m = -1;
    if constexpr (SPLIT) {
        __syncthreads();
        if (tid < S) {
            const PartHead &h = own;
            f.blocks[tid][0] = h.blocks[0];
            f.blocks[tid][1] = h.blocks[1];
            for (int i = 0; i < 4; ++i) atomicOr(f.used + i, (uint32_t)(h.blocks[i >> 1] >> (i & 1) * 32));
            if (h.flags) atomicOr(&f.flags, (uint32_t)h.flags);
        }
    } else {
        const int flags = count_bins<kThreads>(z, 0, V, f.hist, [&]() {
            for (int i = tid; i < kBins / 2; i += kThreads) f.hist[i] = 0;
            __syncthreads();
        });
        if (flags) atomicOr(&f.flags, (uint32_t)flags);
        __syncthreads();
        for (int b = wave; b < kBlocks; b += kWaves)
            if (__ballot(f.hist[b * 64 + lane] != 0) && lane == 0) atomicOr(f.used + (b >> 5), 1u << (b & 31));
    }
    __syncthreads();
    int slots = 0;
    for (int i = 0; i < 4; ++i) slots += __popc(f.used[i]);
    if ((f.flags & 1) || (slots == 0 && !(f.flags & 2))) return no_answer(a, row);
    // (u = 0 and 1 ask for the first and the last token kept, whatever they weigh)
    bool fine = (f.flags & 2) || slots > kSlots || s.u == 0.f || s.u == 1.f;
    const int bins = slots * 128;
    if (!fine) {
        if (tid < 512) f.place[tid] = kSlots * 128;
        __syncthreads();
        if (tid < kBlocks && f.used[tid >> 5] >> (tid & 31) & 1) {
            int at = 0;
            for (int i = 0; i < 4; ++i) {
                const int from = tid - 32 * i;
                at += from >= 32 ? __popc(f.used[i]) : from > 0 ? __popc(f.used[i] & ((1u << from) - 1)) : 0;
            }
            f.block[at] = tid;
            // a positive value's bin is 127 - its mantissa after its place, a negative one's its mantissa
            if (tid < kSide >> 7) f.place[(kHigh >> 7) - 1 - tid] = at * 128;
            else if (tid == kZeroBin >> 7) f.place[0] = at * 128 - 127, f.place[256] = at * 128;
            else if (tid < kBelow >> 7) f.place[256 + (kLow >> 7) + tid - (kNegative >> 7)] = at * 128;
        }
        __syncthreads();
        // a wavefront has every 16th block, two counts a lane; 8 parts of each of its blocks are on their way together
        constexpr int kRounds = kSlots / kWaves;
        uint32_t c0[kRounds] = {}, c1[kRounds] = {};
        if constexpr (SPLIT) {
            uint64_t has[kRounds];               // parts that have counts of the block
            const uint32_t *from[kRounds];
#pragma unroll
            for (int k = 0; k < kRounds; ++k) {
                const int slot = wave + k * kWaves;
                const int b = __builtin_amdgcn_readfirstlane(f.block[min(slot, slots - 1)]);
                has[k] = slot < slots ? __ballot(lane < S && (f.blocks[lane][b >> 6] >> (b & 63) & 1)) : 0;
                from[k] = (const uint32_t *)(part + 64) + b * 64 + lane;
            }
#pragma unroll 1
            while (has[0] | has[1] | has[2]) {
                uint32_t x[kRounds][8];
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int k = 0; k < kRounds; ++k) {
                        x[k][j] = 0;
                        if (has[k]) x[k][j] = from[k][__builtin_ctzll(has[k]) * (parts.bytes / 4)];
                        has[k] &= has[k] - 1;
                    }
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int k = 0; k < kRounds; ++k) c0[k] += x[k][j] & 0xffffu, c1[k] += x[k][j] >> 16;
            }
        } else {
#pragma unroll
            for (int k = 0; k < kRounds; ++k) {
                const int slot = wave + k * kWaves;
                if (slot >= slots) break;
                const uint32_t x = f.hist[f.block[slot] * 64 + lane];
                c0[k] = x & 0xffffu, c1[k] = x >> 16;
            }
        }
#pragma unroll
        for (int k = 0; k < kRounds; ++k) {
            const int i = (wave + k * kWaves) * 64 + lane;
            if (i >= slots * 64) break;
            f.count[2 * i] = c0[k];
            f.count[2 * i + 1] = c1[k];
            const uint64_t any = __ballot((c0[k] | c1[k]) != 0);
            if (any && lane == __builtin_ctzll(any)) atomicMin(&f.first, 2 * i + (c0[k] == 0));
        }
        __syncthreads();
    }
    const auto bin_at = [&](int i) { return f.block[i >> 7] * 128 + (i & 127); };
    double zmax = 0.0;
    const double inv = 1.0 / (double)s.temp;
    int c[kPer], cs = 0, cb = 0, n = 0;
    double ms = 0.0, mb = 0.0, mall = 0.0;
    const int b0 = tid * kPer;
    if (!fine) {
        const int top = bin_at(f.first);
        zmax = (double)value_of(top);
        // values below -2^15 are counted only: their weights vanish, or the row is not for these bins
        const bool below = f.used[kBelow >> 12] >> (kBelow >> 7 & 31) & 1;
        fine = top == kBelow || (below && (zmax + 32768.0) * inv < 800.0);
    }
    if (!fine) {
#pragma unroll 1
        for (int i = tid; i < kSlots * 128 + 256; i += kThreads) {
            const int b = i < bins ? bin_at(i) : kBelow;
            f.weight[i] = b != kBelow && f.count[i] ? exp_below(((double)value_of(b) - zmax) * inv) : 0.0;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            c[i] = b0 + i < bins ? (int)f.count[b0 + i] : 0;
            cs += c[i];
            ms += c[i] ? c[i] * f.weight[b0 + i] : 0.0;
        }
        block_scan(cs, ms, cb, mb, n, mall);
        // ---- where the run ends: a bin, and how many of its tokens belong to it
        if (s.k > 0 && s.k < n && cb < s.k && cb + cs >= s.k) {
            int left = s.k - cb, i = 0;
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                if (i == j && left > c[j]) left -= c[j], ++i;
            f.bin_k = b0 + i;
            f.ties_k = left;
        }
        __syncthreads();
    }
    int end = bins, ties = 0;
    double all = mall;
    // the tokens and the mass of the run: the thread that has its last bin knows them
    const auto measure = [&]() {
        __syncthreads();
        if (end < bins && tid == end / kPer) {
            int above = cb + ties;
            double mass = mb + ties * f.weight[end];
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (b0 + i < end && c[i]) above += c[i], mass += c[i] * f.weight[b0 + i];
            f.above = above;
            f.mass = mass;
        }
        if (end == bins && tid == 0) f.above = n, f.mass = mall;
        __syncthreads();
        all = f.mass;
    };
    if (!fine) {
        if (f.bin_k < kSlots * 128) end = f.bin_k, ties = f.ties_k;
        measure();
        if (s.p < 1.f) {
            const double want = (double)s.p * all;
            double at = mb;
            int hit = kSlots * 128;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                if (!c[i]) continue;
                at += c[i] * f.weight[b0 + i];
                if (at >= want && hit == kSlots * 128) hit = b0 + i;
            }
            if (hit < kSlots * 128) atomicMin(&f.bin_p, hit);
            __syncthreads();
            const int b = f.bin_p;
            if (b <= end && b < bins) {
                if (tid == b / kPer) {
                    double from = mb;
                    int there = 0;
#pragma unroll
                    for (int i = 0; i < kPer; ++i) {
                        if (b0 + i < b && c[i]) from += c[i] * f.weight[b0 + i];
                        if (b0 + i == b) there = c[i];
                    }
                    f.above = (int)fmax(1.0, fmin(ceil((want - from) / f.weight[b]), (double)there));
                }
                __syncthreads();
                ties = b == end ? min(ties, f.above) : f.above;
                end = b;
                __syncthreads();
            }
        }
        if (s.mp > 0.f) {
            int hit = -1;
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (c[i] && f.weight[b0 + i] >= (double)s.mp) hit = b0 + i;
            if (hit >= 0) atomicMax(&f.bin_m, hit);
            __syncthreads();
            if (f.bin_m < end) end = f.bin_m, ties = (int)f.count[end];
        }
        measure();
    }
    if (fine) {
        if constexpr (MANY) {
            if (tid == 0) a.token[row] = kLeft;
        } else {
            __syncthreads();
            sample_fine<uint16_t>(a, row, s, pool.f);
        }
        return;
    }
    const int kept = f.above;
    const double tie_weight = end < bins ? f.weight[end] : 0.0;
    __syncthreads();
    for (int i = end + tid; i < bins; i += kThreads) f.weight[i] = 0.0;
    __syncthreads();
    Drawn d{(double)s.u * all, s.u, ties};
    int begin = 0, stop = V;
    if constexpr (SPLIT) {
        // (two wavefronts a part where there are few)
        const int twice = 2 * S <= kWaves, blocks = min(slots, (end >> 7) + 1);
        for (int q = wave >> twice; q < S; q += kWaves >> twice) {
            Range x{0.0, 0, 0};
            // the part's blocks up to the run's end, by their places here
            bool in = false;
            if (lane < blocks) {
                const int b = f.block[lane];
                in = f.blocks[q][b >> 6] >> (b & 63) & 1;
            }
            uint64_t has = __ballot(in);
            if (twice) has &= wave & 1 ? 0xaaaaaaaaaaaaaaaaull : 0x5555555555555555ull;
            const uint32_t *from = (const uint32_t *)(part + (int64_t)q * parts.bytes + 64) + lane;
#pragma unroll 1
            while (has) {
                uint32_t y[8];
                int at[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    y[j] = 0;
                    at[j] = kSlots * 128;
                    if (has) {
                        const int i = __builtin_ctzll(has);
                        y[j] = from[__builtin_amdgcn_readfirstlane(f.block[i]) * 64];
                        at[j] = i * 128;
                    }
                    has &= has - 1;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int i = at[j] + 2 * lane, n0 = (int)(y[j] & 0xffffu), n1 = (int)(y[j] >> 16);
                    x.mass += n0 * f.weight[i] + n1 * f.weight[i + 1];
                    x.ties += i == end ? n0 : i + 1 == end ? n1 : 0;
                }
            }
            x.mass = wave_sum(x.mass);
            x.ties = wave_sum(x.ties);
            x.kept = x.mass > 0.0;
            if (lane == 0) f.ranges[twice ? 64 + wave : q] = x;
        }
        if (twice) {
            __syncthreads();
            if (tid < S) {
                const Range x = f.ranges[64 + 2 * tid], y = f.ranges[65 + 2 * tid];
                f.ranges[tid] = Range{x.mass + y.mass, x.kept | y.kept, x.ties + y.ties};
            }
        }
        __syncthreads();
        const int q = max(0, pick_range(f.ranges, S, tie_weight, d));
        begin = q * parts.len;
        stop = min(V, begin + parts.len);
    }
    // (values below -2^15 and -inf have a place past the bins, whose weights are 0)
    const auto item = [&](int, uint32_t bits, auto fn) {
        const int at = f.place[bits >> 7] + (int)((bits & 127) ^ (bits & 0x8000u ? 0 : 127));
        const double w = f.weight[at];
        fn(w > 0.0, at == end, w);
    };
    const int token = locate<uint16_t, 4>(z, item, begin, stop, tie_weight, d, f.ranges);
    if (tid == 0) {
        a.token[row] = token;
        if (a.logp) a.logp[row] = (float)(((double)bf16_bits_to_f32(z[token]) - zmax) * inv - log(all));
        if (a.kept) a.kept[row] = kept;
    }
}

}  // namespace

int64_t sample_bytes(const SampleArgs &a, bool bf16) {
    if (a.rows == 0) return 0;
    const Parts p = parts_of(a, bf16);
    return p.count <= 1 || p.count > kMostParts ? 0 : (int64_t)a.rows * p.count * p.bytes;
}

hipError_t launch_sample(const SampleArgs &a, bool bf16, hipStream_t st) {
    const Parts p = parts_of(a, bf16);
    const auto run = [&](auto kernel) {
        kernel<<<a.rows, kThreads, 0, st>>>(a);
        return hipGetLastError();
    };
    const auto run_parts = [&](auto first, auto second) {
        first<<<dim3(a.rows, p.count), kPartThreads, 0, st>>>(a, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        second<<<a.rows, kThreads, 0, st>>>(a, p);
        return hipGetLastError();
    };
    if (p.count > 1 && p.bytes == sizeof(PartHead))
        return bf16 ? run_parts(sample_masses_kernel<uint16_t>, sample_all_kernel<uint16_t>)
                    : run_parts(sample_masses_kernel<float>, sample_all_kernel<float>);
    if (!bf16) return run(sample_fine_kernel<float, false>);
    if (p.count > kMostParts) return run(sample_fine_kernel<uint16_t, false>);   // (more than 4 million tokens)
    if (p.count == 1) {
        sample_coarse_kernel<false, false><<<a.rows, kThreads, 0, st>>>(a, p);
        return hipGetLastError();
    }
    if (a.rows <= kChipUnits) return run_parts(sample_counts_kernel, sample_coarse_kernel<true, false>);
    const hipError_t e = run_parts(sample_counts_kernel, sample_coarse_kernel<true, true>);
    return e != hipSuccess ? e : run(sample_fine_kernel<uint16_t, true>);
}

}  // namespace olive
