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
// Masses are 64-bit: a token changes where the error of the sums passes u times their total over a
// border, and a row has as many borders as tokens.
#include <type_traits>

#include "rows.hpp"
#include "tokens_internal.hpp"

namespace olive {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kCell = 512;                       // tokens that a wavefront looks at together, 8 a lane

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
struct PartHead {
    uint64_t blocks[2];                          // blocks that hold counts
    int32_t flags;                               // bit 0: a bad value, bit 1: one without a bin
    int32_t pad;
};
constexpr int64_t kPartBytes = kBins * 2 + 64;   // head, then 16-bit counts
constexpr int kMostParts = 64, kMostPart = 65024;

struct Parts { int32_t count, len; };

Parts parts_of(int32_t rows, int32_t vocab) {
    int64_t s = 1024 / rows, least = (vocab + kMostPart - 1) / kMostPart;
    if (vocab <= 16384) s = 1;
    if (s > (vocab + 4095) / 4096) s = (vocab + 4095) / 4096;
    if (s > kMostParts) s = kMostParts;
    if (s < least) s = least;
    const int64_t len = ((vocab + s - 1) / s + kCell - 1) / kCell * kCell;
    return Parts{(int32_t)((vocab + len - 1) / len), (int32_t)len};
}

// 8 values from i on (none past `end`), at any alignment of their type
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Eight { T v[8]; };

template <typename T>
__device__ __forceinline__ Eight<T> load_eight(const T *z, int i, int end) {
    if (i + 8 <= end) return *(const Eight<T> *)(z + i);
    Eight<T> x;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if constexpr (sizeof(T) == 2) x.v[j] = i + j < end ? z[i + j] : (T)0xff80u;
        else x.v[j] = i + j < end ? z[i + j] : kNegInf;
    }
    return x;
}

// Counts of [begin, end) of a row into 16-bit bins (two to a word); the flags of its odd values.
template <int THREADS>
__device__ __forceinline__ int count_bins(const uint16_t *z, int begin, int end, uint32_t *hist) {
    int flags = 0;
    for (int i = begin + (int)threadIdx.x * 8; i < end; i += THREADS * 8) {
        const Eight<uint16_t> x = load_eight(z, i, end);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int b = bin_of(x.v[j]);
            if (b >= 0) atomicAdd(hist + (b >> 1), 1u << ((b & 1) * 16));
            else flags |= b == kBad ? 1 : b == kOdd ? 2 : 0;
        }
    }
    return flags;
}

constexpr int kPartThreads = 512;

__global__ __launch_bounds__(kPartThreads) void sample_parts_kernel(SampleArgs a, Parts p) {
    __shared__ uint32_t hist[kBins / 2];
    __shared__ uint32_t used[4], flags;
    const int64_t row = blockIdx.x;
    const int part = blockIdx.y;
    for (int i = threadIdx.x; i < kBins / 2; i += kPartThreads) hist[i] = 0;
    if (threadIdx.x < 4) used[threadIdx.x] = 0;
    if (threadIdx.x == 4) flags = 0;
    __syncthreads();
    const int begin = part * p.len, end = min(a.vocab, begin + p.len);
    const int f = count_bins<kPartThreads>((const uint16_t *)a.logits.p + row * a.logits.st, begin, end, hist);
    if (f) atomicOr(&flags, (uint32_t)f);
    __syncthreads();
    char *to = a.work + (row * p.count + part) * kPartBytes;
    const int lane = threadIdx.x & 63;
    for (int b = threadIdx.x >> 6; b < kBlocks; b += kPartThreads / 64) {
        const uint32_t c = hist[b * 64 + lane];
        if (!__ballot(c != 0)) continue;
        ((uint32_t *)(to + 64))[b * 64 + lane] = c;
        if (lane == 0) atomicOr(used + (b >> 5), 1u << (b & 31));
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        PartHead *h = (PartHead *)to;
        h->blocks[0] = used[0] | (uint64_t)used[1] << 32;
        h->blocks[1] = used[2] | (uint64_t)used[3] << 32;
        h->flags = (int32_t)flags;
    }
}

// ------------------------------------------------------------------------- block-wide steps
// The sums over the threads before this one, and over all, of a count and a mass.
__device__ __forceinline__ void block_scan(int c, double m, int &cb, double &mb, int &call, double &mall) {
    __shared__ int jc[kWaves];
    __shared__ double jm[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int cs = c;
    double ms = m;
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(cs, o);
        const double v = __shfl_up(ms, o);
        if (lane >= o) cs += u, ms += v;
    }
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
    mb = before + __shfl_up(ms, 1);
    if (lane == 0) mb = before;
}

struct Settings {
    float u, temp, p, mp;
    int k;
    bool ok;
};

__device__ __forceinline__ Settings settings_of(const SampleArgs &a, int row) {
    Settings s;
    s.u = a.uniform[row];
    s.temp = a.temperature ? a.temperature[row] : 1.f;
    s.p = a.top_p ? a.top_p[row] : 1.f;
    s.mp = a.min_p ? a.min_p[row] : 0.f;
    s.k = a.top_k ? a.top_k[row] : 0;
    s.ok = s.u >= 0.f && s.u <= 1.f && s.temp >= 0.f && s.temp < __builtin_inff() && s.p == s.p && s.mp == s.mp;
    if (s.temp == 0.f || s.mp > 1.f) s.k = 1, s.p = 1.f, s.mp = 0.f;   // the first token alone
    if (s.temp == 0.f) s.temp = 1.f;
    return s;
}

__device__ __forceinline__ void no_answer(const SampleArgs &a, int row) {
    if (threadIdx.x != 0) return;
    a.token[row] = -1;
    if (a.logp) a.logp[row] = __builtin_nanf("");
    if (a.kept) a.kept[row] = 0;
}

// Where the token lies: ranges of [begin, end) by their kept masses, at most 128 at a time, then
// the 512 tokens of one. `src(i, end, f)` calls f(j, kept, tie, weight) for the 8 tokens of a lane
// from i on; of the ties the first `ties` in order are kept.
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
    int before = t;
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(before, o);
        if (lane >= o) before += u;
    }
    before -= t;
    double own = 0.0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        ties[i] = min(max(d.ties - before, 0), x[i].ties);
        before += x[i].ties;
        kept[i] = x[i].kept + ties[i];
        mass[i] = x[i].mass + ties[i] * w;
        own += mass[i];
    }
    double run = own;
    for (int o = 1; o < 64; o <<= 1) {
        const double u = __shfl_up(run, o);
        if (lane >= o) run += u;
    }
    double at = __shfl_up(run, 1);
    if (lane == 0) at = 0.0;
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
    found = __shfl(found, src);
    d.want = __shfl(left, src);
    d.ties = __shfl(found & 1 ? ties[1] : ties[0], src);
    return found;
}

template <typename Src>
__device__ __forceinline__ int locate(const Src &src, int begin, int end, double tie_weight, Drawn d, Range *ranges) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    while (end - begin > kCell) {
        const int step = max(kCell, ((end - begin + kRanges - 1) / kRanges + kCell - 1) / kCell * kCell);
        const int n = (end - begin + step - 1) / step;
        __syncthreads();                         // (the ranges before are read)
        for (int r = wave; r < n; r += kWaves) {
            Range x{0.0, 0, 0};
            const int e = min(end, begin + (r + 1) * step);
            for (int i = begin + r * step; i < e; i += kCell)
                src(i + lane * 8, e, [&](int, bool kept, bool tie, double w) {
                    x.mass += kept ? w : 0.0;
                    x.kept += kept;
                    x.ties += tie;
                });
            for (int o = 32; o > 0; o >>= 1) {
                x.mass += __shfl_xor(x.mass, o);
                x.kept += __shfl_xor(x.kept, o);
                x.ties += __shfl_xor(x.ties, o);
            }
            if (lane == 0) ranges[r] = x;
        }
        __syncthreads();
        const int r = max(0, pick_range(ranges, n, tie_weight, d));
        begin += r * step;
        end = min(end, begin + step);
    }
    // 8 tokens a lane, every wavefront for itself
    Range own{0.0, 0, 0};
    src(begin + lane * 8, end, [&](int, bool kept, bool tie, double w) {
        own.mass += kept ? w : 0.0;
        own.ties += tie;
    });
    int before = own.ties;
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(before, o);
        if (lane >= o) before += u;
    }
    before -= own.ties;
    own.mass += min(max(d.ties - before, 0), own.ties) * tie_weight;
    double at = own.mass;
    for (int o = 1; o < 64; o <<= 1) {
        const double u = __shfl_up(at, o);
        if (lane >= o) at += u;
    }
    at = __shfl_up(at, 1);
    if (lane == 0) at = 0.0;
    int found = -1, last = -1;
    src(begin + lane * 8, end, [&](int j, bool kept, bool tie, double w) {
        const bool keep = kept || (tie && before < d.ties);
        before += tie;
        if (!keep) return;
        at += tie ? tie_weight : w;
        last = begin + lane * 8 + j;
        if (found < 0 && (d.u == 0.f || (d.u < 1.f && at > d.want))) found = last;
    });
    uint64_t hit = __ballot(found >= 0);
    if (hit) return __shfl(found, __builtin_ctzll(hit));
    hit = __ballot(last >= 0);
    return __shfl(last, hit ? 63 - __builtin_clzll(hit) : 0);
}

// ------------------------------------------------------------------------------ fine bins
constexpr int kFineBins = 2048, kFineList = 4096;

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
    uint64_t mass[kFineBins];                    // in fixed point, relative to the bin's edge
    double edge[kFineBins];                      // e^(-b / 32)
    uint32_t key[kFineList], index[kFineList];
    uint32_t dcount[256];
    uint64_t dmass[256];
    Range ranges[kRanges];
    uint32_t top, n, bad, listed, least;
    int bin, bin_p;
    double before;                               // mass above a bin
    int above;                                   // tokens above it
};

// An end of the run: tokens of the bins before `bin`, and those of it at or above `comp`.
struct Edge {
    int bin;
    uint64_t comp;                               // value, then the index from the last to the first
    int kept;
    double mass;
};

template <typename T>
__device__ void sample_fine(const SampleArgs &a, int row, const Settings &s, FinePool &f) {
    const T *z = (const T *)a.logits.p + row * a.logits.st;
    const int tid = threadIdx.x, V = a.vocab;
    const auto each = [&](auto fn) {             // every token that is not -inf: fn(value, index)
        for (int i = tid * 8; i < V; i += kThreads * 8) {
            const Eight<T> x = load_eight(z, i, V);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float v = RowElem<T>::get(x.v[j]) + 0.f;     // (-0 and 0 are the same value)
                if (!(v == kNegInf)) fn(v, i + j);
            }
        }
    };
    for (int i = tid; i < kFineBins; i += kThreads) f.count[i] = 0, f.mass[i] = 0, f.edge[i] = exp(-i / 32.0);
    if (tid == 0) f.top = 0, f.n = 0, f.bad = 0;
    __syncthreads();
    uint32_t top = 0, n = 0, bad = 0;
    each([&](float v, int) {
        bad |= !(v < __builtin_inff());
        top = max(top, f2ord(v));
        ++n;
    });
    for (int o = 32; o > 0; o >>= 1) {
        top = max(top, (uint32_t)__shfl_xor((int)top, o));
        n += __shfl_xor((int)n, o);
    }
    if ((tid & 63) == 0) {
        atomicMax(&f.top, top);
        atomicAdd(&f.n, n);
    }
    if (bad) atomicOr(&f.bad, 1u);
    __syncthreads();
    if (f.bad || f.n == 0 || !s.ok) return no_answer(a, row);

    const double zmax = (double)ord2f(f.top), inv = 1.0 / (double)s.temp;
    const int total = (int)f.n;
    int bits = 0;
    while ((V >> bits) > 0) ++bits;
    const double unit = ldexp(1.0, 62 - bits), back = ldexp(1.0, bits - 62);
    const auto scaled = [&](float v) { return (zmax - (double)v) * inv; };
    const auto bin_at = [&](double t) { return t < 63.96875 ? (int)(t * 32.0) : kFineBins - 1; };
    const auto rel = [&](double t, int b) {      // weight relative to the bin's edge
        const double x = t - b * 0.03125;
        return b < kFineBins - 1 ? exp_small(x) : exp(-x);
    };
    each([&](float v, int) {
        const double t = scaled(v);
        const int b = bin_at(t);
        atomicAdd(f.count + b, 1u);
        if (b < kFineBins - 1) atomicAdd((unsigned long long *)f.mass + b, (unsigned long long)(rel(t, b) * unit + 0.5));
    });
    __syncthreads();
    int c[2], cb, call;
    double m[2], mb, mall;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        c[i] = (int)f.count[2 * tid + i];
        m[i] = (double)f.mass[2 * tid + i] * back * f.edge[2 * tid + i];
    }
    block_scan(c[0] + c[1], m[0] + m[1], cb, mb, call, mall);

    // The tokens of bin b in order until `count` of them, or until their mass is `mass` (relative to the bin's
    // edge): the last one's value and index, how many they are and their mass.
    const auto refine = [&](int b, bool by_mass, int count, double mass) {
        const bool list = f.count[b] <= (uint32_t)kFineList;
        if (tid == 0) f.listed = 0;
        __syncthreads();
        if (list) {
            each([&](float v, int i) {
                if (bin_at(scaled(v)) != b) return;
                const uint32_t at = atomicAdd(&f.listed, 1u);
                f.key[at] = f2ord(v);
                f.index[at] = i;
            });
        }
        uint64_t prefix = 0, most = 0;
        Edge e{b, 0, 0, 0.0};
        const double want = mass * unit;
        for (int shift = 48; shift >= 0; shift -= 8) {
            if (tid < 256) f.dcount[tid] = 0, f.dmass[tid] = 0;
            __syncthreads();
            const auto add = [&](uint32_t key, int i) {
                const uint64_t comp = (uint64_t)key << 24 | (0xffffff - (uint32_t)i);
                if ((comp >> shift >> 8) != prefix) return;
                const int d = 255 - (int)(comp >> shift & 255);
                atomicAdd(f.dcount + d, 1u);
                if (b < kFineBins - 1)
                    atomicAdd((unsigned long long *)f.dmass + d,
                              (unsigned long long)(rel(scaled(ord2f(key)), b) * unit + 0.5));
            };
            if (list) for (int i = tid; i < (int)f.listed; i += kThreads) add(f.key[i], f.index[i]);
            else each([&](float v, int i) { if (bin_at(scaled(v)) == b) add(f2ord(v), i); });
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
            int cr = cs;
            uint64_t mr = ms;
            for (int o = 1; o < 64; o <<= 1) {
                const int u = __shfl_up(cr, o);
                const uint64_t v = __shfl_up((unsigned long long)mr, o);
                if (lane >= o) cr += u, mr += v;
            }
            cr -= cs, mr -= ms;
            int digit = -1, there = -1;          // where it ends; the last digit that has any
            int c_at = 0, c_there = 0, n_at = 0, n_there = 0;
            uint64_t m_at = 0, m_there = 0, w_at = 0, w_there = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (dc[i] > 0) {
                    there = 4 * lane + i, c_there = cr, m_there = mr, n_there = dc[i], w_there = dm[i];
                    const bool ends = by_mass ? (double)(most + mr + dm[i]) >= want : e.kept + cr + dc[i] >= count;
                    if (digit < 0 && ends) digit = there, c_at = cr, m_at = mr, n_at = dc[i], w_at = dm[i];
                }
                cr += dc[i], mr += dm[i];
            }
            uint64_t hit = __ballot(digit >= 0);
            int src;
            if (hit) {
                src = __builtin_ctzll(hit);
            } else {
                hit = __ballot(there >= 0);
                src = 63 - __builtin_clzll(hit);
                digit = there, c_at = c_there, m_at = m_there, n_at = n_there, w_at = w_there;
            }
            digit = __shfl(digit, src);
            e.kept += __shfl(c_at, src);
            most += __shfl((unsigned long long)m_at, src);
            n_at = __shfl(n_at, src);
            w_at = __shfl((unsigned long long)w_at, src);
            prefix = prefix << 8 | (uint64_t)(255 - digit);
            __syncthreads();
            if (n_at == 1 || (!by_mass && e.kept + n_at == count)) {     // all of this digit
                e.comp = prefix << shift;
                e.kept += n_at;
                most += w_at;
                break;
            }
        }
        e.mass = (double)most * back * f.edge[b];
        return e;
    };
    // the cumulative count and mass before bin b
    const auto before = [&](int b, int &above, double &mass) {
        __syncthreads();
        if (tid == b >> 1) {
            f.above = cb + (b & 1 ? c[0] : 0);
            f.before = mb + (b & 1 ? m[0] : 0.0);
        }
        __syncthreads();
        above = f.above;
        mass = f.before;
    };
    Edge end{kFineBins, 0, total, mall};
    const auto cut = [&](const Edge &e) {
        if (e.bin < end.bin || (e.bin == end.bin && e.comp > end.comp)) end = e;
    };
    if (s.k > 0 && s.k < total) {
        if (tid == 0) f.bin = 0;
        __syncthreads();
        if (cb < s.k && cb + c[0] + c[1] >= s.k) f.bin = 2 * tid + (cb + c[0] < s.k);
        __syncthreads();
        const int b = f.bin;
        int above;
        double mass;
        before(b, above, mass);
        Edge e = refine(b, false, s.k - above, 0.0);
        e.kept += above;
        e.mass += mass;
        cut(e);
    }
    if (s.p < 1.f) {
        const double want = (double)s.p * end.mass;
        __syncthreads();
        if (tid == 0) f.bin_p = kFineBins;
        __syncthreads();
        const int b0 = mb + m[0] >= want && c[0] ? 2 * tid : mb + m[0] + m[1] >= want && c[1] ? 2 * tid + 1 : kFineBins;
        if (b0 < kFineBins) atomicMin(&f.bin_p, b0);
        __syncthreads();
        const int b = f.bin_p;
        if (b < kFineBins - 1 && b <= end.bin) {
            int above;
            double mass;
            before(b, above, mass);
            Edge e = refine(b, true, 0, (want - mass) / f.edge[b]);
            e.kept += above;
            e.mass += mass;
            cut(e);
        }
    }
    if (s.mp > 0.f) {
        const int b = bin_at(-log((double)s.mp));
        __syncthreads();
        if (tid == 0) f.least = 0xffffffffu, f.listed = 0, f.dmass[0] = 0;
        __syncthreads();
        each([&](float v, int) {
            const double t = scaled(v);
            if (bin_at(t) != b || !(exp(-t) >= (double)s.mp)) return;
            atomicMin(&f.least, f2ord(v));
            atomicAdd(&f.listed, 1u);
            if (b < kFineBins - 1) atomicAdd((unsigned long long *)f.dmass, (unsigned long long)(rel(t, b) * unit + 0.5));
        });
        __syncthreads();
        int above;
        double mass;
        before(b, above, mass);
        // (a comp that no token reaches where the bin has none)
        Edge e{b, f.listed ? (uint64_t)f.least << 24 : ~0ull, above + (int)f.listed, mass + (double)f.dmass[0] * back * f.edge[b]};
        __syncthreads();
        cut(e);
    }
    const auto src = [&](int i, int e, auto fn) {
        const Eight<T> x = load_eight(z, i, e);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float v = RowElem<T>::get(x.v[j]) + 0.f;
            const double t = scaled(v);
            const int b = bin_at(t);
            const bool kept = v > kNegInf && (b < end.bin || (b == end.bin && ((uint64_t)f2ord(v) << 24 | (0xffffff - (uint32_t)(i + j))) >= end.comp));
            fn(j, kept, false, kept && b < kFineBins - 1 ? f.edge[b] * rel(t, b) : 0.0);
        }
    };
    const int token = locate(src, 0, V, 0.0, Drawn{(double)s.u * end.mass, s.u, 0}, f.ranges);
    if (tid == 0) {
        a.token[row] = token;
        if (a.logp) a.logp[row] = (float)(-scaled(RowElem<T>::get(z[token])) - log(end.mass));
        if (a.kept) a.kept[row] = end.kept;
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_fine_kernel(SampleArgs a) {
    __shared__ FinePool f;
    sample_fine<T>(a, blockIdx.x, settings_of(a, blockIdx.x), f);
}

// ---------------------------------------------------------------------------- coarse bins
struct CoarsePool {
    double weight[kSlots * 128];
    uint32_t count[kSlots * 128];
    uint64_t blocks[kMostParts][2];
    Range ranges[kRanges];
    uint32_t used[4], flags;
    uint8_t slot[kBlocks], block[kSlots];
    int first, bin_k, ties_k, bin_p, bin_m, above;
    double mass;
};
struct CoarseRow : CoarsePool { uint32_t hist[kBins / 2]; };   // of a row that is counted here

template <bool SPLIT>
__global__ __launch_bounds__(kThreads) void sample_coarse_kernel(SampleArgs a, Parts parts) {
    using Pool = std::conditional_t<SPLIT, CoarsePool, CoarseRow>;
    __shared__ union Shared {
        Pool c;
        FinePool f;
        __device__ Shared() {}
    } pool;
    Pool &f = pool.c;
    constexpr int kPer = kSlots * 128 / kThreads;
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int V = a.vocab, S = parts.count;
    const uint16_t *z = (const uint16_t *)a.logits.p + row * a.logits.st;
    const char *part = a.work + (int64_t)row * S * kPartBytes;
    const Settings s = settings_of(a, row);

    // ---- the blocks in use, and the counts of their bins
    if (tid < 4) f.used[tid] = 0;
    if (tid == 4) f.flags = 0, f.first = kSlots * 128, f.bin_k = f.bin_p = kSlots * 128, f.bin_m = -1;
    if constexpr (!SPLIT)
        for (int i = tid; i < kBins / 2; i += kThreads) f.hist[i] = 0;
    __syncthreads();
    if constexpr (SPLIT) {
        if (tid < S) {
            const PartHead h = *(const PartHead *)(part + tid * kPartBytes);
            f.blocks[tid][0] = h.blocks[0];
            f.blocks[tid][1] = h.blocks[1];
            for (int i = 0; i < 4; ++i) atomicOr(f.used + i, (uint32_t)(h.blocks[i >> 1] >> (i & 1) * 32));
            if (h.flags) atomicOr(&f.flags, (uint32_t)h.flags);
        }
    } else {
        const int flags = count_bins<kThreads>(z, 0, V, f.hist);
        if (flags) atomicOr(&f.flags, (uint32_t)flags);
        __syncthreads();
        for (int b = wave; b < kBlocks; b += kWaves)
            if (__ballot(f.hist[b * 64 + lane] != 0) && lane == 0) atomicOr(f.used + (b >> 5), 1u << (b & 31));
    }
    __syncthreads();
    int slots = 0;
    for (int i = 0; i < 4; ++i) slots += __popc(f.used[i]);
    if ((f.flags & 1) || slots == 0 || !s.ok) return no_answer(a, row);
    bool fine = (f.flags & 2) || slots > kSlots;
    const int bins = slots * 128;
    if (!fine) {
        if (tid < kBlocks) {
            int at = 0;
            for (int i = 0; i < 4; ++i) {
                const int from = tid - 32 * i;
                at += from >= 32 ? __popc(f.used[i]) : from > 0 ? __popc(f.used[i] & ((1u << from) - 1)) : 0;
            }
            const bool in = f.used[tid >> 5] >> (tid & 31) & 1;
            f.slot[tid] = in ? at : 255;
            if (in) f.block[at] = tid;
        }
        __syncthreads();
        for (int i = tid; i < slots * 64; i += kThreads) {
            const int b = f.block[i >> 6], pair = b * 64 + (i & 63);
            uint32_t c0 = 0, c1 = 0;
            if constexpr (SPLIT) {
                for (int q = 0; q < S; ++q) {
                    if (!(f.blocks[q][b >> 6] >> (b & 63) & 1)) continue;
                    const uint32_t x = ((const uint32_t *)(part + q * kPartBytes + 64))[pair];
                    c0 += x & 0xffffu;
                    c1 += x >> 16;
                }
            } else {
                c0 = f.hist[pair] & 0xffffu;
                c1 = f.hist[pair] >> 16;
            }
            f.count[2 * i] = c0;
            f.count[2 * i + 1] = c1;
            if (c0 | c1) atomicMin(&f.first, 2 * i + (c0 == 0));
        }
        __syncthreads();
    }
    const auto bin_at = [&](int i) { return f.block[i >> 7] * 128 + (i & 127); };
    double zmax = 0.0;
    const double t = (double)s.temp;
    int c[kPer], cs = 0, cb = 0, n = 0;
    double ms = 0.0, mb = 0.0, mall = 0.0;
    const int b0 = tid * kPer;
    if (!fine) {
        const int top = bin_at(f.first);
        zmax = (double)value_of(top);
        // values below -2^15 are counted only: their weights vanish, or the row is not for these bins
        const bool below = f.used[kBelow >> 12] >> (kBelow >> 7 & 31) & 1;
        fine = top == kBelow || (below && (zmax + 32768.0) / t < 800.0);
    }
    if (!fine) {
        for (int i = tid; i < bins; i += kThreads) {
            const int b = bin_at(i);
            f.weight[i] = f.count[i] && b != kBelow ? exp(((double)value_of(b) - zmax) / t) : 0.0;
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
        // some of the values below -2^15, and they matter for the token: their order does
        fine = end < bins && bin_at(end) == kBelow && (s.u == 0.f || s.u == 1.f) && ties < (int)f.count[end];
    }
    if (fine) {
        __syncthreads();
        return sample_fine<uint16_t>(a, row, s, pool.f);
    }
    const int kept = f.above;
    const double tie_weight = end < bins ? f.weight[end] : 0.0;
    Drawn d{(double)s.u * all, s.u, ties};
    int begin = 0, stop = V;
    if constexpr (SPLIT) {
        for (int q = wave; q < S; q += kWaves) {
            Range x{0.0, 0, 0};
            const uint32_t *hist = (const uint32_t *)(part + q * kPartBytes + 64);
            for (int i = lane; i < slots * 64 && 2 * (i - lane) <= end; i += 64) {
                const int b = f.block[i >> 6];
                if (!(f.blocks[q][b >> 6] >> (b & 63) & 1)) continue;
                const uint32_t y = hist[b * 64 + (i & 63)];
                const int n0 = (int)(y & 0xffffu), n1 = (int)(y >> 16);
                if (2 * i < end && n0) x.mass += n0 * f.weight[2 * i], x.kept += n0;
                if (2 * i + 1 < end && n1) x.mass += n1 * f.weight[2 * i + 1], x.kept += n1;
                x.ties += 2 * i == end ? n0 : 2 * i + 1 == end ? n1 : 0;
            }
            for (int o = 32; o > 0; o >>= 1) {
                x.mass += __shfl_xor(x.mass, o);
                x.kept += __shfl_xor(x.kept, o);
                x.ties += __shfl_xor(x.ties, o);
            }
            if (lane == 0) f.ranges[q] = x;
        }
        __syncthreads();
        const int q = max(0, pick_range(f.ranges, S, tie_weight, d));
        begin = q * parts.len;
        stop = min(V, begin + parts.len);
    }
    const auto src = [&](int i, int e, auto fn) {
        const Eight<uint16_t> x = load_eight(z, i, e);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int b = bin_of(x.v[j]);
            const int at = b >= 0 ? f.slot[b >> 7] * 128 + (b & 127) : 1 << 20;
            fn(j, at < end, at == end, at < end ? f.weight[at] : 0.0);
        }
    };
    const int token = locate(src, begin, stop, tie_weight, d, f.ranges);
    if (tid == 0) {
        a.token[row] = token;
        if (a.logp) a.logp[row] = (float)(((double)bf16_bits_to_f32(z[token]) - zmax) / t - log(all));
        if (a.kept) a.kept[row] = kept;
    }
}

}  // namespace

int64_t sample_bytes(const SampleArgs &a, bool bf16) {
    if (!bf16 || a.rows == 0) return 0;
    const Parts p = parts_of(a.rows, a.vocab);
    return p.count == 1 || p.count > kMostParts ? 0 : (int64_t)a.rows * p.count * kPartBytes;
}

hipError_t launch_sample(const SampleArgs &a, bool bf16, hipStream_t st) {
    if (!bf16) {
        sample_fine_kernel<float><<<a.rows, kThreads, 0, st>>>(a);
        return hipGetLastError();
    }
    const Parts p = parts_of(a.rows, a.vocab);
    if (p.count > kMostParts) {
        sample_fine_kernel<uint16_t><<<a.rows, kThreads, 0, st>>>(a);
        return hipGetLastError();
    }
    if (p.count == 1) {
        sample_coarse_kernel<false><<<a.rows, kThreads, 0, st>>>(a, p);
        return hipGetLastError();
    }
    sample_parts_kernel<<<dim3(a.rows, p.count), kPartThreads, 0, st>>>(a, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    sample_coarse_kernel<true><<<a.rows, kThreads, 0, st>>>(a, p);
    return hipGetLastError();
}

}  // namespace olive
