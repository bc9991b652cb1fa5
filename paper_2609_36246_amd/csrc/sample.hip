// The next token of rows of logits: temperature, top-k, top-p, min-p, from given numbers.
//
// A workgroup takes a row. What is kept is a run of the tokens in order (value, then index), so it
// is described by its last value and how many tokens of that value belong to it; the value is
// found bit by bit, from the counts or the masses of the tokens above a candidate.
#include "rows.hpp"
#include "tokens_internal.hpp"

namespace olive {
namespace {

constexpr int kThreads = 1024;

template <typename V>
__device__ __forceinline__ V block_sum(V v) {
    __shared__ V join[kThreads / 64];
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) join[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
    for (int i = 0; i < kThreads / 64; ++i) v += join[i];
    return v;
}

// The sum over the threads before this one, and over all.
template <typename V>
__device__ __forceinline__ V block_scan(V v, V &all) {
    __shared__ V join[kThreads / 64];
    const int lane = threadIdx.x & 63;
    V s = v;
    for (int o = 1; o < 64; o <<= 1) {
        const V u = __shfl_up(s, o);
        if (lane >= o) s += u;
    }
    __syncthreads();
    if (lane == 63) join[threadIdx.x >> 6] = s;
    __syncthreads();
    V before = 0;
    all = 0;
    for (int i = 0; i < kThreads / 64; ++i) {
        if (i < (int)(threadIdx.x >> 6)) before += join[i];
        all += join[i];
    }
    return before + (s - v);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
    const int row = blockIdx.x;
    const T *z = (const T *)a.logits.p + row * a.logits.st;
    // (-0 and 0 are the same value)
    const auto key_of = [&](int i) { return f2ord(RowElem<T>::get(z[i]) + 0.f); };
    const uint32_t kNone = f2ord(kNegInf);

    uint32_t top = 0;
    int n = 0, bad = 0;
    for (int i = threadIdx.x; i < a.vocab; i += kThreads) {
        const uint32_t k = key_of(i);
        const float x = ord2f(k);
        bad += !(x < __builtin_inff());
        n += k > kNone;
        top = max(top, k);
    }
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    __shared__ uint32_t tops[kThreads / 64];
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    n = block_sum(n);
    bad = block_sum(bad);
    for (int i = 0; i < kThreads / 64; ++i) top = max(top, tops[i]);

    const float u = a.uniform[row], temp = a.temperature ? a.temperature[row] : 1.f;
    float p = a.top_p ? a.top_p[row] : 1.f, mp = a.min_p ? a.min_p[row] : 0.f;
    int k = a.top_k ? a.top_k[row] : 0;
    if (bad || n == 0 || !(u >= 0.f && u <= 1.f) || !(temp >= 0.f && temp < __builtin_inff()) || p != p || mp != mp) {
        if (threadIdx.x == 0) {
            a.token[row] = -1;
            if (a.logp) a.logp[row] = __builtin_nanf("");
            if (a.kept) a.kept[row] = 0;
        }
        return;
    }
    const double zmax = (double)ord2f(top), t = temp > 0.f ? (double)temp : 1.0;
    if (temp == 0.f || mp > 1.f) k = 1, p = 1.f, mp = 0.f;
    const auto weight = [&](uint32_t key) { return exp(((double)ord2f(key) - zmax) / t); };
    const auto count = [&](uint64_t least) {     // tokens with at least this key
        int c = 0;
        for (int i = threadIdx.x; i < a.vocab; i += kThreads) c += key_of(i) >= least;
        return block_sum(c);
    };
    const auto mass = [&](uint64_t least) {
        double m = 0.0;
        for (int i = threadIdx.x; i < a.vocab; i += kThreads) {
            const uint32_t key = key_of(i);
            if (key >= least && key > kNone) m += weight(key);
        }
        return block_sum(m);
    };
    // kept: the tokens above the value `last`, and the first `ties` of that value
    uint32_t last = kNone;
    int ties = 0, above = n;
    if (k > 0 && k < n) {
        last = 0;
        for (int b = 31; b >= 0; --b)
            if (count(last | 1u << b) >= k) last |= 1u << b;
        above = count((uint64_t)last + 1);
        ties = k - above;
    }
    if (p < 1.f) {
        const double want = (double)p * (mass((uint64_t)last + 1) + (ties > 0 ? ties * weight(last) : 0.0));
        uint32_t key = 0;
        for (int b = 31; b >= 0; --b)
            if ((key | 1u << b) <= top && mass(key | 1u << b) >= want) key |= 1u << b;
        if (key > last || (key == last && ties > 0)) {
            above = count((uint64_t)key + 1);
            const int there = key == last ? ties : count(key) - above;
            const double before = mass((uint64_t)key + 1);
            ties = max(1, (int)fmin(ceil((want - before) / weight(key)), (double)there));
            last = key;
        }
    }
    if (mp > 0.f) {
        uint32_t key = 0;                        // the largest value whose weight is too small
        for (int b = 31; b >= 0; --b)
            if ((key | 1u << b) < top && !(weight(key | 1u << b) >= (double)mp)) key |= 1u << b;
        if (key >= last) {
            last = key;
            ties = 0;
            above = count((uint64_t)key + 1);
        }
    }
    const double all = mass((uint64_t)last + 1) + (ties > 0 ? ties * weight(last) : 0.0);
    const double want = (double)u * all;
    double before = 0.0;
    int seen = 0, newest = -1;
    __shared__ int found;
    if (threadIdx.x == 0) found = 0x7fffffff;
    __syncthreads();
    for (int i0 = 0; i0 < a.vocab; i0 += kThreads) {
        const int i = i0 + threadIdx.x;
        const uint32_t key = i < a.vocab ? key_of(i) : 0;
        int all_t;
        const int rank = seen + block_scan((int)(key == last), all_t);
        seen += all_t;
        const bool keep = key > last || (key == last && rank < ties);
        const double w = keep ? weight(key) : 0.0;
        double all_w;
        const double c = before + block_scan(w, all_w) + w;
        before += all_w;
        if (keep && (u == 0.f || (u < 1.f && c > want))) atomicMin(&found, i);
        if (keep) newest = i;
        __syncthreads();
        if (found != 0x7fffffff) break;
    }
    if (found == 0x7fffffff) {                   // u = 1: the last one kept
        __syncthreads();
        if (threadIdx.x == 0) found = -1;
        __syncthreads();
        atomicMax(&found, newest);
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        a.token[row] = found;
        if (a.logp) a.logp[row] = (float)(((double)ord2f(key_of(found)) - zmax) / t - log(all));
        if (a.kept) a.kept[row] = above + ties;
    }
}

}  // namespace

int64_t sample_bytes(const SampleArgs &, bool) { return 0; }

hipError_t launch_sample(const SampleArgs &a, bool bf16, hipStream_t st) {
    if (bf16) sample_kernel<uint16_t><<<a.rows, kThreads, 0, st>>>(a);
    else sample_kernel<float><<<a.rows, kThreads, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace olive
