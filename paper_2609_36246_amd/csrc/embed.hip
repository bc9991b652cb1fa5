// Rows of an embedding table by tokens, and the table's gradient by sorted tokens.
//
// The gradient: tokens are sorted with their positions (in tiles of 2048 in LDS, then up to 64 sorted
// segments are merged at a time), the sorted list is cut into blocks of equal length, and a wavefront adds
// the rows of a block, 16 bytes a lane, run by run. A run inside a block goes to the table at once;
// of one that crosses a border each block leaves a partial row, which a last pass adds in order. So a
// token that is everywhere is shared by many wavefronts, and the order of additions does not depend on
// what runs when. Bound by memory: 29500 rows of 2048 bf16 (of 32768 tokens) added to a gradient of
// 151936 fp32 rows take 103 us, 76 of them the sums (4.0 TB/s; a row's table row is asked for
// with the row that ends its sum: the call takes 109 where it is asked for at the sum's end), 8 the sort, 10
// the merge and 5 the last pass; written whole, 8192 tokens of 1536 take 213 us (192 for sums and zeros, 4.9
// TB/s). 32768 rows of 2048 by their tokens: 30 us.
#include "rows.hpp"
#include "tokens_internal.hpp"
#include "wave_ops.hpp"

namespace olive {
namespace {

__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// ------------------------------------------------------------------------------------ rows
// Wavefront w: token w / chunks, lots (w % chunks) * per ... of its row.
template <typename T, bool TAIL>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a, int chunks, int per) {
    constexpr int L = kLot<T>;
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)block_index() * 4 + wave_index();
    const int64_t t = w / chunks;
    if (t >= a.tokens) return;
    const int begin = (int)(w % chunks) * per, end = min(a.width, begin + per);
    const int id = a.ids[t];
    const bool there = id >= 0 && id < a.vocab;
    const T *src = (const T *)a.table.p + (there ? id : 0) * a.table.st;
    T *dst = (T *)a.out.p + t * a.out.st;
    for (int i = begin + lane * L; i < end; i += 64 * L) {
        float x[L];
        if (there) {
            if constexpr (TAIL) unpack_lot<T>(load_lot(src, i, end, 0), x);
            else unpack_lot<T>(read_lot(src + i), x);
#pragma unroll
            for (int j = 0; j < L; ++j) x[j] *= a.scale;
        } else {
#pragma unroll
            for (int j = 0; j < L; ++j) x[j] = id < 0 ? 0.f : __builtin_nanf("");
        }
        if constexpr (TAIL) store_lot(dst, i, end, pack_lot<T>(x));
        else write_lot(dst + i, pack_lot<T>(x), a.stream);
    }
}

// ------------------------------------------------------------------------------------ sort
constexpr int kTile = 2048, kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kRounds = kTile / kSortThreads, kDigit = 9;
constexpr int kFan = 64;                         // segments that a pass merges into one

// A token's place in the order: its id, `vocab` for those that have no gradient.
__device__ __forceinline__ uint32_t key_of(const EmbedArgs &a, int id) {
    return id >= 0 && id < a.vocab ? (uint32_t)id : (uint32_t)a.vocab;
}

// Sorts a tile by a digit of the key at a time (at most 9 bits, as many each), stably: a wavefront has 128
// tokens, ranks 64 of them at a time by comparing digits (a ballot a bit), and keeps its own
// counts. 18 bits take two passes, 8 us in all (three passes on tiles of 4096: 15): a chain of waits.
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(EmbedArgs a, uint32_t *keys, int32_t *places, int bits,
                                                                  int digit) {
    __shared__ uint32_t key[2][kTile];
    __shared__ uint16_t place[2][kTile];
    __shared__ uint32_t count[kSortWaves][1 << kDigit];
    __shared__ uint32_t join[kSortWaves];
    constexpr int kPer = (kSortWaves << kDigit) / kSortThreads, kSplit = kSortWaves / kPer;
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_index();
    const int first = blockIdx.x * kTile, n = min(kTile, a.tokens - first);
    const uint32_t mask = (1u << digit) - 1;
    for (int i = tid; i < kTile; i += kSortThreads) {
        key[0][i] = i < n ? key_of(a, a.ids[first + i]) : 0xffffffffu;
        place[0][i] = (uint16_t)i;
    }
    int from = 0;
    for (int shift = 0; shift < bits; shift += digit, from ^= 1) {
        for (int i = tid; i < kSortWaves << kDigit; i += kSortThreads) (&count[0][0])[i] = 0;
        __syncthreads();
        uint32_t k[kRounds], p[kRounds], rank[kRounds];
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            k[r] = key[from][(wave * kRounds + r) * 64 + lane];
            p[r] = place[from][(wave * kRounds + r) * 64 + lane];
        }
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const uint32_t d = k[r] >> shift & mask;
            uint64_t same = ~0ull;
#pragma unroll
            for (int b = 0; b < kDigit; ++b) {
                const bool set = d >> b & 1;
                const uint64_t m = __ballot(set);
                same &= set ? m : ~m;
            }
            const int lead = __builtin_ctzll(same);
            uint32_t before = 0;
            if (lane == lead) before = atomicAdd(&count[wave][d], (uint32_t)__popcll(same));
            rank[r] = __shfl(before, lead) + (uint32_t)__popcll(same & ((1ull << lane) - 1));
        }
        __syncthreads();
        // counts before: of smaller digits, then of the same digit in wavefronts before
        uint32_t c[kPer], s = 0;
        const int d0 = tid / kSplit, w0 = tid % kSplit * kPer;
#pragma unroll
        for (int i = 0; i < kPer; ++i) s += c[i] = count[w0 + i][d0];
        uint32_t at = wave_scan(s);
        if (lane == 63) join[wave] = at;
        __syncthreads();
        at -= s;
        for (int i = 0; i < wave; ++i) at += join[i];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            count[w0 + i][d0] = at;
            at += c[i];
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const uint32_t to = count[wave][k[r] >> shift & mask] + rank[r];
            key[from ^ 1][to] = k[r];
            place[from ^ 1][to] = (uint16_t)p[r];
        }
        __syncthreads();
    }
    for (int i = tid; i < n; i += kSortThreads) {
        keys[first + i] = key[from][i];
        places[first + i] = first + place[from][i];
    }
}

// Merges groups of up to kFan sorted segments of `len`: a token moves on by the number of tokens of
// the group's other segments before it. A workgroup has kWindow tokens of one segment; four threads a
// token search a quarter of the segments each, two side by side: first among 64 keys of each segment
// that lie in LDS, then between two of them. (A search is a chain of waits: of 16 segments of 2048 without
// the keys in LDS 12.6 us a pass.)
constexpr int kWindow = 256, kSamples = 64;

__global__ __launch_bounds__(4 * kWindow) void embed_merge_kernel(EmbedArgs a, const uint32_t *keys, const int32_t *places,
                                                                  uint32_t *keys_to, int32_t *places_to, int64_t len) {
    __shared__ uint32_t samples[kFan][kSamples + 1];
    __shared__ int32_t moves[4][kWindow];
    const int p = threadIdx.x % kWindow, quarter = threadIdx.x / kWindow;
    const int64_t first = (int64_t)blockIdx.x * kWindow, group = first / (len * kFan) * (len * kFan);
    const int own = (int)((first - group) / len), stride = (int)(len / kSamples);
    const int segments = (int)min((int64_t)kFan, (a.tokens - group + len - 1) / len);
    const bool live = first + p < a.tokens;
    const uint32_t k = live ? keys[first + p] : 0;
    for (int i = threadIdx.x; i < segments * kSamples; i += 4 * kWindow) {
        const int64_t at = group + i / kSamples * len + i % kSamples * stride;
        samples[i / kSamples][i % kSamples] = at < a.tokens ? keys[at] : 0xffffffffu;
    }
    __syncthreads();
    int move = 0;
    if (live)
        for (int s0 = quarter; s0 < segments; s0 += 8) {
            int64_t start[2];
            int lo[2], left[2];
            uint32_t want[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int s = s0 + 4 * i;
                const bool there = s < segments && s != own;
                start[i] = group + (there ? s : own) * len;
                want[i] = k + (s < own);                     // (of the segments before also the equal ones)
                int m = 0;                                   // samples before
#pragma unroll
                for (int step = kSamples; step > 0; step >>= 1)
                    if (there && m + step <= kSamples && samples[s][m + step - 1] < want[i]) m += step;
                lo[i] = m > 0 ? (m - 1) * stride + 1 : 0;
                left[i] = m > 0 ? max(0, (int)min((int64_t)stride - 1, min(len, a.tokens - start[i]) - lo[i])) : 0;
            }
            while (left[0] | left[1]) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int half = left[i] >> 1;
                    const bool less = left[i] > 0 && keys[start[i] + lo[i] + half] < want[i];
                    lo[i] = less ? lo[i] + half + 1 : lo[i];
                    left[i] = less ? left[i] - half - 1 : half;
                }
            }
            move += lo[0] + lo[1];
        }
    moves[quarter][p] = move;
    __syncthreads();
    if (quarter || !live) return;
    const int64_t to = first + p - own * len + moves[0][p] + moves[1][p] + moves[2][p] + moves[3][p];
    keys_to[to] = k;
    places_to[to] = places[first + p];
}

// ------------------------------------------------------------------------------------ sums
// N elements of TT at any alignment.
template <typename TT, int N>
struct Piece {
    static constexpr int kWords = N * (int)sizeof(TT) / 4;
    struct __attribute__((packed, aligned(sizeof(TT)))) Loose { uint32_t w[kWords]; };
    static __device__ __forceinline__ void get(const TT *p, float (&x)[N]) {
        const Loose u = *(const Loose *)p;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if constexpr (sizeof(TT) == 4) x[j] = __uint_as_float(u.w[j]);
            else x[j] = __uint_as_float(j & 1 ? u.w[j >> 1] & 0xffff0000u : u.w[j >> 1] << 16);
        }
    }
    static __device__ __forceinline__ void put(TT *p, const float (&x)[N]) {
        Loose u;
#pragma unroll
        for (int j = 0; j < kWords; ++j) {
            if constexpr (sizeof(TT) == 4) u.w[j] = __float_as_uint(x[j]);
            else u.w[j] = pack_bf16x2(x[2 * j], x[2 * j + 1]);
        }
        *(Loose *)p = u;
    }
};

// A lane's N columns from c on of a table's row: what is there, where the sums are added to it.
template <typename TT, int N, bool TAIL>
__device__ __forceinline__ void from_table(const EmbedArgs &a, uint32_t id, int c, float (&x)[N]) {
    const TT *row = (const TT *)a.table.p + id * a.table.st;
    if (c + N <= a.width) {
        Piece<TT, N>::get(row + c, x);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = TAIL && j < N - 1 && c + j < a.width ? RowElem<TT>::get(row[c + j]) : 0.f;
    }
}
// And what goes there: scale * sum + x.
template <typename TT, int N, bool TAIL>
__device__ __forceinline__ void to_table(const EmbedArgs &a, uint32_t id, int c, const float (&sum)[N], float (&x)[N]) {
    TT *row = (TT *)a.table.p + id * a.table.st;
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = fmaf(sum[j], a.scale, x[j]);
    if (c + N <= a.width) {
        Piece<TT, N>::put(row + c, x);
    } else if (TAIL) {
#pragma unroll
        for (int j = 0; j < N - 1; ++j)
            if (c + j < a.width) row[c + j] = RowElem<TT>::put(x[j]);
    }
}

template <typename T, bool TAIL>
__device__ __forceinline__ Lot load_grad(const EmbedArgs &a, int place, int c) {
    const T *row = (const T *)a.out.p + place * a.out.st;
    if constexpr (TAIL) return load_lot(row, c, a.width, 0);
    if (c < a.width) return read_lot(row + c);
    return Lot{{0, 0, 0, 0}};
}

constexpr int kAhead = 8;

struct Sorted {
    const uint32_t *keys;
    const int32_t *places;
    float *part;                                 // [blocks][2][width rounded up to a lane's columns]
    int rows, blocks, chunks;                    // sorted tokens a block; columns' chunks
    int64_t sums;                                // workgroups of sums, before those that write zeros
};

// A wavefront: the sums of one block's runs in one chunk of the columns. Behind them, wavefronts that
// write zeros into the rows of 64 ids each that do not occur.
template <typename T, typename TT, bool TAIL>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedArgs a, Sorted s) {
    constexpr int L = kLot<T>;
    const int lane = threadIdx.x & 63;
    const int64_t g = block_index();
    if (g >= s.sums) {
        const int64_t r0 = ((g - s.sums) * 4 + wave_index()) * 64, r = r0 + lane;
        if (r0 >= a.vocab) return;
        int lo = 0, left = a.tokens;
        while (left > 0) {
            const int half = left >> 1;
            const bool less = s.keys[lo + half] < (uint32_t)r;
            lo = less ? lo + half + 1 : lo;
            left = less ? left - half - 1 : half;
        }
        uint64_t absent = __ballot(r < a.vocab && !(lo < a.tokens && s.keys[lo] == (uint32_t)r));
        constexpr int N = 16 / (int)sizeof(TT);
        for (; absent; absent &= absent - 1) {
            TT *row = (TT *)a.table.p + (r0 + __builtin_ctzll(absent)) * a.table.st;
            for (int c = lane * N; c < a.width; c += 64 * N) {
                if (c + N <= a.width) {
                    write_lot(row + c, Lot{{0, 0, 0, 0}});
                } else {
                    for (int j = c; j < a.width; ++j) row[j] = (TT)0;
                }
            }
        }
        return;
    }
    const int64_t w = g * 4 + wave_index();
    const int b = (int)(w / s.chunks), c = ((int)(w % s.chunks) * 64 + lane) * L;
    if (b >= s.blocks) return;
    const int64_t p0 = (int64_t)b * s.rows;
    const int n = (int)min((int64_t)s.rows, a.tokens - p0);
    const uint32_t key = lane < n ? s.keys[p0 + lane] : 0xffffffffu;
    const int place = lane < n ? s.places[p0 + lane] : 0;
    const uint32_t prev = p0 > 0 ? s.keys[p0 - 1] : 0xffffffffu, next = p0 + n < a.tokens ? s.keys[p0 + n] : 0xffffffffu;
    const int there = __popcll(__ballot(key < (uint32_t)a.vocab));       // (the others are at the end)
    if (there == 0) return;
    // kAhead rows on their way together, and the table's rows of the runs that end among them
    float sum[L] = {};
#pragma unroll 1
    for (int e0 = 0; e0 < there; e0 += kAhead) {
        Lot x[kAhead];
        float old[kAhead][L];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int e = min(e0 + j, there - 1);
            x[j] = load_grad<T, TAIL>(a, wave_read(place, e), c);
            const uint32_t k = wave_read(key, e);
#pragma unroll
            for (int i = 0; i < L; ++i) old[j][i] = 0.f;
            if (a.accumulate && (e == there - 1 || wave_read(key, min(e + 1, 63)) != k))
                from_table<TT, L, TAIL>(a, k, c, old[j]);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int e = e0 + j;
            if (e >= there) break;
            const uint32_t k = wave_read(key, e);
            float v[L];
            unpack_lot<T>(x[j], v);
#pragma unroll
            for (int i = 0; i < L; ++i) sum[i] += v[i];
            if (e < there - 1 && wave_read(key, e + 1) == k) continue;
            const bool from_before = k == prev, goes_on = e == n - 1 && k == next;
            if (from_before || goes_on) {
                Piece<float, L>::put(s.part + ((int64_t)b * 2 + !from_before) * s.chunks * 64 * L + c, sum);
            } else {
                to_table<TT, L, TAIL>(a, k, c, sum, old[j]);
            }
#pragma unroll
            for (int i = 0; i < L; ++i) sum[i] = 0.f;
        }
    }
}

// Adds the sums of a workgroup's four wavefronts, in order, in the first one (of which it says so).
template <int L>
__device__ __forceinline__ bool add_waves(float (&sum)[L]) {
    __shared__ float join[3][64][L + 1];
    const int lane = threadIdx.x & 63, wave = wave_index();
    if (wave)
#pragma unroll
        for (int j = 0; j < L; ++j) join[wave - 1][lane][j] = sum[j];
    __syncthreads();
    if (wave) return false;
#pragma unroll
    for (int i = 0; i < 3; ++i)
#pragma unroll
        for (int j = 0; j < L; ++j) sum[j] += join[i][lane][j];
    return true;
}

// The runs that cross a border: the block where one begins adds what the blocks have left of it.
template <typename T, typename TT, bool TAIL>
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedArgs a, Sorted s) {
    constexpr int L = kLot<T>;
    const int64_t g = block_index();
    const int b = (int)(g / s.chunks), lane = threadIdx.x & 63, wave = wave_index();
    const int c = ((int)(g % s.chunks) * 64 + lane) * L;
    if (b + 1 >= s.blocks) return;
    const int64_t p0 = (int64_t)b * s.rows, p1 = p0 + s.rows;
    const uint32_t run = s.keys[p1 - 1];
    if (run >= (uint32_t)a.vocab || s.keys[p1] != run || (p0 > 0 && s.keys[p0 - 1] == run)) return;
    // blocks after this one whose first token is of the run
    int more = 1;
    for (int64_t i = b + 2; i < s.blocks; i += 64) {
        const uint64_t in = __ballot(i + lane < s.blocks && s.keys[(i + lane) * s.rows] == run);
        more += __popcll(in);
        if (in != ~0ull) break;
    }
    const auto part = [&](int64_t block, int slot) { return s.part + (block * 2 + slot) * s.chunks * 64 * L + c; };
    float sum[L] = {};
    if (wave == 0) Piece<float, L>::get(part(b, 1), sum);
#pragma unroll 4
    for (int i = wave; i < more; i += 4) {
        float x[L];
        Piece<float, L>::get(part(b + 1 + i, 0), x);
#pragma unroll
        for (int j = 0; j < L; ++j) sum[j] += x[j];
    }
    if (!add_waves(sum)) return;
    float x[L] = {};
    if (a.accumulate) from_table<TT, L, TAIL>(a, run, c, x);
    to_table<TT, L, TAIL>(a, run, c, sum, x);
}

template <typename TT>
__global__ __launch_bounds__(256) void embed_zero_kernel(EmbedArgs a) {
    constexpr int N = 16 / (int)sizeof(TT);
    for (int64_t r = blockIdx.x; r < a.vocab; r += gridDim.x) {
        TT *row = (TT *)a.table.p + r * a.table.st;
        for (int c = threadIdx.x * N; c < a.width; c += 256 * N) store_lot(row, c, a.width, Lot{{0, 0, 0, 0}});
    }
}
// Few tokens: the workgroup of a token's first occurrence finds the others, 64 tokens a wavefront, and adds
// their rows. Bound by waits: 1024 drawn of 32000 as text is, 2048 wide, 8 us, all the same 27 (by
// one wavefront, a row at a time, 16 and 193; sorted, 22 and 18).
template <typename T, typename TT, bool TAIL>
__global__ __launch_bounds__(256) void embed_few_kernel(EmbedArgs a, int chunks) {
    constexpr int L = kLot<T>;
    const int lane = threadIdx.x & 63, wave = wave_index();
    const int t = (int)blockIdx.x / chunks, c = ((int)blockIdx.x % chunks * 64 + lane) * L;
    const int id = a.ids[t];
    if (id < 0 || id >= a.vocab) return;
    bool before = false;
    for (int s = wave * 64; s < t; s += 256) before |= s + lane < t && a.ids[s + lane] == id;
    if (__syncthreads_or(before)) return;
    float sum[L] = {};
    for (int s = t + wave * 64; s < a.tokens; s += 256) {
        uint64_t m = __ballot(s + lane < a.tokens && a.ids[s + lane] == id);
        while (m) {
            Lot x[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                x[j] = Lot{{0, 0, 0, 0}};
                if (m) x[j] = load_grad<T, TAIL>(a, s + __builtin_ctzll(m), c);
                m &= m - 1;
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                float v[L];
                unpack_lot<T>(x[j], v);
#pragma unroll
                for (int i = 0; i < L; ++i) sum[i] += v[i];
            }
        }
    }
    if (!add_waves(sum)) return;
    float x[L] = {};
    if (a.accumulate) from_table<TT, L, TAIL>(a, (uint32_t)id, c, x);
    to_table<TT, L, TAIL>(a, (uint32_t)id, c, sum, x);
}

// ---------------------------------------------------------------------------------- launches
constexpr int kFew = 1024;                       // tokens up to which the first occurrences are looked for

// Sorted tokens a block: few where there are few tokens, so that wavefronts are enough, more where the partial
// rows of the borders would be many. Added to fp32 rows of 2048, by 16, 32 and 64 a block: 4096 tokens 30, 38
// and 55 us, 8192 38, 41 and 56, 16384 52, 53 and 61, 32768 98, 91 and 93, 65536 183, 178 and 170; to rows of
// 512, 8192 tokens 28, 37 and 52, 32768 43, 46 and 61, 131072 132, 122 and 124.
int block_rows(int64_t tokens) { return tokens >= 32768 ? 64 : tokens >= 8192 ? 32 : 16; }
int64_t up16(int64_t n) { return (n + 15) & ~(int64_t)15; }

struct Layout { int64_t keys[2], places[2], part, bytes; };

Layout layout_of(const EmbedArgs &a) {
    Layout l{};
    if (a.tokens <= kFew) return l;
    const int64_t n = up16((int64_t)a.tokens * 4), rows = block_rows(a.tokens);
    const int64_t blocks = (a.tokens + rows - 1) / rows, columns = ((int64_t)a.width + 511) / 512 * 512;
    l.keys[0] = 0, l.places[0] = n, l.keys[1] = 2 * n, l.places[1] = 3 * n;
    l.part = 4 * n;
    l.bytes = l.part + blocks * 2 * columns * (int64_t)sizeof(float);
    return l;
}

template <typename T>
hipError_t forward(const EmbedArgs &a, hipStream_t st) {
    constexpr int per = 64 * kLot<T>;
    const int chunks = (a.width + per - 1) / per;
    const dim3 grid = grid_of(((int64_t)a.tokens * chunks + 3) / 4);
    if (a.width % kLot<T>) embed_kernel<T, true><<<grid, 256, 0, st>>>(a, chunks, per);
    else embed_kernel<T, false><<<grid, 256, 0, st>>>(a, chunks, per);
    return hipGetLastError();
}

template <typename T, typename TT, bool TAIL>
hipError_t backward(const EmbedArgs &a, hipStream_t st) {
    const int per = 64 * kLot<T>, chunks = (a.width + per - 1) / per;
    if (a.tokens <= kFew) {
        if (!a.accumulate) {
            embed_zero_kernel<TT><<<a.vocab < 8192 ? a.vocab : 8192, 256, 0, st>>>(a);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess || a.tokens == 0) return e;
        }
        embed_few_kernel<T, TT, TAIL><<<a.tokens * chunks, 256, 0, st>>>(a, chunks);
        return hipGetLastError();
    }
    const Layout l = layout_of(a);
    uint32_t *keys[2] = {(uint32_t *)(a.work + l.keys[0]), (uint32_t *)(a.work + l.keys[1])};
    int32_t *places[2] = {(int32_t *)(a.work + l.places[0]), (int32_t *)(a.work + l.places[1])};
    int bits = 0;
    while (((int64_t)a.vocab >> bits) > 0) ++bits;
    const int tiles = (a.tokens + kTile - 1) / kTile;
    const int passes = (bits + kDigit - 1) / kDigit, digit = (bits + passes - 1) / passes;
    embed_sort_kernel<<<tiles, kSortThreads, 0, st>>>(a, keys[0], places[0], bits, digit);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    int at = 0;
    for (int64_t len = kTile; len < a.tokens; len *= kFan, at ^= 1) {
        embed_merge_kernel<<<(a.tokens + kWindow - 1) / kWindow, 4 * kWindow, 0, st>>>(a, keys[at], places[at], keys[at ^ 1], places[at ^ 1], len);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    Sorted s{};
    s.keys = keys[at];
    s.places = places[at];
    s.part = (float *)(a.work + l.part);
    s.rows = block_rows(a.tokens);
    s.blocks = (a.tokens + s.rows - 1) / s.rows;
    s.chunks = chunks;
    s.sums = ((int64_t)s.blocks * chunks + 3) / 4;
    const int64_t zeros = a.accumulate ? 0 : ((int64_t)a.vocab + 255) / 256;
    embed_sum_kernel<T, TT, TAIL><<<grid_of(s.sums + zeros), 256, 0, st>>>(a, s);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    embed_join_kernel<T, TT, TAIL><<<grid_of((int64_t)s.blocks * chunks), 256, 0, st>>>(a, s);
    return hipGetLastError();
}

template <typename T, typename TT>
hipError_t backward(const EmbedArgs &a, hipStream_t st) {
    return a.width % kLot<T> ? backward<T, TT, true>(a, st) : backward<T, TT, false>(a, st);
}

}  // namespace

int64_t embed_backward_bytes(const EmbedArgs &a) { return layout_of(a).bytes; }

hipError_t launch_embed(const EmbedArgs &a, bool bf16, hipStream_t st) {
    return bf16 ? forward<uint16_t>(a, st) : forward<float>(a, st);
}
hipError_t launch_embed_backward(const EmbedArgs &a, bool bf16, bool table_bf16, hipStream_t st) {
    if (bf16) return table_bf16 ? backward<uint16_t, uint16_t>(a, st) : backward<uint16_t, float>(a, st);
    return table_bf16 ? backward<float, uint16_t>(a, st) : backward<float, float>(a, st);
}

}  // namespace olive
