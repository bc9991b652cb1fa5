// Pieces of the bf16 attention kernels on matrix instructions: the LDS tile of keys or query
// rows with its swizzle, the asynchronous loads into it, and the operand reads out of it.
//
// A tile row holds one head of one token: DP elements (head_dim rounded up to 64, 128 or
// 256) in 16-byte chunks. Chunk c of row r lies in slot c ^ swz(r). The two operand reads
// are then free of bank conflicts: ds_read_b128 of one chunk of 16 consecutive rows, and
// the transposing ds_read_b64_tr_b16 of 4 consecutive rows x 4 consecutive chunks.
#pragma once

#include "attn_seq.hpp"
#include "mfma_pipe.hpp"
#include "olive_device.hpp"

namespace olive {

typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));

#define OLIVE_LDS(T, addr) (*(__attribute__((address_space(3))) T *)(uintptr_t)(uint32_t)(addr))

template <int DP>
struct TileRow {
    static constexpr int CHUNKS = DP / 8;            // 16-byte chunks of a row
    static constexpr int BYTES = DP * 2;
    static constexpr int PER_DMA = 1024 / BYTES;     // rows of a wavefront's 1-KiB load
    static __device__ __forceinline__ int swz(int r) {
        return DP == 64 ? ((((r >> 1) & 1) << 2) | ((r >> 2) & 3))
                        : (((r & 3) << 2) | ((r >> 2) & 3));
    }
};

// Waits for this wavefront's loads into LDS, then for the workgroup's.
__device__ __forceinline__ void tile_barrier() {
    compiler_fence();
    __builtin_amdgcn_s_waitcnt(vmcnt_lgkm0_imm(0));
    __builtin_amdgcn_s_barrier();
    compiler_fence();
}

__device__ __forceinline__ int64_t uniform64(int64_t v) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
    const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)v >> 32));
    return (int64_t)(((uint64_t)hi << 32) | lo);
}

// dma16_sv (mfma_pipe.hpp) from a base that is the same for every lane, wherever it is held.
template <int OFF>
__device__ __forceinline__ void dma16_from(const char *base, uint32_t voff, uint32_t la) {
    dma16_sv<OFF>((const char *)uniform64((int64_t)base), voff, la);
}

// dma16 (mfma_pipe.hpp) with 4 bytes a lane.
__device__ __forceinline__ void dma4(const char *g, uint32_t la) {
    la = __builtin_amdgcn_readfirstlane(la);
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(la), "v"(g) : "memory", "m0");
#pragma clang diagnostic pop
}

// No scalar load is pending from here on: beside one, every wait for an LDS read would have to
// be a wait for all of them.
__device__ __forceinline__ void scalar_loads_done() { __builtin_amdgcn_s_waitcnt(0xC07F); }

// The larger of the two halves' values of a lane pair l, l + 32.
__device__ __forceinline__ float max_of_halves(float x) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// Keeps an address in its register: the compiler would otherwise form it again at each use
// rather than add a constant to it in the read.
__device__ __forceinline__ uint32_t pinned(uint32_t x) {
    asm("" : "+v"(x));
    return x;
}

// First operand (rows x K) of a 32-row block: row lane % 32, chunk 2 step + lane / 32.
template <int DP>
struct RowReader {
    uint32_t at[DP / 16];
    __device__ __forceinline__ void open(uint32_t base, int lane) {
        const int r = lane & 31;
#pragma unroll
        for (int s = 0; s < DP / 16; ++s)
            at[s] = pinned(base + r * TileRow<DP>::BYTES + (((2 * s + (lane >> 5)) ^ TileRow<DP>::swz(r)) << 4));
    }
    __device__ __forceinline__ bf16x8 read(int step, int offset) const { return OLIVE_LDS(bf16x8, at[step] + offset); }
    __device__ __forceinline__ void write(int step, int offset, bf16x8 x) const { OLIVE_LDS(bf16x8, at[step] + offset) = x; }
};

// First operand transposed (elements x rows) of a 16-row block: lane % 32 is the element
// 32 db + lane % 32, the 8 values are rows 4 (lane / 32) + 0..3 and 8 more: the rows whose
// results a lane of the same half holds in 8 registers of a 32 x 32 product.
template <int DP>
struct ColReader {
    uint32_t at[DP / 32][2];
    __device__ __forceinline__ void open(uint32_t base, int lane) {
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r = 8 * j + 4 * (lane >> 5) + ((lane & 15) >> 2);
                const int c = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
                at[d][j] = pinned(base + r * TileRow<DP>::BYTES + ((c ^ TileRow<DP>::swz(r)) << 4) + (lane & 1) * 8);
            }
    }
    __device__ __forceinline__ bf16x8 read(int db, int offset) const {
        const shortx4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(&OLIVE_LDS(shortx4, at[db][0] + offset));
        const shortx4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16(&OLIVE_LDS(shortx4, at[db][1] + offset));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

template <int N> struct Const { static constexpr int value = N; };

// Registers 8 m .. 8 m + 7 of a 32 x 32 product as the second operand of the next one.
__device__ __forceinline__ bf16x8 pack8(const floatx16 &s, int m) {
    uintx4 u;
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] = pack_bf16x2(s[8 * m + 2 * j], s[8 * m + 2 * j + 1]);
    return __builtin_bit_cast(bf16x8, u);
}

__device__ __forceinline__ floatx16 mfma(bf16x8 a, bf16x8 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ floatx16 zero16() { return (floatx16)(0.f); }

// Row of a 32 x 32 product that register i of a lane holds.
__device__ __forceinline__ int acc_row(int i, int lane) { return 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3); }

// A query row (one head of one token): rows are token major, the heads of a key head's group
// within.
__device__ __forceinline__ const uint16_t *head_row(const HeadsArg &h, int64_t t, int64_t head) {
    return (const uint16_t *)h.p + t * h.st + head * h.sh;
}

// The same 8-element chunks of a row as read_row gives, from memory (zeros past d).
__device__ __forceinline__ bf16x8 load_chunk(const uint16_t *row, int c, int nch) {
    uintx4 u = {0u, 0u, 0u, 0u};
    if (c < nch) u = *(const uintx4 *)(row + 8 * c);
    return __builtin_bit_cast(bf16x8, u);
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
// Tiles of n >= 0 keys or rows (the tile is a power of two known at compile time).
template <int TILE>
__device__ __forceinline__ int tiles_of(int n) { return (int)(((unsigned)n + TILE - 1) / TILE); }

inline int padded(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

// Consecutive workgroups go to the 8 dies in turn, each with a cache of its own. Runs of `run`
// consecutive units, which read the same keys or rows, go to one die, the runs to the dies in
// turn: a die that got one long stretch of units would get all the long ones.
struct DieOrder {
    int32_t units, blocks;
    Div run;
    static DieOrder of(int64_t units) {
        const int64_t r = units / 64, run = r < 1 ? 1 : r > 16 ? 16 : r;
        return DieOrder{(int32_t)units, (int32_t)(ceil_div(units, 8 * run) * 8 * run), Div::of(run)};
    }
    // >= units: nothing to do
    __device__ __forceinline__ int unit(int block) const {
        const int i = block >> 3, q = run.quot(i);
        return (q * 8 + (block & 7)) * (int)run.d + run.rem(i, q);
    }
};

// The row tiles of a sequence in chunks of a die's run, the last chunk of all sequences and heads
// first: under a causal mask the last rows see the most keys, and what starts late is short.
// (Sequence by sequence a fifth of the chip waited for the last ones: ragged prompts of 1200 to
// 6000 tokens, 16 heads of 64, 269 us, in this order 244, both on one card.)
constexpr int kRowChunk = 16;
struct RowOrder {
    int tiles, chunks;
    Div chunk;
    static RowOrder of(int64_t tiles) {
        const int64_t c = tiles < 1 ? 1 : tiles < kRowChunk ? tiles : kRowChunk;
        return RowOrder{(int)tiles, (int)ceil_div(tiles, c), Div::of(c)};
    }
    int64_t units() const { return (int64_t)chunks * chunk.d; }   // of a sequence, absent ones among them
    // Tile `in` of the i-th chunk in that order; -1: there is none.
    __device__ __forceinline__ int tile(int i, int in) const {
        const int t = (chunks - 1 - i) * (int)chunk.d + (int)chunk.d - 1 - in;
        return t < tiles ? t : -1;
    }
};

// Tiles [t0, t1) of part i of n.
__device__ __forceinline__ void part_range(int tiles, const Div &n, int i, int &t0, int &t1) {
    const int q = n.quot(tiles), r = n.rem(tiles, q);
    t0 = i * q + min(i, r);
    t1 = t0 + q + (i < r);
}

// One of two views, field by field: a reference that is chosen at run time would put all of a
// kernel's arguments into memory.
__device__ __forceinline__ HeadsArg pick(bool first, HeadsArg x, HeadsArg y) {
    return HeadsArg{first ? x.p : y.p, first ? x.st : y.st, first ? x.sh : y.sh};
}

// (a pointer that went through integers would be read as one that might point into LDS, and
// every wait for an LDS read beside such a load is a wait for all)
__device__ __forceinline__ const __attribute__((address_space(1))) int32_t *global_int(const int32_t *p) {
    return (const __attribute__((address_space(1))) int32_t *)p;
}

// What one workgroup does.
struct Work {
    SeqView s;
    int rows;                        // query rows of the range that begins at token s.q0
    int r0;                          // first of this workgroup's
    int kvh, part;
    int pt;                          // prefix tiles come first
    int t0, t1;
};

// The same for every lane, which the compiler cannot always tell from where it came from.
__device__ __forceinline__ int uniform32(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ void make_uniform(Work &w) {
    w.s.q0 = uniform32(w.s.q0);
    w.s.n = uniform32(w.s.n);
    w.s.plen = uniform32(w.s.plen);
    w.s.slen = uniform32(w.s.slen);
    w.s.pstart = uniform64(w.s.pstart);
    w.s.sstart = uniform64(w.s.sstart);
    w.s.pages = (const int32_t *)uniform64((int64_t)w.s.pages);
    w.s.bad = uniform32(w.s.bad);
    w.rows = uniform32(w.rows);
    w.r0 = uniform32(w.r0);
    w.kvh = uniform32(w.kvh);
    w.part = uniform32(w.part);
    w.pt = uniform32(w.pt);
    w.t0 = uniform32(w.t0);
    w.t1 = uniform32(w.t1);
}

// Keys and values on their way into LDS. A wavefront loads KT / 4 rows of each of a tile; rows
// past the end are copies of the last one (their scores are masked).
template <int DP, int KT>
struct Loader {
    using R = TileRow<DP>;
    static constexpr int N = KT / 4 / R::PER_DMA;    // loads of a wavefront, keys and values each
    static constexpr int BYTES = KT * R::BYTES;      // of the tile's keys; the values follow
    // the segment being read, prefix or suffix (wave-uniform)
    const char *k, *v;                               // its first key's head
    int64_t kst, vst;                                // bytes between keys
    int len, tile0;                                  // its keys, its first tile's index
    bool paged;
    int shift;                                       // log2 of the page size, or -1
    int32_t page[N];                                 // table entries of the next tile's rows
    bool bad = false;

    __device__ __forceinline__ void open(const AttnArgs &a, const Work &w, bool pre) {
        const HeadsArg kh = pick(pre, a.kp, a.ks), vh = pick(pre, a.vp, a.vs);
        const int64_t at = pre ? w.s.pstart : w.s.sstart;
        kst = kh.st * 2;
        vst = vh.st * 2;
        k = kh.p + (int64_t)w.kvh * kh.sh * 2 + at * kst;
        v = vh.p + (int64_t)w.kvh * vh.sh * 2 + at * vst;
        len = pre ? w.s.plen : w.s.slen;
        tile0 = pre ? 0 : w.pt;
        paged = !pre && w.s.pages;
        shift = (a.page_size & (a.page_size - 1)) == 0 ? 31 - __clz(a.page_size | 1) : -1;
    }
    static __device__ __forceinline__ int row(int n) {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        return wave * (KT / 4) + n * R::PER_DMA + lane / R::CHUNKS;
    }
    __device__ __forceinline__ int page_of(const AttnArgs &a, int j) const {
        return shift >= 0 ? j >> shift : j / a.page_size;
    }
    // Asks for the table entries of tile t; they are there at the next barrier.
    __device__ __forceinline__ void look_up(const AttnArgs &a, const Work &w, int t) {
        if (!w.s.pages || t < w.pt || t >= w.t1) return;
        const int j0 = (t - w.pt) * KT;
#pragma unroll
        for (int n = 0; n < N; ++n) page[n] = global_int(w.s.pages)[page_of(a, min(j0 + row(n), w.s.slen - 1))];
    }
    // Tile t to stage offset AT of the ring that begins at `ring`.
    template <int AT>
    __device__ __forceinline__ void issue(const AttnArgs &a, const Work &w, int t, uint32_t ring) {
        if (t == w.pt && t != w.t0) open(a, w, false);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int nch = a.d / 8, j0 = (t - tile0) * KT, last = len - 1 - j0;
        ring += wave * (KT / 4) * R::BYTES;
        if (paged) {
            each<AT>([&](auto n, int ch) {
                const int j = j0 + min(row(n.value), last);
                int64_t at = (int64_t)page[n.value] * a.page_size;
                if (at < 0 || at > a.suffix_rows - a.page_size) {
                    bad = true;
                    at = 0;
                } else {
                    at += j - page_of(a, j) * a.page_size;
                }
                if (ch < nch) {
                    dma16_at<n.to>(k + at * kst + ch * 16, ring);
                    dma16_at<n.to + BYTES>(v + at * vst + ch * 16, ring);
                }
            });
            return;
        }
        // the launcher takes strides for which a tile's offsets fit 32 bits
        const char *kt = k + j0 * kst, *vt = v + j0 * vst;
        if (last >= KT - 1) {
            const uint32_t ro = row(0) * (uint32_t)kst, vo = row(0) * (uint32_t)vst;
            each<AT>([&](auto n, int ch) {
                if (ch < nch) {
                    dma16_from<n.to>(kt + n.value * R::PER_DMA * kst, ro + ch * 16, ring);
                    dma16_from<n.to + BYTES>(vt + n.value * R::PER_DMA * vst, vo + ch * 16, ring);
                }
            });
        } else {
            each<AT>([&](auto n, int ch) {
                const uint32_t r = min(row(n.value), last);
                if (ch < nch) {
                    dma16_from<n.to>(kt, r * (uint32_t)kst + ch * 16, ring);
                    dma16_from<n.to + BYTES>(vt, r * (uint32_t)vst + ch * 16, ring);
                }
            });
        }
    }

  private:
    template <int I, int TO>
    struct Load { static constexpr int value = I, to = TO; };
    // f(load, chunk of the row that this lane takes) for each of the wavefront's loads; the
    // slots past head_dim keep their zeros
    template <int AT, int I = 0, typename F>
    static __device__ __forceinline__ void each(F f) {
        if constexpr (I < N) {
            f(Load<I, AT + I * 1024>{}, (threadIdx.x & (R::CHUNKS - 1)) ^ R::swz(row(I)));
            each<AT, I + 1>(f);
        }
    }
};

}  // namespace olive
