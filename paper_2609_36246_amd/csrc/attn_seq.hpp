// How the attention kernels find the rows of a sequence and of a group, with the checks that
// keep every access inside the buffers whatever the device arrays hold.
#pragma once

#include "layers_internal.hpp"

namespace olive {

// The keys that a range of query tokens reads.
struct SeqView {
    int32_t q0;          // first query token
    int32_t n;           // query tokens
    int32_t plen, slen;  // keys of the prefix and of the suffix
    int64_t pstart;      // row of the prefix's first key
    int64_t sstart;      // packed suffixes: row of the first key
    const int32_t *pages;
    int32_t group, group_end;   // the sequences of its group
    int32_t keys;        // keys of the suffix where it lies in the buffers, whatever else is wrong
    bool skip;           // the query rows themselves are out of order: nothing is written
    bool bad;            // something else is out of range: the rows get NaN
};

// The last i in [0, n) with a[i] <= x, or 0: `a` does not decrease, and if it does the result is
// still in range. 64 entries a step, for a whole wavefront that asks for the same x.
__device__ __forceinline__ int last_at_most(const int32_t *a, int n, int x) {
    const int lane = threadIdx.x & 63;
    int lo = 0;
    while (n > 1) {
        const int step = (n + 63) >> 6, i = lo + lane * step;
        const int k = __popcll(__ballot(lane * step < n && a[i] <= x)) - 1;
        if (k > 0) {
            lo += k * step;
            n -= k * step;
        }
        n = n < step ? n : step;
    }
    return lo;
}
// The group of sequence b (empty groups lie before it), and the sequence of query token t.
__device__ __forceinline__ int group_of(const AttnArgs &a, int b) {
    return last_at_most(a.group_seqs, a.groups, b);
}
__device__ __forceinline__ int seq_of(const AttnArgs &a, int t) { return last_at_most(a.cu_q, a.seqs, t); }

__device__ __forceinline__ bool prefix_ok(const AttnArgs &a, int64_t len, int64_t start) {
    return len >= 0 && len <= a.max_prefix && (len == 0 || (start >= 0 && start <= a.prefix_rows - len));
}
__device__ __forceinline__ bool prefix_ok(const AttnArgs &a, int g) {
    return prefix_ok(a, a.prefix_len[g], a.prefix_start[g]);
}

// The group of sequence b: where it lies among the sequences, and its prefix.
struct GroupView {
    int32_t first, end, plen;
    int64_t pstart;
};
__device__ __forceinline__ GroupView load_group(const AttnArgs &a, int b) {
    GroupView v;
    if (a.groups < 64) {
        // one round of loads instead of three that wait for each other
        const int lane = threadIdx.x & 63, g = min(lane, a.groups - 1);
        const int at = a.group_seqs[min(lane, a.groups)], plen = a.prefix_len[g];
        const int64_t pstart = a.prefix_start[g];
        const int k = max(0, __popcll(__ballot(lane < a.groups && at <= b)) - 1);
        v.first = __builtin_amdgcn_readlane(at, k);
        v.end = __builtin_amdgcn_readlane(at, k + 1);
        v.plen = __builtin_amdgcn_readlane(plen, k);
        v.pstart = (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(pstart >> 32), k) << 32) |
                             (uint32_t)__builtin_amdgcn_readlane((int)pstart, k));
        return v;
    }
    const int g = group_of(a, b);
    v.first = a.group_seqs[g];
    v.end = a.group_seqs[g + 1];
    v.plen = a.prefix_len[g];
    v.pstart = a.prefix_start[g];
    return v;
}

__device__ __forceinline__ SeqView load_seq(const AttnArgs &a, int b) {
    SeqView s;
    const int32_t q0 = a.cu_q[b], q1 = a.cu_q[b + 1];
    s.slen = a.suffix_len[b];
    s.sstart = a.pages || !a.suffix_start ? 0 : a.suffix_start[b];
    const GroupView g = load_group(a, b);
    s.skip = q0 < 0 || q1 < q0 || q1 > a.total_q;
    s.q0 = s.skip ? 0 : q0;
    s.n = s.skip ? 0 : q1 - q0;
    s.bad = s.n > a.max_q || g.first > b || g.end <= b || !prefix_ok(a, g.plen, g.pstart);
    s.group = g.first;
    s.group_end = g.end;
    s.plen = g.plen;
    s.pstart = g.pstart;
    s.pages = nullptr;
    bool inside = s.slen >= 0 && s.slen <= a.max_suffix;
    if (inside && s.slen > 0) {
        if (a.pages) {
            s.pages = a.pages + (int64_t)b * a.table_stride;
            inside = a.suffix_rows >= a.page_size;
        } else {
            inside = s.sstart >= 0 && s.sstart <= a.suffix_rows - s.slen;
        }
    }
    s.keys = inside ? s.slen : 0;
    s.bad |= !inside;
    if (s.bad) s.plen = s.slen = 0;
    return s;
}

// Whether sequence b is not left out and has query token t.
__device__ __forceinline__ bool has_token(const AttnArgs &a, int b, int t) {
    const int32_t q0 = a.cu_q[b], q1 = a.cu_q[b + 1];
    return q0 >= 0 && q0 <= t && t < q1 && q1 <= a.total_q;
}
// Whether any sequence has (for a whole wavefront that asks for the same t). All of them are
// looked through where the one that the order of cu_q leads to has not.
__device__ __forceinline__ bool any_has_token(const AttnArgs &a, int t) {
    if (has_token(a, seq_of(a, t), t)) return true;
    bool any = false;
    for (int b = threadIdx.x & 63; b < a.seqs; b += 64) any |= has_token(a, b, t);
    return __any(any);
}

// The query tokens [q0, q1) of the sequences [b0, b1): whether these entries are in order.
__device__ __forceinline__ bool group_tokens(const AttnArgs &a, int b0, int b1, int &q0, int &q1) {
    q0 = q1 = 0;
    if (b0 < 0 || b1 < b0 || b1 > a.seqs) return false;
    q0 = a.cu_q[b0];
    q1 = a.cu_q[b1];
    return q0 >= 0 && q0 <= q1 && q1 <= a.total_q;
}
// The same, and whether all entries between are in order (a whole wavefront asks).
__device__ __forceinline__ bool group_in_order(const AttnArgs &a, int b0, int b1, int &q0, int &q1) {
    if (!group_tokens(a, b0, b1, q0, q1)) return false;
    bool ok = true;
    for (int b = b0 + (threadIdx.x & 63); b < b1; b += 64) ok &= a.cu_q[b] <= a.cu_q[b + 1];
    return __all(ok);
}
// Whether the tokens of a sequence lie among those of its group (group_tokens): the first lane of
// a pair holds the group's first entry, the second its last one, and each says what its own says.
__device__ __forceinline__ int32_t group_entry(const AttnArgs &a, const SeqView &s) {
    if (s.group < 0 || s.group_end > a.seqs) return -1;
    return a.cu_q[threadIdx.x & 1 ? s.group_end : s.group];
}
__device__ __forceinline__ bool entry_holds(const AttnArgs &a, const SeqView &s, int32_t entry) {
    return threadIdx.x & 1 ? s.q0 + s.n <= entry && entry <= a.total_q : 0 <= entry && entry <= s.q0;
}

// Row of suffix token j (0 <= j < slen). A page outside the buffer sets `bad` and gives row 0.
__device__ __forceinline__ int64_t suffix_row(const AttnArgs &a, const SeqView &s, int j,
                                              bool &bad) {
    if (!s.pages) return s.sstart + j;
    const int pg = j / a.page_size;
    const int64_t row = (int64_t)s.pages[pg] * a.page_size;
    if (row < 0 || row > a.suffix_rows - a.page_size) {
        bad = true;
        return 0;
    }
    return row + (j - pg * a.page_size);
}

// Suffix tokens that query i of a sequence sees.
__device__ __forceinline__ int suffix_seen(const SeqView &s, int i) {
    const int c = s.slen - s.n + i + 1;
    return c < 0 ? 0 : c < s.slen ? c : s.slen;
}

}  // namespace olive
