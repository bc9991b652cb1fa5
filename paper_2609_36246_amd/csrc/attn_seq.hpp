// How the attention kernels find the rows of a sequence and of a group, with the checks that
// keep every access inside the buffers whatever the device arrays hold.
#pragma once

#include "layers_internal.hpp"

namespace olive {

// The keys that a range of query tokens reads.
struct SeqView {
    int64_t q0;          // first query token
    int32_t n;           // query tokens
    int32_t plen, slen;  // keys of the prefix and of the suffix
    int64_t pstart;      // row of the prefix's first key
    int64_t sstart;      // packed suffixes: row of the first key
    const int32_t *pages;
    bool skip;           // the query rows themselves are out of order: nothing is written
    bool bad;            // something else is out of range: the rows get NaN
};

// The last group that begins at or before sequence b (empty groups lie before it).
__device__ __forceinline__ int group_of(const AttnArgs &a, int b) {
    int lo = 0, hi = a.groups - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.group_seqs[mid] <= b) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// The sequence that query token t belongs to: the last one that begins at or before t.
__device__ __forceinline__ int seq_of(const AttnArgs &a, int64_t t) {
    int lo = 0, hi = a.seqs - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.cu_q[mid] <= t) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ bool prefix_ok(const AttnArgs &a, int g) {
    const int64_t len = a.prefix_len[g], start = a.prefix_start[g];
    return len >= 0 && len <= a.max_prefix && (len == 0 || (start >= 0 && start <= a.prefix_rows - len));
}

__device__ __forceinline__ SeqView load_seq(const AttnArgs &a, int b) {
    SeqView s;
    const int64_t q0 = a.cu_q[b], q1 = a.cu_q[b + 1];
    s.skip = q0 < 0 || q1 < q0 || q1 > a.total_q;
    s.q0 = s.skip ? 0 : q0;
    s.n = s.skip ? 0 : (int32_t)(q1 - q0);
    const int g = group_of(a, b);
    s.bad = s.n > a.max_q || a.group_seqs[g] > b || a.group_seqs[g + 1] <= b || !prefix_ok(a, g);
    s.plen = s.bad ? 0 : a.prefix_len[g];
    s.pstart = s.bad ? 0 : a.prefix_start[g];
    s.slen = a.suffix_len[b];
    s.sstart = 0;
    s.pages = nullptr;
    if (s.slen < 0 || s.slen > a.max_suffix) {
        s.bad = true;
    } else if (s.slen > 0) {
        if (a.pages) {
            s.pages = a.pages + (int64_t)b * a.table_stride;
            s.bad |= a.suffix_rows < a.page_size;
        } else {
            s.sstart = a.suffix_start[b];
            s.bad |= s.sstart < 0 || s.sstart > a.suffix_rows - s.slen;
        }
    }
    if (s.bad) s.plen = s.slen = 0;
    return s;
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
