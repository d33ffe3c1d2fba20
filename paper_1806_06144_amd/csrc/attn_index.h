// Index arithmetic of the attention kernels, for host and device: everything
// that stands between a value read from device memory (starts, lengths, page
// numbers) and an address.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define EP_HD __host__ __device__ __forceinline__
#else
#define EP_HD inline
#endif

namespace ep {

EP_HD int clamp_i(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

// Rows start[b] .. start[b + 1] - 1 of `tokens`, whatever start holds.
EP_HD void held_range(int begin, int end, int tokens, int& first, int& count) {
    first = clamp_i(begin, 0, tokens);
    count = clamp_i(end, first, tokens) - first;
}

// A sequence's length, within what its row of the table can address.
EP_HD int held_length(int length, int64_t cols, int page_shift) {
    const int64_t most = cols << page_shift;
    return length < 0 ? 0 : length > most ? (int)most : length;
}

// The first tile of sequence b among tiles of `size` rows, per rows a token:
// each sequence gets at least as many tiles as it needs, the last ends at
// most at tokens per / size + batch.
EP_HD int64_t first_tile(int start, int tokens, int b, int per, int size) {
    return (int64_t)clamp_i(start, 0, tokens) * per / size + b;
}

// floor(r / group) for r group < 2^32; magic = 2^32 / group, rounded up.
EP_HD unsigned group_magic(int group) {
    return (unsigned)(((int64_t(1) << 32) + group - 1) / group);
}
EP_HD int row_token(int r, int group, unsigned magic) {
    return group == 1 ? r : (int)(((uint64_t)(unsigned)r * magic) >> 32);
}

// Page of token j (j within the table), or -1 where its number is none of the
// cache's.
EP_HD int page_of(const int* table, int64_t cols, int b, int pages, int shift, int64_t j) {
    const int page = table[b * cols + (j >> shift)];
    return (unsigned)page < (unsigned)pages ? page : -1;
}
// Place of token j in its page, counted in tokens from the first page's start.
EP_HD int64_t page_slot(int page, int shift, int64_t j) {
    return ((int64_t)page << shift) + (j & ((int64_t(1) << shift) - 1));
}

// Keys that the query of token t (position t + off) sees: lo .. hi - 1.
EP_HD int visible_hi(int t, int off, int m, int causal) {
    return causal ? clamp_i(t + off + 1, 0, m) : m;
}
EP_HD int visible_lo(int t, int off, int window) {
    const int lo = t + off + 1 - window;
    return window && lo > 0 ? lo : 0;
}
// Rows that see key j: from .. to - 1 (n tokens of `group` rows).
EP_HD int seen_from(int j, int off, int n, int group, int causal) {
    return causal ? clamp_i(j - off, 0, n) * group : 0;
}
EP_HD int seen_to(int j, int off, int n, int group, int window) {
    const int64_t t = (int64_t)j - off + window;
    return (!window || t > n ? n : t < 0 ? 0 : (int)t) * group;
}

}  // namespace ep
