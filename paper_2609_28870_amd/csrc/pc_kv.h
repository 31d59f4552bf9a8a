// What the operators over a paged cache of KV blocks share (gfx950, wave64).
// Not part of the ABI.
#pragma once

#include "pc_internal.h"

namespace pc {

// Exact quotient of n < 2^31 by a divisor fixed on the host: with 2^(s - 1) < d
// <= 2^s and mul = ceil(2^(31 + s) / d), n * (mul * d - 2^(31 + s)) < 2^(31 + s).
struct FastDiv {
    uint32_t mul, shift, d;
    __device__ __forceinline__ uint32_t div(uint32_t n) const { return (uint32_t)(((uint64_t)n * mul) >> shift); }
};
inline FastDiv fast_div(uint32_t d) {
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;
    return FastDiv{(uint32_t)(((1ull << (31 + s)) + d - 1) / d), 31 + s, d};
}

// The cache as the kernels see it; strides in bytes.
struct KvView {
    char *k, *v;
    const float *k_scale, *v_scale;   // nullptr: not 8-bit
    uint64_t sp, sh, st;              // page, head, slot
    uint32_t n_pages, n_kv, dim, page;
    FastDiv by_page;
};

// A launch holds fewer than 2^32 threads.
inline bool launch_fits(uint64_t groups, uint32_t threads) { return groups < (1ull << 32) / threads; }

// whether two ranges of memory share a byte
inline bool overlap(const void *a, uint64_t a_bytes, const void *b, uint64_t b_bytes) {
    const uint64_t x = (uint64_t)(uintptr_t)a, y = (uint64_t)(uintptr_t)b;
    return a_bytes && b_bytes && (x < y ? y - x < a_bytes : x - y < b_bytes);
}

pc_status kv_view(const pc_kv_cache *c, KvView *v);   // checks the descriptor
size_t type_size(uint32_t dtype);                     // 0: no such type

// Rows of sequence s inside the chunk arrays, its length, and the slot of its first row
// (negative: rows before slot 0); a table entry that does not fit (decreasing, past n_q)
// counts as no rows.
struct Seq {
    uint32_t first, rows, len;
    int32_t slot;
};
__device__ __forceinline__ Seq load_seq(const uint32_t *__restrict__ q_off, const uint32_t *__restrict__ kv_len, uint32_t s,
                                        uint32_t n_q, uint32_t max_kv, bool *bad) {
    const uint32_t a = q_off[s], b = q_off[s + 1], l = kv_len[s];
    const bool ok = a <= b && b <= n_q;
    *bad = !ok || l > max_kv;
    const uint32_t rows = ok ? b - a : 0u, len = l < max_kv ? l : max_kv;
    return Seq{a, rows, len, (int32_t)(len - rows)};
}

// sequence of chunk row t: the last s with q_off[s] <= t
__device__ __forceinline__ uint32_t seq_of(const uint32_t *__restrict__ q_off, uint32_t n_seqs, uint32_t t) {
    uint32_t lo = 0, hi = n_seqs;   // q_off[lo] <= t < q_off[hi]
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (q_off[mid] <= t) lo = mid; else hi = mid;
    }
    return lo;
}

}  // namespace pc
