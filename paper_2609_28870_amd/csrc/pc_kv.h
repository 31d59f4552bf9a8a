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
    uint8_t *k_exp, *v_exp;           // nullptr: not 4-bit; of the 16 bytes of codes from byte b on at b / 16
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

// Two arrays [n_rows][n_heads] of runs of `width` bytes: whether they are one, and whether they
// share memory.  In one range they are known not to if their strides agree and one lies in the
// other's gaps, between its runs or between blocks of them.
struct Entries {
    const void *base;
    uint64_t row, head;   // strides in bytes
};
bool same_strides(const Entries &x, const Entries &y, uint64_t n_rows, uint64_t n_heads);
bool entries_overlap(const Entries &x, const Entries &y, uint64_t n_rows, uint64_t n_heads, uint64_t width);

pc_status kv_view(const pc_kv_cache *c, KvView *v);          // checks the descriptor
uint64_t bytes_of(uint32_t dtype, uint64_t elements);        // 0: no such type

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

// slot of row t of sequence s, negative if it has none: by the length as it is, so that one above
// max_kv moves no row to another's slot
__device__ __forceinline__ int64_t slot_of_row(const uint32_t *__restrict__ kv_len, uint32_t max_kv, uint32_t s, const Seq &q, uint32_t t) {
    const int64_t slot = (int64_t)kv_len[s] - q.rows + (t - q.first);
    return slot < (int64_t)max_kv ? slot : -1;
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

// sequence of chunk row t, by a whole wave: the first that ends past it (or the last one)
__device__ __forceinline__ uint32_t wave_seq_of(const uint32_t *__restrict__ q_off, uint32_t n_seqs, uint32_t t) {
    const uint32_t lane = threadIdx.x & (WAVE - 1);
    uint32_t lo = 0, n = n_seqs;   // one of lo .. lo + n - 1
    while (n > 1) {
        const uint32_t step = (n + WAVE - 1) / WAVE;
        const bool in = lane * step < n;
        const uint32_t end = in ? q_off[lo + min((lane + 1) * step, n)] : 0;
        const uint32_t past = min((uint32_t)__popcll(ballot(in && end <= t)) * step, n - 1);
        lo += past;
        n = min(step, n - past);
        if (step == 1) break;
    }
    return lo;
}

// Where new rows go.
struct Chunks {
    KvView kv;
    const uint32_t *table, *kv_len, *q_off;
    uint64_t table_stride;
    uint32_t n_seqs, n_rows, max_kv;
};

// Whether anything of an append does not fit, by one workgroup: it looks at every
// sequence and every page that the call writes (a lane per page, 64 sequences at
// a time), so that no launch is spent on clearing a word that the others would set.
// No row's slot may be max_pos or more (where slots are positions).
__device__ __forceinline__ bool chunks_bad(const Chunks &a, uint32_t max_pos) {
    const int lane = threadIdx.x & (WAVE - 1), wave = threadIdx.x / WAVE, waves = blockDim.x / WAVE;
    bool any = threadIdx.x == 0 && (a.q_off[0] != 0 || a.q_off[a.n_seqs] != a.n_rows);
    for (uint32_t s0 = wave * WAVE; s0 < a.n_seqs; s0 += waves * WAVE) {
        const uint32_t s = s0 + lane;
        uint32_t from = 0, pages = 0;
        bool bad = false;
        if (s < a.n_seqs) {
            const Seq q = load_seq(a.q_off, a.kv_len, s, a.n_rows, a.max_kv, &bad);
            bad |= q.rows > q.len || (q.rows && q.len > max_pos);
            if (q.rows && q.len) {
                from = a.kv.by_page.div(q.rows < q.len ? q.len - q.rows : 0);
                pages = a.kv.by_page.div(q.len - 1) + 1 - from;
            }
        }
        any |= bad;
        // Pages are counted in 32 bits, which rows that overlap (offsets that decrease) could pass, and
        // the loop below would not end; but then the status is known.
        if (ballot(bad)) continue;
        const uint32_t end = wave_incl_scan(pages), all = (uint32_t)__shfl((int)end, WAVE - 1, WAVE);
        for (uint32_t p0 = 0; p0 < all; p0 += WAVE) {
            const uint32_t p = p0 + lane;
            int at = 0;   // sequence of page p: the first lane whose end is past it
#pragma unroll
            for (int step = WAVE / 2; step; step /= 2)
                if ((uint32_t)__shfl((int)end, at + step - 1, WAVE) <= p) at += step;
            at = at < WAVE ? at : WAVE - 1;
            const uint32_t e = (uint32_t)__shfl((int)end, at, WAVE), n = (uint32_t)__shfl((int)pages, at, WAVE),
                           f = (uint32_t)__shfl((int)from, at, WAVE);
            if (p < all) any |= a.table[(uint64_t)(s0 + at) * a.table_stride + f + (p - (e - n))] >= a.kv.n_pages;
        }
    }
    return any;
}

__device__ __forceinline__ float to_float(uint32_t bits, bool bf16) {
    if (bf16) return __uint_as_float(bits << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}
// four values to four 8-bit codes
__device__ __forceinline__ uint32_t to_e4m3(float x0, float x1, float x2, float x3, float scale) {
    float x[4] = {x0, x1, x2, x3};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float y = x[i] / scale;
        x[i] = y != y ? y : fminf(fmaxf(y, -448.f), 448.f);
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
    return (uint32_t)w;
}

// The position rotation as the kernels see it.
struct Turn {
    const float2 *table;     // [n_pos][half] cosine and sine
    const uint32_t *pos;     // of every row, or nullptr: its slot
    uint32_t n_pos, half;    // half: pairs of a head
    float sign;              // -1: transposed
};
enum class Layout { HALVES, PAIRS, ANY };   // ANY: halves, whatever their size
struct Queries {
    const char *x;           // nullptr: none
    char *out;
    uint64_t x_row, x_head, o_row, o_head;   // bytes
    uint32_t n_heads;
};
// New tokens through the kernels of pc_rope.hip: turned (turn.half > 0), or as they are into a cache
// of 4 bits.
pc_status append_turned(const Chunks &c, uint32_t cache_dtype, const Entries &k, const Entries &v, uint32_t dtype, const Turn &turn,
                        Layout layout, const Queries &q, int32_t *status, hipStream_t st);

}  // namespace pc
