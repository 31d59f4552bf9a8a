// The pieces that the attention kernels over the paged cache share: matrix
// products, the work list, tiles of keys and values.  Not part of the ABI.
#pragma once

#include <type_traits>

#include "pc_kv.h"

namespace pc {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float MINUS_INF = -__builtin_inff();

// A row's weights are exp2(score - ref + TOP), ref a maximum of the scores so far that
// may lag behind by SLACK: most tiles that bring a slightly larger one need no
// rescaling of the sums (the factor cancels in sum p v / sum p).
struct Bf16 {
    static constexpr float TOP = 0.f, SLACK = 8.f;
    static __device__ __forceinline__ f32x16 mfma(uint4 a, uint4 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float x, float y) {
        const bf16x2 v = {(__bf16)x, (__bf16)y};
        return __builtin_bit_cast(uint32_t, v);
    }
    template <bool HI>
    static __device__ __forceinline__ uint32_t from_e4m3(uint32_t w) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HI));
    }
    template <int BYTE>
    static __device__ __forceinline__ uint32_t from_e2m1(uint32_t w, float scale) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, BYTE));
    }
    static constexpr uint32_t SIGNS = 0x80008000u, EXPONENT = 0x7F80u;
    static __device__ __forceinline__ float value(uint32_t bits) { return __uint_as_float(bits << 16); }
};
struct F16 {
    // f16 has five exponent bits: at most 2^15, and down to 2^-25 of ref normal numbers
    static constexpr float TOP = 11.f, SLACK = 4.f;
    static __device__ __forceinline__ f32x16 mfma(uint4 a, uint4 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float x, float y) {
        const f16x2 v = {(_Float16)x, (_Float16)y};
        return __builtin_bit_cast(uint32_t, v);
    }
    template <bool HI>
    static __device__ __forceinline__ uint32_t from_e4m3(uint32_t w) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HI));
    }
    template <int BYTE>
    static __device__ __forceinline__ uint32_t from_e2m1(uint32_t w, float scale) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, BYTE));
    }
    static constexpr uint32_t SIGNS = 0x80008000u, EXPONENT = 0x7C00u;
    static __device__ __forceinline__ float value(uint32_t bits) {
        return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
    }
};

// How the cache holds its values: in the queries' type, as 8-bit or as 4-bit codes.
enum class Held { SAME, E4M3, E2M1 };
// bytes of n elements
template <Held H>
constexpr __host__ __device__ __forceinline__ uint32_t held_bytes(uint32_t n) {
    return H == Held::SAME ? 2 * n : H == Held::E4M3 ? n : n / 2;
}

// The scale of a block of 4-bit codes is the exponent byte of a number: the conversions take
// that field alone (0 as 2^-127, 255 as NaN).
__device__ __forceinline__ float scale_of(uint32_t exponent) { return __uint_as_float(exponent << 23); }
// eight 4-bit codes as a piece of eight elements
template <class T>
__device__ __forceinline__ uint4 expand(uint32_t w, float scale) {
    return make_uint4(T::template from_e2m1<0>(w, scale), T::template from_e2m1<1>(w, scale), T::template from_e2m1<2>(w, scale),
                      T::template from_e2m1<3>(w, scale));
}
// sixteen 8-bit codes as two pieces of eight elements
template <class T>
__device__ __forceinline__ void expand(uint4 x, uint4 *lo, uint4 *hi) {
    *lo = make_uint4(T::template from_e4m3<false>(x.x), T::template from_e4m3<true>(x.x),
                     T::template from_e4m3<false>(x.y), T::template from_e4m3<true>(x.y));
    *hi = make_uint4(T::template from_e4m3<false>(x.z), T::template from_e4m3<true>(x.z),
                     T::template from_e4m3<false>(x.w), T::template from_e4m3<true>(x.w));
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
// the same lane of the other half of the wave
__device__ __forceinline__ void both_halves(float x, float *lower, float *upper) {
    const uint32_t b = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    *lower = __uint_as_float(r[0]);
    *upper = __uint_as_float(r[1]);
}
__device__ __forceinline__ float max_of_halves(float x) {
    float a, b;
    both_halves(x, &a, &b);
    return fmaxf(a, b);
}
__device__ __forceinline__ float sum_of_halves(float x) {
    float a, b;
    both_halves(x, &a, &b);
    return a + b;
}

// Keys and values of 16-bit elements lie in LDS as rows of D, in pieces of 16
// bytes.  LDS has 64 banks of 4 bytes: 16 lanes' pieces, or 32 lanes' 8 bytes, at a
// time.  Keys are read as a column of pieces over 16 consecutive rows, values (transposed) as
// four neighbouring pieces of four consecutive rows.  Piece c of row k is at c ^ spread(k):
// both then meet every bank once, and so do writes of whole rows or columns.
template <int D>
constexpr __device__ __forceinline__ uint32_t spread(uint32_t row) {
    return D == 64 ? (row >> 1 & 1) << 2 | (row >> 2 & 3) : (row & 3) << 2 | (row >> 2 & 3);
}
template <int D>
__device__ __forceinline__ uint32_t piece_at(uint32_t row, uint32_t c) {
    return row * (D * 2) + ((c ^ spread<D>(row)) * 16);
}
// four keys of one value dimension a lane: the 16 lanes of a group fetch 8 bytes each
// of four rows of 16 elements and get a column each
__device__ __forceinline__ uint2 read_transposed(const char *p) {
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p));
}
// Where this lane fetches values: of the 16 keys at hand, rows 4 half + lane % 16 / 4 (lo) and 8
// further (hi) of dimensions 32 b + 16 (lane / 16 % 2) + 4 (lane % 4) .. + 3.  The spread has
// four bits (two pairs of blocks are 256 bytes apart), so a few numbers a lane serve all
// rows and blocks: at[b % 4] + b / 4 * 256.
template <int D>
struct ValueAt {
    uint32_t lo[D == 64 ? 2 : 4], hi[D == 64 ? 2 : 4];
    __device__ __forceinline__ ValueAt() {
        const uint32_t lane = threadIdx.x & (WAVE - 1), row = 4 * (lane / 32) + lane % 16 / 4;
#pragma unroll
        for (uint32_t b = 0; b < (D == 64 ? 2 : 4); ++b) {
            const uint32_t c = 4 * b + 2 * (lane / 16 % 2) + lane % 4 / 2;
            lo[b] = piece_at<D>(row, c) + lane % 2 * 8;
            hi[b] = piece_at<D>(row + 8, c) + lane % 2 * 8;
        }
    }
};
// Where this lane finds its key (or query row) lane % 32 of a tile, step i of its dimensions.
template <int D>
struct RowAt {
    uint32_t at[D == 64 ? 4 : 8];
    __device__ __forceinline__ RowAt() {
        const uint32_t lane = threadIdx.x & (WAVE - 1);
#pragma unroll
        for (uint32_t i = 0; i < (D == 64 ? 4 : 8); ++i)
            at[i] = piece_at<D>(lane % 32, 4 * (i / 2) + 2 * (lane / 32) + i % 2);
    }
    __device__ __forceinline__ uint4 read(const char *tile, int i) const {
        return *(const uint4 *)(tile + at[i % (D == 64 ? 4 : 8)] + i / 8 * 256);
    }
};

// ------------------------------------------------------------------ arguments

struct AttnArgs {
    KvView kv;
    const uint32_t *table, *kv_len, *q_off;
    uint64_t table_stride;
    uint32_t n_seqs, n_rows, max_q, max_kv;
    const char *q;               // strides in bytes
    char *out;
    uint64_t q_row, q_head, o_row, o_head;
    float *lse;                  // user's, or nullptr
    const float *weight;
    float *weight_out;
    uint64_t weight_stride;
    uint32_t n_heads, group;
    FastDiv by_group;
    float scale;
    uint32_t causal, window;
    uint32_t by_16;              // 16 slots from a multiple of 16 share a page, their strides small
    // the work list
    uint32_t target;             // items wanted
    uint32_t least;              // tiles of an item, at least
    uint32_t cut_first;          // the ranges of sequences that are cut come first: what is left for the end is smaller
    uint32_t even;               // a sequence's ranges are of one length, not all but the last as long as they may be
    uint32_t row_tile, key_tile; // rows, keys
    uint32_t slots;              // partial results that fit
    uint32_t slot_rows;
    // workspace
    int32_t *status;
    float *part;                 // [slot][row][padded dim]
    float2 *part_ml;             // [slot][row] maximum (base 2), sum
    float *lse2;                 // [row][head] base 2, for the weights
    float *scores;               // [seq][kv head][row][score_stride] base 2 (few rows, with weights)
    uint64_t score_stride;
    float *weight_part;          // [row part][seq][kv head][max_kv]
    uint32_t weight_parts;
};

// Keys that rows i0 .. i1 of a sequence see between them: [lo, hi).
struct Range {
    uint32_t lo, hi;
};
__device__ __forceinline__ Range seen(const AttnArgs &a, const Seq &q, uint32_t i0, uint32_t i1) {
    const int64_t j0 = q.slot;
    int64_t hi = a.causal ? j0 + i1 + 1 : (int64_t)q.len, lo = a.window ? j0 + i0 - (int64_t)a.window + 1 : 0;
    if (hi > (int64_t)q.len) hi = q.len;
    if (lo < 0) lo = 0;
    if (hi < lo) hi = lo;
    return Range{(uint32_t)lo, (uint32_t)hi};
}
// slots that row i sees: first .. last (none if last < first)
__device__ __forceinline__ void seen_by_row(const AttnArgs &a, const Seq &q, uint32_t i, int32_t *first, int32_t *last) {
    const int64_t x = (int64_t)q.slot + i;
    const int64_t lo = a.window ? x - (int64_t)a.window + 1 : 0;
    *first = lo > 0 ? (lo < 0x7FFFFFFF ? (int32_t)lo : 0x7FFFFFFF) : 0;
    *last = a.causal && x < (int64_t)q.len ? (x < 0 ? -1 : (int32_t)x) : (int32_t)q.len - 1;
}

// ------------------------------------------------------------------ work list
// An item is a tile of rows (a row is a token and one of the query heads that
// share a key/value head) against a range of key tiles.  Every workgroup works
// the list out from the lengths, which only the device knows: the tiles of
// all sequences divided by the items wanted give the length of a range, so that a
// few long sequences fill the chip as well as many short ones.
struct Shape {   // one sequence's part of the list
    Seq q;
    Range keys;
    uint32_t row_tiles, key_tiles;
};
__device__ __forceinline__ Shape shape_of(const AttnArgs &a, uint32_t s) {
    Shape h;
    bool bad;
    h.q = load_seq(a.q_off, a.kv_len, s, a.n_rows, a.max_kv, &bad);
    if (h.q.rows > a.max_q) h.q.rows = a.max_q;   // the first ones, at the slots that they have
    h.keys = h.q.rows ? seen(a, h.q, 0, h.q.rows - 1) : Range{0, 0};
    h.keys.lo &= ~(a.key_tile - 1);   // a power of two
    h.row_tiles = (uint32_t)(((uint64_t)h.q.rows * a.group + a.row_tile - 1) / a.row_tile);
    h.key_tiles = (h.keys.hi - h.keys.lo + a.key_tile - 1) / a.key_tile;
    return h;
}
struct Item {
    uint32_t seq, head, row_tile, split;
    uint32_t splits, length;   // ranges of the sequence, tiles in each
    uint32_t slot;             // of the partial result (splits > 1)
    Shape shape;
    bool there;
};
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }
__device__ __forceinline__ uint32_t from_lane(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }

// What `key` counts: items; tiles of rows of every head (whatever their ranges); sequences.
enum class By { ITEM, TILE, SEQ };
template <By BY, bool EVEN = false>   // EVEN: where ranges may be
__device__ __forceinline__ Item find_item(const AttnArgs &a, uint32_t key) {
    const int lane = threadIdx.x & (WAVE - 1);
    Item it;
    it.there = false;
    uint64_t tiles = 0;
    Shape h;
    for (uint32_t s0 = 0; s0 < a.n_seqs; s0 += WAVE) {
        if (s0 + lane < a.n_seqs) {
            h = shape_of(a, s0 + lane);
            tiles += (uint64_t)h.row_tiles * h.key_tiles;
        }
    }
#pragma unroll
    for (int step = 1; step < WAVE; step *= 2) tiles += __shfl_xor((unsigned long long)tiles, step, WAVE);
    const uint64_t len = (tiles * a.kv.n_kv + a.target - 1) / a.target;
    const uint32_t longest = uniform(len > a.least ? (uint32_t)(len < 0x7FFFFFFFu ? len : 0x7FFFFFFFu) : a.least);
    uint64_t base = 0, slot = 0;
    const int classes = BY != By::SEQ && a.cut_first ? 2 : 1;
#pragma unroll 1
    for (int whole = 0; whole < classes; ++whole) {
        for (uint32_t s0 = 0; s0 < a.n_seqs; s0 += WAVE) {
            const uint32_t s = s0 + lane;
            uint32_t items = 0, splits = 1, count = 0, length = longest;
            if (s < a.n_seqs) {
                if (a.n_seqs > WAVE) h = shape_of(a, s);
                splits = (h.key_tiles + length - 1) / length;
                splits = splits ? splits : 1;
                if (EVEN && a.even && splits > 1) {
                    length = (h.key_tiles + splits - 1) / splits;
                    splits = (h.key_tiles + length - 1) / length;
                }
                const uint64_t n = (uint64_t)h.row_tiles * splits * a.kv.n_kv;
                items = n < (1u << 25) ? (uint32_t)n : 1u << 25;
                if (classes == 1 || (splits == 1) == (whole == 1)) count = BY == By::ITEM ? items : h.row_tiles * a.kv.n_kv;
            }
            const uint32_t partial = splits > 1 ? items : 0, slot_end = wave_incl_scan(partial);
            const uint32_t end = BY == By::SEQ ? 0 : wave_incl_scan(count);
            int at;
            if (BY == By::SEQ) at = key - s0 < WAVE ? (int)(key - s0) : WAVE;
            else at = __popcll(ballot(base + end <= key));
            at = (int)uniform((uint32_t)at);
            if (at < WAVE && s0 + at < a.n_seqs) {
                it.there = true;
                it.seq = s0 + at;
                it.splits = from_lane(splits, at);
                it.length = EVEN ? from_lane(length, at) : longest;
                it.shape.q.first = from_lane(h.q.first, at);
                it.shape.q.rows = from_lane(h.q.rows, at);
                it.shape.q.len = from_lane(h.q.len, at);
                it.shape.q.slot = (int32_t)from_lane((uint32_t)h.q.slot, at);
                it.shape.keys.lo = from_lane(h.keys.lo, at);
                it.shape.keys.hi = from_lane(h.keys.hi, at);
                it.shape.row_tiles = from_lane(h.row_tiles, at);
                it.shape.key_tiles = from_lane(h.key_tiles, at);
                it.slot = (uint32_t)slot + from_lane(slot_end - partial, at);
                it.head = it.row_tile = it.split = 0;
                if (BY != By::SEQ) {
                    // heads first (neighbouring workgroups are on different XCDs, so with 2, 4 or 8
                    // heads an L2 holds one or few heads' keys), then rows, the last ones first
                    // (they see the most keys), then ranges
                    const uint32_t i = key - (uint32_t)(base + from_lane(end - count, at));
                    const uint32_t j = i / a.kv.n_kv;
                    it.head = i - j * a.kv.n_kv;
                    it.split = j / it.shape.row_tiles;
                    it.row_tile = it.shape.row_tiles - 1 - (j - it.split * it.shape.row_tiles);
                    if (BY == By::ITEM) it.slot += i;
                }
                return it;
            }
            base += from_lane(end, WAVE - 1);
            if (!whole) slot += from_lane(slot_end, WAVE - 1);
        }
    }
    return it;
}
// slot of an item, from the sequence's first (found by tile or by sequence)
__device__ __forceinline__ uint32_t slot_of(const AttnArgs &a, const Item &it, uint32_t head, uint32_t row_tile, uint32_t split) {
    return it.slot + (split * it.shape.row_tiles + (it.shape.row_tiles - 1 - row_tile)) * a.kv.n_kv + head;
}

// ------------------------------------------------------------------ rows

// Elements of a query with the sign of the scores' factor; a factor of zero leaves zeros, and NaN
// of what is not finite.
template <class T>
__device__ __forceinline__ uint32_t times_zero(uint32_t w) {
    return ((w & T::EXPONENT) == T::EXPONENT ? 0x7FFFu : 0) | ((w >> 16 & T::EXPONENT) == T::EXPONENT ? 0x7FFF0000u : 0);
}
template <class T, int N>
__device__ __forceinline__ void sign_query(uint4 (&q)[N], uint32_t flip, bool zero) {
    if (zero) {   // rare, and apart, so that the loads before are one run
#pragma unroll
        for (int i = 0; i < N; ++i)
            q[i] = make_uint4(times_zero<T>(q[i].x), times_zero<T>(q[i].y), times_zero<T>(q[i].z), times_zero<T>(q[i].w));
    }
#pragma unroll
    for (int i = 0; i < N; ++i) q[i] = make_uint4(q[i].x ^ flip, q[i].y ^ flip, q[i].z ^ flip, q[i].w ^ flip);
}
// A row's query as the right operand of scores^T = K Q^T: step s holds dimensions
// 32 (s / 2) + 16 half + 8 (s % 2) .. + 7, the order in which keys are read, too
// (the sum over dimensions takes any order that both operands share).
constexpr __device__ __forceinline__ uint32_t dim_of_step(uint32_t step, uint32_t half) {
    return 32 * (step / 2) + 16 * half + 8 * (step % 2);
}
template <class T, int D, bool FULL>
__device__ __forceinline__ void load_query(const AttnArgs &a, const char *row, bool there, uint32_t half, uint32_t flip,
                                           bool zero, uint4 (&q)[D / 16]) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
        const uint32_t d = dim_of_step(s, half);
        q[s] = make_uint4(0, 0, 0, 0);
        if (there && (FULL || d < a.kv.dim)) q[s] = *(const uint4 *)(row + d * 2);
    }
    sign_query<T>(q, flip, zero);
}

// SLACK in units of scores that are taken times c > 0; finite, so that a first score always
// passes a maximum of -inf by it
template <class T>
__device__ __forceinline__ float slack_of(float c) { return fminf(T::SLACK / c, 3e38f); }

// softmax state of the rows of a wave: lane % 32 is the row; the maximum is
// common to both halves, the sum is each half's own until the end.  Scores are taken
// times c, and `slack` is slack_of(c).
template <class T, int D>
struct Rows {
    f32x16 o[D / 32];
    float m, l;
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int b = 0; b < D / 32; ++b) o[b] = f32x16(0.f);
        m = MINUS_INF;
        l = 0.f;
    }
    // scores of 32 * B keys -> weights packed as the right operand of O^T += V^T P^T
    template <int B>
    __device__ __forceinline__ void weigh(f32x16 (&s)[B], float c, float slack, uint4 (&p)[2 * B]) {
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < B; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[b][r]);
        top = max_of_halves(top);
        if (ballot(top > m + slack)) {
            // a row that has seen nothing keeps a sum of 0: exp2(-inf - 0)
            const float next = fmaxf(m, top), f = exp2_fast((m - (next == MINUS_INF ? 0.f : next)) * c);
            l *= f;
#pragma unroll
            for (int b = 0; b < D / 32; ++b) o[b] *= f;
            m = next;
        }
        const float ref = m == MINUS_INF ? 0.f : m;
        const float shift = T::TOP - ref * c;
        float sum = 0.f;
#pragma unroll
        for (int b = 0; b < B; ++b) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[b][r] = exp2_fast(fmaf(s[b][r], c, shift));
#pragma unroll
            for (int r = 0; r < 16; r += 4) sum += (s[b][r] + s[b][r + 1]) + (s[b][r + 2] + s[b][r + 3]);
#pragma unroll
            for (int t = 0; t < 2; ++t)
                p[2 * b + t] = make_uint4(T::pack(s[b][8 * t], s[b][8 * t + 1]), T::pack(s[b][8 * t + 2], s[b][8 * t + 3]),
                                          T::pack(s[b][8 * t + 4], s[b][8 * t + 5]), T::pack(s[b][8 * t + 6], s[b][8 * t + 7]));
        }
        l += sum;
    }
    // O^T += V^T P^T over 16 keys, the first of them at `v`
    __device__ __forceinline__ void add(const char *v, const ValueAt<D> &at, uint4 p) {
#pragma unroll
        for (int b = 0; b < D / 32; ++b) {
            const uint2 lo = read_transposed(v + at.lo[b % 4] + b / 4 * 256), hi = read_transposed(v + at.hi[b % 4] + b / 4 * 256);
            o[b] = T::mfma(make_uint4(lo.x, lo.y, hi.x, hi.y), p, o[b]);
        }
    }
};

// key of score register r in its block of 32
__device__ __forceinline__ uint32_t key_of(uint32_t r, uint32_t half) { return 8 * (r / 4) + 4 * half + r % 4; }

// The factor of scores (base 2) for head h, as a positive number: its sign, or a
// zero, goes to the queries.
__device__ __forceinline__ float score_factor(const AttnArgs &a, uint32_t h, uint32_t *flip, bool *zero) {
    float c = a.scale * LOG2E;
    if (a.kv.k_scale) c *= a.kv.k_scale[h];
    *zero = c == 0.f;
    *flip = c < 0.f ? 0x80008000u : 0u;
    return *zero ? 1.f : fabsf(c);
}

// ------------------------------------------------------------ keys and values

// address of a slot's entry in `base`, the page taken as is (it is below n_pages)
__device__ __forceinline__ uint64_t entry_at(const KvView &kv, uint32_t page, uint32_t off, uint32_t head) {
    return page * kv.sp + off * kv.st + head * kv.sh;
}
// a table entry that does not fit reads page 0 (the join reports it)
__device__ __forceinline__ uint32_t page_of(const KvView &kv, uint32_t entry) { return entry < kv.n_pages ? entry : 0; }

// x with the elements that are not finite zeroed; *any is set if there are any
template <class T>
__device__ __forceinline__ uint32_t drop_not_finite(uint32_t w, bool *any) {
    const bool lo = (w & T::EXPONENT) == T::EXPONENT, hi = (w >> 16 & T::EXPONENT) == T::EXPONENT;
    *any |= lo | hi;
    return (lo ? 0 : w & 0xFFFFu) | (hi ? 0 : w & 0xFFFF0000u);
}
template <class T>
__device__ __forceinline__ uint4 drop_not_finite(uint4 x, bool *any) {
    return make_uint4(drop_not_finite<T>(x.x, any), drop_not_finite<T>(x.y, any), drop_not_finite<T>(x.z, any),
                      drop_not_finite<T>(x.w, any));
}

// log2 of a row's sum of exponentials, from its maximum and its sum relative to that.  A sum of
// zero is a row that sees nothing (or scores of -inf alone); the maximum does not say so:
// it passes over NaN, which is in the sum.
template <class T>
__device__ __forceinline__ float log_sum(float m, float l) {
    return l == 0.f ? MINUS_INF : m + __log2f(l) - T::TOP;
}

// ------------------------------------------------------------------ 4 bits

// The path for few rows over a cache in 4 bits (pc_attn4.hip): max_rows of a sequence and head; scores are kept
// where a.scores is there.
uint32_t rows4_resident(uint32_t dim, uint32_t max_rows);   // workgroups that the chip holds at once
pc_status attn_rows4(const AttnArgs &a, bool bf16, uint32_t dim, uint32_t max_rows, dim3 items, hipStream_t st);

}  // namespace pc
