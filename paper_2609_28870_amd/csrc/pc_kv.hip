// The paged cache of KV blocks: new tokens written into it (pc_kv_append), and
// sequences cut to the tokens with the most accumulated attention weight
// (pc_kv_evict).
#include "pc_kv.h"

namespace pc {

size_t type_size(uint32_t dtype) {
    switch (dtype) {
    case PC_BF16:
    case PC_F16: return 2;
    case PC_FP8_E4M3: return 1;
    }
    return 0;
}

pc_status kv_view(const pc_kv_cache *c, KvView *v) {
    if (!c || !c->k || !c->v) return PC_ERR_INVALID;
    const size_t size = type_size(c->dtype);
    if (!size) return PC_ERR_INVALID;
    const bool scaled = c->dtype == PC_FP8_E4M3;
    if (scaled != (c->k_scale != nullptr) || scaled != (c->v_scale != nullptr)) return PC_ERR_INVALID;
    if (c->page_size < 1 || c->page_size > PC_MAX_PAGE || c->n_kv_heads < 1 || c->n_kv_heads > PC_MAX_HEADS)
        return PC_ERR_INVALID;
    if (c->head_dim < 16 || c->head_dim > PC_MAX_HEAD_DIM || c->head_dim % 16 || c->n_pages < 1) return PC_ERR_INVALID;
    if (c->n_pages == PC_NONE) return PC_ERR_TOO_LARGE;
    // every access is of 16 bytes at a multiple of 16
    const uint64_t bits = (uint64_t)(uintptr_t)c->k | (uint64_t)(uintptr_t)c->v | c->stride_page * size |
                          c->stride_head * size | c->stride_slot * size;
    if (bits % 16) return PC_ERR_INVALID;
    *v = KvView{(char *)c->k, (char *)c->v, c->k_scale, c->v_scale, c->stride_page * size, c->stride_head * size,
                c->stride_slot * size, c->n_pages, c->n_kv_heads, c->head_dim, c->page_size, fast_div(c->page_size)};
    return PC_OK;
}

// ------------------------------------------------------------------- append
// A copy with an index: bound by memory, or for a few tokens by the one launch
// and its chain of loads (the row's sequence, its length, its page).

constexpr uint32_t APPEND_ROWS = 4;   // of a wave, where rows share one

struct AppendArgs {
    KvView kv;
    const uint32_t *table, *kv_len, *q_off;
    uint64_t table_stride;
    uint32_t n_seqs, n_rows, max_kv;
    const char *k, *v;   // strides in bytes
    uint64_t k_row, k_head, v_row, v_head;
    int32_t *status;
    FastDiv by_head;     // 16-byte pieces of one head's cache entry
    FastDiv by_token;    // and of a token's
    uint32_t pieces;     // of one token
};

// One word for the whole call, by the first workgroup: it looks at every
// sequence and every page that the call writes (a lane per page, 64 sequences at
// a time), so that no launch is spent on clearing a word that the others would set.
__device__ void append_status(const AppendArgs &a) {
    __shared__ int32_t wrong;
    if (threadIdx.x == 0) wrong = 0;
    __syncthreads();
    const int lane = threadIdx.x & (WAVE - 1), wave = threadIdx.x / WAVE, waves = blockDim.x / WAVE;
    bool any = threadIdx.x == 0 && (a.q_off[0] != 0 || a.q_off[a.n_seqs] != a.n_rows);
    for (uint32_t s0 = wave * WAVE; s0 < a.n_seqs; s0 += waves * WAVE) {
        const uint32_t s = s0 + lane;
        uint32_t from = 0, pages = 0;
        bool bad = false;
        if (s < a.n_seqs) {
            const Seq q = load_seq(a.q_off, a.kv_len, s, a.n_rows, a.max_kv, &bad);
            bad |= q.rows > q.len;
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
    if (any) wrong = DEV_ERR_BAD_LAYOUT;
    __syncthreads();
    if (threadIdx.x == 0) *a.status = wrong;
}

// slot of row t of sequence s, negative if it has none: by the length as it is, so that one above
// max_kv moves no row to another's slot
__device__ __forceinline__ int64_t slot_of_row(const AppendArgs &a, uint32_t s, const Seq &q, uint32_t t) {
    const int64_t slot = (int64_t)a.kv_len[s] - q.rows + (t - q.first);
    return slot < (int64_t)a.max_kv ? slot : -1;
}

__device__ __forceinline__ float to_float(uint32_t bits, bool bf16) {
    if (bf16) return __uint_as_float(bits << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}

// four elements (two words) to four codes
template <bool BF16>
__device__ __forceinline__ uint32_t to_e4m3(uint32_t a, uint32_t b, float scale) {
    float x[4] = {to_float(a & 0xFFFF, BF16), to_float(a >> 16, BF16), to_float(b & 0xFFFF, BF16), to_float(b >> 16, BF16)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float y = x[i] / scale;
        x[i] = y != y ? y : fminf(fmaxf(y, -448.f), 448.f);
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
    return (uint32_t)w;
}

// A wave a row, so that the row's chain of loads is all there is and its addresses are
// scalar.  MODE 0: the types agree; 1, 2: an 8-bit cache from bf16, f16.
// bf16, 4 heads of 128: 256 rows 2.8 us, 8,192 rows 7.5 us (33 MB, 4.5 TB/s).
template <int MODE>
__global__ __launch_bounds__(256) void append_few_kernel(AppendArgs a) {
    if (blockIdx.x == 0) {
        append_status(a);
        return;
    }
    const int lane = threadIdx.x & (WAVE - 1);
    const uint32_t t = (blockIdx.x - 1) * (256 / WAVE) + threadIdx.x / WAVE;
    if (t >= a.n_rows) return;
    const uint32_t s = seq_of(a.q_off, a.n_seqs, t);
    bool bad;
    const Seq q = load_seq(a.q_off, a.kv_len, s, a.n_rows, a.max_kv, &bad);
    if (t < q.first || t - q.first >= q.rows) return;
    const int64_t slot = slot_of_row(a, s, q, t);
    if (slot < 0) return;
    const uint32_t at = a.kv.by_page.div((uint32_t)slot), off = (uint32_t)slot - at * a.kv.page;
    const uint32_t page = a.table[(uint64_t)s * a.table_stride + at];
    if (page >= a.kv.n_pages) return;
    const uint64_t to = page * a.kv.sp + off * a.kv.st;
    for (uint32_t p = lane; p < a.pieces; p += WAVE) {
        const uint32_t h = a.by_head.div(p), c = p - h * a.by_head.d;
        const uint64_t dst = to + h * a.kv.sh + c * 16;
        const uint4 *k = (const uint4 *)(a.k + t * a.k_row + h * a.k_head) + c * (MODE ? 2 : 1);
        const uint4 *v = (const uint4 *)(a.v + t * a.v_row + h * a.v_head) + c * (MODE ? 2 : 1);
        if (MODE == 0) {
            const uint4 x = *k, y = *v;
            *(uint4 *)(a.kv.k + dst) = x;
            *(uint4 *)(a.kv.v + dst) = y;
        } else {
            const uint4 x0 = k[0], x1 = k[1], y0 = v[0], y1 = v[1];
            const float ks = a.kv.k_scale[h], vs = a.kv.v_scale[h];
            *(uint4 *)(a.kv.k + dst) = make_uint4(to_e4m3<MODE == 1>(x0.x, x0.y, ks), to_e4m3<MODE == 1>(x0.z, x0.w, ks),
                                                  to_e4m3<MODE == 1>(x1.x, x1.y, ks), to_e4m3<MODE == 1>(x1.z, x1.w, ks));
            *(uint4 *)(a.kv.v + dst) = make_uint4(to_e4m3<MODE == 1>(y0.x, y0.y, vs), to_e4m3<MODE == 1>(y0.z, y0.w, vs),
                                                  to_e4m3<MODE == 1>(y1.x, y1.y, vs), to_e4m3<MODE == 1>(y1.z, y1.w, vs));
        }
    }
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

// Four rows to a wave, whose lanes take the 16-byte pieces of their cache entries, so that
// the chain's wait is shared and no lane idles where a row has few of them.
// 21,100 rows of bf16 into an 8-bit cache (4 heads of 128, 65 MB): 18 us, 3.6 TB/s (a
// row a wave: 24.5).
template <int MODE>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
    constexpr int TOKENS = APPEND_ROWS;
    if (blockIdx.x == 0) {
        append_status(a);
        return;
    }
    const uint32_t lane = threadIdx.x & (WAVE - 1);
    const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / WAVE));
    const uint32_t t0 = ((blockIdx.x - 1) * (256 / WAVE) + wave) * TOKENS;
    if (t0 >= a.n_rows) return;
    const uint32_t s0 = wave_seq_of(a.q_off, a.n_seqs, t0), rows = min((uint32_t)TOKENS, a.n_rows - t0);
    constexpr int AT_ONCE = MODE ? 1 : 2, IN = MODE ? 2 : 1;   // 64 bytes a lane
    for (uint32_t p0 = lane; p0 < rows * a.pieces; p0 += AT_ONCE * WAVE) {
        uint4 x[AT_ONCE][IN], y[AT_ONCE][IN];
        uint64_t to[AT_ONCE];
        uint32_t head[AT_ONCE];
        bool there[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const uint32_t p = p0 + u * WAVE, i = min(a.by_token.div(p), rows - 1), t = t0 + i;
            const uint32_t of = p - i * a.pieces, h = a.by_head.div(of), c = of - h * a.by_head.d;
            uint32_t s = s0;   // or a later one, behind any number of empty ones
            if (s + 1 < a.n_seqs && a.q_off[s + 1] <= t) s += 1 + seq_of(a.q_off + s + 1, a.n_seqs - s - 1, t);
            bool bad;
            const Seq q = load_seq(a.q_off, a.kv_len, s, a.n_rows, a.max_kv, &bad);
            const int64_t slot = slot_of_row(a, s, q, t);
            there[u] = p < rows * a.pieces && t >= q.first && t - q.first < q.rows && slot >= 0;
            if (!there[u]) continue;
            const uint32_t at = a.kv.by_page.div((uint32_t)slot), off = (uint32_t)slot - at * a.kv.page;
            const uint32_t page = a.table[(uint64_t)s * a.table_stride + at];
            there[u] = page < a.kv.n_pages;
            to[u] = page * a.kv.sp + off * a.kv.st + h * a.kv.sh + c * 16;
            head[u] = h;
            const uint4 *k = (const uint4 *)(a.k + t * a.k_row + h * a.k_head) + c * IN;
            const uint4 *v = (const uint4 *)(a.v + t * a.v_row + h * a.v_head) + c * IN;
#pragma unroll
            for (int j = 0; j < IN; ++j) {
                x[u][j] = k[j];
                y[u][j] = v[j];
            }
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            if (!there[u]) continue;
            if (MODE) {
                constexpr int HI = IN - 1;
                const float ks = a.kv.k_scale[head[u]], vs = a.kv.v_scale[head[u]];
                const uint4 x0 = x[u][0], x1 = x[u][HI], y0 = y[u][0], y1 = y[u][HI];
                *(uint4 *)(a.kv.k + to[u]) = make_uint4(to_e4m3<MODE == 1>(x0.x, x0.y, ks), to_e4m3<MODE == 1>(x0.z, x0.w, ks),
                                                        to_e4m3<MODE == 1>(x1.x, x1.y, ks), to_e4m3<MODE == 1>(x1.z, x1.w, ks));
                *(uint4 *)(a.kv.v + to[u]) = make_uint4(to_e4m3<MODE == 1>(y0.x, y0.y, vs), to_e4m3<MODE == 1>(y0.z, y0.w, vs),
                                                        to_e4m3<MODE == 1>(y1.x, y1.y, vs), to_e4m3<MODE == 1>(y1.z, y1.w, vs));
            } else {
                *(uint4 *)(a.kv.k + to[u]) = x[u][0];
                *(uint4 *)(a.kv.v + to[u]) = y[u][0];
            }
        }
    }
}

// Rows share a wave where their pieces (of 16 bytes in the cache) leave most of one idle.  Us of a wave
// a row / of four rows a wave, in 24 sequences:
//   8-bit cache    8 pieces: 64 rows 6.6 / 3.4, 8,192 rows 11.5 / 5.9;  16: 4.0 / 3.4, 10.3 / 6.3;
//                  32: 64 rows 3.8 / 5.1, 2,048 rows 5.1 / 5.4, 8,192 rows 11.1 / 8.0;  48: 3.8 / 6.7, 7.4 / 8.0
//                  (4,096), 12.2 / 11.4;  64: 13.6 / 15.2 (8,192), 37.5 / 39.8 (32,768)
//   16-bit cache   8 pieces: 16,384 rows 9.8 / 17.3, 65,536 rows 35.4 / 32.5 (256 sequences: 32.1 / 23.1);
//                  32: 10.8 / 19.2, 38.4 / 40.5 (34.8 / 29.7);  64: 13.9 / 23.0, 60.9 / 62.9 (62.9 / 63.5)
// And 2^26 rows, a wave each, are more than a launch holds.
static bool append_many(uint32_t n_rows, uint32_t pieces, bool f8) {
    if (n_rows >= 1u << 26) return true;
    if (f8) return pieces <= 16 || (pieces < 64 && n_rows >= 8192);
    return pieces <= 32 && n_rows >= 65536;
}
static uint64_t append_groups(uint32_t n_rows, bool many) {
    const uint32_t per = (many ? APPEND_ROWS : 1) * (256 / WAVE);
    return 1 + ((uint64_t)n_rows + per - 1) / per;
}

template <int MODE>
static pc_status append_run(const AppendArgs &a, bool many, hipStream_t st) {
    const dim3 grid((unsigned)append_groups(a.n_rows, many));
    if (many) PC_LAUNCH(K_KV_APPEND, append_kernel<MODE>, grid, dim3(256), 0, st, a);
    else PC_LAUNCH(K_KV_APPEND, append_few_kernel<MODE>, grid, dim3(256), 0, st, a);
    return PC_OK;
}

// -------------------------------------------------------------------- evict

struct EvictArgs {
    KvView kv;
    const uint32_t *table, *kv_len, *dst_table;
    uint64_t table_stride, dst_stride, weight_stride;
    uint32_t n_seqs, max_kv, budget, recent;
    const float *weight;
    uint32_t *kept, *new_len;
    float *weight_out;
    int32_t *status;
    FastDiv by_piece;   // 16-byte pieces of one entry
};

// floats as integers of the same order; the zeros are one value, and so are the NaN, above all others
__device__ __forceinline__ uint32_t order_of(float f) {
    if (f != f) return 0xFFFFFFFFu;
    const uint32_t b = __float_as_uint(f + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

constexpr int SELECT_THREADS = 1024, SELECT_WAVES = SELECT_THREADS / WAVE;
constexpr uint32_t DIGITS = 2048;   // bins of a histogram

// Adds this lane's digit to the histogram.  Weights are heavy-tailed and often tied, so
// most lanes of a wave meet in one bin, where atomics would follow each other: the
// first lane adds for all that have its digit, the others for themselves.
__device__ __forceinline__ void count_digit(uint32_t *hist, bool in, uint32_t digit) {
    const uint64_t all = ballot(in);
    if (!all) return;
    const uint32_t lead = (uint32_t)__ffsll((unsigned long long)all) - 1;
    const bool same = in & (digit == (uint32_t)__builtin_amdgcn_readlane((int)digit, (int)lead));
    const uint32_t n = (uint32_t)__popcll(ballot(same)), lane = threadIdx.x & (WAVE - 1);
    if (in & (!same | (lane == lead))) atomicAdd(&hist[digit], same ? n : 1u);
}

// What one (sequence, head) keeps: `need` of the first `cand` slots, and all behind them.
struct EvictRow {
    uint32_t s, h, cand, need, n;
    const float *w;
    uint32_t *kept;
    float *wout;   // or nullptr
};
__device__ __forceinline__ EvictRow evict_row(const EvictArgs &a, uint32_t row) {
    EvictRow r;
    r.s = row / a.kv.n_kv;
    r.h = row - r.s * a.kv.n_kv;
    const uint32_t len = min(a.kv_len[r.s], a.max_kv);
    r.n = min(len, a.budget);
    const uint32_t late = min(a.recent, r.n);
    r.cand = len - late;
    r.need = r.n - late;
    r.w = a.weight + (uint64_t)row * a.weight_stride;
    r.kept = a.kept + (uint64_t)row * a.budget;
    r.wout = a.weight_out ? a.weight_out + (uint64_t)row * a.budget : nullptr;
    return r;
}
// the call's status word (the pages are the move's to check), by one workgroup
__device__ __forceinline__ void evict_status(const EvictArgs &a) {
    bool bad = false;
    for (uint32_t i = threadIdx.x; i < a.n_seqs; i += SELECT_THREADS) bad |= a.kv_len[i] > a.max_kv;
    const int any = __syncthreads_or(bad);
    if (threadIdx.x == 0) *a.status = any ? DEV_ERR_BAD_LAYOUT : 0;
}
// the places that need no choice: the last slots, and none behind them (part of `parts`)
__device__ __forceinline__ void place_rest(const EvictArgs &a, const EvictRow &e, uint32_t part, uint32_t parts) {
    if (e.h == 0 && part == 0 && threadIdx.x == 0) a.new_len[e.s] = e.n;
    for (uint32_t r = e.need + part * SELECT_THREADS + threadIdx.x; r < a.budget; r += parts * SELECT_THREADS) {
        const uint32_t j = e.cand + (r - e.need);
        e.kept[r] = r < e.n ? j : NONE;
        if (e.wout) e.wout[r] = r < e.n ? e.w[j] : 0.f;
    }
}
// This thread's slots j0 + 64 i: their weights, and the keys that order them.  Key 0 is no
// weight's: slots past the candidates.
template <int N>
struct SlotKeys {
    float x[N];
    uint32_t key[N];
    __device__ __forceinline__ SlotKeys(const EvictRow &e, uint32_t j0) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = e.w[min(j0 + i * WAVE, e.cand - 1)];
#pragma unroll
        for (int i = 0; i < N; ++i) key[i] = j0 + i * WAVE < e.cand ? order_of(x[i]) : 0;
    }
};
// digit number 0, 1 or 2 of a key, from the top
__device__ __forceinline__ uint32_t digit_shift(int digit) { return digit == 0 ? 21 : digit == 1 ? 10 : 0; }
template <int N>
__device__ __forceinline__ void count_digits(uint32_t *hist, const uint32_t (&key)[N], int digit, uint32_t known) {
    const uint32_t shift = digit_shift(digit), bins = digit == 2 ? 1024 : 2048;
    const uint32_t mask = digit == 0 ? 0 : digit == 1 ? ~0u << 21 : ~0u << 10;
    hist[threadIdx.x] = hist[threadIdx.x + SELECT_THREADS] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) count_digit(hist, (key[i] != 0) & ((key[i] & mask) == known), key[i] >> shift & (bins - 1));
    __syncthreads();
}
// The digit of the `equal`-th largest key, from the counts of two digits a thread (the
// largest digits first); *equal becomes its place among the keys of that digit.
__device__ __forceinline__ uint32_t pick_digit(uint32_t hi, uint32_t lo, uint32_t *equal, uint32_t *tmp) {
    __shared__ uint32_t pick, left;
    uint32_t total;
    const uint32_t above = block_excl_scan(hi + lo, tmp, &total);
    if (above < *equal && above + hi + lo >= *equal) {
        const bool first = above + hi >= *equal;
        pick = DIGITS - 1 - 2 * threadIdx.x - (first ? 0 : 1);
        left = *equal - above - (first ? 0 : hi);
    }
    __syncthreads();
    *equal = left;
    return pick;
}
// The kept ones of a workgroup's keys to their places, from `at` on: those above floor_key, and
// `quota` at most of those equal to it.  A wave's slots are consecutive, and so are the waves'.
template <int N>
__device__ __forceinline__ void place_kept(const EvictRow &e, const SlotKeys<N> &slots, uint32_t j0, uint32_t floor_key, uint32_t at,
                                           uint32_t quota) {
    __shared__ uint32_t above_of[SELECT_WAVES], ties_of[SELECT_WAVES];
    const uint32_t(&key)[N] = slots.key;
    const uint32_t tid = threadIdx.x, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid / WAVE));
    uint32_t above = 0, ties = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        above += (uint32_t)__popcll(ballot(key[i] > floor_key));
        ties += (uint32_t)__popcll(ballot((key[i] != 0) & (key[i] == floor_key)));
    }
    if (tid % WAVE == 0) {
        above_of[wave] = above;
        ties_of[wave] = ties;
    }
    __syncthreads();
    for (uint32_t i = 0; i < wave; ++i) {
        const uint32_t t = min(ties_of[i], quota);
        at += above_of[i] + t;
        quota -= t;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bool tie = (key[i] != 0) & (key[i] == floor_key);
        const uint64_t tied = ballot(tie);
        const bool keep = (key[i] > floor_key) | (tie & (mbcnt_acc(tied, 0) < quota));
        quota -= min(quota, (uint32_t)__popcll(tied));
        const uint64_t all = ballot(keep);
        if (keep) {
            const uint32_t r = at + mbcnt_acc(all, 0);
            if (r < e.need) {   // also where another stream changes the weights between two launches
                e.kept[r] = j0 + i * WAVE;
                if (e.wout) e.wout[r] = slots.x[i];
            }
        }
        at += (uint32_t)__popcll(all);
    }
}

// The selection: the need-th largest weight by digits of 11, 11 and 10 bits (a histogram
// each), then the kept slots in order.  Bound by one compute unit's instructions, about
// 25 a slot and pass, and by a few waits.

// Rows of up to 8192 slots: one workgroup per (sequence, head), the keys in registers.
// 4 rows of 4,099 slots: 10 us (reading them again for each pass of 8-bit digits: 17.5).
constexpr int ROW_KEYS = 8;
__global__ __launch_bounds__(SELECT_THREADS) void evict_select_kernel(EvictArgs a) {
    __shared__ uint32_t hist[DIGITS], tmp[SELECT_WAVES];
    if (blockIdx.x == 0) evict_status(a);
    const EvictRow e = evict_row(a, blockIdx.x);
    place_rest(a, e, 0, 1);
    if (!e.need) return;
    const uint32_t tid = threadIdx.x, j0 = tid / WAVE * (ROW_KEYS * WAVE) + tid % WAVE;
    const SlotKeys<ROW_KEYS> slots(e, j0);
    uint32_t floor_key = 0, equal = 0;   // keys above floor_key stay, and `equal` of those at it
    if (e.need < e.cand) {
        equal = e.need;
#pragma unroll 1   // small code: of a few-microsecond call much is the first fetch of its instructions
        for (int digit = 0; digit < 3; ++digit) {
            count_digits(hist, slots.key, digit, floor_key);
            floor_key |= pick_digit(hist[DIGITS - 1 - 2 * tid], hist[DIGITS - 2 - 2 * tid], &equal, tmp) << digit_shift(digit);
        }
    }
    place_kept(e, slots, j0, floor_key, 0, equal);
}

// Longer rows: a workgroup per segment of 16384 slots, and a launch per digit, since
// the segments have to meet: each phase adds up its row's histograms of the digit before
// and counts the next; the last one places.  What a segment needs to know of those
// before it (the keys above the digit) follows from their histograms.
// 16 sequences of 4 heads, 303k slots, the longest 65,536: 33 us in four launches (one workgroup a row: 60, keys
// in registers, or 71).
constexpr int SEGMENT_KEYS = 16;
constexpr uint32_t SEGMENT = SEGMENT_KEYS * SELECT_THREADS;
struct EvictSplit {
    uint32_t segments;   // of a row
    uint64_t all;        // of the call
    uint32_t *hist;      // [2][row][segment][digit], used in turn
    uint32_t *above;     // [2][row][segment] keys above the first and second digit
    uint2 *state;        // [2][row] digits known, place among the keys that have them
};
template <int PHASE>
__global__ __launch_bounds__(SELECT_THREADS) void evict_split_kernel(EvictArgs a, EvictSplit b) {
    __shared__ uint32_t hist[DIGITS], tmp[SELECT_WAVES];
    __shared__ uint32_t tied;
    const uint32_t row = blockIdx.x / b.segments, segment = blockIdx.x - row * b.segments, tid = threadIdx.x;
    if (PHASE == 0 && blockIdx.x == 0) evict_status(a);
    const EvictRow e = evict_row(a, row);
    if (PHASE == 3) place_rest(a, e, segment, b.segments);
    if (!e.need || segment * SEGMENT >= e.cand) return;
    const bool all = e.need == e.cand;
    if (PHASE < 3 && all) return;
    const uint32_t j0 = segment * SEGMENT + tid / WAVE * (SEGMENT_KEYS * WAVE) + tid % WAVE;
    const SlotKeys<SEGMENT_KEYS> slots(e, j0);
    if (all) {
        place_kept(e, slots, j0, 0, segment * SEGMENT, 0);
        return;
    }
    uint32_t floor_key = 0, equal = e.need;
    uint32_t before = 0, tied_before = 0;   // of the segments before: keys that stay, keys at floor_key
    if (PHASE > 0) {
        if (PHASE > 1) {
            const uint2 x = b.state[(uint64_t)(PHASE - 2) * (b.all / b.segments) + row];
            floor_key = x.x;
            equal = x.y;
        }
        const uint32_t *level = b.hist + ((uint64_t)((PHASE - 1) % 2) * b.all + (uint64_t)row * b.segments) * DIGITS;
        const uint32_t there = (e.cand + SEGMENT - 1) / SEGMENT, digit = DIGITS - 1 - 2 * tid;   // and the one below
        uint32_t hi = 0, lo = 0, mine_hi = 0, mine_lo = 0;   // mine: this segment's, at last those before it
#pragma unroll 4
        for (uint32_t g = 0; g < there; ++g) {
            const uint2 x = *(const uint2 *)(level + (uint64_t)g * DIGITS + digit - 1);
            hi += x.y;
            lo += x.x;
            const bool count = PHASE < 3 ? g == segment : g < segment;
            mine_hi += count ? x.y : 0;
            mine_lo += count ? x.x : 0;
        }
        const uint32_t pick = pick_digit(hi, lo, &equal, tmp);
        floor_key |= pick << digit_shift(PHASE - 1);
        if (PHASE == 3 && (pick == digit || pick == digit - 1)) tied = pick == digit ? mine_hi : mine_lo;
        uint32_t above;
        block_excl_scan((digit > pick ? mine_hi : 0) + (digit - 1 > pick ? mine_lo : 0), tmp, &above);
        if (PHASE < 3) {
            if (tid == 0) b.above[(uint64_t)(PHASE - 1) * b.all + blockIdx.x] = above;
            if (tid == 0 && segment == 0) b.state[(uint64_t)(PHASE - 1) * (b.all / b.segments) + row] = make_uint2(floor_key, equal);
        } else {
            before = above;
            for (uint32_t g = 0; g < segment; ++g)
                before += b.above[(uint64_t)row * b.segments + g] + b.above[b.all + (uint64_t)row * b.segments + g];
            tied_before = tied;
        }
    }
    if (PHASE < 3) {
        count_digits(hist, slots.key, PHASE, floor_key);
        uint32_t *out = b.hist + ((uint64_t)(PHASE % 2) * b.all + blockIdx.x) * DIGITS;
        out[tid] = hist[tid];
        out[tid + SELECT_THREADS] = hist[tid + SELECT_THREADS];
        return;
    }
    place_kept(e, slots, j0, floor_key, before + min(tied_before, equal), equal - min(tied_before, equal));
}

constexpr uint32_t MOVE_SLOTS = 64;   // slots of one (sequence, head) per workgroup

// Keys and values of the kept slots, each a run of 16-byte pieces: bound by memory.  (Pieces
// looked up and loaded four at a time took 100 us for what this does in 84, and 9 for 4.)
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a, uint32_t groups) {
    const uint32_t row = blockIdx.x / groups, r0 = (blockIdx.x - row * groups) * MOVE_SLOTS;
    const uint32_t s = row / a.kv.n_kv, h = row - s * a.kv.n_kv;
    const uint32_t n = min(min(a.kv_len[s], a.max_kv), a.budget);
    if (r0 >= n) return;
    const uint32_t slots = min(MOVE_SLOTS, n - r0), pieces = slots * a.by_piece.d;
    for (uint32_t p = threadIdx.x; p < pieces; p += 256) {
        const uint32_t i = a.by_piece.div(p), c = p - i * a.by_piece.d, r = r0 + i;
        const uint32_t j = min(a.kept[(uint64_t)row * a.budget + r], a.max_kv - 1);   // in bounds whatever else is written there
        const uint32_t js = a.kv.by_page.div(j), rs = a.kv.by_page.div(r);
        const uint32_t from = a.table[(uint64_t)s * a.table_stride + js], to = a.dst_table[(uint64_t)s * a.dst_stride + rs];
        if (from >= a.kv.n_pages || to >= a.kv.n_pages) {
            atomicOr(a.status, DEV_ERR_BAD_LAYOUT);
            continue;
        }
        const uint64_t src = from * a.kv.sp + h * a.kv.sh + (j - js * a.kv.page) * a.kv.st + c * 16;
        const uint64_t dst = to * a.kv.sp + h * a.kv.sh + (r - rs * a.kv.page) * a.kv.st + c * 16;
        const uint4 x = *(const uint4 *)(a.kv.k + src), y = *(const uint4 *)(a.kv.v + src);
        *(uint4 *)(a.kv.k + dst) = x;
        *(uint4 *)(a.kv.v + dst) = y;
    }
}

static bool evict_split(uint32_t max_kv) { return max_kv > (uint32_t)ROW_KEYS * SELECT_THREADS; }
static size_t evict_carve(char *ws, uint64_t rows, uint32_t max_kv, int32_t **status, EvictSplit *b) {
    Carver c{ws, 0};
    *status = c.take<int32_t>(WS_HEADER / 4);
    if (evict_split(max_kv)) {
        b->segments = (max_kv + SEGMENT - 1) / SEGMENT;
        b->all = rows * b->segments;
        b->hist = c.take<uint32_t>(2 * b->all * DIGITS);
        b->above = c.take<uint32_t>(2 * b->all);
        b->state = c.take<uint2>(2 * rows);
    }
    return c.off;
}

// whether a result shares memory with another, or with the weights that are still read
static bool evict_overlaps(uint32_t rows, uint32_t n_seqs, uint32_t max_kv, const float *weight, uint64_t weight_stride, uint32_t budget,
                           const uint32_t *kept, const float *weight_out, const uint32_t *new_len) {
    const uint64_t out = (uint64_t)rows * budget * 4, in = rows && max_kv ? ((rows - 1) * weight_stride + max_kv) * 4 : 0;
    const void *base[4] = {weight, kept, new_len, weight_out};
    const uint64_t bytes[4] = {in, out, n_seqs * 4ull, weight_out ? out : 0};
    for (int i = 0; i < 4; ++i)
        for (int j = i + 1; j < 4; ++j)
            if (overlap(base[i], bytes[i], base[j], bytes[j])) return true;
    return false;
}

}  // namespace pc

extern "C" {

size_t pc_kv_append_ws(void) { return pc::WS_HEADER; }

pc_status pc_kv_append(const pc_kv_cache *cache, const uint32_t *page_table, uint64_t table_stride,
                       const uint32_t *kv_len, const uint32_t *q_off, uint32_t n_seqs, uint32_t n_rows,
                       uint32_t max_kv, const void *k, uint64_t k_stride_row, uint64_t k_stride_head,
                       const void *v, uint64_t v_stride_row, uint64_t v_stride_head, uint32_t dtype, void *ws,
                       size_t ws_bytes, void *stream) {
    using namespace pc;
    AppendArgs a;
    const pc_status ok = kv_view(cache, &a.kv);
    if (ok != PC_OK) return ok;
    if (dtype != PC_BF16 && dtype != PC_F16) return PC_ERR_INVALID;
    if (cache->dtype != dtype && cache->dtype != PC_FP8_E4M3) return PC_ERR_INVALID;
    const bool f8 = cache->dtype == PC_FP8_E4M3;
    a.by_head = fast_div((uint32_t)(a.kv.dim * type_size(cache->dtype) / 16));
    a.pieces = a.by_head.d * a.kv.n_kv;
    a.by_token = fast_div(a.pieces);
    const bool many = append_many(n_rows, a.pieces, f8);
    if (n_seqs >= 0x80000000u || n_rows >= 0x80000000u || max_kv > 0x7FFF0000u || !launch_fits(append_groups(n_rows, many), 256))
        return PC_ERR_TOO_LARGE;
    if (max_kv > table_stride * a.kv.page) return PC_ERR_INVALID;
    if (!kv_len || !q_off || (max_kv && !page_table) || (n_rows && (!k || !v))) return PC_ERR_INVALID;
    if (((uint64_t)(uintptr_t)k | (uint64_t)(uintptr_t)v | k_stride_row * 2 | k_stride_head * 2 | v_stride_row * 2 |
         v_stride_head * 2) % 16)
        return PC_ERR_INVALID;
    if (n_seqs == 0 && n_rows) return PC_ERR_INVALID;
    if (!ws || ws_bytes < pc_kv_append_ws()) return PC_ERR_WORKSPACE;
    const hipStream_t st = (hipStream_t)stream;
    a.table = page_table;
    a.kv_len = kv_len;
    a.q_off = q_off;
    a.table_stride = table_stride;
    a.n_seqs = n_seqs;
    a.n_rows = n_rows;
    a.max_kv = max_kv;
    a.k = (const char *)k;
    a.v = (const char *)v;
    a.k_row = k_stride_row * 2;
    a.k_head = k_stride_head * 2;
    a.v_row = v_stride_row * 2;
    a.v_head = v_stride_head * 2;
    a.status = (int32_t *)ws;
    if (!f8) return append_run<0>(a, many, st);
    return dtype == PC_BF16 ? append_run<1>(a, many, st) : append_run<2>(a, many, st);
}

size_t pc_kv_evict_ws(uint32_t n_seqs, uint32_t n_kv_heads, uint32_t max_kv) {
    pc::EvictSplit b;
    int32_t *status;
    return pc::evict_carve(nullptr, (uint64_t)n_seqs * n_kv_heads, max_kv, &status, &b);
}

pc_status pc_kv_evict(const pc_kv_cache *cache, const uint32_t *page_table, uint64_t table_stride,
                      const uint32_t *kv_len, uint32_t n_seqs, uint32_t max_kv, const float *weight,
                      uint64_t weight_stride, uint32_t budget, uint32_t recent, const uint32_t *dst_table,
                      uint64_t dst_stride, uint32_t *kept, float *weight_out, uint32_t *new_len, void *ws,
                      size_t ws_bytes, void *stream) {
    using namespace pc;
    EvictArgs a;
    const pc_status ok = kv_view(cache, &a.kv);
    if (ok != PC_OK) return ok;
    if (budget < 1 || recent > budget) return PC_ERR_INVALID;
    if (max_kv > 0x7FFF0000u || budget > 0x7FFF0000u || (uint64_t)n_seqs * a.kv.n_kv > 0x7FFFFFFFu) return PC_ERR_TOO_LARGE;
    if (max_kv > weight_stride) return PC_ERR_INVALID;
    if (n_seqs && (!kv_len || !kept || !new_len || (max_kv && !weight))) return PC_ERR_INVALID;
    if (dst_table && (max_kv > table_stride * a.kv.page || budget > dst_stride * a.kv.page || (max_kv && !page_table)))
        return PC_ERR_INVALID;
    EvictSplit b;
    const uint32_t rows = n_seqs * a.kv.n_kv, groups = (budget < max_kv ? budget : max_kv) / MOVE_SLOTS + 1;
    const size_t need = evict_carve((char *)ws, rows, max_kv, &a.status, &b);
    if (!launch_fits(evict_split(max_kv) ? b.all : rows, SELECT_THREADS) || (dst_table && !launch_fits((uint64_t)rows * groups, 256)))
        return PC_ERR_TOO_LARGE;
    if (!ws || ws_bytes < need) return PC_ERR_WORKSPACE;
    if (evict_overlaps(rows, n_seqs, max_kv, weight, weight_stride, budget, kept, weight_out, new_len)) return PC_ERR_INVALID;
    const hipStream_t st = (hipStream_t)stream;
    if (n_seqs == 0) return fill_u32((uint32_t *)ws, 0, 1, st);
    a.table = page_table;
    a.kv_len = kv_len;
    a.dst_table = dst_table;
    a.table_stride = table_stride;
    a.dst_stride = dst_stride;
    a.weight_stride = weight_stride;
    a.n_seqs = n_seqs;
    a.max_kv = max_kv;
    a.budget = budget;
    a.recent = recent;
    a.weight = weight;
    a.kept = kept;
    a.new_len = new_len;
    a.weight_out = weight_out;
    a.by_piece = fast_div((uint32_t)(a.kv.dim * type_size(cache->dtype) / 16));
    if (evict_split(max_kv)) {
        const dim3 grid((unsigned)b.all);
        PC_LAUNCH(K_KV_EVICT_SELECT, evict_split_kernel<0>, grid, dim3(SELECT_THREADS), 0, st, a, b);
        PC_LAUNCH(K_KV_EVICT_SELECT, evict_split_kernel<1>, grid, dim3(SELECT_THREADS), 0, st, a, b);
        PC_LAUNCH(K_KV_EVICT_SELECT, evict_split_kernel<2>, grid, dim3(SELECT_THREADS), 0, st, a, b);
        PC_LAUNCH(K_KV_EVICT_SELECT, evict_split_kernel<3>, grid, dim3(SELECT_THREADS), 0, st, a, b);
    } else {
        PC_LAUNCH(K_KV_EVICT_SELECT, evict_select_kernel, dim3(rows), dim3(SELECT_THREADS), 0, st, a);
    }
    if (dst_table) PC_LAUNCH(K_KV_EVICT_MOVE, evict_move_kernel, dim3(rows * groups), dim3(256), 0, st, a, groups);
    return PC_OK;
}

}  // extern "C"
