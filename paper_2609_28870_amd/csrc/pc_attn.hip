// Attention of new tokens over the paged cache (pc_attn_paged): the path for few
// rows (decode, drafted tokens), the path for chunks, the join of partial results
// and the accumulated weights.
#include <math.h>

#include <type_traits>

#include "pc_attn.h"

namespace pc {

// Values that are not finite, in tiles whose keys some rows see and some do not: the
// matrix product would carry 0 * inf = NaN to rows that do not see the key.  Such a
// tile is worked on without them, and where there were any they are added here, after
// the loop, to the rows that see them: key by key, the scores formed again.  Rare,
// so written for size.  `query` is this lane's row of 16-bit elements.
template <class T, Held H, int D, class Query>
__device__ __forceinline__ void add_not_finite(Rows<T, D> &state, const AttnArgs &a, uint32_t seq, uint32_t head, uint32_t key,
                                               int32_t first, int32_t last, float c, Query query) {
    const uint32_t lane = threadIdx.x & (WAVE - 1), half = lane / 32;
    const uint32_t at = a.kv.by_page.div(key), page = page_of(a.kv, a.table[(uint64_t)seq * a.table_stride + at]);
    const uint64_t entry = entry_at(a.kv, page, key - at * a.kv.page, head);
    auto element = [&](bool value, uint32_t d) {
        const char *x = (value ? a.kv.v : a.kv.k) + entry + held_bytes<H>(d);
        if (H == Held::E4M3) return T::value(T::template from_e4m3<false>(*(const uint8_t *)x) & 0xFFFF);
        if (H == Held::E2M1) {
            const float scale = scale_of((value ? a.kv.v_exp : a.kv.k_exp)[entry / 16 + d / 32]);
            return T::value(T::template from_e2m1<0>(*(const uint8_t *)x >> 4 * (d % 2), scale) & 0xFFFF);
        }
        return T::value(*(const uint16_t *)x);
    };
    bool odd = false;
    for (uint32_t d = lane; d < a.kv.dim; d += WAVE) odd |= !(fabsf(element(true, d)) < __builtin_inff());
    if (!ballot(odd)) return;
    float s = 0.f;
#pragma unroll 1
    for (uint32_t d = half; d < a.kv.dim; d += 2) s = fmaf(T::value(query(d)), element(false, d), s);
    s = sum_of_halves(s);
    const float p = exp2_fast(fmaf(s, c, T::TOP - state.m * c));
    const bool visible = (int32_t)key >= first && (int32_t)key <= last;
    if constexpr (H == Held::E2M1) {
        // four codes are two bytes, and a block has one scale
        const char *x = a.kv.v + entry + 2 * half;
        const uint8_t *exponents = a.kv.v_exp + entry / 16;
#pragma unroll
        for (int b = 0; b < D / 32; ++b) {
            if (32u * b >= a.kv.dim) break;
            const float scale = scale_of(exponents[b]);
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const uint32_t w = *(const uint16_t *)(x + 16 * b + r);
                const uint32_t lo = T::template from_e2m1<0>(w, scale), hi = T::template from_e2m1<1>(w, scale);
                const float y[4] = {T::value(lo & 0xFFFF), T::value(lo >> 16), T::value(hi & 0xFFFF), T::value(hi >> 16)};
#pragma unroll
                for (int i = 0; i < 4; ++i) state.o[b][r + i] += visible && !(fabsf(y[i]) < __builtin_inff()) ? p * y[i] : 0.f;
                __asm__ volatile("" ::: "memory");   // few of the loads at once: the registers are full
            }
        }
        return;
    }
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const uint32_t d = 32 * b + key_of(r, half);
            const float x = element(true, d < a.kv.dim ? d : 0);
            state.o[b][r] += visible && !(fabsf(x) < __builtin_inff()) ? p * x : 0.f;
            if (r % 4 == 3) __asm__ volatile("" ::: "memory");   // few of the loads at once: the registers are full
        }
}

// A row's result: whole (its sequence is one item long), or a part for the join.
template <class T, int D>
__device__ __forceinline__ void write_rows(const AttnArgs &a, const Item &it, const f32x16 (&o)[D / 32], float m, float l,
                                           uint32_t at, uint32_t t, uint32_t head, uint32_t half) {
    if (it.splits > 1) {
        if (it.slot >= a.slots) return;
        const uint64_t row = (uint64_t)it.slot * a.slot_rows + at;
        if (half == 0) a.part_ml[row] = make_float2(m, l);
#pragma unroll
        for (int b = 0; b < D / 32; ++b)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *(float4 *)(a.part + row * D + 32 * b + key_of(r, half)) =
                    make_float4(o[b][r], o[b][r + 1], o[b][r + 2], o[b][r + 3]);
        return;
    }
    const float base2 = log_sum<T>(m, l);
    const float f = l == 0.f ? 0.f : (a.kv.v_scale ? a.kv.v_scale[it.head] : 1.f) / l;
    if (half == 0) {
        if (a.lse) a.lse[(uint64_t)t * a.n_heads + head] = base2 * LN2;
        if (a.lse2) a.lse2[(uint64_t)t * a.n_heads + head] = base2;
    }
    char *out = a.out + (uint64_t)t * a.o_row + head * a.o_head;
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const uint32_t d = 32 * b + key_of(r, half);
            if (d < a.kv.dim)
                *(uint2 *)(out + 2 * d) = make_uint2(T::pack(o[b][r] * f, o[b][r + 1] * f), T::pack(o[b][r + 2] * f, o[b][r + 3] * f));
        }
}

// ------------------------------------------------------------------ few rows

// At most 32 rows (new tokens times the query heads that share a key/value head)
// of a sequence against a range of its keys.  Bound by the bytes of keys and
// values: a wave takes 32 keys at a time on its own (every fourth such tile of the
// item), the next tile's bytes on their way to its registers meanwhile.  Keys
// go straight into the matrix product, a lane per key; values pass through
// LDS for the transposed read.  The four waves' results are joined in LDS.
// FULL: the head has D dimensions, and no piece of a key is past them.
// 32 over 4 heads of 128, 1.05M keys in 8 even sequences: bf16 384 us, 8-bit 194 us (5.6 TB/s; a
// plain read of 4 GiB: 6.3); 618k keys in 63 uneven ones, bf16, 254 us (5.0 TB/s: ranges end at different
// times); one token over 1,537 keys 11 us, a chain of dependent loads.
template <class T, Held H, int D, bool FULL, bool WEIGHTS>
__global__ __launch_bounds__(256, D <= 128 ? 2 : 1) void rows_kernel(AttnArgs a) {
    constexpr bool F8 = H == Held::E4M3;
    constexpr int PIECES = F8 ? D / 32 : D / 16;   // 16 bytes, of one lane's half of a key
    __shared__ __attribute__((aligned(16))) char tiles[4 * 32 * D * 2];
    __shared__ __attribute__((aligned(16))) char queries[32 * D * 2];   // the same for all waves
    __shared__ float2 join_ml[2][64];
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = 0;
    const Item it = find_item<By::ITEM>(a, blockIdx.x);
    if (!it.there) return;
    const uint32_t lane = threadIdx.x & (WAVE - 1), half = lane / 32, wave = uniform(threadIdx.x / WAVE), col = lane % 32;
    const Seq &sq = it.shape.q;
    const uint32_t rows = sq.rows * a.group;
    uint32_t flip;
    bool zero;
    const float c = score_factor(a, it.head, &flip, &zero);
    // this lane's row
    const bool valid = col < rows;
    const uint32_t token = a.by_group.div(col), head = it.head * a.group + (col - token * a.group);
    int32_t first = 0, last = 0x7FFFFFFF;
    if (valid) seen_by_row(a, sq, token, &first, &last);
    int32_t all_first = first, all_last = last;   // keys that every row sees
#pragma unroll
    for (int step = 1; step < 32; step *= 2) {
        all_first = max(all_first, __shfl_xor(all_first, step, WAVE));
        all_last = min(all_last, __shfl_xor(all_last, step, WAVE));
    }
    all_first = (int32_t)uniform((uint32_t)all_first);
    all_last = (int32_t)uniform((uint32_t)all_last);
    const uint32_t t_end = min(it.shape.key_tiles, (it.split + 1) * it.length);
    uint32_t t = it.split * it.length + wave;
    const uint32_t *table = a.table + (uint64_t)it.seq * a.table_stride;
    char *tile = tiles + wave * (32 * D * 2);
    Rows<T, D> state;
    state.clear();
    uint4 k[PIECES], v[PIECES];
    uint64_t at = 0;
    uint32_t entry = 0, off = 0;
    auto look_up = [&](uint32_t tt) {
        const uint32_t j = min(it.shape.keys.lo + tt * 32 + col, it.shape.keys.hi - 1), p = a.kv.by_page.div(j);
        off = j - p * a.kv.page;
        entry = table[p];
    };
    auto load = [&](const char *base, uint4 (&x)[PIECES]) {
        const char *p = base + at + half * (F8 ? 16 : 32);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const uint32_t o = F8 ? 32 * i : 2 * dim_of_step(i, 0);
            // past the head's dimensions: its first ones
            if (FULL || o + half * (F8 ? 16 : 32) < a.kv.dim * (F8 ? 1 : 2)) x[i] = *(const uint4 *)(p + o);
            else x[i] = *(const uint4 *)(base + at);
        }
    };
    if (t < t_end) look_up(t);
    uint4 q[D / 64];
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
        const uint32_t r = (threadIdx.x + 256 * i) / (D / 8), d = threadIdx.x % (D / 8) * 8, n = a.by_group.div(r);
        q[i] = make_uint4(0, 0, 0, 0);
        if (r < rows && (FULL || d < a.kv.dim))
            q[i] = *(const uint4 *)(a.q + (uint64_t)(sq.first + n) * a.q_row + (it.head * a.group + (r - n * a.group)) * a.q_head + d * 2);
    }
    if (t < t_end) {
        at = entry_at(a.kv, page_of(a.kv, entry), off, it.head);
        load(a.kv.k, k);
        load(a.kv.v, v);
        if (t + 4 < t_end) look_up(t + 4);
    }
    sign_query<T>(q, flip, zero);
#pragma unroll
    for (int i = 0; i < D / 64; ++i)
        *(uint4 *)(queries + piece_at<D>((threadIdx.x + 256 * i) / (D / 8), threadIdx.x % (D / 8))) = q[i];
    __syncthreads();
    bool odd = false;   // a value that is not finite was left out of a tile
    const RowAt<D> q_at;
    const ValueAt<D> v_at;
    const float slack = slack_of<T>(c);
    auto query = [&](int i) { return q_at.read(queries, i); };
    for (; t < t_end; t += 4) {
        const bool more = t + 4 < t_end;
        const uint32_t k0 = it.shape.keys.lo + t * 32;
        const bool full = (int32_t)k0 >= all_first && (int32_t)k0 + 31 <= all_last;
        f32x16 s[1];
        if (!FULL) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
                if ((F8 ? 32 * i + 16 * half : dim_of_step(i, half)) >= a.kv.dim) k[i] = make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            if (F8) {
                uint4 x, y;
                expand<T>(k[i / 2], &x, &y);
                s[0] = T::mfma(i % 2 ? y : x, query(i), i ? s[0] : f32x16(0.f));
            } else {
                s[0] = T::mfma(k[i % PIECES], query(i), i ? s[0] : f32x16(0.f));
            }
        }
        if (more) {
            at = entry_at(a.kv, page_of(a.kv, entry), off, it.head);
            load(a.kv.k, k);
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const uint32_t n = F8 ? 4 * i + 2 * half : dim_of_step(i, half) / 8;
            auto put = [&](uint4 x, int e) {
                if (!full) x = drop_not_finite<T>(x, &odd);
                *(uint4 *)(tile + piece_at<D>(col, n + e)) = x;
            };
            if (F8) {
                uint4 x, y;
                expand<T>(v[i], &x, &y);
                put(x, 0);
                put(y, 1);
            } else {
                put(v[i], 0);
            }
        }
        if (more) {
            load(a.kv.v, v);
            if (t + 8 < t_end) look_up(t + 8);
        }
        if (!full) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int32_t key = (int32_t)(k0 + key_of(r, half));
                if (key < first || key > last) s[0][r] = MINUS_INF;
            }
        }
        if (WEIGHTS && valid) {
            float *w = a.scores + (((uint64_t)it.seq * a.kv.n_kv + it.head) * a.slot_rows + col) * a.score_stride + k0 + 4 * half;
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *(float4 *)(w + 2 * r) = make_float4(s[0][r] * c, s[0][r + 1] * c, s[0][r + 2] * c, s[0][r + 3] * c);
        }
        uint4 p[2];
        state.template weigh<1>(s, c, slack, p);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        state.add(tile, v_at, p[0]);
        state.add(tile + 16 * D * 2, v_at, p[1]);
        __builtin_amdgcn_wave_barrier();
    }
    if (ballot(odd)) {
        for (t = it.split * it.length + wave; t < t_end; t += 4) {
            const uint32_t k0 = it.shape.keys.lo + t * 32;
            if ((int32_t)k0 >= all_first && (int32_t)k0 + 31 <= all_last) continue;
            for (uint32_t key = k0; key < min(k0 + 32, it.shape.keys.hi); ++key)
                add_not_finite<T, H, D>(state, a, it.seq, it.head, key, first, last, c, [&](uint32_t d) {
                    return *(const uint16_t *)(queries + piece_at<D>(col, d / 8) + d % 8 * 2);
                });
        }
    }
    float m = state.m == MINUS_INF ? MINUS_INF : state.m * c, l = sum_of_halves(state.l);
    // waves 2 and 3 to 0 and 1, then 1 to 0
    for (int from = 2; from >= 1; from /= 2) {
        __syncthreads();
        float *buf = (float *)tiles + (wave % from) * (32 * D);
        if (wave >= (uint32_t)from && wave < 2u * from) {
            join_ml[wave % from][lane] = make_float2(m, l);
#pragma unroll
            for (int b = 0; b < D / 32; ++b)
#pragma unroll
                for (int r = 0; r < 16; r += 4)
                    *(float4 *)(buf + ((b * 4 + r / 4) * WAVE + lane) * 4) =
                        make_float4(state.o[b][r], state.o[b][r + 1], state.o[b][r + 2], state.o[b][r + 3]);
        }
        __syncthreads();
        if (wave < (uint32_t)from) {
            const float2 ml = join_ml[wave][lane];
            const float top = fmaxf(m, ml.x), ref = top == MINUS_INF ? 0.f : top;
            const float f = exp2_fast(m - ref), g = exp2_fast(ml.x - ref);
            m = top;
            l = l * f + ml.y * g;
#pragma unroll
            for (int b = 0; b < D / 32; ++b)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const float4 x = *(const float4 *)(buf + ((b * 4 + r / 4) * WAVE + lane) * 4);
                    state.o[b][r] = state.o[b][r] * f + x.x * g;
                    state.o[b][r + 1] = state.o[b][r + 1] * f + x.y * g;
                    state.o[b][r + 2] = state.o[b][r + 2] * f + x.z * g;
                    state.o[b][r + 3] = state.o[b][r + 3] * f + x.w * g;
                }
        }
    }
    if (wave || !valid) return;
    write_rows<T, D>(a, it, state.o, m, l, col, sq.first + token, head, half);
}

// ------------------------------------------------------------------ chunks

constexpr int CHUNK_WAVES = 4, CHUNK_WAVES_WIDE = 8;
// keys of a tile: with 256 dimensions half as many, so that the registers hold out
constexpr __host__ __device__ int chunk_keys(int d) { return d <= 128 ? 64 : 32; }

// 32 rows a wave against a range of keys, in tiles of 64 keys that the workgroup
// shares through LDS (two buffers: the next tile is loaded to registers while this one is
// worked on, and written to the other buffer).  W waves: four and two workgroups to a
// compute unit, or eight, which load and write half as much a wave for rows that last.
// Bound by the matrix products and the exponentials between them: 2,048 tokens over
// 32,768 (bf16, 32 over 4 heads of 128) 1,060 to 1,094 us on five devices, 974 to 1,005 TFLOP/s
// (four waves: a tenth more time); the matrix cores are busy in 43% of the cycles, vector
// instructions issued in 42%.
template <class T, Held H, int D, bool FULL, int W>
__global__ __launch_bounds__(W * WAVE, D <= 128 ? 2 : 1) void chunk_kernel(AttnArgs a) {
    constexpr int THREADS = W * WAVE, ROWS = 32 * W;
    constexpr int CHUNK_KEYS = chunk_keys(D), BLOCKS = CHUNK_KEYS / 32;
    constexpr bool CODES = H != Held::SAME;
    constexpr int PER_ROW = CODES ? D / 16 : D / 8;         // pieces of a cache entry: 16 bytes (of 4-bit codes 8)
    constexpr int PIECES = CHUNK_KEYS * PER_ROW / THREADS;      // of one thread
    constexpr int TILE = CHUNK_KEYS * D * 2;
    static_assert(PIECES * THREADS == CHUNK_KEYS * PER_ROW, "whole pieces");
    __shared__ __attribute__((aligned(16))) char lds[2][2][TILE];
    __shared__ uint32_t odd;   // a value that is not finite was left out of a tile
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = 0;
    const Item it = find_item<By::ITEM>(a, blockIdx.x);
    if (!it.there) return;
    const uint32_t tid = threadIdx.x, lane = tid & (WAVE - 1), half = lane / 32, wave = uniform(tid / WAVE), col = lane % 32;
    const Seq &sq = it.shape.q;
    const uint32_t rows = sq.rows * a.group, r0 = it.row_tile * ROWS, row = r0 + wave * 32 + col;
    uint32_t flip;
    bool zero;
    const float c = score_factor(a, it.head, &flip, &zero);
    const bool valid = row < rows;
    const uint32_t token = a.by_group.div(valid ? row : 0), head = it.head * a.group + (valid ? row - token * a.group : 0);
    int32_t first = 0, last = 0x7FFFFFFF;
    if (valid) seen_by_row(a, sq, token, &first, &last);
    int32_t all_first = first, all_last = last;   // keys that every row of the wave sees
#pragma unroll
    for (int step = 1; step < 32; step *= 2) {
        all_first = max(all_first, __shfl_xor(all_first, step, WAVE));
        all_last = min(all_last, __shfl_xor(all_last, step, WAVE));
    }
    all_first = (int32_t)uniform((uint32_t)all_first);
    all_last = (int32_t)uniform((uint32_t)all_last);
    // the tile's own keys, and those that all its rows see, inside the item's range
    const uint32_t i0 = a.by_group.div(r0), i1 = a.by_group.div(min(r0 + ROWS, rows) - 1);
    const Range own = seen(a, sq, i0, i1);
    int32_t wg_first, wg_last, unused;
    seen_by_row(a, sq, i1, &wg_first, &unused);
    seen_by_row(a, sq, i0, &unused, &wg_last);
    const uint32_t from = it.shape.keys.lo + it.split * it.length * CHUNK_KEYS;
    const uint64_t past = (uint64_t)from + (uint64_t)it.length * CHUNK_KEYS;
    const uint32_t k_lo = max(from, own.lo & ~(CHUNK_KEYS - 1u)), k_hi = (uint32_t)min((uint64_t)own.hi, past);
    uint4 q[D / 16];
    load_query<T, D, FULL>(a, a.q + (uint64_t)(sq.first + token) * a.q_row + head * a.q_head, valid, half, flip, zero, q);
    const uint32_t *table = a.table + (uint64_t)it.seq * a.table_stride;

    typedef std::conditional_t<H == Held::E2M1, uint2, uint4> Piece;
    Piece k[PIECES], v[PIECES];
    uint32_t ke[PIECES], ve[PIECES];   // exponent bytes of 4-bit codes' scales
    // Where a page holds whole groups of 16 slots, a wave's rows of a piece lie in one group and
    // its address is one number for the wave: the table's entries are read 64 groups at a time,
    // a lane each, and the arithmetic is scalar.  Else every thread finds its rows' pages.
    const uint32_t n_piece = tid % PER_ROW;
    const bool past_dim = !FULL && n_piece * sizeof(Piece) >= held_bytes<H>(a.kv.dim);
    const uint32_t o_piece = past_dim ? 0 : n_piece * (uint32_t)sizeof(Piece), o_lane = lane / PER_ROW * (uint32_t)a.kv.st + o_piece;
    const uint32_t g_last = (k_hi - 1) / 16;
    uint32_t groups = 0, groups_next = 0, g0 = k_lo / 16;   // entries of groups g0 + lane, g0 + 64 + lane
    uint32_t entry[PIECES], off[PIECES];
    auto look_up_groups = [&](uint32_t g) { return table[a.kv.by_page.div(min(g + lane, g_last) * 16)]; };
    auto look_up = [&](uint32_t k0) {
        if (a.by_16) return;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const uint32_t j = min(k0 + (tid + THREADS * i) / PER_ROW, k_hi - 1), p = a.kv.by_page.div(j);
            off[i] = j - p * a.kv.page;
            entry[i] = table[p];
        }
    };
    auto load = [&](uint32_t k0) {
        if (a.by_16) {
            if (k0 / 16 - g0 >= WAVE) {
                g0 += WAVE;
                groups = groups_next;
                groups_next = look_up_groups(g0 + WAVE);
            }
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const uint32_t r = (wave * WAVE + THREADS * i) / PER_ROW, g = min(k0 / 16 + r / 16, g_last), slot = g * 16;
                const uint32_t p = a.kv.by_page.div(slot);
                const uint32_t page = page_of(a.kv, from_lane(groups, (int)(g - g0)));
                const uint64_t at = entry_at(a.kv, page, slot - p * a.kv.page + r % 16, it.head);
                k[i] = *(const Piece *)(a.kv.k + at + o_lane);
                v[i] = *(const Piece *)(a.kv.v + at + o_lane);
                if (H == Held::E2M1) {
                    ke[i] = a.kv.k_exp[at / 16 + o_lane / 16];
                    ve[i] = a.kv.v_exp[at / 16 + o_lane / 16];
                }
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const uint64_t at = entry_at(a.kv, page_of(a.kv, entry[i]), off[i], it.head) + o_piece;
            k[i] = *(const Piece *)(a.kv.k + at);
            v[i] = *(const Piece *)(a.kv.v + at);
            if (H == Held::E2M1) {
                ke[i] = a.kv.k_exp[at / 16];
                ve[i] = a.kv.v_exp[at / 16];
            }
        }
    };
    auto is_edge = [&](uint32_t k0) {
        return (int32_t)k0 < wg_first || (int32_t)(k0 + CHUNK_KEYS - 1) > wg_last || k0 + CHUNK_KEYS > k_hi;
    };
    if (tid == 0) odd = 0;
    __syncthreads();
    uint32_t to[CODES ? 2 : 1];   // this thread's places in a tile
#pragma unroll
    for (int e = 0; e < (CODES ? 2 : 1); ++e) to[e] = piece_at<D>(tid / PER_ROW, n_piece * (CODES ? 2 : 1) + e);
    auto store = [&](int buf, uint32_t k0) {
        const bool edge = is_edge(k0);
        bool mine = false;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            // rows a multiple of 16 on have the same spread, those 8 on another by 2
            const uint32_t at = THREADS / PER_ROW * i * D * 2, turn = THREADS / PER_ROW == 8 && i % 2 ? 32 : 0;
            auto put = [&](uint4 x, uint4 y, int e) {
                if (past_dim) x = make_uint4(0, 0, 0, 0);
                if (edge) {   // slots past the end may hold anything
                    if (k0 + (tid + THREADS * i) / PER_ROW >= k_hi) y = make_uint4(0, 0, 0, 0);
                    y = drop_not_finite<T>(y, &mine);
                }
                const uint32_t o = (to[e] ^ turn) + at;
                *(uint4 *)(lds[buf][0] + o) = x;
                *(uint4 *)(lds[buf][1] + o) = y;
            };
            if constexpr (H == Held::E2M1) {
                const float x = scale_of(ke[i]), y = scale_of(ve[i]);
                put(expand<T>(k[i].x, x), expand<T>(v[i].x, y), 0);
                put(expand<T>(k[i].y, x), expand<T>(v[i].y, y), 1);
            } else if constexpr (H == Held::E4M3) {
                uint4 x0, x1, y0, y1;
                expand<T>(k[i], &x0, &x1);
                expand<T>(v[i], &y0, &y1);
                put(x0, y0, 0);
                put(x1, y1, 1);
            } else {
                put(k[i], v[i], 0);
            }
        }
        if (mine) odd = 1;
    };
    const RowAt<D> k_at;
    const ValueAt<D> v_at;
    const float slack = slack_of<T>(c);
    Rows<T, D> state;
    state.clear();
    if (k_lo < k_hi) {
        if (a.by_16) {
            groups = look_up_groups(g0);
            groups_next = look_up_groups(g0 + WAVE);
        }
        look_up(k_lo);
        load(k_lo);
        if (k_lo + CHUNK_KEYS < k_hi) look_up(k_lo + CHUNK_KEYS);
        store(0, k_lo);
        __syncthreads();
    }
    int buf = 0;
    for (uint32_t k0 = k_lo; k0 < k_hi; k0 += CHUNK_KEYS) {
        const uint32_t next = k0 + CHUNK_KEYS;
        if (next < k_hi) {
            load(next);
            if (next + CHUNK_KEYS < k_hi) look_up(next + CHUNK_KEYS);
        }
        const char *kt = lds[buf][0], *vt = lds[buf][1];
        f32x16 s[BLOCKS];
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
                s[b] = T::mfma(k_at.read(kt + 32 * b * D * 2, i), q[i], i ? s[b] : f32x16(0.f));
        if ((int32_t)k0 < all_first || (int32_t)(k0 + CHUNK_KEYS - 1) > all_last || next > k_hi) {
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int32_t key = (int32_t)(k0 + 32 * b + key_of(r, half));
                    if (key < first || key > last || key >= (int32_t)k_hi) s[b][r] = MINUS_INF;
                }
        }
        uint4 p[2 * BLOCKS];
        state.template weigh<BLOCKS>(s, c, slack, p);
#pragma unroll
        for (int t = 0; t < 2 * BLOCKS; ++t) state.add(vt + 16 * t * D * 2, v_at, p[t]);
        if (next < k_hi) store(buf ^ 1, next);
        __syncthreads();
        buf ^= 1;
    }
    if (odd) {
        const char *row_q = a.q + (uint64_t)(sq.first + token) * a.q_row + head * a.q_head;
        for (uint32_t k0 = k_lo; k0 < k_hi; k0 += CHUNK_KEYS) {
            if (!is_edge(k0)) continue;
            for (uint32_t key = k0; key < min(k0 + CHUNK_KEYS, k_hi); ++key)
                add_not_finite<T, H, D>(state, a, it.seq, it.head, key, first, last, c, [&](uint32_t d) {
                    return zero ? 0u : *(const uint16_t *)(row_q + 2 * d) ^ (flip & 0x8000u);
                });
        }
    }
    if (!valid) return;
    const float m = state.m == MINUS_INF ? MINUS_INF : state.m * c;
    const float l = sum_of_halves(state.l);
    write_rows<T, D>(a, it, state.o, m, l, row - r0, sq.first + token, head, half);
}

// -------------------------------------------------------------------- join

constexpr uint32_t WEIGH_KEYS = 1024;   // keys of one (sequence, head) per workgroup

// A row's maximum (base 2) and sum over its parts, by the lanes of a team of `team`
// consecutive lanes (every lane gets them).
__device__ __forceinline__ float2 join_stats(const AttnArgs &a, const Item &it, uint32_t head, uint32_t tile, uint32_t at,
                                             uint32_t lane, uint32_t team) {
    float m = MINUS_INF, l = 0.f;
    for (uint32_t p = lane; p < it.splits; p += team) {
        const uint32_t slot = slot_of(a, it, head, tile, p);
        const float2 x = slot < a.slots ? a.part_ml[(uint64_t)slot * a.slot_rows + at] : make_float2(MINUS_INF, 0.f);
        const float top = fmaxf(m, x.x), ref = top == MINUS_INF ? 0.f : top;
        l = l * exp2_fast(m - ref) + x.y * exp2_fast(x.x - ref);
        m = top;
    }
    for (uint32_t step = 1; step < team; step *= 2) {
        const float m2 = __shfl_xor(m, step, WAVE), l2 = __shfl_xor(l, step, WAVE);
        const float top = fmaxf(m, m2), ref = top == MINUS_INF ? 0.f : top;
        l = l * exp2_fast(m - ref) + l2 * exp2_fast(m2 - ref);
        m = top;
    }
    return make_float2(m, l);
}

// The parts of some rows of a tile, `teams` of D / 4 lanes to a row, each over every
// teams-th part; and the whole call's status, for which the workgroups share the
// table's entries.  Behind those workgroups, with few rows: the weights, from the scores.
// Bound by its waits (list, statistics, parts): 6 us for one row, 8 for a decode batch; with the weights of
// 64 uneven sequences of up to 32,768 slots (79 MB of scores read, 43 MB of weights read and written) 32.
template <class T, int D, bool EVEN, bool WEIGH>   // WEIGH: the launch has workgroups for weights
__global__ __launch_bounds__(256) void join_kernel(AttnArgs a, uint32_t teams, uint32_t joins, uint32_t row_blocks,
                                                   uint32_t key_blocks) {
    constexpr uint32_t LANES = D / 4, ALL = 256 / LANES;
    __shared__ float4 sums[256];
    __shared__ float stats[32];
    __shared__ int2 sees[32];   // first and last slot
    const uint32_t tid = threadIdx.x;
    if (!WEIGH || blockIdx.x < joins) {
        // status
        bool bad = false;
        if (blockIdx.x == 0 && tid == 0) bad = a.q_off[0] != 0 || a.q_off[a.n_seqs] != a.n_rows;
        const uint32_t share = joins > a.n_seqs ? joins / a.n_seqs : 1;   // workgroups to a sequence
        for (uint32_t b = blockIdx.x; b < a.n_seqs * share; b += joins) {
            const uint32_t s = b / share, part = b - s * share;
            bool wrong;
            const Seq q = load_seq(a.q_off, a.kv_len, s, a.n_rows, a.max_kv, &wrong);
            bad |= wrong || q.rows > a.max_q || q.rows > q.len;
            if (!q.rows) continue;
            const Range r = seen(a, q, 0, q.rows - 1);
            if (r.lo >= r.hi) continue;
            const uint32_t p1 = a.kv.by_page.div(r.hi - 1);
            for (uint32_t p = a.kv.by_page.div(r.lo) + part * 256 + tid; p <= p1; p += share * 256)
                bad |= a.table[(uint64_t)s * a.table_stride + p] >= a.kv.n_pages;
        }
        if (bad) atomicOr(a.status, DEV_ERR_BAD_LAYOUT);
        // join
        const uint32_t tile = blockIdx.x / row_blocks;
        const Item it = find_item<By::TILE, EVEN>(a, tile);
        if (!it.there || it.splits < 2) return;
        const uint32_t at = tid / LANES, lane = tid % LANES, team = at % teams, step = ALL / teams;
        const uint32_t r0 = it.row_tile * a.row_tile, rows = min(a.row_tile, it.shape.q.rows * a.group - r0);
        for (uint32_t from = (blockIdx.x - tile * row_blocks) * step; from < rows; from += row_blocks * step) {
            const bool there = from + at / teams < rows;
            const uint32_t row = there ? from + at / teams : from;
            const uint32_t part0 = slot_of(a, it, it.head, it.row_tile, 0), apart = it.shape.row_tiles * a.kv.n_kv;
            // four parts from p on, every teams-th: one that saw nothing has the maximum -inf and holds
            // zeros, and so does one that is not there
            auto parts = [&](uint32_t p, float2 (&y)[4], float4 (&x)[4]) {
#pragma unroll
                for (uint32_t u = 0; u < 4; ++u) {
                    const uint32_t slot = part0 + min(p + u * teams, it.splits - 1) * apart;
                    const uint64_t i = (uint64_t)min(slot, a.slots - 1) * a.slot_rows + row;
                    y[u] = a.part_ml[i];
                    x[u] = *(const float4 *)(a.part + i * D + lane * 4);
                    if (p + u * teams >= it.splits || slot >= a.slots) {
                        y[u] = make_float2(MINUS_INF, 0.f);
                        x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
                    }
                }
            };
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
            auto add = [&](const float2 (&y)[4], const float4 (&x)[4], float ref) {
#pragma unroll
                for (uint32_t u = 0; u < 4; ++u) {
                    const float f = exp2_fast(y[u].x - ref);   // 0 for a part whose scores are all NaN: 0 * NaN stays NaN
                    sum = make_float4(sum.x + x[u].x * f, sum.y + x[u].y * f, sum.z + x[u].z * f, sum.w + x[u].w * f);
                }
            };
            float2 ml, y[4];
            float4 x[4];
            if (teams == 1 && it.splits <= 4) {   // all there is, in one wait
                parts(0, y, x);
                ml = make_float2(fmaxf(fmaxf(y[0].x, y[1].x), fmaxf(y[2].x, y[3].x)), 0.f);
                const float ref = ml.x == MINUS_INF ? 0.f : ml.x;
#pragma unroll
                for (uint32_t u = 0; u < 4; ++u) ml.y += y[u].y * exp2_fast(y[u].x - ref);
                add(y, x, ref);
            } else {
                ml = join_stats(a, it, it.head, it.row_tile, row, lane, LANES);
                const float ref = ml.x == MINUS_INF ? 0.f : ml.x;
                for (uint32_t p = team; p < it.splits; p += 4 * teams) {
                    parts(p, y, x);
                    add(y, x, ref);
                }
            }
            if (teams > 1) {
                __syncthreads();
                sums[tid] = sum;
                __syncthreads();
            }
            if (team || !there) continue;
            for (uint32_t i = 1; i < teams; ++i) {
                const float4 x = sums[tid + i * LANES];
                sum = make_float4(sum.x + x.x, sum.y + x.y, sum.z + x.z, sum.w + x.w);
            }
            const float f = ml.y == 0.f ? 0.f : (a.kv.v_scale ? a.kv.v_scale[it.head] : 1.f) / ml.y;
            const float base2 = log_sum<T>(ml.x, ml.y);
            const uint32_t i = a.by_group.div(r0 + row), t = it.shape.q.first + i, e = it.head * a.group + (r0 + row - i * a.group);
            if (lane == 0) {
                if (a.lse) a.lse[(uint64_t)t * a.n_heads + e] = base2 * LN2;
                if (a.lse2) a.lse2[(uint64_t)t * a.n_heads + e] = base2;
            }
            if (lane * 4 < a.kv.dim)
                *(uint2 *)(a.out + (uint64_t)t * a.o_row + e * a.o_head + lane * 8) =
                    make_uint2(T::pack(sum.x * f, sum.y * f), T::pack(sum.z * f, sum.w * f));
        }
        return;
    }
    if constexpr (!WEIGH) return;
    // weights of WEIGH_KEYS keys of one (sequence, head) from the scores
    const uint32_t b = blockIdx.x - joins, s = b / (key_blocks * a.kv.n_kv), hk = b - s * key_blocks * a.kv.n_kv;
    const uint32_t h = hk / key_blocks;
    // Neighbouring workgroups are on different XCDs, and the first keys are there in every sequence: each row begins
    // one block later, so that no XCD gets the same blocks of all of them (64 sequences with room for
    // 32,768 slots, a multiple of eight blocks: 48 us, rotated 32).
    const uint32_t block = (hk - h * key_blocks + s * a.kv.n_kv + h) % key_blocks, k0 = block * WEIGH_KEYS;
    const Shape shape = shape_of(a, s);
    const Seq &q = shape.q;
    const uint32_t rows = q.rows * a.group;
    // four keys a thread, so that a row's scores are one load (rows of them begin at multiples of 32)
    static_assert(WEIGH_KEYS == 4 * 256, "four keys a thread");
    const uint64_t row = (uint64_t)s * a.kv.n_kv + h;
    const uint32_t j = k0 + 4 * tid, end = min(a.max_kv, q.len);
    float old[4], sum[4] = {0.f, 0.f, 0.f, 0.f};
    const uint64_t at = row * a.weight_stride + j;
    const bool pieces = ((uint64_t)(uintptr_t)a.weight_out | (uint64_t)(uintptr_t)a.weight | a.weight_stride * 4) % 16 == 0;
    if (a.weight && pieces && j + 4 <= end) {
        const float4 w = *(const float4 *)(a.weight + at);
        old[0] = w.x, old[1] = w.y, old[2] = w.z, old[3] = w.w;
    } else {
#pragma unroll
        for (uint32_t n = 0; n < 4; ++n) old[n] = a.weight && j + n < end ? a.weight[at + n] : 0.f;
    }
    if (k0 < shape.keys.hi && k0 + WEIGH_KEYS > shape.keys.lo) {   // else no row sees any of them
        const bool scored = j < shape.keys.hi && j + 4 > shape.keys.lo;
        const float *x = a.scores + row * a.slot_rows * a.score_stride + (scored ? j : shape.keys.lo);
        // the first rows' scores are on their way while the statistics are found
        constexpr uint32_t FIRST = 8;
        float4 z[FIRST];
#pragma unroll
        for (uint32_t i = 0; i < FIRST; ++i) z[i] = *(const float4 *)(x + min(i, rows - 1) * a.score_stride);
        const Item it = find_item<By::SEQ, EVEN>(a, s);
        const uint32_t r = tid / 8;   // 32 teams of 8
        if (r < rows) {
            const uint32_t i = a.by_group.div(r);
            float base2;
            if (it.splits > 1) {
                const float2 ml = join_stats(a, it, h, 0, r, tid % 8, 8);
                base2 = log_sum<T>(ml.x, ml.y);
            } else {
                base2 = a.lse2[(uint64_t)(q.first + i) * a.n_heads + h * a.group + (r - i * a.group)];
            }
            if (tid % 8 == 0) {
                stats[r] = base2 == MINUS_INF ? __builtin_inff() : base2;   // a row without a weight: exp2(-inf)
                seen_by_row(a, q, i, &sees[r].x, &sees[r].y);
            }
        }
        __syncthreads();
        auto add = [&](uint32_t i, float4 z) {
            const float y[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
            for (uint32_t n = 0; n < 4; ++n) {
                const float e = exp2_fast(y[n] - stats[i]);   // NaN of a broken row: for what it sees
                sum[n] += (((int32_t)(j + n) >= sees[i].x) & ((int32_t)(j + n) <= sees[i].y)) ? e : 0.f;
            }
        };
#pragma unroll
        for (uint32_t i = 0; i < FIRST; ++i)
            if (i < rows) add(i, z[i]);
#pragma unroll 8
        for (uint32_t i = FIRST; i < rows; ++i) add(i, *(const float4 *)(x + i * a.score_stride));
    }
#pragma unroll
    for (uint32_t n = 0; n < 4; ++n) sum[n] = j + n < end ? old[n] + sum[n] : 0.f;
    if (pieces && j + 4 <= a.max_kv) {
        *(float4 *)(a.weight_out + at) = make_float4(sum[0], sum[1], sum[2], sum[3]);
    } else {
#pragma unroll
        for (uint32_t n = 0; n < 4; ++n)
            if (j + n < a.max_kv) a.weight_out[at + n] = sum[n];
    }
}

// ----------------------------------------------------------------- weights

constexpr int WEIGHT_KEYS = 256, WEIGHT_ROWS = 64;

// Of a chunk: 256 keys against all rows that see them (or one part of the
// rows), 64 keys a wave in registers as the right operand of scores = Q K^T, the rows
// passing through LDS.  With the statistics known there is no running maximum: a
// register holds one row, so a key's sum is a sum over registers.  Bound by the
// matrix products and exponentials (matrix cores busy in 36% of the cycles, vector instructions
// issued in 57%): 2 x 1,024 tokens over 16,384 (bf16, 32 over 4 heads of 128) 390 us, 680
// TFLOP/s; the attention before it, of twice the products, takes some 500.
template <class T, Held H, int D, bool FULL>
__global__ __launch_bounds__(256, D <= 128 ? 2 : 1) void weight_kernel(AttnArgs a, uint32_t key_blocks) {
    constexpr int PIECES = D / 8 * WEIGHT_ROWS / 256;
    constexpr int TILE = WEIGHT_ROWS * D * 2;
    __shared__ __attribute__((aligned(16))) char lds[2][TILE];
    __shared__ __attribute__((aligned(16))) float base2[2][WEIGHT_ROWS];
    __shared__ __attribute__((aligned(16))) int2 sees[2][WEIGHT_ROWS];   // first and last slot
    const uint32_t tid = threadIdx.x, lane = tid & (WAVE - 1), half = lane / 32, wave = uniform(tid / WAVE), col = lane % 32;
    uint32_t b = blockIdx.x;
    const uint32_t h = b % a.kv.n_kv;
    b /= a.kv.n_kv;
    const uint32_t part = b % a.weight_parts;
    b /= a.weight_parts;
    const uint32_t s = b / key_blocks, k0 = (b - s * key_blocks) * WEIGHT_KEYS;
    const Shape shape = shape_of(a, s);
    const Seq &q = shape.q;
    const uint64_t out_row = (uint64_t)s * a.kv.n_kv + h;
    uint32_t flip;
    bool zero;
    const float c = score_factor(a, h, &flip, &zero);
    float sum[2] = {0.f, 0.f};
    const uint32_t k_lo = max(k0, shape.keys.lo), k_hi = min(min(k0 + WEIGHT_KEYS, shape.keys.hi), q.len);
    if (k_lo < k_hi) {
        // rows (token, head of the group) that see any of the keys, and this part of them
        const int64_t j0 = q.slot;
        int64_t i_lo = a.causal ? (int64_t)k_lo - j0 : 0, i_hi = a.window ? (int64_t)k_hi - 1 + a.window - j0 : q.rows;
        i_lo = i_lo < 0 ? 0 : i_lo > (int64_t)q.rows ? (int64_t)q.rows : i_lo;
        i_hi = i_hi < i_lo ? i_lo : i_hi > (int64_t)q.rows ? (int64_t)q.rows : i_hi;
        const uint32_t r_all = (uint32_t)i_lo * a.group, r_past = (uint32_t)i_hi * a.group;
        const uint32_t tiles = (r_past - r_all + WEIGHT_ROWS - 1) / WEIGHT_ROWS;
        const uint32_t each = (tiles + a.weight_parts - 1) / a.weight_parts;
        const uint32_t r_lo = min(r_past, r_all + part * each * WEIGHT_ROWS), r_hi = min(r_past, r_lo + each * WEIGHT_ROWS);
        // this lane's two keys
        uint4 k[2][D / 16];
        const uint32_t *table = a.table + (uint64_t)s * a.table_stride;
        if (r_lo < r_hi) {
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const uint32_t j = min(k0 + wave * 64 + 32 * n + col, k_hi - 1), p = a.kv.by_page.div(j);
                const uint64_t entry = entry_at(a.kv, page_of(a.kv, table[p]), j - p * a.kv.page, h);
                const char *base = a.kv.k + entry;
#pragma unroll
                for (int i = 0; i < D / 16; i += H == Held::SAME ? 1 : 2) {
                    const uint32_t d = dim_of_step(i, half);
                    const bool in = FULL || d < a.kv.dim;
                    const char *from = base + (in ? held_bytes<H>(d) : 0);
                    const uint32_t all = in ? ~0u : 0;
                    if constexpr (H == Held::E2M1) {
                        const uint2 x = *(const uint2 *)from;
                        const float s = scale_of(a.kv.k_exp[entry / 16 + (in ? d / 32 : 0)]);
                        k[n][i] = expand<T>(x.x & all, in ? s : 1.f);
                        k[n][i + 1] = expand<T>(x.y & all, in ? s : 1.f);
                    } else {
                        uint4 x = *(const uint4 *)from;
                        x = make_uint4(x.x & all, x.y & all, x.z & all, x.w & all);
                        if constexpr (H == Held::E4M3) expand<T>(x, &k[n][i], &k[n][i + 1]);
                        else k[n][i] = x;
                    }
                }
            }
            // the scale's sign, or its zero, goes to the keys; and they are waited for here, else
            // every pass of the loop would wait for all its loads
            const uint32_t all = zero ? 0 : ~0u;
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    uint4 &x = k[n][i];
                    x = make_uint4((x.x ^ flip) & all, (x.y ^ flip) & all, (x.z ^ flip) & all, (x.w ^ flip) & all);
                    __asm__ volatile("" : "+v"(x.x), "+v"(x.y), "+v"(x.z), "+v"(x.w));
                }
        }
        const uint32_t n_piece = tid % (D / 8);
        const RowAt<D> q_at;
        const bool no_piece = !FULL && n_piece * 8 >= a.kv.dim;
        uint4 x[PIECES];
        float base = 0.f;
        int2 see = make_int2(0, -1);
        // whether a row of the 64 from r0 on is not there or does not see one of keys from .. to
        auto masks = [&](uint32_t r0, int32_t from, int32_t to) {
            const int64_t x0 = j0 + a.by_group.div(r0), x1 = j0 + a.by_group.div(min(r0 + WEIGHT_ROWS, r_hi) - 1);
            return (a.causal && to > x0) || (a.window && (int64_t)from <= x1 - (int64_t)a.window) || to >= (int32_t)k_hi ||
                   r0 + WEIGHT_ROWS > r_hi;
        };
        // rows past the end are the last one's bytes (and masked); nothing here waits for what it loads
        auto load = [&](uint32_t r0) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const uint32_t r = min(r0 + (tid + 256 * i) / (D / 8), r_hi - 1);
                const uint32_t t = a.by_group.div(r), e = h * a.group + (r - t * a.group);
                x[i] = *(const uint4 *)(a.q + (uint64_t)(q.first + t) * a.q_row + e * a.q_head + (no_piece ? 0 : n_piece * 16));
            }
            if (tid < WEIGHT_ROWS) {
                const uint32_t r = min(r0 + tid, r_hi - 1), t = a.by_group.div(r), e = h * a.group + (r - t * a.group);
                base = a.lse2[(uint64_t)(q.first + t) * a.n_heads + e];
                if (masks(r0, (int32_t)k0, (int32_t)k0 + WEIGHT_KEYS - 1)) {   // of any wave's keys
                    seen_by_row(a, q, t, &see.x, &see.y);
                    if (r0 + tid >= r_hi) see.y = -1;
                }
            }
        };
        auto store = [&](int buf) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
                *(uint4 *)(lds[buf] + piece_at<D>((tid + 256 * i) / (D / 8), n_piece)) = no_piece ? make_uint4(0, 0, 0, 0) : x[i];
            if (tid < WEIGHT_ROWS) {
                base2[buf][tid] = base == MINUS_INF ? __builtin_inff() : base;   // a row that sees nothing: exp2(-inf)
                sees[buf][tid] = see;
            }
        };
        const int32_t w_first = (int32_t)(k0 + wave * 64), w_last = w_first + 63;   // the wave's keys
        // 64 rows; `masked` where a row of them does not see a key of the wave's
        auto add_rows = [&](auto masked, int buf) {
#pragma unroll
            for (int m = 0; m < WEIGHT_ROWS / 32; ++m) {
                f32x16 z[2];
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    const uint4 y = q_at.read(lds[buf] + 32 * m * D * 2, i);
#pragma unroll
                    for (int n = 0; n < 2; ++n) z[n] = T::mfma(y, k[n][i], i ? z[n] : f32x16(0.f));
                }
                float g[2] = {0.f, 0.f};
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const float4 l = *(const float4 *)&base2[buf][32 * m + key_of(r, half)];
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        float e[4] = {exp2_fast(fmaf(z[n][r], c, -l.x)), exp2_fast(fmaf(z[n][r + 1], c, -l.y)),
                                      exp2_fast(fmaf(z[n][r + 2], c, -l.z)), exp2_fast(fmaf(z[n][r + 3], c, -l.w))};
                        if (masked.value) {
                            const int32_t key = w_first + 32 * n + (int32_t)col;
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int2 see = sees[buf][32 * m + key_of(r, half) + i];
                                if (key >= (int32_t)k_hi || key < see.x || key > see.y) e[i] = 0.f;
                            }
                        }
                        g[n] += (e[0] + e[1]) + (e[2] + e[3]);
                    }
                }
                sum[0] += g[0];
                sum[1] += g[1];
            }
        };
        if (r_lo < r_hi) {
            load(r_lo);
            store(0);
        }
        __syncthreads();
        int buf = 0;
        for (uint32_t r0 = r_lo; r0 < r_hi; r0 += WEIGHT_ROWS) {
            const bool more = r0 + WEIGHT_ROWS < r_hi;
            if (more) load(r0 + WEIGHT_ROWS);
            if (masks(r0, w_first, w_last))
                add_rows(std::true_type{}, buf);
            else
                add_rows(std::false_type{}, buf);
            if (more) store(buf ^ 1);
            __syncthreads();
            buf ^= 1;
        }
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const float w = sum_of_halves(sum[n]);
        const uint32_t j = k0 + wave * 64 + 32 * n + col;
        if (half || j >= a.max_kv) continue;
        if (a.weight_parts > 1) {
            a.weight_part[((uint64_t)part * a.n_seqs * a.kv.n_kv + out_row) * a.max_kv + j] = w;
        } else {
            const float old = a.weight && j < q.len ? a.weight[out_row * a.weight_stride + j] : 0.f;
            a.weight_out[out_row * a.weight_stride + j] = j < q.len ? old + w : 0.f;
        }
    }
}

__global__ __launch_bounds__(256) void weight_sum_kernel(AttnArgs a, uint32_t key_blocks) {
    const uint32_t row = blockIdx.x / key_blocks, s = row / a.kv.n_kv;
    const uint32_t j = (blockIdx.x - row * key_blocks) * 256 + threadIdx.x;
    if (j >= a.max_kv) return;
    float w = 0.f;
    if (j < a.kv_len[s]) {
        w = a.weight ? a.weight[(uint64_t)row * a.weight_stride + j] : 0.f;
        float sum = 0.f;
        for (uint32_t p = 0; p < a.weight_parts; ++p)
            sum += a.weight_part[((uint64_t)p * a.n_seqs * a.kv.n_kv + row) * a.max_kv + j];
        w += sum;
    }
    a.weight_out[(uint64_t)row * a.weight_stride + j] = w;
}

// ---------------------------------------------------------------------- host

constexpr uint32_t ROWS_MOST = 32;           // rows of the path for few rows
constexpr uint32_t ROWS_ITEMS = 1024;
// Chunks: one round of the chip, 512 workgroups of four waves, or 256 of eight.  The wide ones take
// one to three sequences of at least 2,048 rows (tokens times heads of a group) for each of them, with
// room for 8,192 slots, in heads of 65 to 128 dimensions: 6% faster in the mean of 122 such shapes (all
// types, 1 to 12 key/value heads, 8,192 and 32,768 keys; 2,048 tokens over 32,768: 1,068 us, 1,177
// narrow), 22% slower at worst.  The 230 shapes measured below those bounds were 2% slower, 46% at
// worst (three sequences of 1,024 rows); a cache that does not use its room, 4%.
// Smaller items, those of cut sequences first, fill the gaps that uneven lengths leave: of twelve
// sequences on whose rows are under 7/8 of what max_q allows 640 items are wanted (12 sequences: 1%
// slower in the mean of 38 shapes, of which they take 0.82 to 1.17 of the time; 14 to 48: 3% faster in the
// mean of 150).  Of fewer sequences they took 4% more time, and of even ones up to 56%: each
// is cut into one part more than the round holds.
constexpr uint32_t CHUNK_ITEMS = 512, CHUNK_ITEMS_WIDE = 256, CHUNK_ITEMS_RAGGED = 640, RAGGED_SEQS = 12;
constexpr uint32_t WIDE_SEQS = 3, WIDE_ROWS = 2048, WIDE_KEYS = 8192;
constexpr uint32_t ROWS_LEAST = 8, CHUNK_LEAST = 4;   // tiles of an item: 256 keys
// Few rows with weights: up to 2^30 scores (rows times room) are kept, a workspace of 4 GiB.  Above
// that the weights take the chunks' second pass over the keys, which is slower but keeps
// none (32 sequences of 32,768 keys, 8 heads: 32 rows a head 1,468 us with 1 GB of scores and
// 1,508 without; uneven lengths 387 and 537; 64 of 4 heads with 8 rows each 1,055 and 1,466).
constexpr uint64_t SCORES_MOST = 1ull << 30;
constexpr uint32_t WEIGHT_ITEMS = 4096;   // with 1024, two rounds of the chip, uneven ends took a quarter of the time

struct AttnPlan {
    bool few, wide, ragged, scores;
    uint32_t row_tile, dim, items, slots, slot_rows, weight_parts, key_blocks;
    uint64_t score_stride, score_room;   // scores of a row, and of the call that the workspace holds
};
static AttnPlan attn_plan(uint32_t n_seqs, uint32_t n_rows, uint32_t max_q, uint32_t max_kv, uint32_t n_heads, uint32_t n_kv,
                          uint32_t dim, bool weights) {
    AttnPlan p;
    const uint32_t group = n_heads / n_kv;
    p.few = (uint64_t)max_q * group <= ROWS_MOST;
    p.dim = dim <= 64 ? 64 : dim <= 128 ? 128 : 256;
    const uint64_t most = (uint64_t)max_q * group;   // rows of a sequence and head
    p.wide = !p.few && p.dim == 128 && n_seqs <= WIDE_SEQS && most >= (uint64_t)WIDE_ROWS * n_seqs && max_kv >= WIDE_KEYS;
    p.ragged = !p.few && n_seqs >= RAGGED_SEQS && (uint64_t)n_rows * 8 < (uint64_t)n_seqs * max_q * 7;
    p.row_tile = p.few ? ROWS_MOST : 32 * (p.wide ? CHUNK_WAVES_WIDE : CHUNK_WAVES);
    p.items = p.few ? ROWS_ITEMS : p.wide ? CHUNK_ITEMS_WIDE : p.ragged ? CHUNK_ITEMS_RAGGED : CHUNK_ITEMS;
    // an item that is a part has more than half an item's tiles: at most two per item wanted (and
    // a workspace for many rows holds out for fewer, uneven ones)
    p.slots = 2 * (!p.few && n_seqs >= RAGGED_SEQS ? CHUNK_ITEMS_RAGGED : p.items);
    p.slot_rows = p.few ? (max_q ? max_q : 1) * group : p.row_tile;
    p.score_stride = ((uint64_t)max_kv + 31) / 32 * 32;
    // a workspace for some bounds holds out for lower ones, so above SCORES_MOST it does not shrink
    const uint64_t score_rows = p.few && weights ? (uint64_t)n_seqs * n_kv * p.slot_rows : 0;
    const bool fit = score_rows <= SCORES_MOST && score_rows * p.score_stride <= SCORES_MOST;
    p.scores = p.few && weights && fit;
    p.score_room = fit ? score_rows * p.score_stride : SCORES_MOST;
    p.key_blocks = (uint32_t)(((uint64_t)max_kv + WEIGHT_KEYS - 1) / WEIGHT_KEYS);
    const uint64_t blocks = (uint64_t)n_seqs * n_kv * (p.key_blocks ? p.key_blocks : 1);
    const uint64_t tiles = ((uint64_t)max_q * group + WEIGHT_ROWS - 1) / WEIGHT_ROWS;
    uint64_t parts = blocks ? WEIGHT_ITEMS / blocks : 1;
    parts = parts < tiles / 4 ? parts : tiles / 4;
    p.weight_parts = (uint32_t)(parts < 1 ? 1 : parts > 16 ? 16 : parts);
    return p;
}
static size_t attn_carve(AttnArgs *a, const AttnPlan &p, char *ws, uint32_t n_seqs, uint32_t n_rows, uint32_t max_kv,
                         uint32_t n_heads, uint32_t n_kv, bool weights) {
    Carver c{ws, 0};
    a->status = c.take<int32_t>(WS_HEADER / 4);
    a->part = c.take<float>((size_t)p.slots * p.slot_rows * p.dim);
    a->part_ml = c.take<float2>((size_t)p.slots * p.slot_rows);
    a->lse2 = nullptr;
    a->scores = a->weight_part = nullptr;
    if (weights) {
        a->lse2 = c.take<float>((size_t)n_rows * n_heads);
        if (p.few) a->scores = c.take<float>(p.score_room);
        else if (p.weight_parts > 1) a->weight_part = c.take<float>((size_t)p.weight_parts * n_seqs * n_kv * max_kv);
    }
    a->slots = p.slots;
    a->slot_rows = p.slot_rows;
    a->score_stride = p.score_stride;
    a->weight_parts = p.weight_parts;
    return c.off;
}

// Workgroups of the call's launches.
struct AttnGrids {
    uint64_t items;      // as many as there can be: the ones wanted, and one more for every tile of rows
    uint32_t teams, row_blocks, key_blocks;   // of the join
    uint64_t joins, weigh;                    // its two kinds of workgroups
    uint64_t weights, sums;                   // of the weights' second pass
};
static AttnGrids attn_grids(const AttnPlan &p, const AttnArgs &a, uint64_t tiles) {
    AttnGrids g;
    g.items = a.target + tiles;
    // few joins take several teams to a row (a decode batch: 8.7 us in 1,008 workgroups, 13 in
    // 2,016); many are walked by at most 2048 workgroups, or one
    // a tile (most of them find whole results and end)
    const uint32_t all = 256 / (p.dim / 4);
    g.teams = all;
    while (g.teams > 1 && tiles * p.slot_rows * g.teams / all > 1024) g.teams /= 2;
    g.row_blocks = (p.slot_rows * g.teams + all - 1) / all;
    while (g.row_blocks > 1 && tiles * g.row_blocks > 2048) g.row_blocks = (g.row_blocks + 1) / 2;
    g.key_blocks = (uint32_t)(((uint64_t)a.max_kv + WEIGH_KEYS - 1) / WEIGH_KEYS);
    g.joins = tiles * g.row_blocks;
    g.weigh = p.scores ? (uint64_t)a.n_seqs * a.kv.n_kv * g.key_blocks : 0;
    g.sums = a.weight_out && !p.scores ? (uint64_t)a.n_seqs * a.kv.n_kv * p.key_blocks : 0;
    g.weights = g.sums * p.weight_parts;
    return g;
}
static bool attn_fits(const AttnGrids &g, const AttnPlan &p) {
    return launch_fits(g.items, p.few ? 256 : p.row_tile / 32 * WAVE) && launch_fits(g.joins + g.weigh, 256) && launch_fits(g.weights, 256);
}

template <class T, Held H, int D, bool FULL>
static pc_status attn_run(const AttnArgs &a, const AttnPlan &p, const AttnGrids &g, hipStream_t st) {
    const dim3 items((unsigned)g.items);
    if (p.few) {
        if constexpr (H == Held::E2M1) {
            const pc_status ok = attn_rows4(a, std::is_same<T, Bf16>::value, D, p.slot_rows, items, st);
            if (ok != PC_OK) return ok;
        } else {
            if (p.scores) PC_LAUNCH(K_ATTN_ROWS, (rows_kernel<T, H, D, FULL, true>), items, dim3(256), 0, st, a);
            else PC_LAUNCH(K_ATTN_ROWS, (rows_kernel<T, H, D, FULL, false>), items, dim3(256), 0, st, a);
        }
    } else if (p.wide) {
        constexpr int W = D == 128 ? CHUNK_WAVES_WIDE : CHUNK_WAVES;
        PC_LAUNCH(K_ATTN_CHUNK, (chunk_kernel<T, H, D, FULL, W>), items, dim3(W * WAVE), 0, st, a);
    } else {
        PC_LAUNCH(K_ATTN_CHUNK, (chunk_kernel<T, H, D, FULL, CHUNK_WAVES>), items, dim3(CHUNK_WAVES * WAVE), 0, st, a);
    }
    const dim3 joins((unsigned)(g.joins + g.weigh));
    constexpr bool EVEN = H == Held::E2M1;
    if (g.weigh)
        PC_LAUNCH(K_ATTN_JOIN, (join_kernel<T, D, EVEN, true>), joins, dim3(256), 0, st, a, g.teams, (uint32_t)g.joins, g.row_blocks,
                  g.key_blocks);
    else
        PC_LAUNCH(K_ATTN_JOIN, (join_kernel<T, D, EVEN, false>), joins, dim3(256), 0, st, a, g.teams, (uint32_t)g.joins, g.row_blocks,
                  g.key_blocks);
    if (g.weights) {
        PC_LAUNCH(K_ATTN_WEIGHT, (weight_kernel<T, H, D, FULL>), dim3((unsigned)g.weights), dim3(256), 0, st, a, p.key_blocks);
        if (p.weight_parts > 1) PC_LAUNCH(K_ATTN_WEIGHT, weight_sum_kernel, dim3((unsigned)g.sums), dim3(256), 0, st, a, p.key_blocks);
    }
    return PC_OK;
}
template <class T, Held H>
static pc_status attn_dim(const AttnArgs &a, const AttnPlan &p, const AttnGrids &g, hipStream_t st) {
    const bool full = a.kv.dim == p.dim;
    if (p.dim == 64) return full ? attn_run<T, H, 64, true>(a, p, g, st) : attn_run<T, H, 64, false>(a, p, g, st);
    if (p.dim == 128) return full ? attn_run<T, H, 128, true>(a, p, g, st) : attn_run<T, H, 128, false>(a, p, g, st);
    return full ? attn_run<T, H, 256, true>(a, p, g, st) : attn_run<T, H, 256, false>(a, p, g, st);
}

template <class T>
static pc_status attn_held(const AttnArgs &a, const AttnPlan &p, const AttnGrids &g, Held held, hipStream_t st) {
    if (held == Held::E2M1) return attn_dim<T, Held::E2M1>(a, p, g, st);
    return held == Held::E4M3 ? attn_dim<T, Held::E4M3>(a, p, g, st) : attn_dim<T, Held::SAME>(a, p, g, st);
}

}  // namespace pc

extern "C" {

size_t pc_attn_paged_ws(uint32_t n_seqs, uint32_t n_rows, uint32_t max_q, uint32_t max_kv, uint32_t n_heads,
                        uint32_t n_kv_heads, uint32_t head_dim, int with_weight) {
    using namespace pc;
    if (!n_heads || !n_kv_heads || n_heads % n_kv_heads) return WS_HEADER;
    AttnArgs a;
    const AttnPlan p = attn_plan(n_seqs, n_rows, max_q, max_kv, n_heads, n_kv_heads, head_dim, with_weight != 0);
    return attn_carve(&a, p, nullptr, n_seqs, n_rows, max_kv, n_heads, n_kv_heads, with_weight != 0);
}

pc_status pc_attn_paged(const pc_kv_cache *cache, const uint32_t *page_table, uint64_t table_stride,
                        const uint32_t *kv_len, const uint32_t *q_off, uint32_t n_seqs, uint32_t n_rows,
                        uint32_t max_q, uint32_t max_kv, const void *q, uint64_t q_stride_row,
                        uint64_t q_stride_head, uint32_t dtype, uint32_t n_heads, float scale, uint32_t flags,
                        uint32_t window, void *out, uint64_t out_stride_row, uint64_t out_stride_head, float *lse,
                        const float *weight, float *weight_out, uint64_t weight_stride, void *ws, size_t ws_bytes,
                        void *stream) {
    using namespace pc;
    AttnArgs a;
    const pc_status ok = kv_view(cache, &a.kv);
    if (ok != PC_OK) return ok;
    if (dtype != PC_BF16 && dtype != PC_F16) return PC_ERR_INVALID;
    if (cache->dtype != dtype && cache->dtype != PC_FP8_E4M3 && cache->dtype != PC_FP4_E2M1) return PC_ERR_INVALID;
    if (!n_heads || n_heads > PC_MAX_HEADS || n_heads % a.kv.n_kv || flags & ~PC_ATTN_CAUSAL || !isfinite(scale))
        return PC_ERR_INVALID;
    if (max_kv > 0x7FFF0000u || (uint64_t)n_rows * n_heads > 0x7FFFFFFFu || (uint64_t)max_q * n_heads > 0x7FFFFFFFu)
        return PC_ERR_TOO_LARGE;
    if (max_kv > table_stride * a.kv.page || (weight_out && max_kv > weight_stride) || (weight && !weight_out))
        return PC_ERR_INVALID;
    if (n_rows && (!n_seqs || !max_q || !q || !out)) return PC_ERR_INVALID;
    if (n_seqs && (!kv_len || !q_off || (max_kv && !page_table))) return PC_ERR_INVALID;
    if (((uint64_t)(uintptr_t)q | (uint64_t)(uintptr_t)out | q_stride_row * 2 | q_stride_head * 2 | out_stride_row * 2 |
         out_stride_head * 2) % 16)
        return PC_ERR_INVALID;
    const AttnPlan p = attn_plan(n_seqs, n_rows, max_q, max_kv, n_heads, a.kv.n_kv, a.kv.dim, weight_out != nullptr);
    const size_t need = attn_carve(&a, p, (char *)ws, n_seqs, n_rows, max_kv, n_heads, a.kv.n_kv, weight_out != nullptr);
    const hipStream_t st = (hipStream_t)stream;
    a.table = page_table;
    a.kv_len = kv_len;
    a.q_off = q_off;
    a.table_stride = table_stride;
    a.n_seqs = n_seqs;
    a.n_rows = n_rows;
    a.max_q = max_q;
    a.max_kv = max_kv;
    a.q = (const char *)q;
    a.out = (char *)out;
    a.q_row = q_stride_row * 2;
    a.q_head = q_stride_head * 2;
    a.o_row = out_stride_row * 2;
    a.o_head = out_stride_head * 2;
    a.lse = lse;
    a.weight = weight;
    a.weight_out = weight_out;
    a.weight_stride = weight_stride;
    a.n_heads = n_heads;
    a.group = n_heads / a.kv.n_kv;
    a.by_group = fast_div(a.group);
    a.scale = scale;
    a.causal = flags & PC_ATTN_CAUSAL;
    a.window = window;
    a.by_16 = a.kv.page % 16 == 0 && a.kv.st < (1u << 24);
    if (!p.scores) a.scores = nullptr;   // the workspace may have room for them all the same
    a.target = p.items;
    a.cut_first = p.ragged;   // few rows: items are alike but for the last (drafted tokens 28 us, cut first 31)
    a.even = cache->dtype == PC_FP4_E2M1 && p.few;
    if (a.even) {
        // One round of the chip, less the half range more that every uneven sequence and head is likely to make (618k
        // keys in 63 of them 139 -> 82 us).  Even ones make none or a whole one, and where they all make one the second
        // round is mostly empty: 32,768 keys over 4 heads of 128 for 16 / 20 / 24 / 28 / 32 sequences 61 / 99 / 94 / 140 /
        // 125 us.
        const uint32_t round = rows4_resident(p.dim, p.slot_rows), halves = (uint32_t)((uint64_t)n_seqs * a.kv.n_kv / 2 < round / 2
                                                                                           ? n_seqs * a.kv.n_kv / 2 : round / 2);
        a.target = round - halves;
    }
    a.least = p.few ? ROWS_LEAST : CHUNK_LEAST * 64 / chunk_keys(p.dim);
    a.row_tile = p.row_tile;
    a.key_tile = p.few ? 32 : chunk_keys(p.dim);
    // tiles of rows of every head, at most
    const uint64_t tiles = (p.few ? n_seqs : (uint64_t)n_rows * a.group / p.row_tile + n_seqs) * (uint64_t)a.kv.n_kv;
    const AttnGrids g = attn_grids(p, a, tiles);
    if (tiles * p.slot_rows + a.target > 0x7FFFFFFFu || !attn_fits(g, p)) return PC_ERR_TOO_LARGE;
    if (!ws || ws_bytes < need) return PC_ERR_WORKSPACE;
    const Entries from{q, a.q_row, a.q_head}, to{out, a.o_row, a.o_head};
    // in place, a row's query is read before its result is written, but for the weights' own pass
    const bool in_place = q == out && same_strides(from, to, n_rows, n_heads) && !weight_out;
    if (!in_place && entries_overlap(from, to, n_rows, n_heads, 2ull * a.kv.dim)) return PC_ERR_INVALID;
    const uint64_t weight_bytes = max_kv && n_seqs ? (((uint64_t)n_seqs * a.kv.n_kv - 1) * weight_stride + max_kv) * 4 : 0;
    if (weight && weight != weight_out && overlap(weight, weight_bytes, weight_out, weight_bytes)) return PC_ERR_INVALID;
    if (n_seqs == 0) return fill_u32((uint32_t *)ws, 0, 1, st);
    const Held held = cache->dtype == PC_FP8_E4M3 ? Held::E4M3 : cache->dtype == PC_FP4_E2M1 ? Held::E2M1 : Held::SAME;
    return dtype == PC_BF16 ? attn_held<Bf16>(a, p, g, held, st) : attn_held<F16>(a, p, g, held, st);
}

}  // extern "C"
