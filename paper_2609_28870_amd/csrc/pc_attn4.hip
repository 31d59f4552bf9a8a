// Attention of few new tokens over a cache in 4 bits: a kernel of its own, for a
// tile of keys is a quarter of the bytes while its products, exponentials and
// conversions stay, so that they, and not memory, would bound a path written for more.
#include "pc_attn.h"

namespace pc {

typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma16(Bf16, uint4 a, uint4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16(F16, uint4 a, uint4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// over the four lanes of a wave with the same lane % 16
__device__ __forceinline__ float max_of_quarters(float x) {
    const uint32_t b = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    return max_of_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float sum_of_quarters(float x) {
    const uint32_t b = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    return sum_of_halves(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// Values of a tile lie in LDS as rows of D 16-bit elements, in pieces of 16 bytes, piece c of row k at
// c ^ spread16(k).  They are written by 16 lanes at a time, the same piece of 16 rows, and read
// (transposed) by 32, two pieces of eight rows: both meet every bank once.
template <int D>
constexpr __device__ __forceinline__ uint32_t spread16(uint32_t row) {
    return D == 64 ? (row >> 1 & 3) << 1 | (row >> 3 & 1) : (row & 7) << 1 | (row >> 3 & 1);
}

// What a lane holds of a key: of every 128 dimensions the 32 of a block (of 64 dimensions 16, half a
// block), word w of piece i the eight from dim_of(i, w, lane / 16) on, which are its part of one
// step of the products (any order of the dimensions serves that keys and queries share).
template <int D>
constexpr __device__ __forceinline__ uint32_t dim_of(uint32_t i, uint32_t w, uint32_t quarter) {
    return 128 * i + (D == 64 ? 16 : 32) * quarter + 8 * w;
}

template <int D>
struct Rows16 {   // softmax state of 16 rows: lane % 16 is the row; the sum is each lane's own until the end
    f32x4 o[D / 16];
    float m, l;
};

// As add_not_finite of the other paths: key by key, the values that are not finite to the rows that see them.
template <class T, int D, class Query>
__device__ __forceinline__ void add_not_finite16(Rows16<D> &state, const AttnArgs &a, uint32_t seq, uint32_t head, uint32_t key,
                                                 int32_t first, int32_t last, float c, Query query) {
    const uint32_t lane = threadIdx.x & (WAVE - 1), quarter = lane / 16;
    const uint32_t at = a.kv.by_page.div(key), page = page_of(a.kv, a.table[(uint64_t)seq * a.table_stride + at]);
    const uint64_t entry = entry_at(a.kv, page, key - at * a.kv.page, head);
    auto element = [&](const char *codes, const uint8_t *exponents, uint32_t d) {
        const uint32_t w = *(const uint8_t *)(codes + entry + d / 2);
        return T::value(T::template from_e2m1<0>(w >> 4 * (d % 2), scale_of(exponents[entry / 16 + d / 32])) & 0xFFFF);
    };
    bool odd = false;
    for (uint32_t d = lane; d < a.kv.dim; d += WAVE) odd |= !(fabsf(element(a.kv.v, a.kv.v_exp, d)) < __builtin_inff());
    if (!ballot(odd)) return;
    float s = 0.f;
#pragma unroll 1
    for (uint32_t d = quarter; d < a.kv.dim; d += 4) s = fmaf(T::value(query(d)), element(a.kv.k, a.kv.k_exp, d), s);
    s = sum_of_quarters(s);
    const float p = exp2_fast(fmaf(s, c, T::TOP - state.m * c));
    const bool visible = (int32_t)key >= first && (int32_t)key <= last;
    const char *v = a.kv.v + entry + 2 * quarter;   // four codes are two bytes
#pragma unroll
    for (int b = 0; b < D / 16; ++b) {
        if (16u * b >= a.kv.dim) break;
        const float scale = scale_of(a.kv.v_exp[entry / 16 + b / 2]);
        const uint32_t w = *(const uint16_t *)(v + 8 * b);
        const uint32_t lo = T::template from_e2m1<0>(w, scale), hi = T::template from_e2m1<1>(w, scale);
        const float y[4] = {T::value(lo & 0xFFFF), T::value(lo >> 16), T::value(hi & 0xFFFF), T::value(hi >> 16)};
#pragma unroll
        for (int i = 0; i < 4; ++i) state.o[b][i] += visible && !(fabsf(y[i]) < __builtin_inff()) ? p * y[i] : 0.f;
        __asm__ volatile("" ::: "memory");   // few of the loads at once
    }
}

// Waves of a SIMD, and so workgroups of a compute unit, that the registers hold: a tile of 16 rows more takes those
// of one.
constexpr __host__ __device__ uint32_t rows4_waves(uint32_t dim, uint32_t tiles) {
    return (dim == 64 ? 4 : dim == 128 ? 3 : 2) - (tiles - 1);
}

// At most 16 R rows of a sequence (new tokens times the query heads that share a key/value head) against a range of
// its keys.  A wave takes 32 keys at a time on its own (every fourth such tile of the item), the next
// tile's codes on their way meanwhile.  Products are of 16 rows, so that a group of eight
// heads pays for 16, not 32; queries stay in registers, keys are widened straight into them,
// values pass through LDS for the transposed read.
// Where 16 slots share a page (by_16) a table entry is read for 16 keys, 32 tiles ahead, and
// the address is one number for the wave; else every lane looks its key's up (63 uneven sequences: pages of 16, 24 and 64
// slots 88 to 90 us, of one slot 207).
// Bound by memory: 32 over 4 heads of 128, 1.05M keys in 8 even sequences (570 MB) 106 us, 5.4 TB/s; 618k in 63
// uneven ones 70 us, 4.8 TB/s (two tiles on their way instead of one: 2% slower, with 160 registers for
// 138); one token over 1,537 keys 9 us, a chain of dependent loads.
template <class T, int D, bool FULL, int R, bool BY_16>
__global__ __launch_bounds__(256, rows4_waves(D, R)) void rows4_kernel(AttnArgs a) {
    constexpr int PIECES = D == 256 ? 2 : 1, WORDS = D == 64 ? 2 : 4, STEPS = PIECES * WORDS;
    __shared__ __attribute__((aligned(16))) char tiles[4 * 32 * D * 2];
    __shared__ float2 join_ml[2][R][64];
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = 0;
    const Item it = find_item<By::ITEM, true>(a, blockIdx.x);
    if (!it.there) return;
    const uint32_t lane = threadIdx.x & (WAVE - 1), wave = uniform(threadIdx.x / WAVE), col = lane % 16, quarter = lane / 16;
    const Seq &sq = it.shape.q;
    const uint32_t rows = sq.rows * a.group;
    uint32_t flip;
    bool zero;
    const float c = score_factor(a, it.head, &flip, &zero);
    // this lane's rows, the slots that they see, and those that every row sees
    int32_t first[R], last[R], all_first = 0, all_last = 0x7FFFFFFF;
    auto query_at = [&](uint32_t row) {
        const uint32_t token = a.by_group.div(row);
        return a.q + (uint64_t)(sq.first + token) * a.q_row + (it.head * a.group + (row - token * a.group)) * a.q_head;
    };
#pragma unroll
    for (int n = 0; n < R; ++n) {
        const uint32_t row = 16 * n + col, token = a.by_group.div(row < rows ? row : 0);
        first[n] = 0;
        last[n] = 0x7FFFFFFF;
        if (row < rows) seen_by_row(a, sq, token, &first[n], &last[n]);
        all_first = max(all_first, first[n]);
        all_last = min(all_last, last[n]);
    }
#pragma unroll
    for (int step = 1; step < 16; step *= 2) {
        all_first = max(all_first, __shfl_xor(all_first, step, WAVE));
        all_last = min(all_last, __shfl_xor(all_last, step, WAVE));
    }
    all_first = (int32_t)uniform((uint32_t)all_first);
    all_last = (int32_t)uniform((uint32_t)all_last);
    const uint32_t t0 = it.split * it.length + wave, t_end = min(it.shape.key_tiles, (it.split + 1) * it.length);
    const uint32_t *table = a.table + (uint64_t)it.seq * a.table_stride;
    char *tile = tiles + wave * (32 * D * 2);

    typedef std::conditional_t<D == 64, uint2, uint4> Piece;
    Piece k[2][PIECES], v[2][PIECES];          // of keys col and 16 + col
    uint32_t ke[2][PIECES], ve[2][PIECES];     // their scales
    const uint32_t g_last = (it.shape.keys.hi - 1) / 16;
    uint32_t groups = 0, groups_next = 0, g0 = 0;   // table entries of tiles g0 + lane / 2 (of this wave), half lane % 2
    auto look_up_groups = [&](uint32_t n) {
        const uint32_t g = it.shape.keys.lo / 16 + 2 * (t0 + 4 * (n + lane / 2)) + lane % 2;
        return table[a.kv.by_page.div(min(g, g_last) * 16)];
    };
    uint32_t entry[2] = {0, 0}, off[2] = {0, 0};
    auto look_up = [&](uint32_t t) {
        if (BY_16) return;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const uint32_t j = min(it.shape.keys.lo + t * 32 + 16 * b + col, it.shape.keys.hi - 1), p = a.kv.by_page.div(j);
            off[b] = j - p * a.kv.page;
            entry[b] = table[p];
        }
    };
    // this lane's part of an entry; past the head's dimensions the first ones
    const uint32_t o_codes = FULL || dim_of<D>(0, 0, quarter) < a.kv.dim ? dim_of<D>(0, 0, quarter) / 2 : 0;
    const uint32_t o_row = col * (uint32_t)a.kv.st + o_codes;
    uint64_t at[2];
    auto locate = [&](uint32_t n, uint32_t t) {
        if (BY_16) {
            if (n - g0 >= WAVE / 2) {
                g0 += WAVE / 2;
                groups = groups_next;
                groups_next = look_up_groups(g0 + WAVE / 2);
            }
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const uint32_t slot = min(it.shape.keys.lo / 16 + 2 * t + b, g_last) * 16, p = a.kv.by_page.div(slot);
                at[b] = entry_at(a.kv, page_of(a.kv, from_lane(groups, (int)(2 * (n - g0) + b))), slot - p * a.kv.page, it.head);
            }
            return;
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) at[b] = entry_at(a.kv, page_of(a.kv, entry[b]), off[b], it.head);
    };
    auto load = [&](const char *codes, const uint8_t *exponents, Piece (&x)[2][PIECES], uint32_t (&e)[2][PIECES]) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const uint32_t o = BY_16 ? o_row : o_codes;
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const bool in = FULL || i == 0 || dim_of<D>(i, 0, quarter) < a.kv.dim;
                x[b][i] = *(const Piece *)(codes + at[b] + o + (in ? 64 * i : 0));
                e[b][i] = exponents[at[b] / 16 + o / 16 + (in ? 4 * i : 0)];
            }
        }
    };
    if (t0 < t_end) {
        if (BY_16) {
            groups = look_up_groups(0);
            groups_next = look_up_groups(WAVE / 2);
        }
        look_up(t0);
    }
    uint4 q[R][STEPS];
#pragma unroll
    for (int n = 0; n < R; ++n)
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const uint32_t d = dim_of<D>(s / WORDS, s % WORDS, quarter);
            q[n][s] = make_uint4(0, 0, 0, 0);
            if (16u * n + col < rows && (FULL || d < a.kv.dim)) q[n][s] = *(const uint4 *)(query_at(16 * n + col) + d * 2);
        }
    if (t0 < t_end) {
        locate(0, t0);
        load(a.kv.k, a.kv.k_exp, k, ke);
        load(a.kv.v, a.kv.v_exp, v, ve);
        look_up(min(t0 + 4, t_end - 1));
    }
#pragma unroll
    for (int n = 0; n < R; ++n) sign_query<T>(q[n], flip, zero);
    bool odd = false;   // a value that is not finite was left out of a tile
    const float slack = slack_of<T>(c);
    Rows16<D> state[R];
#pragma unroll
    for (int n = 0; n < R; ++n) {
#pragma unroll
        for (int b = 0; b < D / 16; ++b) state[n].o[b] = f32x4(0.f);
        state[n].m = MINUS_INF;
        state[n].l = 0.f;
    }
    auto word = [](Piece x, int i) {
        if constexpr (D == 64) return i ? x.y : x.x;
        else return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w;
    };
    // where this lane writes its values, and where it reads: four keys 4 quarter + (0 .. 3) of dimension col of 16
    const uint32_t w_row = col * (D * 2), w_spread = spread16<D>(col) * 16;
    const uint32_t r_row = 4 * quarter + col / 4, r_at = r_row * (D * 2) + (((lane % 4 / 2) ^ spread16<D>(r_row)) * 16) + lane % 2 * 8;
    for (uint32_t n = 0, t = t0; t < t_end; ++n, t += 4) {
        const bool more = t + 4 < t_end;
        const uint32_t k0 = it.shape.keys.lo + t * 32;
        const bool full = (int32_t)k0 >= all_first && (int32_t)k0 + 31 <= all_last;
        f32x4 s[R][2];
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const uint4 x = expand<T>(word(k[b][i / WORDS], i % WORDS), scale_of(ke[b][i / WORDS]));
                // queries are zero past the head's dimensions, and what is read there is a number unless a scale is not
                const bool past = !FULL && dim_of<D>(i / WORDS, i % WORDS, quarter) >= a.kv.dim;
                const uint4 y = past ? make_uint4(0, 0, 0, 0) : x;
#pragma unroll
                for (int r = 0; r < R; ++r) s[r][b] = mfma16(T{}, y, q[r][i], i ? s[r][b] : f32x4(0.f));
            }
        if (more) {
            locate(n + 1, t + 4);
            load(a.kv.k, a.kv.k_exp, k, ke);
        }
        auto value_at = [&](int b, int i, int w) {
            return (uint4 *)(tile + b * (16 * D * 2) + w_row + (dim_of<D>(i, w, quarter) / 8 * 16 ^ w_spread));
        };
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
#pragma unroll
                for (int w = 0; w < WORDS; ++w) *value_at(b, i, w) = expand<T>(word(v[b][i], w), scale_of(ve[b][i]));
        if (!full) {   // seldom, and apart, in few registers
#pragma unroll 1
            for (int n = 0; n < 2 * STEPS; ++n) {
                uint4 *x = value_at(n / STEPS, n % STEPS / WORDS, n % WORDS);
                *x = drop_not_finite<T>(*x, &odd);
            }
        }
        if (more) {
            load(a.kv.v, a.kv.v_exp, v, ve);
            if (t + 8 < t_end) look_up(t + 8);
        }
        uint4 p[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (!full) {
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int32_t key = (int32_t)(k0 + 16 * b + 4 * quarter + i);
                        if (key < first[r] || key > last[r]) s[r][b][i] = MINUS_INF;
                    }
            }
            if (a.scores && 16u * r + col < rows) {
                float *w = a.scores + (((uint64_t)it.seq * a.kv.n_kv + it.head) * a.slot_rows + 16 * r + col) * a.score_stride + k0 + 4 * quarter;
#pragma unroll
                for (int b = 0; b < 2; ++b)
                    *(float4 *)(w + 16 * b) = make_float4(s[r][b][0] * c, s[r][b][1] * c, s[r][b][2] * c, s[r][b][3] * c);
            }
            Rows16<D> &st = state[r];
            float top = s[r][0][0];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, s[r][b][i]);
            top = max_of_quarters(top);
            if (ballot(top > st.m + slack)) {
                // a row that has seen nothing keeps a sum of 0: exp2(-inf - 0)
                const float next = fmaxf(st.m, top), f = exp2_fast((st.m - (next == MINUS_INF ? 0.f : next)) * c);
                st.l *= f;
#pragma unroll
                for (int b = 0; b < D / 16; ++b) st.o[b] *= f;
                st.m = next;
            }
            const float ref = st.m == MINUS_INF ? 0.f : st.m, shift = T::TOP - ref * c;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll
                for (int i = 0; i < 4; ++i) s[r][b][i] = exp2_fast(fmaf(s[r][b][i], c, shift));
                st.l += (s[r][b][0] + s[r][b][1]) + (s[r][b][2] + s[r][b][3]);
            }
            p[r] = make_uint4(T::pack(s[r][0][0], s[r][0][1]), T::pack(s[r][0][2], s[r][0][3]), T::pack(s[r][1][0], s[r][1][1]),
                              T::pack(s[r][1][2], s[r][1][3]));
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int b = 0; b < D / 16; ++b) {
            const char *x = tile + (r_at ^ (b % 8 * 32)) + b / 8 * 256;
            const uint2 lo = read_transposed(x), hi = read_transposed(x + 16 * D * 2);
#pragma unroll
            for (int r = 0; r < R; ++r) state[r].o[b] = mfma16(T{}, make_uint4(lo.x, lo.y, hi.x, hi.y), p[r], state[r].o[b]);
        }
        __builtin_amdgcn_wave_barrier();
    }
    if (ballot(odd)) {
        uint32_t row = col;
        __asm__ volatile("" : "+v"(row));   // found anew here, not kept through the loop above
        for (uint32_t t = t0; t < t_end; t += 4) {
            const uint32_t k0 = it.shape.keys.lo + t * 32;
            if ((int32_t)k0 >= all_first && (int32_t)k0 + 31 <= all_last) continue;
            for (uint32_t key = k0; key < min(k0 + 32, it.shape.keys.hi); ++key)
#pragma unroll
                for (int r = 0; r < R; ++r)
                    add_not_finite16<T, D>(state[r], a, it.seq, it.head, key, first[r], last[r], c, [&](uint32_t d) {
                        return zero ? 0u : *(const uint16_t *)(query_at(min(16 * r + row, rows - 1)) + 2 * d) ^ (flip & 0x8000u);
                    });
        }
    }
    float m[R], l[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        m[r] = state[r].m == MINUS_INF ? MINUS_INF : state[r].m * c;
        l[r] = sum_of_quarters(state[r].l);
    }
    // waves 2 and 3 to 0 and 1, then 1 to 0
    for (int from = 2; from >= 1; from /= 2) {
        __syncthreads();
        float *buf = (float *)tiles + (wave % from) * (R * D * 16);
        if (wave >= (uint32_t)from && wave < 2u * from) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                join_ml[wave % from][r][lane] = make_float2(m[r], l[r]);
#pragma unroll
                for (int b = 0; b < D / 16; ++b) *(f32x4 *)(buf + ((r * (D / 16) + b) * WAVE + lane) * 4) = state[r].o[b];
            }
        }
        __syncthreads();
        if (wave < (uint32_t)from) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float2 ml = join_ml[wave][r][lane];
                const float top = fmaxf(m[r], ml.x), ref = top == MINUS_INF ? 0.f : top;
                const float f = exp2_fast(m[r] - ref), g = exp2_fast(ml.x - ref);
                m[r] = top;
                l[r] = l[r] * f + ml.y * g;
#pragma unroll
                for (int b = 0; b < D / 16; ++b)
                    state[r].o[b] = state[r].o[b] * f + *(const f32x4 *)(buf + ((r * (D / 16) + b) * WAVE + lane) * 4) * g;
            }
        }
    }
    if (wave) return;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t row = 16 * r + col;
        if (row >= rows) continue;
        if (it.splits > 1) {
            if (it.slot >= a.slots) continue;
            const uint64_t part = (uint64_t)it.slot * a.slot_rows + row;
            if (quarter == 0) a.part_ml[part] = make_float2(m[r], l[r]);
#pragma unroll
            for (int b = 0; b < D / 16; ++b) *(f32x4 *)(a.part + part * D + 16 * b + 4 * quarter) = state[r].o[b];
            continue;
        }
        const uint32_t token = a.by_group.div(row), t = sq.first + token, head = it.head * a.group + (row - token * a.group);
        const float base2 = log_sum<T>(m[r], l[r]), f = l[r] == 0.f ? 0.f : 1.f / l[r];
        if (quarter == 0) {
            if (a.lse) a.lse[(uint64_t)t * a.n_heads + head] = base2 * LN2;
            if (a.lse2) a.lse2[(uint64_t)t * a.n_heads + head] = base2;
        }
        char *out = a.out + (uint64_t)t * a.o_row + head * a.o_head;
#pragma unroll
        for (int b = 0; b < D / 16; ++b) {
            const uint32_t d = 16 * b + 4 * quarter;
            if (FULL || d < a.kv.dim)
                *(uint2 *)(out + 2 * d) = make_uint2(T::pack(state[r].o[b][0] * f, state[r].o[b][1] * f),
                                                     T::pack(state[r].o[b][2] * f, state[r].o[b][3] * f));
        }
    }
}

uint32_t rows4_resident(uint32_t dim, uint32_t max_rows) { return 256 * rows4_waves(dim, max_rows <= 16 ? 1 : 2); }

template <class T, int D, bool FULL>
static pc_status rows4_run(const AttnArgs &a, uint32_t max_rows, dim3 items, hipStream_t st) {
    if (max_rows <= 16) {
        if (a.by_16) PC_LAUNCH(K_ATTN_ROWS, (rows4_kernel<T, D, FULL, 1, true>), items, dim3(256), 0, st, a);
        else PC_LAUNCH(K_ATTN_ROWS, (rows4_kernel<T, D, FULL, 1, false>), items, dim3(256), 0, st, a);
    } else {
        if (a.by_16) PC_LAUNCH(K_ATTN_ROWS, (rows4_kernel<T, D, FULL, 2, true>), items, dim3(256), 0, st, a);
        else PC_LAUNCH(K_ATTN_ROWS, (rows4_kernel<T, D, FULL, 2, false>), items, dim3(256), 0, st, a);
    }
    return PC_OK;
}
template <class T, int D>
static pc_status rows4_dim(const AttnArgs &a, uint32_t max_rows, dim3 items, hipStream_t st) {
    return a.kv.dim == D ? rows4_run<T, D, true>(a, max_rows, items, st) : rows4_run<T, D, false>(a, max_rows, items, st);
}
template <class T>
static pc_status rows4_type(const AttnArgs &a, uint32_t dim, uint32_t max_rows, dim3 items, hipStream_t st) {
    if (dim == 64) return rows4_dim<T, 64>(a, max_rows, items, st);
    return dim == 128 ? rows4_dim<T, 128>(a, max_rows, items, st) : rows4_dim<T, 256>(a, max_rows, items, st);
}
pc_status attn_rows4(const AttnArgs &a, bool bf16, uint32_t dim, uint32_t max_rows, dim3 items, hipStream_t st) {
    return bf16 ? rows4_type<Bf16>(a, dim, max_rows, items, st) : rows4_type<F16>(a, dim, max_rows, items, st);
}

}  // namespace pc
