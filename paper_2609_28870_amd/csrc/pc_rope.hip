// Rotary positions: tables of their cosines and sines (pc_rope_table), rows turned
// by them (pc_rope), and new tokens written into the paged cache with the rotation
// applied on the way (pc_kv_append_rope); and every append into a cache of 4 bits.
#include <math.h>

#include "pc_kv.h"

namespace pc {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

template <bool BF>
__device__ __forceinline__ void unpack(uint4 x, float (&f)[8]) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = to_float(w[i] & 0xFFFF, BF);
        f[2 * i + 1] = to_float(w[i] >> 16, BF);
    }
}
template <bool BF>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
    if (BF) {
        const bf16x2 v = {(__bf16)x, (__bf16)y};
        return __builtin_bit_cast(uint32_t, v);
    }
    const f16x2 v = {(_Float16)x, (_Float16)y};
    return __builtin_bit_cast(uint32_t, v);
}
template <bool BF>
__device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    return make_uint4(pack2<BF>(f[0], f[1]), pack2<BF>(f[2], f[3]), pack2<BF>(f[4], f[5]), pack2<BF>(f[6], f[7]));
}

// x c + y s.  For 16-bit results 32 bits are enough (two roundings of 2^-24 before one of 2^-8 or
// 2^-11).  Codes of 8 and 4 bits take the sum in 64 bits, rounded to 32 (a product of a
// 16-bit and a 32-bit number is exact in 64, so the sum has one rounding there): what is next to a border between two
// codes is then on the same side for whoever computes it in 64 bits.
template <bool EXACT>
__device__ __forceinline__ float turned(float x, float y, float c, float s) {
    if (EXACT) return (float)fma((double)x, (double)c, (double)y * (double)s);
    float r = fmaf(x, c, y * s);
    // rounded to 32 bits here: a fused sum that rounds to float16 at once, where the compiler finds
    // one, would make the same element differ between two kernels
    __asm__("" : "+v"(r));
    return r;
}

// ------------------------------------------------------------------- table

constexpr double TWO_OVER_PI = 0.63661977236758134308, HALF_PI = 1.57079632679489661923, HALF_PI_REST = 6.12323399573676603587e-17;

struct Frequencies {
    double f[PC_MAX_HEAD_DIM / 2];
};

// Cosine and sine of the product p f, p a whole number below 2^32: the product and what its rounding
// leaves, less a multiple of pi/2 (exact in the fused sums), then their series up to r^14 and
// r^13.  |r| is at most pi/4, but for large products: near 2^48, the largest, their own rounding and the
// quotient's add up to 0.08.  The first terms left out are r^15 / 15! and r^16 / 16!: 2.1e-14 at pi/4, 1e-13 at 0.87.
__device__ __forceinline__ double2 turn_by(double p, double f) {
    const double a = p * f, n = rint(a * TWO_OVER_PI);
    const double r = fma(-n, HALF_PI, a) + fma(-n, HALF_PI_REST, fma(p, f, -a)), z = r * r;
    double s = 1.0 / 6227020800.0, c = -1.0 / 87178291200.0;
    s = fma(s, z, -1.0 / 39916800.0);
    s = fma(s, z, 1.0 / 362880.0);
    s = fma(s, z, -1.0 / 5040.0);
    s = fma(s, z, 1.0 / 120.0);
    s = fma(s, z, -1.0 / 6.0);
    s = fma(s * z, r, r);
    c = fma(c, z, 1.0 / 479001600.0);
    c = fma(c, z, -1.0 / 3628800.0);
    c = fma(c, z, 1.0 / 40320.0);
    c = fma(c, z, -1.0 / 720.0);
    c = fma(c, z, 1.0 / 24.0);
    c = fma(c, z, -0.5);
    c = fma(c, z, 1.0);
    // n modulo 4, which is below 2^51: from the bits of n + 1.5 * 2^52
    const uint32_t quarter = (uint32_t)__double_as_longlong(n + 6755399441055744.0);
    const double x = (quarter & 1) ? s : c, y = (quarter & 1) ? c : s;
    return make_double2(((quarter + 1) & 2) ? -x : x, (quarter & 2) ? -y : y);
}

// A thread keeps its frequency over POSITIONS positions, `together` apart: the first angle and the
// step are worked out, the others are the one turned by the other, four products in 64 bits, each off by
// 2^-52 more.  (All of them worked out: 18.2 us for 131,072 positions of 64 pairs, bound by 64-bit arithmetic.)
constexpr int POSITIONS = 16;
__global__ __launch_bounds__(256) void rope_table_kernel(Frequencies freq, uint32_t half, uint32_t together, uint32_t first, uint32_t n_pos,
                                                         double magnitude, float2 *__restrict__ out) {
    const uint32_t at = threadIdx.x / half, d = threadIdx.x - at * half;
    if (at >= together) return;
    const double f = freq.f[d];
    uint32_t p = blockIdx.x * (together * POSITIONS) + at;   // below 2^32: the last group starts inside the table
    if (p >= n_pos) return;
    const double2 step = turn_by(together, f);
    double2 x = turn_by((double)first + (double)p, f);
    x = make_double2(x.x * magnitude, x.y * magnitude);
    float2 *to = out + (uint64_t)p * half + d;
#pragma unroll
    for (int i = 0; i < POSITIONS; ++i) {
        *to = make_float2((float)x.x, (float)x.y);
        if (n_pos - p <= together) return;
        p += together;
        to += together * half;
        x = make_double2(fma(x.x, step.x, -(x.y * step.y)), fma(x.y, step.x, x.x * step.y));
    }
}

// -------------------------------------------------------------------- rows

// Where a workgroup's threads are: a unit is what one thread turns of one head (eight dimensions
// and their partners, or one and its partner in layouts of any size), then the pieces
// that stay as they are.  A thread takes the same unit of every `apart`-th head, so that
// it reads its cosines once.  Halves of a part that is no multiple of 16 (Layout::ANY) go two bytes at a time,
// what does not turn among them: 16,384 rows of 20 heads of 96, 24 turned 76 us (in place, where only those move, 13),
// 32 turned 31 (14).
struct Shape {
    uint32_t units, turning;   // of a head; of them, those that turn
    uint32_t apart;            // threads to a unit of a row
    FastDiv by_unit, by_row;   // units, units * apart
    uint32_t rows;             // of a workgroup
};

constexpr int AT_ONCE = 4;   // heads whose loads are on their way together

template <bool BF, Layout L, class Pos>
__device__ __forceinline__ void turn_rows(const Queries &q, const Turn &turn, const Shape &g, uint32_t t0, uint32_t rows, Pos pos_of) {
    for (uint32_t p = threadIdx.x; p < rows * g.by_row.d; p += 256) {
        const uint32_t i = g.by_row.div(p), r = p - i * g.by_row.d, h0 = g.by_unit.div(r), u = r - h0 * g.units;
        const uint64_t t = t0 + i;
        const uint32_t pos = pos_of(i);
        if (pos >= turn.n_pos) continue;
        const float2 *angles = turn.table + (uint64_t)pos * turn.half;
        const bool turns = u < g.turning;
        const char *x = q.x + t * q.x_row + h0 * q.x_head;
        char *out = q.out + t * q.o_row + h0 * q.o_head;
        const uint64_t x_step = g.apart * q.x_head, o_step = g.apart * q.o_head;
        if (L == Layout::ANY) {
            const uint32_t a = turns ? u : u + turn.half, b = turns ? u + turn.half : a;
            const float2 cs = turns ? angles[u] : make_float2(1.f, 0.f);
            for (uint32_t h = h0; h < q.n_heads; h += g.apart, x += x_step, out += o_step) {
                const uint16_t xa = *(const uint16_t *)(x + 2 * a), xb = *(const uint16_t *)(x + 2 * b);
                if (!turns) {
                    *(uint16_t *)(out + 2 * a) = xa;
                    continue;
                }
                const float fa = to_float(xa, BF), fb = to_float(xb, BF), s = cs.y * turn.sign;
                const uint32_t y = pack2<BF>(turned<false>(fa, fb, cs.x, -s), turned<false>(fb, fa, cs.x, s));
                *(uint16_t *)(out + 2 * a) = (uint16_t)y;
                *(uint16_t *)(out + 2 * b) = (uint16_t)(y >> 16);
            }
            continue;
        }
        constexpr int N = L == Layout::HALVES ? 8 : 4;   // angles of a unit
        const uint32_t a = L == Layout::HALVES && !turns ? 16 * u + 16 * (turn.half / 8) : 16 * u, b = a + 2 * turn.half;   // bytes
        float c[N], s[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const uint32_t n = N * u + j;
            const float2 cs = turns && n < turn.half ? angles[n] : make_float2(1.f, 0.f);
            c[j] = cs.x;
            s[j] = cs.y * turn.sign;
        }
        for (uint32_t h = h0; h < q.n_heads; h += AT_ONCE * g.apart) {
            uint4 xa[AT_ONCE], xb[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const char *y = h + k * g.apart < q.n_heads ? x + k * x_step : x;
                xa[k] = *(const uint4 *)(y + a);
                if (L == Layout::HALVES && turns) xb[k] = *(const uint4 *)(y + b);
            }
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                if (h + k * g.apart >= q.n_heads) break;
                char *to = out + k * o_step;
                if (turns) {
                    float fa[8], ya[8];
                    unpack<BF>(xa[k], fa);
                    if (L == Layout::HALVES) {
                        float fb[8], yb[8];
                        unpack<BF>(xb[k], fb);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            ya[j] = turned<false>(fa[j], fb[j], c[j % N], -s[j % N]);
                            yb[j] = turned<false>(fb[j], fa[j], c[j % N], s[j % N]);
                        }
                        *(uint4 *)(to + b) = pack<BF>(yb);
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const bool there = 4 * u + j < turn.half;   // of the last piece some may not turn
                            ya[2 * j] = there ? turned<false>(fa[2 * j], fa[2 * j + 1], c[j % N], -s[j % N]) : fa[2 * j];
                            ya[2 * j + 1] = there ? turned<false>(fa[2 * j + 1], fa[2 * j], c[j % N], s[j % N]) : fa[2 * j + 1];
                        }
                    }
                    *(uint4 *)(to + a) = pack<BF>(ya);
                } else {
                    *(uint4 *)(to + a) = xa[k];
                }
            }
            x += AT_ONCE * x_step;
            out += AT_ONCE * o_step;
        }
    }
}

// whether a position of the call's rows is past the table, by this workgroup's part of them
__device__ __forceinline__ bool positions_bad(const uint32_t *__restrict__ pos, uint32_t n_pos, uint32_t n_rows) {
    uint32_t most = 0;
    for (uint32_t t = threadIdx.x; t < n_rows; t += 8 * 256) {
        uint32_t x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = pos[min(t + 256 * i, n_rows - 1)];
#pragma unroll
        for (int i = 0; i < 8; ++i) most = max(most, x[i]);
    }
    return most >= n_pos;
}

// A read and a write of the rows, the angles from a cache: bound by memory (16,384 rows of 32 heads of 128,
// 271 MB: 44 us in passes over the same rows, 51 over others each time).
template <bool BF, Layout L>
__global__ __launch_bounds__(256) void rope_kernel(Queries q, Turn turn, Shape g, uint32_t n_rows, int32_t *status, uint32_t cleared) {
    const uint32_t block = cleared ? blockIdx.x : blockIdx.x - 1;
    if (!cleared && blockIdx.x == 0) {
        const int any = __syncthreads_or(turn.pos && n_rows && positions_bad(turn.pos, turn.n_pos, n_rows));
        if (threadIdx.x == 0) *status = any ? DEV_ERR_BAD_LAYOUT : 0;
        return;
    }
    const uint32_t t0 = block * g.rows, rows = min(g.rows, n_rows - t0);
    if (cleared && turn.pos && threadIdx.x < rows && turn.pos[t0 + threadIdx.x] >= turn.n_pos) atomicOr(status, DEV_ERR_BAD_LAYOUT);
    turn_rows<BF, L>(q, turn, g, t0, rows, [&](uint32_t i) { return turn.pos ? turn.pos[t0 + i] : t0 + i; });
}

// ------------------------------------------------------------------ append

constexpr uint32_t GROUP_ROWS = 64;   // at most, of a workgroup

struct AppendTurnedArgs {
    Chunks c;
    const char *k, *v;               // strides in bytes
    uint64_t k_row, k_head, v_row, v_head;
    Turn turn;
    Queries q;
    Shape g;                         // of the queries
    int32_t *status;
    FastDiv by_head, by_token;       // pieces of a head's entry, and of a token's
    uint32_t rows, groups;           // of a workgroup that writes keys and values, and those workgroups
    uint32_t cleared;                // the status word is cleared, and every row's position reported by its workgroup
};

// Where rows t0 .. t0 + rows - 1 go (bytes from the cache's start) and their positions, by the
// first wave: ~0 and PC_NONE of a row that has none.
__device__ __forceinline__ void find_places(const AppendTurnedArgs &a, uint32_t t0, uint32_t rows, bool pages, uint64_t *to, uint32_t *pos) {
    if (threadIdx.x >= WAVE) return;
    const Chunks &c = a.c;
    const uint32_t lane = threadIdx.x, t = t0 + min(lane, rows - 1);
    uint32_t p = a.turn.pos ? a.turn.pos[t] : 0;
    uint64_t at = ~0ull;
    if (pages || !a.turn.pos) {
        const uint32_t s0 = wave_seq_of(c.q_off, c.n_seqs, t0);
        // the ends of the 64 sequences from there on, a lane each; a row is behind those that are not past it
        const uint32_t end = s0 + 1 + lane < c.n_seqs ? c.q_off[s0 + 1 + lane] : 0xFFFFFFFFu;
        uint32_t behind = 0;
        for (uint32_t i = 0; i < rows; ++i) {
            const uint32_t n = (uint32_t)__popcll(ballot(end <= t0 + i));
            behind = lane == i ? n : behind;
        }
        uint32_t s = min(s0 + behind, c.n_seqs - 1);
        if (behind == WAVE && s + 1 < c.n_seqs && c.q_off[s + 1] <= t) s += 1 + seq_of(c.q_off + s + 1, c.n_seqs - s - 1, t);
        bool bad;
        const Seq q = load_seq(c.q_off, c.kv_len, s, c.n_rows, c.max_kv, &bad);
        const int64_t slot = slot_of_row(c.kv_len, c.max_kv, s, q, t);
        const bool there = t >= q.first && t - q.first < q.rows && slot >= 0;
        if (!a.turn.pos) p = there ? (uint32_t)slot : PC_NONE;
        if (pages && there && (!a.turn.half || p < a.turn.n_pos)) {
            const uint32_t n = c.kv.by_page.div((uint32_t)slot), off = (uint32_t)slot - n * c.kv.page;
            const uint32_t page = c.table[(uint64_t)s * c.table_stride + n];
            if (page < c.kv.n_pages) at = page * c.kv.sp + off * c.kv.st;
        }
    }
    if (lane < rows) {
        if (pages) to[lane] = at;
        pos[lane] = p;
    }
}

// Eight values from dimension d of a key's row on, turned by the angles of its position.
template <bool BF, Layout L, bool EXACT>
__device__ __forceinline__ void turned_piece(const char *row, uint32_t d, const Turn &turn, const float2 *__restrict__ angles, float (&y)[8]) {
    float x[8];
    unpack<BF>(*(const uint4 *)(row + 2 * d), x);
    const uint32_t half = turn.half;
    if (d >= 2 * half) {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = x[j];
    } else if (L == Layout::PAIRS) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t n = d / 2 + j;
            y[2 * j] = x[2 * j];
            y[2 * j + 1] = x[2 * j + 1];
            if (n < half) {
                const float2 cs = angles[n];
                y[2 * j] = turned<EXACT>(x[2 * j], x[2 * j + 1], cs.x, -cs.y);
                y[2 * j + 1] = turned<EXACT>(x[2 * j + 1], x[2 * j], cs.x, cs.y);
            }
        }
    } else if (L == Layout::HALVES) {
        const bool second = d >= half;
        const uint32_t n = second ? d - half : d;
        float other[8];
        unpack<BF>(*(const uint4 *)(row + 2 * (second ? n : d + half)), other);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float2 cs = angles[n + j];
            y[j] = turned<EXACT>(x[j], other[j], cs.x, second ? cs.y : -cs.y);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t e = d + j;
            y[j] = x[j];
            if (e < 2 * half) {
                const bool second = e >= half;
                const uint32_t n = second ? e - half : e;
                const float2 cs = angles[n];
                const float other = to_float(*(const uint16_t *)(row + 2 * (second ? n : e + half)), BF);
                y[j] = turned<EXACT>(x[j], other, cs.x, second ? cs.y : -cs.y);
            }
        }
    }
}

// 32 values as 4-bit codes (steps of a half up to 2, of 1 up to 4, and 6), the low half of a byte first, and the exponent byte of
// their scale.  It is the power of two that leaves the largest below 7, so that no code is off by
// more than half a step; bounded to what the type's numbers hold (6 times the largest one is
// finite, half the smallest one a number).  NaN takes its block with it.
template <bool BF>
__device__ __forceinline__ uint4 to_e2m1(const float (&y)[32], uint32_t *exponent) {
    float top = 0.f;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        top = fmaxf(top, fabsf(y[i]));
        nan |= y[i] != y[i];
    }
    int e = (int)((__float_as_uint(top) + 0x200000u) >> 23) - 2;
    e = min(max(e, BF ? 1 : 104), BF ? 252 : 140);
    *exponent = nan ? 255 : (uint32_t)e;
    const float scale = __uint_as_float((uint32_t)e << 23);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, y[8 * i], y[8 * i + 1], scale, 0);
        w[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[i], y[8 * i + 2], y[8 * i + 3], scale, 1);
        w[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[i], y[8 * i + 4], y[8 * i + 5], scale, 2);
        w[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[i], y[8 * i + 6], y[8 * i + 7], scale, 3);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// One launch: a workgroup for the status word, then keys and values, a 16-byte piece of the
// cache a thread, then queries.  CACHE: PC_FP8_E4M3, PC_FP4_E2M1, or the new tokens' own type.
// Bound by memory, or for a few tokens by the launch and the chain of loads to a row's page: 268 MB of
// ragged chunks into 4 bits 58 us (4.6 TB/s), into 8 bits 62; 256 single tokens 5 us.
template <bool BF, Layout L, uint32_t CACHE>
__global__ __launch_bounds__(256) void append_turned_kernel(AppendTurnedArgs a) {
    __shared__ uint64_t to[GROUP_ROWS];
    __shared__ uint32_t pos[GROUP_ROWS];
    const Chunks &c = a.c;
    if (blockIdx.x == 0) {
        const bool listed = a.turn.pos != nullptr, turns = a.turn.half != 0;
        bool bad = chunks_bad(c, turns && !listed ? a.turn.n_pos : 0xFFFFFFFFu);
        if (listed && !a.cleared && c.n_rows) bad |= positions_bad(a.turn.pos, a.turn.n_pos, c.n_rows);
        const int any = __syncthreads_or(bad);
        if (threadIdx.x == 0) {
            if (!a.cleared) *a.status = any ? DEV_ERR_BAD_LAYOUT : 0;
            else if (any) atomicOr(a.status, DEV_ERR_BAD_LAYOUT);
        }
        return;
    }
    if (blockIdx.x > a.groups) {
        const uint32_t t0 = (blockIdx.x - 1 - a.groups) * a.g.rows, rows = min(a.g.rows, c.n_rows - t0);
        find_places(a, t0, rows, false, to, pos);
        __syncthreads();
        turn_rows<BF, L>(a.q, a.turn, a.g, t0, rows, [&](uint32_t i) { return pos[i]; });
        return;
    }
    const uint32_t t0 = (blockIdx.x - 1) * a.rows, rows = min(a.rows, c.n_rows - t0);
    find_places(a, t0, rows, true, to, pos);
    if (a.cleared && threadIdx.x < rows && a.turn.pos && a.turn.pos[t0 + threadIdx.x] >= a.turn.n_pos) atomicOr(a.status, DEV_ERR_BAD_LAYOUT);
    __syncthreads();
    constexpr uint32_t E = CACHE == PC_FP4_E2M1 ? 32 : CACHE == PC_FP8_E4M3 ? 16 : 8;   // elements of a piece
    const uint32_t pieces = rows * a.by_token.d;   // keys', then values'
    for (uint32_t p = threadIdx.x; p < 2 * pieces; p += 256) {
        const bool value = p >= pieces;
        const uint32_t r = value ? p - pieces : p, i = a.by_token.div(r), of = r - i * a.by_token.d;
        const uint32_t h = a.by_head.div(of), n = of - h * a.by_head.d;
        if (to[i] == ~0ull) continue;
        const uint64_t dst = to[i] + h * c.kv.sh + n * 16, t = t0 + i;
        const char *row = value ? a.v + t * a.v_row + h * a.v_head : a.k + t * a.k_row + h * a.k_head;
        char *base = value ? c.kv.v : c.kv.k;
        if (CACHE == PC_BF16 && value) {
            *(uint4 *)(base + dst) = *(const uint4 *)(row + 16 * n);
            continue;
        }
        float y[E];
#pragma unroll
        for (uint32_t j = 0; j < E / 8; ++j) {
            float x[8];
            if (value) unpack<BF>(*(const uint4 *)(row + 2 * (E * n + 8 * j)), x);
            else turned_piece<BF, L, E != 8>(row, E * n + 8 * j, a.turn, a.turn.table + (uint64_t)pos[i] * a.turn.half, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[8 * j + e] = x[e];
        }
        if constexpr (CACHE == PC_FP4_E2M1) {
            uint32_t e;
            const uint4 w = to_e2m1<BF>(y, &e);
            *(uint4 *)(base + dst) = w;
            (value ? c.kv.v_exp : c.kv.k_exp)[dst / 16] = (uint8_t)e;
        } else if constexpr (CACHE == PC_FP8_E4M3) {
            const float s = (value ? c.kv.v_scale : c.kv.k_scale)[h];
            *(uint4 *)(base + dst) = make_uint4(to_e4m3(y[0], y[1], y[2], y[3], s), to_e4m3(y[4], y[5], y[6], y[7], s),
                                                to_e4m3(y[8], y[9], y[10], y[11], s), to_e4m3(y[12], y[13], y[14], y[15], s));
        } else {
            *(uint4 *)(base + dst) = pack<BF>(y);
        }
    }
}

// ---------------------------------------------------------------------- host

// Threads of a call for its queries up to which a thread takes one head; above, AT_ONCE of them (32 heads of 128 in
// bf16, one a thread and four: 64 rows 2.9 and 3.6 us, 512 rows 4.4 and 4.7, 1,024 rows 6.2 and 6.0, 4,096
// rows 19.6 and 16.3, 16,384 rows 63 and 51).
constexpr uint64_t ONE_HEAD = 1u << 18;
// A workgroup looks at 2,048 positions in the time that the others move half a megabyte; above
// these many rows each reports its own, and a launch before clears the word.
constexpr uint32_t ROWS_LOOKED_AT = 32768;

static Shape shape_of(const Turn &turn, Layout layout, uint32_t dim, uint32_t n_heads, uint64_t n_rows, bool in_place) {
    Shape g;
    const uint32_t rot = 2 * turn.half;
    if (layout == Layout::ANY) {
        g.turning = turn.half;
        g.units = turn.half + (in_place ? 0 : dim - rot);
    } else if (layout == Layout::HALVES) {
        g.turning = turn.half / 8;
        g.units = g.turning + (in_place ? 0 : (dim - rot) / 8);
    } else {
        g.turning = (rot + 7) / 8;
        g.units = in_place ? g.turning : dim / 8;
    }
    const bool few = n_rows * n_heads * g.units <= ONE_HEAD;
    g.apart = few ? n_heads : (n_heads + AT_ONCE - 1) / AT_ONCE;
    g.by_unit = fast_div(g.units);
    g.by_row = fast_div(g.units * g.apart);
    g.rows = 256 / g.by_row.d;
    g.rows = g.rows < 1 ? 1 : g.rows > GROUP_ROWS ? GROUP_ROWS : g.rows;
    return g;
}
static uint64_t groups_of(uint64_t rows, uint32_t each) { return (rows + each - 1) / each; }

template <bool BF, Layout L>
static pc_status append_layout(const AppendTurnedArgs &a, uint32_t cache, dim3 grid, hipStream_t st) {
    if (cache == PC_FP4_E2M1) PC_LAUNCH(K_KV_APPEND_TURNED, (append_turned_kernel<BF, L, PC_FP4_E2M1>), grid, dim3(256), 0, st, a);
    else if (cache == PC_FP8_E4M3) PC_LAUNCH(K_KV_APPEND_TURNED, (append_turned_kernel<BF, L, PC_FP8_E4M3>), grid, dim3(256), 0, st, a);
    else PC_LAUNCH(K_KV_APPEND_TURNED, (append_turned_kernel<BF, L, PC_BF16>), grid, dim3(256), 0, st, a);
    return PC_OK;
}
template <bool BF>
static pc_status append_type(const AppendTurnedArgs &a, Layout l, uint32_t cache, dim3 grid, hipStream_t st) {
    if (l == Layout::HALVES) return append_layout<BF, Layout::HALVES>(a, cache, grid, st);
    if (l == Layout::PAIRS) return append_layout<BF, Layout::PAIRS>(a, cache, grid, st);
    return append_layout<BF, Layout::ANY>(a, cache, grid, st);
}

pc_status append_turned(const Chunks &c, uint32_t cache_dtype, const Entries &k, const Entries &v, uint32_t dtype, const Turn &turn,
                        Layout layout, const Queries &q, int32_t *status, hipStream_t st) {
    AppendTurnedArgs a;
    a.c = c;
    a.k = (const char *)k.base;
    a.v = (const char *)v.base;
    a.k_row = k.row;
    a.k_head = k.head;
    a.v_row = v.row;
    a.v_head = v.head;
    a.turn = turn;
    a.q = q;
    a.status = status;
    a.by_head = fast_div((uint32_t)(bytes_of(cache_dtype, c.kv.dim) / 16));
    a.by_token = fast_div(a.by_head.d * c.kv.n_kv);
    a.rows = 128 / a.by_token.d;
    a.rows = a.rows < 1 ? 1 : a.rows > GROUP_ROWS ? GROUP_ROWS : a.rows;
    const uint64_t kv_groups = groups_of(c.n_rows, a.rows);
    uint64_t q_groups = 0;
    if (q.x) {
        a.g = shape_of(turn, layout, c.kv.dim, q.n_heads, c.n_rows, q.x == q.out);
        q_groups = groups_of(c.n_rows, a.g.rows);
    }
    if (!launch_fits(1 + kv_groups + q_groups, 256)) return PC_ERR_TOO_LARGE;
    a.groups = (uint32_t)kv_groups;
    a.cleared = turn.pos && c.n_rows > ROWS_LOOKED_AT;
    if (a.cleared) {
        const pc_status ok = fill_u32((uint32_t *)status, 0, 1, st);
        if (ok != PC_OK) return ok;
    }
    const dim3 grid((unsigned)(1 + kv_groups + q_groups));
    return dtype == PC_BF16 ? append_type<true>(a, layout, cache_dtype, grid, st) : append_type<false>(a, layout, cache_dtype, grid, st);
}

template <bool BF>
static pc_status rope_type(const Queries &q, const Turn &turn, const Shape &g, Layout l, uint32_t n_rows, int32_t *status, uint32_t cleared,
                           dim3 grid, hipStream_t st) {
    if (l == Layout::HALVES) PC_LAUNCH(K_ROPE, (rope_kernel<BF, Layout::HALVES>), grid, dim3(256), 0, st, q, turn, g, n_rows, status, cleared);
    else if (l == Layout::PAIRS) PC_LAUNCH(K_ROPE, (rope_kernel<BF, Layout::PAIRS>), grid, dim3(256), 0, st, q, turn, g, n_rows, status, cleared);
    else PC_LAUNCH(K_ROPE, (rope_kernel<BF, Layout::ANY>), grid, dim3(256), 0, st, q, turn, g, n_rows, status, cleared);
    return PC_OK;
}

// checks a rotation for heads of `dim` dimensions
static pc_status turn_of(const pc_rotation *r, uint32_t dim, uint32_t flags_allowed, Turn *turn, Layout *layout) {
    if (!r || !r->table || (uint64_t)(uintptr_t)r->table % 8) return PC_ERR_INVALID;
    if (r->rot_dim < 2 || r->rot_dim % 2 || r->rot_dim > dim || r->n_pos < 1 || r->flags & ~flags_allowed) return PC_ERR_INVALID;
    if (r->n_pos == PC_NONE) return PC_ERR_TOO_LARGE;
    *turn = Turn{(const float2 *)r->table, r->pos, r->n_pos, r->rot_dim / 2, r->flags & PC_ROPE_TRANSPOSE ? -1.f : 1.f};
    *layout = r->flags & PC_ROPE_INTERLEAVED ? Layout::PAIRS : r->rot_dim % 16 ? Layout::ANY : Layout::HALVES;
    return PC_OK;
}
static bool aligned(const void *p, uint64_t row, uint64_t head) { return ((uint64_t)(uintptr_t)p | row * 2 | head * 2) % 16 == 0; }

// whether the runs of an array that is written share no memory: the heads of a row in a block, or the rows of a head
static bool runs_apart(const Entries &x, uint64_t n_rows, uint64_t n_heads, uint64_t width) {
    if (n_rows < 2 || n_heads < 2) return (n_rows < 2 || x.row >= width) && (n_heads < 2 || x.head >= width);
    return x.head <= x.row ? x.head >= width && x.row >= (n_heads - 1) * x.head + width
                           : x.row >= width && x.head >= (n_rows - 1) * x.row + width;
}

// Whether two arrays of rows may share memory, the one of x_heads, the other of y_heads heads: known not to where the
// heads of a row make a block each and the blocks lie apart, or where heads of one stride lie in each other's gaps (each
// head's query, key and value beside each other), which more heads than there are cannot change.
static bool rows_overlap(Entries x, uint64_t x_heads, Entries y, uint64_t y_heads, uint64_t n_rows, uint64_t width) {
    const uint64_t x_bytes = (x_heads - 1) * x.head + width, y_bytes = (y_heads - 1) * y.head + width;
    if (!n_rows || !overlap(x.base, (n_rows - 1) * x.row + x_bytes, y.base, (n_rows - 1) * y.row + y_bytes)) return false;
    if (n_rows > 1 && x.row == y.row && x.row) {
        const uint64_t apart = (uint64_t)(uintptr_t)y.base - (uint64_t)(uintptr_t)x.base, back = 0 - apart;
        const uint64_t d = (int64_t)apart < 0 ? (x.row - back % x.row) % x.row : apart % x.row;
        if (d >= x_bytes && d + y_bytes <= x.row) return false;
    }
    if (x_heads < 2) x.head = y.head;   // the stride of one head is anything
    if (y_heads < 2) y.head = x.head;
    return entries_overlap(x, y, n_rows, x_heads < y_heads ? y_heads : x_heads, width);
}

}  // namespace pc

extern "C" {

pc_status pc_rope_table(const double *freq, uint32_t n_freq, uint64_t first, uint64_t n_pos, double magnitude, float *table, void *stream) {
    using namespace pc;
    if (!freq || n_freq < 1 || n_freq > PC_MAX_HEAD_DIM / 2 || !isfinite(magnitude)) return PC_ERR_INVALID;
    Frequencies f;
    for (uint32_t i = 0; i < PC_MAX_HEAD_DIM / 2; ++i) {
        f.f[i] = i < n_freq ? freq[i] : 0.0;
        if (!(fabs(f.f[i]) <= 65536.0)) return PC_ERR_INVALID;
    }
    if (n_pos > 0xFFFFFFFEull || first > 0xFFFFFFFEull || first + n_pos > 0xFFFFFFFEull) return PC_ERR_TOO_LARGE;
    if (n_pos && (!table || (uint64_t)(uintptr_t)table % 8)) return PC_ERR_INVALID;
    if (!n_pos) return PC_OK;
    const uint32_t together = 256 / n_freq;
    const uint64_t groups = groups_of(n_pos, together * POSITIONS);
    if (!launch_fits(groups, 256)) return PC_ERR_TOO_LARGE;
    PC_LAUNCH(K_ROPE_TABLE, rope_table_kernel, dim3((unsigned)groups), dim3(256), 0, (hipStream_t)stream, f, n_freq, together, (uint32_t)first,
              (uint32_t)n_pos, magnitude, (float2 *)table);
    return PC_OK;
}

size_t pc_rope_ws(void) { return pc::WS_HEADER; }

pc_status pc_rope(const pc_rotation *rotation, const void *x, uint64_t x_stride_row, uint64_t x_stride_head, void *out,
                  uint64_t out_stride_row, uint64_t out_stride_head, uint32_t dtype, uint32_t n_rows, uint32_t n_heads, uint32_t head_dim,
                  void *ws, size_t ws_bytes, void *stream) {
    using namespace pc;
    Turn turn;
    Layout layout;
    if (dtype != PC_BF16 && dtype != PC_F16) return PC_ERR_INVALID;
    if (head_dim < 8 || head_dim % 8 || head_dim > PC_MAX_HEAD_DIM || !n_heads || n_heads > PC_MAX_HEADS) return PC_ERR_INVALID;
    const pc_status ok = turn_of(rotation, head_dim, PC_ROPE_INTERLEAVED | PC_ROPE_TRANSPOSE, &turn, &layout);
    if (ok != PC_OK) return ok;
    if (n_rows >= 0x80000000u) return PC_ERR_TOO_LARGE;
    if ((n_rows && (!x || !out)) || !aligned(x, x_stride_row, x_stride_head) || !aligned(out, out_stride_row, out_stride_head))
        return PC_ERR_INVALID;
    if (!turn.pos && n_rows > turn.n_pos) return PC_ERR_INVALID;
    const Queries q{(const char *)x, (char *)out, x_stride_row * 2, x_stride_head * 2, out_stride_row * 2, out_stride_head * 2, n_heads};
    const Entries from{x, q.x_row, q.x_head}, to{out, q.o_row, q.o_head};
    const bool in_place = x == out && same_strides(from, to, n_rows, n_heads);
    const Shape g = shape_of(turn, layout, head_dim, n_heads, n_rows, in_place);
    const uint64_t groups = groups_of(n_rows, g.rows);
    const uint32_t cleared = turn.pos && n_rows > ROWS_LOOKED_AT;
    if (!launch_fits(groups + 1, 256)) return PC_ERR_TOO_LARGE;
    if (!ws || ws_bytes < pc_rope_ws()) return PC_ERR_WORKSPACE;
    if (!runs_apart(to, n_rows, n_heads, 2ull * head_dim)) return PC_ERR_INVALID;
    if (!in_place && entries_overlap(from, to, n_rows, n_heads, 2ull * head_dim)) return PC_ERR_INVALID;
    const hipStream_t st = (hipStream_t)stream;
    if (cleared) {
        const pc_status filled = fill_u32((uint32_t *)ws, 0, 1, st);
        if (filled != PC_OK) return filled;
    }
    const dim3 grid((unsigned)(groups + (cleared ? 0 : 1)));
    return dtype == PC_BF16 ? rope_type<true>(q, turn, g, layout, n_rows, (int32_t *)ws, cleared, grid, st)
                            : rope_type<false>(q, turn, g, layout, n_rows, (int32_t *)ws, cleared, grid, st);
}

size_t pc_kv_append_rope_ws(void) { return pc::WS_HEADER; }

pc_status pc_kv_append_rope(const pc_kv_cache *cache, const uint32_t *page_table, uint64_t table_stride, const uint32_t *kv_len,
                            const uint32_t *q_off, uint32_t n_seqs, uint32_t n_rows, uint32_t max_kv, const pc_rotation *rotation,
                            const void *k, uint64_t k_stride_row, uint64_t k_stride_head, const void *v, uint64_t v_stride_row,
                            uint64_t v_stride_head, const void *q, uint64_t q_stride_row, uint64_t q_stride_head, void *q_out,
                            uint64_t qo_stride_row, uint64_t qo_stride_head, uint32_t n_heads, uint32_t dtype, void *ws, size_t ws_bytes,
                            void *stream) {
    using namespace pc;
    Chunks c;
    const pc_status ok = kv_view(cache, &c.kv);
    if (ok != PC_OK) return ok;
    if (dtype != PC_BF16 && dtype != PC_F16) return PC_ERR_INVALID;
    if (cache->dtype != dtype && cache->dtype != PC_FP8_E4M3 && cache->dtype != PC_FP4_E2M1) return PC_ERR_INVALID;
    Turn turn;
    Layout layout;
    const pc_status fine = turn_of(rotation, c.kv.dim, PC_ROPE_INTERLEAVED, &turn, &layout);
    if (fine != PC_OK) return fine;
    if (n_seqs >= 0x80000000u || n_rows >= 0x80000000u || max_kv > 0x7FFF0000u) return PC_ERR_TOO_LARGE;
    if (max_kv > table_stride * c.kv.page) return PC_ERR_INVALID;
    if (!q_off || (n_seqs && (!kv_len || (max_kv && !page_table))) || (n_rows && (!k || !v))) return PC_ERR_INVALID;
    if (!aligned(k, k_stride_row, k_stride_head) || !aligned(v, v_stride_row, v_stride_head)) return PC_ERR_INVALID;
    if (n_seqs == 0 && n_rows) return PC_ERR_INVALID;
    if ((q != nullptr) != (q_out != nullptr)) return PC_ERR_INVALID;
    Queries queries{};
    if (q) {
        if (!n_heads || n_heads > PC_MAX_HEADS) return PC_ERR_INVALID;
        if (!aligned(q, q_stride_row, q_stride_head) || !aligned(q_out, qo_stride_row, qo_stride_head)) return PC_ERR_INVALID;
        queries = Queries{(const char *)q, (char *)q_out, q_stride_row * 2, q_stride_head * 2, qo_stride_row * 2, qo_stride_head * 2, n_heads};
        const uint64_t run = 2ull * c.kv.dim;
        const Entries from{q, queries.x_row, queries.x_head}, to{q_out, queries.o_row, queries.o_head};
        if (!runs_apart(to, n_rows, n_heads, run)) return PC_ERR_INVALID;
        if (!(q == q_out && same_strides(from, to, n_rows, n_heads)) && entries_overlap(from, to, n_rows, n_heads, run)) return PC_ERR_INVALID;
        // keys and values are read while queries are written
        if (rows_overlap(to, n_heads, Entries{k, k_stride_row * 2, k_stride_head * 2}, c.kv.n_kv, n_rows, run) ||
            rows_overlap(to, n_heads, Entries{v, v_stride_row * 2, v_stride_head * 2}, c.kv.n_kv, n_rows, run))
            return PC_ERR_INVALID;
    }
    if (!ws || ws_bytes < pc_kv_append_rope_ws()) return PC_ERR_WORKSPACE;
    c.table = page_table;
    c.kv_len = kv_len;
    c.q_off = q_off;
    c.table_stride = table_stride;
    c.n_seqs = n_seqs;
    c.n_rows = n_rows;
    c.max_kv = max_kv;
    return append_turned(c, cache->dtype, Entries{k, k_stride_row * 2, k_stride_head * 2}, Entries{v, v_stride_row * 2, v_stride_head * 2},
                         dtype, turn, layout, n_rows ? queries : Queries{}, (int32_t *)ws, (hipStream_t)stream);
}

}  // extern "C"
