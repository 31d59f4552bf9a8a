"""Plain 64-bit forms of the operators over a paged cache (numpy, no code of the
library), and the error bounds that their tests use.

Bounds.  u is the unit roundoff of the output type (2^-8 for bfloat16, 2^-11 for
float16).  A score is a sum of d products accumulated in 32 bits: it is off by at most
(d + 8) 2^-24 times the sum of their magnitudes, plus 2^-22 of itself for the scaling
and the base-2 exponential; call the largest such error of a row e.  Then every weight
is off by a factor of at most 1 + 3 e + 2^-20 against the exact softmax; its rounding to the output
type for the product with v adds a factor 1 + u, the sums in 32 bits 2^-20, and the
result's own rounding u times its magnitude:
    |out - exact| <= u |exact| + (u + 3 e + 2^-19) sum p |v| (+ float16: weights
                     under 2^-29 of the largest lose up to 2^-40 of it each)
    |lse - exact| <= e + 2^-21 (1 + |exact|)
    |weight - exact| <= (3 e + 2^-19 (1 + |lse|)) times the exact sum, + 2^-22 weight
"""
import numpy as np
import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def cache_values(cache_k, cache_v, k_scale, v_scale):
    """What the cache holds, float64 [page, head, slot, dim]."""
    k, v = cache_k.detach().cpu().float().double().numpy(), cache_v.detach().cpu().float().double().numpy()
    if k_scale is not None:
        k = k * k_scale.cpu().double().numpy()[None, :, None, None]
        v = v * v_scale.cpu().double().numpy()[None, :, None, None]
    return k, v


def gather(x, table, n, page):
    """Slots 0 .. n - 1 of one sequence: [head, slot, dim]."""
    ids = table[:(n + page - 1) // page].astype(np.int64)
    y = x[ids].transpose(1, 0, 2, 3).reshape(x.shape[1], -1, x.shape[3])
    return y[:, :n]


def attention(q, k, v, table, kv_len, q_off, scale, causal, window, weight=None, dtype=torch.bfloat16):
    """(out, lse, weight) in 64 bits and the bounds of their errors.  q [rows, heads, dim];
    k, v [page, kv head, slot, dim] float64."""
    q = q.detach().cpu().float().double().numpy()
    rows, heads, dim = q.shape
    page, kvh = k.shape[2], k.shape[1]
    group = heads // kvh
    out, lse = np.zeros_like(q), np.full((rows, heads), -np.inf)
    out_tol, lse_tol = np.zeros_like(q), np.zeros((rows, heads))
    w = None if weight is None else weight.detach().cpu().double().numpy().copy()
    w_tol = None if weight is None else 2.0 ** -22 * np.abs(w)
    u = UNIT[dtype]
    for s in range(len(kv_len)):
        a, b, n = int(q_off[s]), int(q_off[s + 1]), int(kv_len[s])
        if w is not None:
            w[s, :, n:] = 0
        if a == b or n == 0:
            continue
        keys, vals = gather(k, table[s], n, page), gather(v, table[s], n, page)
        pos = n - (b - a) + np.arange(b - a)
        j = np.arange(n)
        see = np.ones((b - a, n), bool)
        if causal:
            see &= j[None] <= pos[:, None]
        if window:
            see &= j[None] > pos[:, None] - window
        for e in range(heads):
            h = e // group
            with np.errstate(invalid="ignore"):
                z = np.where(see, scale * (q[a:b, e] @ keys[h].T), -np.inf)
                size = np.where(see, abs(scale) * (np.abs(q[a:b, e]) @ np.abs(keys[h].T)), 0)
            top = z.max(1)
            some = see.any(1)
            ref = np.where(some, top, 0.0)
            with np.errstate(invalid="ignore", divide="ignore"):
                p = np.exp(z - ref[:, None])
                total = p.sum(1)
                p = np.where(see, p / np.where(some, total, 1)[:, None], 0)
                lse[a:b, e] = np.where(some, ref + np.log(total), -np.inf)
            for i in range(b - a):        # row by row: what a row does not see must not reach it
                out[a + i, e] = p[i, see[i]] @ vals[h][see[i]]
            err = np.nan_to_num((dim + 8) * 2.0 ** -24 * size + 2.0 ** -22 * np.abs(np.where(see, z, 0))).max(1)
            mass = np.stack([p[i, see[i]] @ np.abs(vals[h][see[i]]) for i in range(b - a)])
            out_tol[a:b, e] = u * np.abs(out[a:b, e]) + (u + 3 * err + 2.0 ** -19)[:, None] * mass
            if dtype == torch.float16:
                # weights below the normal range, and results in the format's subnormal range
                out_tol[a:b, e] += n * 2.0 ** -39 * np.abs(np.nan_to_num(vals[h])).max() + 2.0 ** -24
            with np.errstate(invalid="ignore"):
                lse_tol[a:b, e] = err + 2.0 ** -21 * (1 + np.abs(lse[a:b, e]))
            if w is not None:
                l = np.abs(np.where(some, lse[a:b, e], 0))
                w[s, h, :n] += p.sum(0)
                w_tol[s, h, :n] += ((3 * err + 2.0 ** -19 * (1 + l))[:, None] * p).sum(0)
    return (out, lse, w), (out_tol, lse_tol, w_tol)


def evict(weight, kv_len, budget, recent):
    """(kept, their weights, new lengths): the definition, one slot after the other."""
    n_seqs, kvh, _ = weight.shape
    kept = np.full((n_seqs, kvh, budget), -1, np.int64)
    moved = np.zeros((n_seqs, kvh, budget), np.float32)
    new_len = np.minimum(kv_len, budget)
    for s in range(n_seqs):
        n, m = int(kv_len[s]), int(new_len[s])
        late = min(recent, m)
        for h in range(kvh):
            w = weight[s, h, :n - late]
            # NaN first, then large to small, equal ones by slot
            order = sorted(range(n - late), key=lambda j: (not np.isnan(w[j]), -w[j] if not np.isnan(w[j]) else 0, j))
            keep = sorted(order[:m - late]) + list(range(n - late, n))
            kept[s, h, :m] = keep
            moved[s, h, :m] = weight[s, h, keep]
    return kept, moved, new_len


def nearest_e4m3(x):
    """float64 -> the nearest value of the 8-bit grid (4 exponent, 3 fraction bits, largest
    448), ties to the even code; NaN stays NaN."""
    grid = [0.0]
    for e in range(0, 16):
        for f in range(8):
            if e == 15 and f == 7:
                continue
            grid.append((f / 8) * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
    grid = np.array(sorted(set(grid)))        # code order: index parity is the code's last bit
    a = np.minimum(np.abs(x), 448.0)
    i = np.searchsorted(grid, a)
    i = np.clip(i, 1, grid.size - 1)
    lo, hi = grid[i - 1], grid[i]
    up = (hi - a < a - lo) | ((hi - a == a - lo) & (i % 2 == 0))
    return np.where(np.isnan(x), np.nan, np.copysign(np.where(up, hi, lo), x))
