"""Plain 64-bit forms of the position rotation and of 4-bit codes (numpy, no code of the library)."""
import numpy as np
import torch

GRID4 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BOUNDS = {torch.bfloat16: (1, 252), torch.float16: (104, 140)}   # of a scale's exponent byte, by the new tokens' type


def angles(n_pos, rot, base=10000.0, magnitude=1.0):
    """float32 [n_pos, rot / 2, 2]."""
    a = np.multiply.outer(np.arange(n_pos, dtype=np.float64), base ** (np.arange(0, rot, 2) / -rot))
    return torch.from_numpy((magnitude * np.stack([np.cos(a), np.sin(a)], -1)).astype(np.float32)).cuda()


def pair_of(rot, interleaved):
    """First and second dimension of every pair."""
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def turned(x, table, pos, interleaved, transpose=False):
    """x [row, head, dim] turned, in float64, and the sum of the magnitudes of its two products."""
    x, table = np.asarray(x, np.float64), table.cpu().numpy().astype(np.float64)[np.asarray(pos)][:, None]
    c, s = table[..., 0], table[..., 1] * (-1 if transpose else 1)
    a, b = pair_of(2 * table.shape[2], interleaved)
    y, size = x.copy(), np.abs(x)
    with np.errstate(invalid="ignore", over="ignore"):
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
        size[..., a] = np.abs(x[..., a] * c) + np.abs(x[..., b] * s)
        size[..., b] = np.abs(x[..., b] * c) + np.abs(x[..., a] * s)
    return y, size


def to_fp4(y, dtype):
    """What a 4-bit cache holds of float64 values [..., dim]: (values, codes, exponent bytes)."""
    y = np.asarray(y).astype(np.float32).astype(np.float64).reshape(*np.shape(y)[:-1], -1, 32)
    nan = np.isnan(y).any(-1)
    a = np.abs(np.where(np.isnan(y), 0, y))
    top = a.max(-1)
    lo, hi = BOUNDS[dtype]
    e = np.full(top.shape, hi, np.int64)
    for b in range(hi, lo - 1, -1):                          # the smallest power of two that leaves the largest below 7
        e = np.where(top < 7 * 2.0 ** (b - 127), b, e)
    q = np.minimum(a / 2.0 ** (e - 127)[..., None], 6)
    i = np.clip(np.searchsorted(GRID4, q), 1, 7)
    down, up = q - GRID4[i - 1], GRID4[i] - q
    code = np.where((up < down) | ((up == down) & (i % 2 == 0)), i, i - 1)
    value = np.copysign(GRID4[code] * 2.0 ** (e - 127)[..., None], y)
    value = np.where(nan[..., None], np.nan, value)
    return value.reshape(*value.shape[:-2], -1), code, np.where(nan, 255, e)


def pack_fp4(y, dtype):
    """Float values [..., dim] as torch bytes: codes [..., dim / 2] and exponents [..., dim / 32]."""
    value, code, e = to_fp4(y, dtype)
    code = code | np.where(np.signbit(np.asarray(y, np.float64).reshape(code.shape)), 8, 0)
    code = code.reshape(*code.shape[:-2], -1).astype(np.uint8)
    return torch.from_numpy(code[..., ::2] | code[..., 1::2] << 4), torch.from_numpy(e.astype(np.uint8))


def fp4_values(codes, exponents):
    """float64 [..., dim] that bytes stand for."""
    c, e = codes.cpu().view(torch.uint8).numpy(), exponents.cpu().view(torch.uint8).numpy().astype(np.float64)
    c = np.stack([c & 15, c >> 4], -1).reshape(*c.shape[:-1], -1)
    x = GRID4[c & 7] * np.where(c & 8, -1.0, 1.0)
    scale = np.where(e == 255, np.nan, 2.0 ** (e - 127))
    return (x.reshape(*e.shape, 32) * scale[..., None]).reshape(x.shape)
