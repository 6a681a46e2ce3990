"""Rotary positions and attention over latent rows in 64 bits on the CPU, from their definitions.  No code shared with the library."""
import math
from fractions import Fraction

import numpy as np

HALF_STEP = 2.0 ** -8                                             # of bf16


def bf16(x):
    """float32 array rounded to bf16 (finite values)."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)


def turns(rot, base=10000.0, keep=None, factor=1.0):
    """keep: share of each pair that is not divided by factor."""
    t = np.array([base ** (-2.0 * i / rot) / (2 * math.pi) for i in range(rot // 2)])
    return t if keep is None else t * (keep + (1 - keep) / factor)


def angles(pos, t):
    """2 pi frac(pos t), [len(pos)][len(t)]: the products as rational numbers, so that whole turns go exactly."""
    out = np.empty((len(pos), len(t)))
    for i, p in enumerate(pos):
        for j, x in enumerate(t):
            f = Fraction(int(p)) * Fraction(float(x))
            out[i, j] = float(f - round(f)) * 2 * math.pi
    return out


def pairs_of(rot, layout):
    i = np.arange(rot // 2)
    return (i, i + rot // 2) if layout == "halves" else (2 * i, 2 * i + 1)


def rotate(x, pos, t, layout, magnitude=1.0, transposed=False):
    """x [T][...][d]: rotated rows, and |a| + |b| of each channel's pair (0 where nothing turns)."""
    x = np.asarray(x, np.float64)
    a, b = pairs_of(2 * len(t), layout)
    th = angles(pos, t).reshape(len(pos), *[1] * (x.ndim - 2), len(t)) * (-1 if transposed else 1)
    y, size = x.copy(), np.zeros_like(x)
    y[..., a] = magnitude * (x[..., a] * np.cos(th) - x[..., b] * np.sin(th))
    y[..., b] = magnitude * (x[..., b] * np.cos(th) + x[..., a] * np.sin(th))
    size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y, size


def rotation_allowed(y, size, dtype, magnitude=1.0):
    """Cosine and sine are rounded to fp32, one of the two products is, and the sum is: 3 roundings of m (|a| + |b|) at most, and 64-bit arithmetic's own
    (2^-33 of the angle).  Then the result is rounded to its type.  Channels that stay are exact."""
    return 3.01 * 2.0 ** -24 * magnitude * size + np.where(size > 0, (HALF_STEP if dtype == "bf16" else 0) * np.abs(y), 0)


def attend(q, rows, lat, prefix, scale):
    """q [N][H][W] at positions prefix + i over rows [prefix + N][W]: outputs [N][H][lat], sum p |v|, sum (p (v - o))^2, and the largest sum |q| |k| scale."""
    n, h, w = q.shape
    v = rows[:, :lat]
    s = scale * (q.reshape(n * h, w) @ rows.T).reshape(n, h, -1)
    hidden = np.broadcast_to(np.arange(len(rows))[None, None] > prefix + np.arange(n)[:, None, None], s.shape)
    reach = np.where(hidden, 0, scale * (np.abs(q).reshape(n * h, w) @ np.abs(rows).T).reshape(n, h, -1)).max(-1)
    s = np.where(hidden, -np.inf, s)
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    f = p.reshape(n * h, -1)
    o, size, sq, sv = (x.reshape(n, h, lat) for x in (f @ v, f @ np.abs(v), f ** 2 @ v ** 2, f ** 2 @ v))
    spread = (sq - 2 * o * sv + o ** 2 * (p ** 2).sum(-1, keepdims=True)).clip(0)
    return o, size, spread, reach


def elementwise(o, size, reach, w, n):
    """How far an output may be off.  Weights are rounded to bf16, 2^-8 of themselves, and summed as rounded: 2 * 2^-8 sum p |v|.  Scores are w products added up in
    fp32, and scaled: w + 2 roundings of 2^-24 reach (taken twice, with the factor's own), in weight and sum.  Sums over n keys in fp32, and exp2, a merge of
    pieces: (n + 16) 2^-24, numerator and denominator.  The output is rounded once."""
    return HALF_STEP * np.abs(o) + size * (2 * HALF_STEP + 2 * (w + 4) * 2.0 ** -24 * reach[..., None] + 2 * (n + 16) * 2.0 ** -24) + 1e-30


def norm_allowed(o, spread):
    """Of all errors together.  A rounding to bf16 is off by a number spread evenly over half a step to either side: its square is (2^-8 x)^2 / 3 at most on average, for
    the output, and for the weights, whose errors leave sum p e (v - o).  Both are upper ends.  fp32 arithmetic: 6e-6 of the norm (2^-24 sqrt(576) of scores of size 3, twice)."""
    return HALF_STEP * np.sqrt(((o ** 2).sum() + spread.sum()) / 3) + 6e-6 * np.linalg.norm(o)
