"""The 8-bit cache's arithmetic in 64 bits on the CPU, from its definition: rows as e4m3 numbers with a power of two, and attention over
them.  No code shared with the library."""
import numpy as np

E_LO, E_HI = -110, 119

# e4m3 numbers by their byte: four bits of exponent (bias 7), three of mantissa, no infinities, NaN at 0x7F and 0xFF
_b = np.arange(256)
_e, _m = (_b >> 3) & 15, _b & 7
TABLE = np.where(_e > 0, np.ldexp(1 + _m / 8, _e - 7), np.ldexp(_m / 8, -6)) * np.where(_b & 128, -1, 1)
TABLE[[127, 255]] = np.nan


def bf16(x):
    """float32 array rounded to bf16 (finite values)."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)


def quantise(rows):
    """[..., D] numbers -> (bytes [..., D], exponents [...])."""
    x = np.asarray(rows, np.float64)
    finite = np.isfinite(x)
    most = np.where(finite, np.abs(x), 0.0).max(-1)
    e = np.full(most.shape, E_LO)
    for k in range(E_LO, E_HI):                                   # the least exponent that holds the row, by trying
        e = np.where((e == k) & (most > np.ldexp(448.0, k)), k + 1, e)
    y = np.clip(np.where(finite, x, 0.0) * np.ldexp(1.0, -e)[..., None], -448, 448)
    # nearest by the table's positive half: of two as near, the one with an even byte
    pos = TABLE[:127]
    at = np.searchsorted(pos, np.abs(y), side="left").clip(1, 126)
    lo, hi = pos[at - 1], pos[at]
    up = np.where(np.abs(y) - lo == hi - np.abs(y), at % 2 == 0, np.abs(y) - lo > hi - np.abs(y))
    byte = np.where(up, at, at - 1) | np.where(np.signbit(np.where(finite, x, 0.0)), 128, 0)
    return np.where(finite, byte, 127).astype(np.uint8), e


def values(byte, e):
    return TABLE[byte] * np.ldexp(1.0, np.asarray(e))[..., None]


def attend(q, k, v, prefix, scale):
    """q [N][Hq][D] at positions prefix + i over k, v [prefix + N][Hkv][D]: outputs, the weighted sizes sum p |v| and the largest sum
    |q| |k| * scale of a row, all [N][Hq][D] or [N][Hq]."""
    n, hq, d = q.shape
    g = hq // k.shape[1]
    out, size, reach = np.zeros((n, hq, d)), np.zeros((n, hq, d)), np.zeros((n, hq))
    for h in range(hq):
        kh, vh = k[:, h // g], v[:, h // g]
        s = scale * (q[:, h] @ kh.T)
        hidden = np.arange(kh.shape[0])[None, :] > prefix + np.arange(n)[:, None]
        s[hidden] = -np.inf
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        out[:, h], size[:, h] = p @ vh, p @ np.abs(vh)
        reach[:, h] = np.where(hidden, 0, scale * (np.abs(q[:, h]) @ np.abs(kh).T)).max(-1)
    return out, size, reach
