"""The norm that q8_bounds.py allows is one that correct arithmetic keeps and that an output with keys left out does not."""
import numpy as np
import pytest

import q8_bounds
import q8_oracle as Q


def draw(n, seed, d=128, hq=8, hkv=2):
    rng = np.random.default_rng(seed)
    k, v = (Q.values(*Q.quantise(rng.standard_normal((n, hkv, d)) * np.exp2(rng.integers(-2, 3, (n, hkv, 1)) if i else 0))) for i in range(2))
    return Q.bf16(rng.standard_normal((1, hq, d)).astype(np.float32)).astype(np.float64), k, v


def rounded(q, k, v, scale, weights):
    """Attention as bf16 rows have it: weights rounded or not, output rounded."""
    hq, g = q.shape[1], q.shape[1] // k.shape[1]
    out = np.zeros(q.shape)
    for h in range(hq):
        s = scale * (q[:, h] @ k[:, h // g].T)
        p = np.exp(s - s.max())
        if weights:
            p = Q.bf16(p.astype(np.float32)).astype(np.float64)
        out[:, h] = p @ v[:, h // g] / p.sum()
    return Q.bf16(out.astype(np.float32)).astype(np.float64)


@pytest.mark.parametrize("n", [1, 3, 64, 700, 4097, 20000])
def test_correct_roundings_are_allowed_and_missing_keys_are_not(n):
    scale = 0.09
    for seed in range(2):
        q, k, v = draw(n, seed)
        out, spread = q8_bounds.attend(q, k, v, n - 1, scale)
        assert np.allclose(out, Q.attend(q, k, v, n - 1, scale)[0], rtol=0, atol=1e-12)
        for weights in (False, True):
            most = q8_bounds.norm_allowed("bf16", weights, out, spread)
            assert np.linalg.norm(rounded(q, k, v, scale, weights) - out) <= most
            if n < 700:
                continue
            # a step of 64 tokens, a wave's quarter of a segment, a segment, left out or taken twice
            for first, count in ((0, 64), (n // 2, 64), (n - 64, 64), (n // 3, 128), (n // 4, 512 if n > 1000 else 128)):
                keep = np.r_[0:first, first + count:n]
                less = q8_bounds.attend(q, k[keep], v[keep], len(keep) - 1, scale)[0]
                twice = np.r_[0:n, first:first + count]
                more = q8_bounds.attend(q, k[twice], v[twice], len(twice) - 1, scale)[0]
                assert min(np.linalg.norm(x - out) for x in (less, more)) > 3 * most, (n, first, count)
