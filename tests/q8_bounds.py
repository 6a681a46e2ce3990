"""How far the norm of attention's errors over an 8-bit cache may be, from the 64-bit oracle's own quantities, tight enough that a key left out shows.

An output rounded to bf16 is off by a number that is spread evenly over half a step to either side, 2^-8 of the output at most: its square is
(2^-8 o)^2 / 3 at most on average.  Weights rounded to bf16, and summed as rounded, leave sum p_j e_j (v_j - o), with e_j as evenly spread and
independent: sum (2^-8 p_j (v_j - o))^2 / 3 on average.  Both are upper ends (a number just above a power of two; on average half steps are 0.72 of that), so that
over thousands of outputs the sums of squares lie well below.  fp32 arithmetic adds what test_gpu_q8.py allows fp32 rows: 6e-6 of the norm.
Weights in 24 bits (fp32 rows; bf16 decode where rounds() is false) add nothing to that."""
import numpy as np

HALF_STEP = 2.0 ** -8


def rounds(call, d, page, hq, hkv):
    """Whether bf16 rows round their weights (ag_q8.h)."""
    return call != "decode" or (d == 128 and page == 16 and hq <= 16 * hkv)


def attend(q, k, v, prefix, scale):
    """As q8_oracle.attend: outputs, and sum (p (v - o))^2, both [N][Hq][D]."""
    n, hq, d = q.shape
    g = hq // k.shape[1]
    out, spread = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    for h in range(hq):
        kh, vh = k[:, h // g], v[:, h // g]
        s = scale * (q[:, h] @ kh.T)
        s[np.arange(kh.shape[0])[None, :] > prefix + np.arange(n)[:, None]] = -np.inf
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        o = out[:, h] = p @ vh
        spread[:, h] = (p ** 2 @ vh ** 2 - 2 * o * (p ** 2 @ vh) + o ** 2 * (p ** 2).sum(-1, keepdims=True)).clip(0)
    return out, spread


def norm_allowed(dtype, rounded_weights, out, spread):
    of_arithmetic = 6e-6 * np.linalg.norm(out)
    if dtype == "f32":
        return of_arithmetic
    return HALF_STEP * np.sqrt(((out ** 2).sum() + (spread.sum() if rounded_weights else 0)) / 3) + of_arithmetic
