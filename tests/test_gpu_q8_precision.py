"""What attention over an 8-bit cache keeps of its softmax weights, against the 64-bit oracle (q8_oracle.py)."""
import numpy as np
import pytest
import torch

import q8_oracle as Q
from gpu_helpers import i32
from paper_2603_10342_amd import binding as B
from test_gpu_q8 import AG, DEV, TD, Side, decode, resume
from test_q8_dispatch import SHARED_CTX

pytestmark = pytest.mark.gpu


def two_opposite_keys(d, page, hkv, prefix, seed, batch=40):
    """Sessions that end in two keys whose scores differ by 2^-11 to 2^-10 and whose values are +1 and -1, behind one whose score is 0.875 higher
    and whose value is 0, and `prefix` keys of no weight: a row's output is the difference of two nearly equal weights of about 0.4, over their sum."""
    n = prefix + 3
    side = Side("bf16", d, page, hkv, [n] * batch, seed=seed)
    k, v = np.zeros((batch, n, hkv, d), np.float32), np.ones((batch, n, hkv, d), np.float32)
    k[:, :prefix, :, 2] = -4096.0
    k[:, prefix:, :, 0] = 1.0
    k[:, prefix, :, 0], v[:, prefix] = 1.875, 0.0
    k[:, prefix + 2, :, 1] = -Q.bf16(side.rng.uniform(2.0 ** -8, 2.0 ** -7, size=(batch, hkv)).astype(np.float32))
    v[:, prefix + 2] = -1.0
    side.append([n] * batch, k=k.reshape(-1, hkv, d), v=v.reshape(-1, hkv, d))
    return side


def opposite_query(batch, hq, d):
    q = np.zeros((batch, hq, d), np.float32)
    q[:, :, 0] = q[:, :, 2] = 8.0
    q[:, :, 1] = 1.0
    return q


# A relative error e of one weight is e 2^10 to e 2^11 of the result.  Allowed: the result's own rounding to bf16, 2^-8, and 2^-10 for fp32
# arithmetic (scores, exponentials and sums: a few 2^-24 of the weights, up to 2^-11 of the result).  A weight rounded to bf16, up to 2^-8 of
# itself, may take all of the result; as two bf16 terms 2^-6 of it.
LIMIT = 2.0 ** -8 + 2.0 ** -10


@pytest.mark.parametrize("max_ctx", [None, SHARED_CTX])           # one workgroup a pair, and shares
@pytest.mark.parametrize("prefix", [0, 70])
@pytest.mark.parametrize("d,page,hq,hkv", [(64, 64, 8, 2), (64, 16, 4, 4), (128, 32, 8, 2), (80, 32, 5, 1), (96, 16, 4, 2), (112, 16, 2, 1), (192, 16, 4, 2), (256, 16, 6, 2),
                                           (128, 64, 40, 2), (128, 16, 40, 2)])
def test_decode_keeps_its_softmax_weights_in_24_bits(d, page, hq, hkv, prefix, max_ctx):
    """All shapes of bf16 but 128 channels on pages of 16 with up to 16 heads a group."""
    side = two_opposite_keys(d, page, hkv, prefix, seed=61)
    q = opposite_query(40, hq, d)
    got = decode(side, q, hq, 0.125, max_ctx=max_ctx).double().cpu().numpy()
    for s in range(40):
        ref = Q.attend(q[s:s + 1], side.k[s], side.v[s], prefix + 2, 0.125)[0][0]
        assert (np.abs(got[s] - ref) <= LIMIT * np.abs(ref)).all(), (s, float((np.abs(got[s] - ref) / np.abs(ref)).max()))


@pytest.mark.parametrize("d,page,prefix", [(128, 16, 0), (128, 16, 70), (64, 32, 70), (256, 16, 0)])
def test_fp32_rows_over_a_cache_that_bf16_rows_wrote_keep_24_bits_in_every_call(d, page, prefix):
    """The pools hold the same numbers whatever the activations' type: a caller who wants all bits of the weights says so by passing fp32 rows."""
    hq, hkv, batch = 4, 2, 40
    side = two_opposite_keys(d, page, hkv, prefix, seed=62)
    side.dtype, side.cache.dtype = "f32", AG["f32"]
    q = opposite_query(batch, hq, d)
    new, cu, old = i32([1] * batch), i32(np.arange(batch + 1)), i32([prefix + 2] * batch)
    out = torch.full((batch, hq, d), float("nan"), dtype=TD["f32"], device=DEV)
    B.ag_attn_resume_q8(side.cache, side.dev(q), out, side.bt_dev, old, new, cu, batch, 1, prefix + 3, hq, 0.125)
    torch.cuda.synchronize()
    for what, got in (("resume", out), ("decode", decode(side, q, hq, 0.125))):
        got = got.double().cpu().numpy()
        for s in range(batch):
            ref = Q.attend(q[s:s + 1], side.k[s], side.v[s], prefix + 2, 0.125)[0][0]
            assert (np.abs(got[s] - ref) <= 2.0 ** -10 * np.abs(ref)).all(), (what, s)


@pytest.fixture(scope="module")
def few_cus():
    """A stream of eight CUs, on which small batches are many workgroups."""
    stream = B.ag_stream_create_cumask(B.ag_cumask_build(256, 8, 0, 1))
    yield stream
    torch.cuda.synchronize()
    B.ag_stream_destroy(stream)


# Every token of a session has the same value row c: whatever the weights are, the output is c, if they are divided by the sum of what they were
# multiplied as.  c has four significant bits, half a step of bf16 away from rounding to anything else, 2^-9 of itself at least; the sums'
# roundings are (n + 16) 2^-23.  The weights of all keys but one are the same number, so that what rounds it does not average out: up to 2^-8.
@pytest.mark.parametrize("d,page", [(128, 16), (64, 32), (256, 16), (96, 32)])
def test_equal_values_come_out_as_they_are(few_cus, d, page):
    hq, hkv, new = 8, 2, np.array([100, 64, 1, 33])
    n = np.array([700, 300, 130, 33])
    side = Side("bf16", d, page, hkv, n, seed=d)
    t = int(n.sum())
    k, c = np.zeros((t, hkv, d), np.float32), np.zeros((4, hkv, d), np.float32)
    for s, at in enumerate(np.cumsum(n) - n):
        k[at + 1:at + n[s], :, 0] = -1.0
        c[s] = (8 + side.rng.integers(0, 8, (hkv, d))) / 8 * np.exp2(side.rng.integers(-3, 4, (hkv, d))) * side.rng.choice([-1, 1], (hkv, d))
    side.append(n, k=k, v=np.repeat(c, n, 0))
    want = np.repeat(c, hq // hkv, 1)                             # [session][query head][channel]
    q = np.zeros((int(new.sum()), hq, d), np.float32)
    q[:, :, 0] = Q.bf16(side.rng.uniform(0.5, 16, q.shape[:2]).astype(np.float32))       # weights e^(-q / 8): 0.14 to 0.94
    for stream in (None, few_cus):
        got = resume(side, q, new, hq, 0.125, stream=stream).double().cpu().numpy()
        assert np.array_equal(got, np.repeat(want, new, 0)), stream
    for max_ctx in (None, SHARED_CTX):
        for step in range(8):
            got = decode(side, q[4 * step:4 * step + 4], hq, 0.125, max_ctx=max_ctx).double().cpu().numpy()
            assert np.array_equal(got, want), max_ctx


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_the_ends_of_the_documented_range_change_no_bit(few_cus, dtype, d):
    """Queries and keys raised together, or lowered, with a scale that takes it back: the largest scores are 2^125 (d 256: entries up to 2^2.4, so
    2^(112 + 4.8 + 8)) before the scale and as ever behind it.  Values at their ends.  Every rounding is relative: the same bits."""
    lens, new, hq, hkv, scale = [300, 77], [120, 77], 8, 2, d ** -0.5 / 4
    outs = []
    for kp, qp, pv in ((0, 0, 0), (56, 56, 77), (77, 35, -57), (-30, -25, 70), (-57, 0, 0)):
        side = Side(dtype, d, 16, hkv, lens, seed=3)
        old = [n - m for n, m in zip(lens, new)]
        for n in (old, new):
            k, v = (side.draw(sum(n), hkv, d).clip(-5, 5) for _ in range(2))
            side.append(n, k=np.ldexp(k, kp).astype(np.float32), v=np.ldexp(v, pv).astype(np.float32))
        q, s = np.ldexp(side.draw(sum(new), hq, d).clip(-5, 5), qp), float(np.ldexp(scale, -kp - qp))
        got = [resume(side, q, new, hq, s), resume(side, q, new, hq, s, stream=few_cus)]
        got += [decode(side, q[:2], hq, s), decode(side, q[:2], hq, s, max_ctx=SHARED_CTX)]
        outs.append([np.ldexp(x.double().cpu().numpy(), -pv) for x in got])
    for other in outs[1:]:
        for x, y in zip(outs[0], other):
            assert np.isfinite(x).all() and np.array_equal(x, y)
