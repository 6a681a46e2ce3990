"""Attention over an 8-bit cache against the oracle in the norm, tight enough that a step of keys left out shows (q8_bounds.py; test_q8_bounds.py
shows that on the CPU): contexts of many partials, and every kernel at ordinary sizes."""
import numpy as np
import pytest
import torch

import q8_bounds
from test_gpu_q8 import Side, decode, few_cus, resume  # noqa: F401 (a fixture)
from test_q8_dispatch import FOUR_LENS, SHARED_CTX, TILED

pytestmark = pytest.mark.gpu


def check(side, call, page, hq, got, q, prefix, k, v, scale, what):
    """One session's outputs [N][Hq][D]: finite, and their errors' squares and those allowed."""
    out, spread = q8_bounds.attend(q, k, v, prefix, scale)
    assert np.isfinite(got).all(), what
    return np.linalg.norm(got - out), q8_bounds.norm_allowed(side.dtype, q8_bounds.rounds(call, side.d, page, hq, side.hkv), out, spread)


def check_all(found, what):
    err, most = (np.sqrt(sum(x[i] ** 2 for x in found)) for i in range(2))
    assert err <= most, (what, err / most)


# Up to 40 partials a pair: five rounds of the merge's eight behind the first four; 4097 tokens end one token into a step.
@pytest.mark.parametrize("dtype,d,page,hq,hkv", [("bf16", 128, 16, 8, 2), ("bf16", 128, 16, 40, 2), ("bf16", 64, 32, 8, 2), ("bf16", 256, 16, 2, 1), ("f32", 128, 16, 8, 2),
                                                 ("f32", 80, 64, 4, 1)])
def test_decode_of_long_contexts(few_cus, dtype, d, page, hq, hkv):  # noqa: F811
    side = Side(dtype, d, page, hkv, [20000, 9000], seed=d)
    side.append([20000, 9000])
    q = side.draw(2, hq, d)
    scale = d ** -0.5
    for ctx, stream in (([20000, 9000], None), ([4097, 0], None), ([20000, 33], None), ([1, 8999], few_cus)):
        got = decode(side, q, hq, scale, ctx=ctx, max_ctx=20000, stream=stream)
        again = decode(side, q, hq, scale, ctx=ctx, max_ctx=20000, stream=stream, ws_fill=3.0)
        assert torch.equal(got.view(torch.uint8), again.view(torch.uint8))
        got = got.double().cpu().numpy()
        found = []
        for s, n in enumerate(ctx):
            if n == 0:
                assert not got[s].any()
            else:
                found.append(check(side, "decode", page, hq, got[s:s + 1], q[s:s + 1], n - 1, side.k[s][:n], side.v[s][:n], scale, (ctx, s)))
                check_all(found[-1:], (ctx, s))


SHAPES = [(128, 16, 16, 2), (128, 64, 16, 2), (64, 16, 16, 2), (48, 128, 16, 2), (96, 32, 16, 2), (112, 16, 16, 2), (192, 16, 16, 2), (208, 256, 16, 2), (256, 16, 16, 2)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page,hq,hkv", SHAPES)
def test_decode_of_ordinary_contexts(dtype, d, page, hq, hkv):
    ctx = [1100, 700, 64, 1, 333, 897]
    side = Side(dtype, d, page, hkv, ctx, seed=d + 1)
    side.append(ctx)
    q, scale = side.draw(len(ctx), hq, d), d ** -0.5
    for bound in (None, SHARED_CTX):
        got = decode(side, q, hq, scale, max_ctx=bound).double().cpu().numpy()
        found = [check(side, "decode", page, hq, got[s:s + 1], q[s:s + 1], n - 1, side.k[s], side.v[s], scale, s) for s, n in enumerate(ctx)]
        check_all(found, (d, page, bound))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page,hq,hkv", SHAPES)
@pytest.mark.parametrize("lens", ["ragged", "prompts", "long", "four"])
def test_prefill(few_cus, dtype, d, page, hq, hkv, lens):  # noqa: F811
    """By few rows on the whole device, and on eight CUs by whole tiles (fp32: by few rows' four waves)."""
    prefix, new = (np.array(x) for x in {**TILED, "four": FOUR_LENS}[lens])
    side = Side(dtype, d, page, hkv, prefix + new, seed=d + 2)
    if prefix.any():
        side.append(prefix)
    side.append(new)
    q, scale = side.draw(int(new.sum()), hq, d), d ** -0.5
    for stream in (None, few_cus):
        got, at, found = resume(side, q, new, hq, scale, stream=stream).double().cpu().numpy(), 0, []
        for s, n in enumerate(new):
            if n:
                found.append(check(side, "resume", page, hq, got[at:at + n], q[at:at + n], int(prefix[s]), side.k[s], side.v[s], scale, s))
            at += n
        check_all(found, (d, page, lens, stream is not None))
