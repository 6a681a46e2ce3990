"""Calls over an 8-bit cache that its header allows: bounds that are no session's, batches in which nothing is new, queries that are not finite, unused
table entries that name no page, decodes and chunks in one batch."""
import numpy as np
import pytest
import torch

from gpu_helpers import i32
from paper_2603_10342_amd import binding as B
from test_gpu_q8 import AG, DEV, TD, Side, check, check_decode, check_resume, decode, few_cus, resume  # noqa: F401 (a fixture)
from test_q8_dispatch import SHARED_CTX

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(128, 16), (64, 64), (256, 32)])
@pytest.mark.parametrize("sessions", [5, 70])
def test_bounds_that_no_session_reaches(few_cus, dtype, d, page, sessions):  # noqa: F811
    """As a captured call has them: max_new, max_ctx and total_new for more than there is; table entries that no token uses are far outside the pool."""
    hq, hkv, rng = 4, 2, np.random.default_rng(d)
    prefix, new = rng.integers(0, 90, sessions), rng.integers(0, 12 if sessions > 5 else 80, sessions)
    new[1] = 0
    side = Side(dtype, d, page, hkv, prefix + new, seed=d)
    side.append(prefix)
    side.append(new)
    n = side.lens()
    pages, bound = side.bt.shape[1] + 7, int(new.sum()) + 33
    bt = np.full((sessions, pages), 1 << 30, np.int32)
    for s in range(sessions):
        used = -(-n[s] // page)
        bt[s, :used] = side.bt[s, :used]
    bt, max_ctx, scale = i32(bt), pages * page, d ** -0.5
    q = side.draw(bound, hq, d)
    qd, q1 = side.dev(q), side.dev(q[:sessions])
    lens, cu, old, ctx = i32(new), i32(np.concatenate([[0], np.cumsum(new)])), i32(prefix), i32(n)
    ws = torch.full((B.ag_attn_decode_q8_workspace_bytes(sessions, hq, d, SHARED_CTX) // 4,), float("nan"), device=DEV)
    wide = i32(np.pad(bt.cpu().numpy(), ((0, 0), (0, SHARED_CTX // page)), constant_values=1 << 30))
    for stream in (None, few_cus):
        out = torch.full((bound, hq, d), 5.0, dtype=TD[dtype], device=DEV)
        torch.cuda.synchronize()
        B.ag_attn_resume_q8(side.cache, qd, out, bt, old, lens, cu, bound, min(bound, max_ctx), max_ctx, hq, scale, stream)
        torch.cuda.synchronize()
        assert bool((out[int(new.sum()):] == 5.0).all())
        check_resume(side, q, out[:int(new.sum())], new, scale, (d, page, sessions))
        for table, most in ((bt, max_ctx), (wide, SHARED_CTX)):
            one = torch.full((sessions, hq, d), 5.0, dtype=TD[dtype], device=DEV)
            torch.cuda.synchronize()
            B.ag_attn_decode_q8(side.cache, q1, one, table, ctx, most, hq, scale, ws, stream)
            torch.cuda.synchronize()
            check_decode(side, q[:sessions], one, scale, (d, page, sessions, most))
    rows = [torch.full((bound, hkv, d), 5.0, dtype=TD[dtype], device=DEV) for _ in range(2)]
    B.ag_kv_read_q8(side.cache, *rows, bt, old, lens, cu, bound)
    torch.cuda.synchronize()
    for got, want in zip(rows, (side.k, side.v)):
        assert np.array_equal(got[:int(new.sum())].double().cpu().numpy(), np.concatenate([w[p:] for w, p in zip(want, prefix)]))
        assert bool((got[int(new.sum()):] == 5.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nothing_new_in_a_batch_writes_nothing(few_cus, dtype):  # noqa: F811
    side = Side(dtype, 128, 16, 2, [40, 7], seed=1, fill=0x21)
    side.append([40, 7])
    none, cu, old = i32([0, 0]), i32([0, 0, 0]), i32([40, 7])
    before = [x.clone() for x in (side.cache.k_pool, side.cache.v_pool, side.cache.exps)]
    rows = [torch.full((9, 2, 128), 5.0, dtype=TD[dtype], device=DEV) for _ in range(2)]
    q, out = (torch.full((9, 4, 128), 5.0, dtype=TD[dtype], device=DEV) for _ in range(2))
    for stream in (None, few_cus):
        torch.cuda.synchronize()
        B.ag_kv_append_q8(side.cache, *rows, side.bt_dev, old, none, cu, 9, stream)
        B.ag_kv_read_q8(side.cache, *rows, side.bt_dev, old, none, cu, 9, stream)
        B.ag_attn_resume_q8(side.cache, q, out, side.bt_dev, old, none, cu, 9, 9, 40, 4, 0.1, stream)
        B.ag_attn_prefill_q8(side.cache, q, out, side.bt_dev, none, cu, 9, 9, 4, 0.1, stream)
        torch.cuda.synchronize()
        assert all(bool((x == 5.0).all()) for x in (*rows, out))
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(before, (side.cache.k_pool, side.cache.v_pool, side.cache.exps)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(128, 16), (64, 32), (256, 16)])
def test_queries_that_are_not_finite_stay_in_their_rows(few_cus, dtype, d, page):  # noqa: F811
    """A NaN or an infinity in a query of one head: that row of that head is NaN, every other as ever."""
    hq, hkv, prefix, new, scale = 8, 2, np.array([300, 0]), np.array([70, 130]), d ** -0.5
    side = Side(dtype, d, page, hkv, prefix + new, seed=d)
    side.append(prefix)
    side.append(new)
    q = side.draw(int(new.sum()), hq, d)
    bad = [(3, 2, 5, np.nan), (69, 7, 1, np.inf), (70, 0, 0, np.nan), (110, 5, d - 1, -np.inf), (199, 4, 9, np.nan)]
    with_bad, clean = q.copy(), np.ones(q.shape[:2], bool)
    for row, head, ch, x in bad:
        with_bad[row, head, ch] = x
        clean[row, head] = False
    for stream in (None, few_cus):
        got, at = resume(side, with_bad, new, hq, scale, stream=stream).double().cpu().numpy(), 0
        assert np.array_equal(np.isnan(got).all(-1), ~clean) and np.array_equal(np.isnan(got).any(-1), ~clean)
        good = resume(side, q, new, hq, scale, stream=stream).double().cpu().numpy()
        for s, n in enumerate(new):
            o = np.where(clean[at:at + n, :, None], got[at:at + n], good[at:at + n])
            check(dtype, o, q[at:at + n], side.k[s], side.v[s], int(prefix[s]), scale, (d, s))
            at += n
    for max_ctx in (None, SHARED_CTX):
        one = decode(side, with_bad[[3, 70]], hq, scale, max_ctx=max_ctx).double().cpu().numpy()
        assert np.array_equal(np.isnan(one).all(-1), ~clean[[3, 70]]) and np.array_equal(np.isnan(one).any(-1), ~clean[[3, 70]])
        ok = decode(side, q[[3, 70]], hq, scale, max_ctx=max_ctx).double().cpu().numpy()
        assert np.array_equal(one[clean[[3, 70]]], ok[clean[[3, 70]]])


@pytest.mark.parametrize("dtype,d,page", [("bf16", 128, 16), ("bf16", 64, 32), ("f32", 64, 16)])
def test_decodes_and_chunks_in_one_batch(few_cus, dtype, d, page):  # noqa: F811
    """A queue of decodes - chunks of one row - beside a few long chunks and a prompt, as resume takes it: more sessions than a wave scans at once."""
    rng = np.random.default_rng(5)
    prefix, new = rng.integers(1, 900, 90), np.ones(90, int)
    prefix[[3, 40, 77]], new[[3, 40, 77]] = (1500, 0, 700), (130, 260, 64)
    side = Side(dtype, d, page, 2, prefix + new, seed=d)
    side.append(prefix)
    side.append(new)
    q, scale = side.draw(int(new.sum()), 8, d), d ** -0.5
    for stream in (None, few_cus):
        check_resume(side, q, resume(side, q, new, 8, scale, stream=stream), new, scale, (d, page))


def test_the_checker_of_tables_takes_an_8_bit_cache():
    side = Side("f32", 96, 64, 2, [130, 64], seed=1)
    side.append([130, 64])
    lens, none, cu = i32([130, 64]), i32([0, 0]), i32([0, 0, 0])
    B.ag_debug_validate(side.cache, side.bt_dev, lens, none, cu)
    bt = side.bt.copy()
    bt[1, 1] = 1 << 30                                            # not in use
    B.ag_debug_validate(side.cache, i32(bt), lens, none, cu)
    for at, page in (((0, 2), side.cache.num_pages), ((1, 0), -1)):
        bad = bt.copy()
        bad[at] = page
        with pytest.raises(B.AgError, match="outside"):
            B.ag_debug_validate(side.cache, i32(bad), lens, none, cu)
    with pytest.raises(B.AgError, match="cu_new"):
        B.ag_debug_validate(side.cache, side.bt_dev, none, lens, i32([0, 130, 130]))
