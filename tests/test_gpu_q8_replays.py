"""Calls over an 8-bit cache captured and replayed: appends that have something to write, and every prefill kernel (test_q8_replayed_kernels.py)."""
import numpy as np
import pytest
import torch

from gpu_helpers import i32
from paper_2603_10342_amd import binding as B
from test_gpu_q8 import DEV, Side, check_decode, check_resume, few_cus  # noqa: F401 (a fixture)
from test_q8_dispatch import SHARED_CTX
from test_q8_replayed_kernels import REPLAYS

pytestmark = pytest.mark.gpu


def same(a, b):
    return all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype,d,page", [("bf16", 128, 16), ("f32", 64, 32), ("bf16", 96, 64)])
@pytest.mark.parametrize("new", [[1, 1, 1], [16, 37, 2]])
def test_a_replayed_append_writes(dtype, d, page, new):
    """A step - append, decode, resume, read-back - captured once.  Before every replay the pools are as they were before the append, or hold stale bytes in
    the new tokens' place, and the rows are other ones: pools and outputs are those of an eager step with the same rows."""
    hq, hkv, old = 8, 2, [700, 290, 62]
    side = Side(dtype, d, page, hkv, [p + n for p, n in zip(old, new)], seed=9)
    side.append(old)
    c, t, scale = side.cache, sum(new), d ** -0.5
    pools = (c.k_pool, c.v_pool, c.exps)
    before = [x.clone() for x in pools]
    prefix, lens, cu, ctx = i32(old), i32(new), i32(np.concatenate([[0], np.cumsum(new)])), i32([p + n for p, n in zip(old, new)])
    max_ctx = max(p + n for p, n in zip(old, new))
    k, v, q, q1 = (side.dev(side.draw(*s)) for s in ((t, hkv, d), (t, hkv, d), (t, hq, d), (3, hq, d)))
    out, out1, back = torch.empty_like(q), torch.empty_like(q1), [torch.empty_like(k) for _ in range(2)]
    ws = torch.empty(B.ag_attn_decode_q8_workspace_bytes(3, hq, d, max_ctx), dtype=torch.uint8, device=DEV)

    def step():
        B.ag_kv_append_q8(c, k, v, side.bt_dev, prefix, lens, cu, t)
        B.ag_attn_decode_q8(c, q1, out1, side.bt_dev, ctx, max_ctx, hq, scale, ws)
        B.ag_attn_resume_q8(c, q, out, side.bt_dev, prefix, lens, cu, t, max(new), max_ctx, hq, scale)
        B.ag_kv_read_q8(c, *back, side.bt_dev, prefix, lens, cu, t)

    def reset(junk):
        for x, y in zip(pools, before):
            x.view(torch.uint8).copy_(y.view(torch.uint8))
        if junk is not None:                                      # in the slots that the append is to write
            for s, n in enumerate(new):
                pos = np.arange(old[s], old[s] + n)
                page_ids, slots = (torch.from_numpy(x.astype(np.int64)).to(DEV) for x in (side.bt[s, pos // page], pos % page))
                c.k_pool.view(torch.uint8)[page_ids, :, slots // 4, :, slots % 4] = junk
                c.v_pool.view(torch.uint8)[page_ids, :, slots // 16, :, slots % 16] = junk
                c.exps[page_ids, :, 0, (slots & ~15) | ((slots & 3) << 2) | ((slots >> 2) & 3)] = junk
                c.exps[page_ids, :, 1, slots] = junk
        for x in (out, out1, *back):
            x.fill_(float("nan"))
        ws.random_()
        torch.cuda.synchronize()

    step()
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=other):
        step()
    results = (*pools, out, out1, *back)
    seen = []
    for r, junk in enumerate((None, 0xFF, 0x5A, None)):
        for x in (k, v, q, q1):
            x.copy_(side.dev(side.draw(*x.shape)))
        reset(junk)
        step()
        torch.cuda.synchronize()
        eager = [x.clone() for x in results]
        assert not same(eager[:3], before) and not any(bool(torch.isnan(x).any()) for x in eager[3:])
        reset(junk)
        graph.replay()
        torch.cuda.synchronize()
        assert same(results, eager), r
        seen.append(eager)
    assert not same(seen[0][:3], seen[3][:3])


@pytest.mark.parametrize("dtype,d,hq,prefix,new,all_cus,eight", REPLAYS)
def test_replays_of_every_prefill_kernel(few_cus, dtype, d, hq, prefix, new, all_cus, eight):  # noqa: F811
    prefix, new = np.array(prefix), np.array(new)
    side = Side(dtype, d, 16, 2, prefix + new, seed=d)
    if prefix.any():
        side.append(prefix)
    side.append(new)
    n, t, scale = prefix + new, int(new.sum()), d ** -0.5
    host_q, host_q1 = side.draw(t, hq, d), side.draw(len(new), hq, d)
    q, q1 = side.dev(host_q), side.dev(host_q1)
    lens, cu, old, ctx = i32(new), i32(np.concatenate([[0], np.cumsum(new)])), i32(prefix), i32(n)
    bt = i32(np.pad(side.bt, ((0, 0), (0, SHARED_CTX // 16 - side.bt.shape[1]))))
    ws = torch.empty(B.ag_attn_decode_q8_workspace_bytes(len(new), hq, d, SHARED_CTX), dtype=torch.uint8, device=DEV)
    got = [torch.empty_like(q), torch.empty_like(q1)]

    def step():
        B.ag_attn_resume_q8(side.cache, q, got[0], bt, old, lens, cu, t, int(new.max()), int(n.max()), hq, scale)
        B.ag_attn_decode_q8(side.cache, q1, got[1], bt, ctx, SHARED_CTX, hq, scale, ws)

    for stream in (torch.cuda.Stream(), torch.cuda.ExternalStream(few_cus)):
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            step()
        torch.cuda.synchronize()
        eager = [x.clone() for x in got]
        check_resume(side, host_q, eager[0], new, scale, (d, "resume"))
        check_decode(side, host_q1, eager[1], scale, (d, "decode"))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for r in range(3):
            for x in got:
                x.fill_(float("nan"))
            ws.random_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert same(got, eager), r
