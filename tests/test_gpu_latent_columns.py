"""Attention over the latent cache in its widest columns, which short batches take only under a loose bound of their contexts (test_latent_dispatch.py
sees that they do), and in all of them the same numbers."""
import numpy as np
import pytest
import torch

import latent_oracle as O
from gpu_helpers import i32
from paper_2603_10342_amd import binding as B
from test_gpu_latent import DEV, WIDTHS, Side, check_decode, check_resume, decode, resume

pytestmark = pytest.mark.gpu
HEADS = [1, 16, 33, 64, 65, 100, 128, 129, 200]
CTX, NEW = [2, 300, 0, 47, 1024, 33, 640], [2, 13, 0, 1, 20, 33, 5]
LOOSE = 1 << 16


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("page", [16, 128])
def test_heads(heads, page):
    side = Side(512, 64, page, CTX)
    side.append(CTX)
    q = side.draw(len(CTX), heads, side.w)
    check_decode(side, q, 0.04, decode(side, q, 0.04, max_ctx=LOOSE))
    q = side.draw(sum(NEW), heads, side.w)
    check_resume(side, q, NEW, 0.04, resume(side, q, NEW, 0.04, bound=sum(NEW) + 3, max_ctx=LOOSE))


@pytest.mark.parametrize("lat,rd", WIDTHS)
@pytest.mark.parametrize("heads", [24, 128])
def test_widths(lat, rd, heads):
    side = Side(lat, rd, 16, CTX)
    side.append(CTX)
    scale = side.w ** -0.5
    q = side.draw(len(CTX), heads, side.w)
    check_decode(side, q, scale, decode(side, q, scale, max_ctx=LOOSE))
    q = side.draw(sum(NEW), heads, side.w)
    check_resume(side, q, NEW, scale, resume(side, q, NEW, scale, max_ctx=LOOSE))


@pytest.mark.parametrize("heads", [60, 128])
@pytest.mark.parametrize("loose", [300, LOOSE])
def test_rows_that_are_not_finite(heads, loose):
    n, new, at, ch = 300, 70, 270, 77
    bad, clean = Side(512, 64, 16, [n, 50], seed=3), Side(512, 64, 16, [n, 50], seed=3)
    rows = bad.draw(n + 50, bad.w)
    assert (clean.draw(n + 50, clean.w) == rows).all()
    clean.append([n, 50], rows)
    rows = rows.copy()
    rows[at, ch] = float("nan")
    bad.append([n, 50], rows)
    q = bad.draw(new + 5, heads, bad.w)
    got, want = (resume(s, q, [new, 5], 0.04, max_ctx=loose) for s in (bad, clean))
    sees = np.arange(new) + n - new >= at
    assert np.isnan(got[:new][sees]).all()
    assert (got[:new][~sees] == want[:new][~sees]).all() and (got[new:] == want[new:]).all()
    one = decode(bad, q[:2], 0.04, max_ctx=loose)
    assert np.isnan(one[0]).all()
    check_decode(clean, q[:2], 0.04, np.stack([decode(clean, q[:2], 0.04, max_ctx=loose)[0], one[1]]))


def test_scores_that_grow_late():
    """The first tile's scores are far below a later one's: the piece is done again under its largest."""
    side = Side(512, 64, 16, [1500, 40])
    rows = side.draw(1540, side.w) * np.linspace(0.01, 1.0, 1540)[:, None]
    rows[700] *= 20
    side.append([1500, 40], O.bf16(rows.astype(np.float32)))
    for heads in (64, 128):
        q = side.draw(7, heads, side.w, sigma=2.0)
        for loose in (1500, LOOSE):
            check_resume(side, q, [6, 1], 0.3, resume(side, q, [6, 1], 0.3, max_ctx=loose))
            check_decode(side, q[:2], 0.3, decode(side, q[:2], 0.3, max_ctx=loose))


def test_one_workspace_for_every_width():
    """Calls that follow each other in one workspace, of the widest one's size, whatever the one before left there."""
    side = Side(512, 64, 16, CTX)
    side.append(CTX)
    ws = torch.full((max(B.ag_attn_decode_latent_workspace_bytes(len(CTX), 128, 512, LOOSE), B.ag_attn_resume_latent_workspace_bytes(len(CTX), sum(NEW), 128, 512, LOOSE)) // 4,),
                    float("nan"), dtype=torch.float32, device=DEV)
    table, ctx, lens, new, cu = side.table(LOOSE), i32(CTX), i32(np.array(CTX) - NEW), i32(NEW), i32(np.concatenate([[0], np.cumsum(NEW)]))
    for heads, bound in ((128, LOOSE), (16, 1024), (128, 1024), (64, LOOSE), (128, LOOSE)):
        q, chunk = side.draw(len(CTX), heads, side.w), side.draw(sum(NEW), heads, side.w)
        out, rows = (torch.full((n, heads, 512), float("nan"), dtype=torch.bfloat16, device=DEV) for n in (len(CTX), sum(NEW)))
        B.ag_attn_decode_latent(side.cache, side.dev(q), out, table, ctx, bound, heads, 0.04, ws)
        B.ag_attn_resume_latent(side.cache, side.dev(chunk), rows, table, lens, new, cu, sum(NEW), max(NEW), bound, heads, 0.04, ws)
        torch.cuda.synchronize()
        check_decode(side, q, 0.04, out.double().cpu().numpy())
        check_resume(side, chunk, NEW, 0.04, rows.double().cpu().numpy())
