"""Queries and outputs of the wrong type, width or number over a latent cache, by both ways into the library: refused before it, and what fits goes through."""
import pytest
import torch

from gpu_helpers import i32
from paper_2603_10342_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"


def x(*shape, dtype=torch.bfloat16):
    return torch.full(shape, 2.0, dtype=dtype, device=DEV)


def test_queries_and_outputs(monkeypatch):
    cache, bt = B.LatentCache(4, 16, 128, 32, DEV, fill=1.0), i32([[0], [1]])
    ws = torch.empty(max(B.ag_attn_decode_latent_workspace_bytes(2, 8, 128, 5), B.ag_attn_resume_latent_workspace_bytes(2, 2, 8, 128, 5)), dtype=torch.uint8, device=DEV)

    def decode(q, out, heads=4):
        B.ag_attn_decode_latent(cache, q, out, bt, i32([3, 4]), 4, heads, 0.1, ws)

    def resume(q, out, heads=4):
        B.ag_attn_resume_latent(cache, q, out, bt, i32([3, 4]), i32([1, 1]), i32([0, 1, 2]), 2, 1, 5, heads, 0.1, ws)

    assert not isinstance(B._calls(), B._NoCalls)
    for _ in range(2):
        for call in (decode, resume):
            q = x(2, 4, 160)
            for a, b, error in ((q.float(), x(2, 4, 128), TypeError), (q.half(), x(2, 4, 128), TypeError), (q, x(2, 4, 128, dtype=torch.float32), TypeError),
                                (x(2, 4, 128), x(2, 4, 128), ValueError), (q, x(2, 4, 160), ValueError), (x(1, 4, 160), x(2, 4, 128), ValueError), (q, x(1, 4, 128), ValueError),
                                (x(2, 3, 160), x(2, 4, 128), ValueError), (x(4, 4, 128), x(2, 4, 128), ValueError), (q.transpose(0, 1), x(2, 4, 128), ValueError)):
                with pytest.raises(error):
                    call(a, b)
                torch.cuda.synchronize()
                assert bool((b == 2).all())
            for a, b in ((q, x(2, 4, 128)), (x(3, 4, 160), x(5, 4, 128)), (x(2, 640), x(2, 512))):
                call(a, b)
                torch.cuda.synchronize()
                assert bool((b[:2] == 1).all()) and bool((b[2:] == 2).all())
            with pytest.raises(ValueError):
                call(q, x(2, 4, 128), heads=8)
        monkeypatch.setattr(B, "_native", B._NoCalls())
