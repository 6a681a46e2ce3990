"""Rows of another type, width or number that Python refuses of the rotating append before the library sees an address: by ctypes without a GPU, tensors on the host standing
for the card's, and by both ways on it."""
import pytest
import torch

from paper_2603_10342_amd import binding as B
from test_latent_shapes_cpu import Library, Reached


def wrong(x, q, k):
    """(q, q_out, k_new, v_new), and what they raise, of two tokens with four query heads and two KV heads of 64 channels."""
    return [((q.float(), q, k, k), TypeError), ((q, q.half(), k, k), TypeError), ((q, q, k.float(), k), TypeError), ((q, q, k, k.half()), TypeError), ((x(1, 4, 64), q, k, k), ValueError),
            ((q, x(1, 4, 64), k, k), ValueError), ((q, q, x(1, 2, 64), k), ValueError), ((q, q, k, x(1, 2, 64)), ValueError), ((q, x(2, 2, 64), k, k), ValueError),
            ((x(2, 4, 48), q, k, k), ValueError), ((q, q, x(2, 1, 64), k), ValueError), ((q, q, k, x(2, 2, 128)), ValueError), ((None, None, k.float(), k), TypeError), ((None, None, k, x(1, 2, 64)), ValueError)]


def run(cache, rope, rows, device):
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device=device)
    B.ag_kv_append_rope(cache, rope, *rows, i(0, 1).view(1, 2), i(3), i(2), i(0, 2), 2)


def test_without_a_gpu(monkeypatch):
    monkeypatch.setattr(B, "_native", B._NoCalls())
    monkeypatch.setattr(B, "_ptr", lambda t: None if t is None else t.data_ptr())
    monkeypatch.setattr(B, "lib", Library)
    x = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    cache, rope, q, k = B.KVCache(4, 16, 2, 64, B.AG_BF16, "cpu"), B.Rope(torch.zeros(16, dtype=torch.float64)), x(2, 4, 64), x(2, 2, 64)
    for rows in ((q, q, k, k), (None, None, k, k), (x(3, 4, 64), x(5, 4, 64), x(4, 2, 64), x(2, 128))):
        with pytest.raises(Reached):
            run(cache, rope, rows, "cpu")
    for rows, error in wrong(x, q, k):
        with pytest.raises(error):
            run(cache, rope, rows, "cpu")
    full = B.KVCache(4, 16, 2, 64, B.AG_F32, "cpu")
    with pytest.raises(Reached):
        run(full, rope, [t.float() for t in (q, q, k, k)], "cpu")
    with pytest.raises(TypeError, match="float32"):
        run(full, rope, (q, q, k, k), "cpu")


@pytest.mark.gpu
def test_by_both_ways(monkeypatch):
    x = lambda *s: torch.full(s, 2.0, dtype=torch.bfloat16, device="cuda")
    cache, rope, q, k = B.KVCache(4, 16, 2, 64, B.AG_BF16, "cuda", fill=1.0), B.Rope(torch.zeros(16, dtype=torch.float64, device="cuda")), x(2, 4, 64), x(2, 2, 64)
    assert not isinstance(B._calls(), B._NoCalls)
    for _ in range(2):
        for rows, error in wrong(x, q, k):
            with pytest.raises(error):
                run(cache, rope, rows, "cuda")
        torch.cuda.synchronize()
        assert bool((cache.k_pool == 1).all()) and bool((cache.v_pool == 1).all()) and bool((q == 2).all())
        out = x(3, 4, 64) + 1
        run(cache, rope, (x(3, 4, 64), out, x(4, 2, 64), x(2, 128)), "cuda")
        torch.cuda.synchronize()
        assert int((cache.k_pool == 2).sum()) == int((cache.v_pool == 2).sum()) == 2 * 2 * 64 and bool((out[:2] == 2).all()) and bool((out[2] == 3).all())
        cache.k_pool.fill_(1.0), cache.v_pool.fill_(1.0)
        monkeypatch.setattr(B, "_native", B._NoCalls())
