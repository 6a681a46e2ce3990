"""What Python refuses of queries and outputs over a latent cache, whose widths differ, before the library sees an address: without a GPU, by the ctypes path, tensors on
the host standing for the card's."""
import pytest
import torch

from paper_2603_10342_amd import binding as B


class Reached(Exception):
    pass


class Library:
    def __getattr__(self, name):
        raise Reached(name)


@pytest.fixture(autouse=True)
def host(monkeypatch):
    monkeypatch.setattr(B, "_native", B._NoCalls())
    monkeypatch.setattr(B, "_ptr", lambda t: None if t is None else t.data_ptr())
    cache = B.LatentCache(4, 16, 128, 32, "cpu")                       # (asks the library for a row's width)
    monkeypatch.setattr(B, "lib", Library)
    return cache


def x(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def i(*v):
    return torch.tensor(v, dtype=torch.int32)


def decode(cache, q, out, heads=4):
    B.ag_attn_decode_latent(cache, q, out, i(0, 1).view(2, 1), i(3, 4), 4, heads, 0.1, x(64))


def resume(cache, q, out, heads=4):
    B.ag_attn_resume_latent(cache, q, out, i(0, 1).view(2, 1), i(3, 4), i(1, 1), i(0, 1, 2), 2, 1, 5, heads, 0.1, x(64))


@pytest.mark.parametrize("call", [decode, resume])
def test_queries_and_outputs(host, call):
    for q, out in ((x(2, 4, 160), x(2, 4, 128)), (x(5, 4, 160), x(3, 4, 128)), (x(2, 640), x(2, 512))):
        with pytest.raises(Reached):
            call(host, q, out)
    q, out = x(2, 4, 160), x(2, 4, 128)
    for a, b in ((q.float(), out), (q.half(), out), (q, out.float()), (q, out.half())):
        with pytest.raises(TypeError, match="bfloat16"):
            call(host, a, b)
    for a, b in ((x(2, 4, 128), out), (q, x(2, 4, 160)), (x(1, 4, 160), out), (q, x(1, 4, 128)), (x(2, 3, 160), out), (q, x(2, 3, 128)), (x(2, 5, 160), out), (x(2 * 4 * 160), out),
                 (x(4, 4, 128), out), (q, x(4, 160))):
        with pytest.raises(ValueError, match="rows or more"):
            call(host, a, b)
    with pytest.raises(ValueError, match="rows or more"):
        call(host, q, out, heads=8)
