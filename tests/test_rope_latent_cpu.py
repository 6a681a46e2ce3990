"""Rotary positions and the latent cache without a GPU: host-side refusals, which come before any device work (fake pointers, never dereferenced), turns, sizes."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import latent_oracle as O
from paper_2603_10342_amd import binding as B

P = 4096                                                          # an aligned address that nothing reads
BAD, NOT = B.AG_ERR_INVALID_ARG, B.AG_ERR_UNSUPPORTED


def rope(**more):
    f = dict(turns=P, rot_dim=64, layout=B.AG_ROPE_HALVES, magnitude=1.0)
    f.update(more)
    return B.ag_rope(*f.values())


def kv(**more):
    f = dict(k_pool=P, v_pool=P, num_pages=8, page_size=16, num_kv_heads=2, head_dim=128, dtype=B.AG_BF16)
    f.update(more)
    return B.ag_kv_cache(*f.values())


def latent(**more):
    f = dict(pool=P, num_pages=8, page_size=16, latent_dim=512, rope_dim=64)
    f.update(more)
    return B.ag_latent_cache(*f.values())


def ref(x):
    return None if x is None else C.byref(x)


def rows(r=None, dtype=B.AG_BF16, x=P, xt=1024, xh=128, y=2 * P, yt=1024, yh=128, heads=8, d=128, prefix=P, new=P, cu=P, batch=1, total=0, transposed=0):
    return B.lib().ag_rope_rows(ref(r or rope()), dtype, x, xt, xh, y, yt, yh, heads, d, prefix, new, cu, batch, total, transposed, None)


def append(c=None, r=None, q=P, q_out=P, hq=4, k=P, v=P, bt=P, pages=4, prefix=P, new=P, cu=P, batch=1, total=0):
    return B.lib().ag_kv_append_rope(ref(c or kv()), ref(r or rope()), q, q_out, hq, k, v, bt, pages, prefix, new, cu, batch, total, None)


def append_latent(c=None, r=None, lat=P, lt=576, rot=P, rt=576, bt=P, pages=4, prefix=P, new=P, cu=P, batch=1, total=0):
    return B.lib().ag_kv_append_latent(ref(c or latent()), ref(r), lat, lt, rot, rt, bt, pages, prefix, new, cu, batch, total, None)


def decode(c=None, q=P, out=P, bt=P, pages=4, ctx=P, batch=1, max_ctx=64, hq=4, scale=0.1, ws=P, nbytes=1 << 40):
    return B.lib().ag_attn_decode_latent(ref(c or latent()), q, out, bt, pages, ctx, batch, max_ctx, hq, scale, ws, nbytes, None)


def resume(c=None, q=P, out=P, bt=P, pages=4, prefix=P, new=P, cu=P, batch=1, total=16, max_new=16, max_ctx=16, hq=4, scale=0.1, ws=P, nbytes=1 << 40):
    return B.lib().ag_attn_resume_latent(ref(c or latent()), q, out, bt, pages, prefix, new, cu, batch, total, max_new, max_ctx, hq, scale, ws, nbytes, None)


@pytest.mark.parametrize("call", [rows, append, lambda r: append_latent(r=r)])
@pytest.mark.parametrize("field,value,want", [
    ("turns", 0, BAD), ("turns", P + 4, BAD), ("rot_dim", 8, NOT), ("rot_dim", 0, NOT), ("rot_dim", 40, NOT), ("rot_dim", 272, NOT), ("rot_dim", -16, NOT), ("rot_dim", 160, BAD),
    ("layout", 2, NOT), ("layout", -1, NOT), ("magnitude", 0.0, BAD), ("magnitude", -1.0, BAD), ("magnitude", math.nan, BAD), ("magnitude", math.inf, BAD)])
def test_rotations(call, field, value, want):
    assert call(r=rope(**{field: value})) == want and B.lib().ag_last_error()


def test_rows_to_rotate():
    assert rows() == B.AG_OK                                       # nothing to do reaches no device
    for more in (dict(x=0), dict(y=0), dict(prefix=0), dict(new=0), dict(cu=0), dict(batch=0), dict(total=-1), dict(heads=0), dict(heads=1 << 27), dict(d=0), dict(d=60), dict(d=48),
                 dict(x=P + 8), dict(y=P + 2), dict(xt=1028), dict(yh=4), dict(xh=-8), dict(yt=1 << 40), dict(y=P, yh=256)):
        assert rows(**more) == BAD, more
        assert B.lib().ag_last_error()
    assert rows(dtype=2) == NOT and rows(dtype=B.AG_F32, xh=12) == B.AG_OK and rows(dtype=B.AG_F32, xh=6) == BAD
    assert B.lib().ag_rope_rows(None, B.AG_BF16, P, 8, 8, P, 8, 8, 1, 128, P, P, P, 1, 0, 0, None) == BAD


def test_rotating_append():
    assert append() == B.AG_OK and append(q=None, q_out=None, hq=0) == B.AG_OK
    for more in (dict(q=None), dict(q_out=None), dict(q=None, q_out=None), dict(hq=3), dict(hq=0), dict(hq=1 << 18), dict(k=0), dict(v=0), dict(bt=0), dict(prefix=0), dict(new=0), dict(cu=0), dict(batch=0),
                 dict(pages=0), dict(total=-1), dict(k=P + 8), dict(v=P + 2), dict(q=P + 4), dict(q_out=P + 8), dict(c=kv(k_pool=P + 8)), dict(c=kv(num_pages=0)), dict(c=kv(v_pool=0))):
        assert append(**more) == BAD, more
        assert B.lib().ag_last_error()
    for more in (dict(page_size=8), dict(page_size=24), dict(page_size=512), dict(head_dim=100), dict(head_dim=264), dict(dtype=2)):
        assert append(c=kv(**more)) == NOT, more
    assert append(c=kv(head_dim=48)) == BAD                       # fewer channels than turn


CALLS = [append_latent, decode, resume]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("field,value,want", [
    ("latent_dim", 64, NOT), ("latent_dim", 384, NOT), ("latent_dim", 1024, NOT), ("latent_dim", 0, NOT), ("rope_dim", 0, NOT), ("rope_dim", 16, NOT), ("rope_dim", 128, NOT),
    ("page_size", 8, NOT), ("page_size", 24, NOT), ("page_size", 512, NOT), ("page_size", 0, NOT), ("num_pages", 0, BAD), ("pool", 0, BAD), ("pool", P + 8, BAD)])
def test_latent_caches(call, field, value, want):
    assert call(c=latent(**{field: value})) == want and B.lib().ag_last_error()


def test_latent_rows():
    assert append_latent() == B.AG_OK and append_latent(r=rope()) == B.AG_OK and append_latent(lt=512, rt=64) == B.AG_OK
    for more in (dict(lat=0), dict(rot=0), dict(bt=0), dict(prefix=0), dict(new=0), dict(cu=0), dict(batch=0), dict(pages=0), dict(total=-1), dict(lat=P + 8), dict(rot=P + 2), dict(lt=573), dict(rt=4), dict(lt=-8),
                 dict(rt=1 << 40), dict(r=rope(rot_dim=32))):
        assert append_latent(**more) == BAD, more
    with pytest.raises(ValueError, match="128, 256 or 512"):
        B.LatentCache(4, 16, 192, 64, "cpu")
    c = B.LatentCache(4, 32, 256, 32, "cpu", fill=2.0)
    assert c.pool.shape == (4, 32, 320) and c.pool.dtype == torch.bfloat16 and bool((c.pool == 2).all())
    assert [B.ag_latent_row(*w) for w in ((512, 64), (512, 32), (256, 64), (256, 32), (128, 64), (128, 32), (512, 48), (96, 64))] == [576, 576, 320, 320, 192, 192, 0, 0]


@pytest.mark.parametrize("call,bad", [
    (decode, [dict(q=0), dict(out=0), dict(bt=0), dict(ctx=0), dict(q=P + 2), dict(out=P + 8), dict(hq=0), dict(hq=-1), dict(scale=0.0), dict(scale=math.nan), dict(scale=math.inf), dict(max_ctx=65), dict(max_ctx=-1),
              dict(batch=0), dict(pages=0), dict(ws=P + 8)]),
    (resume, [dict(q=0), dict(out=0), dict(bt=0), dict(prefix=0), dict(new=0), dict(cu=0), dict(q=P + 2), dict(out=P + 8), dict(batch=0), dict(pages=0), dict(hq=0), dict(scale=-1.0), dict(max_new=17), dict(max_ctx=15),
              dict(max_ctx=65), dict(total=-1), dict(max_new=-1), dict(ws=P + 4)])])
def test_attention_arguments(call, bad):
    for more in bad:
        assert call(**more) == BAD, more
        assert B.lib().ag_last_error()


def test_workspaces_and_batches_past_one_launch():
    need = B.ag_attn_decode_latent_workspace_bytes(1, 4, 512, 64)
    assert need > 0 and decode(nbytes=need - 1) == B.AG_ERR_WORKSPACE and decode(ws=None) == B.AG_ERR_WORKSPACE
    need = B.ag_attn_resume_latent_workspace_bytes(1, 16, 4, 512, 16)
    assert need > 0 and resume(nbytes=need - 1) == B.AG_ERR_WORKSPACE and resume(ws=None) == B.AG_ERR_WORKSPACE
    assert resume(total=0, max_new=0, max_ctx=0, ws=None, nbytes=0) == B.AG_OK
    for f, args in ((B.ag_attn_decode_latent_workspace_bytes, [(0, 4, 512, 64), (1, 0, 512, 64), (1, 4, 500, 64), (1, 4, 512, -1), (1 << 20, 128, 512, 1 << 20)]),
                    (B.ag_attn_resume_latent_workspace_bytes, [(0, 1, 4, 512, 64), (1, -1, 4, 512, 64), (1, 1, 0, 512, 64), (1, 1, 4, 96, 64), (1, 1, 4, 512, -1), (1, (1 << 31) - 1, 1 << 20, 512, 1 << 20)])):
        assert all(f(*a) == 0 for a in args)
    assert decode(batch=1 << 20, hq=128, pages=1 << 20, max_ctx=1 << 20) == BAD and b"too large" in B.lib().ag_last_error()
    most = (1 << 31) - 1025
    assert decode(pages=1 << 27, max_ctx=most + 1) == BAD and resume(pages=1 << 27, max_ctx=most + 1) == BAD and b"max_ctx" in B.lib().ag_last_error()
    assert B.ag_attn_decode_latent_workspace_bytes(1, 4, 512, most + 1) == 0 and B.ag_attn_decode_latent_workspace_bytes(1, 4, 512, most) > 0


def test_turns():
    np.testing.assert_allclose(B.ag_rope_turns(64).numpy(), O.turns(64), rtol=4e-16)
    np.testing.assert_allclose(B.ag_rope_turns(128, 5e5, B.AG_ROPE_LINEAR, 4.0).numpy(), O.turns(128, 5e5) / 4, rtol=4e-16)
    t = O.turns(64)
    keep = np.clip((4096 * t - 1) / (32 - 1), 0, 1)               # turns over the trained context, from 1 to 32
    got = B.ag_rope_turns(64, 10000.0, B.AG_ROPE_RAMP, 40.0, 4096.0, 1.0, 32.0).numpy()
    np.testing.assert_allclose(got, O.turns(64, keep=keep, factor=40.0), rtol=1e-14)
    assert got[0] == t[0] and abs(got[-1] * 40 / t[-1] - 1) < 1e-15 and ((got < t) & (got > t / 40)).any()
    for more in (dict(rot_dim=0), dict(rot_dim=7), dict(base=0.0), dict(base=math.inf), dict(factor=0.0), dict(factor=math.nan), dict(scaling=B.AG_ROPE_RAMP),
                 dict(scaling=B.AG_ROPE_RAMP, trained_len=4096.0, low=2.0, high=2.0), dict(scaling=B.AG_ROPE_RAMP, trained_len=4096.0, low=-1.0, high=2.0)):
        with pytest.raises(B.AgError) as e:
            B.ag_rope_turns(**{"rot_dim": 64, **more})
        assert e.value.status == BAD
    with pytest.raises(B.AgError) as e:
        B.ag_rope_turns(64, scaling=3)
    assert e.value.status == NOT


def test_the_binding_refuses_what_is_no_device_memory():
    t, x, i = torch.zeros(8, dtype=torch.float64), lambda *s: torch.zeros(s, dtype=torch.bfloat16), lambda *v: torch.tensor(v, dtype=torch.int32)
    with pytest.raises(TypeError, match="fp64"):
        B.Rope(t.float())
    r, bt, lens = B.Rope(t), i(0, 1).view(1, 2), (i(0), i(1), i(0, 1))
    cache, lat = B.KVCache(4, 16, 2, 64, B.AG_BF16, "cpu"), B.LatentCache(4, 16, 128, 32, "cpu")
    for call in (lambda: B.ag_rope_rows(r, x(1, 2, 64), x(1, 2, 64), *lens, 1), lambda: B.ag_kv_append_rope(cache, r, None, None, x(1, 2, 64), x(1, 2, 64), bt, *lens, 1),
                 lambda: B.ag_kv_append_latent(lat, None, x(1, 128), x(1, 32), bt, *lens, 1), lambda: B.ag_attn_decode_latent(lat, x(1, 2, 160), x(1, 2, 128), bt, i(1), 1, 2, 0.1, x(1)),
                 lambda: B.ag_attn_resume_latent(lat, x(1, 2, 160), x(1, 2, 128), bt, *lens, 1, 1, 1, 2, 0.1, x(1))):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    with pytest.raises(ValueError, match="one shape"):
        B.ag_rope_rows(r, x(1, 2, 64), x(1, 3, 64), *lens, 1)
    assert B._calls().kv_append_latent(cache, None, x(1, 128), x(1, 32), bt, *lens, 1, None) is None


def test_oracle_of_rotations_against_complex_numbers():
    t, pos = O.turns(16), np.array([0, 1, 17, 100000])
    x = np.random.default_rng(1).standard_normal((4, 3, 24))
    for layout in ("halves", "pairs"):
        a, b = O.pairs_of(16, layout)
        z = (x[..., a] + 1j * x[..., b]) * 1.5 * np.exp(2j * np.pi * np.outer(pos, t))[:, None]
        y, _ = O.rotate(x, pos, t, layout, 1.5)
        np.testing.assert_allclose(y[..., a] + 1j * y[..., b], z, atol=1e-10)
        assert (y[..., 16:] == x[..., 16:]).all()
        back, _ = O.rotate(y, pos, t, layout, 1 / 1.5, transposed=True)
        np.testing.assert_allclose(back, x, atol=1e-12)
