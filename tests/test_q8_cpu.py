"""The 8-bit cache's host-side refusals, which come before any device work: fake pointers, never dereferenced."""
import ctypes as C

import pytest
import torch

from paper_2603_10342_amd import binding as B

P = 4096                                                          # an aligned address that nothing reads


def cache(**more):
    f = dict(k_pool=P, v_pool=P, exps=P, num_pages=8, page_size=16, num_kv_heads=2, head_dim=128, dtype=B.AG_BF16)
    f.update(more)
    return B.ag_kv_cache_q8(*f.values())


def rows(fn, c, k=P, v=P, bt=P, pages=4, prefix=P, new=P, cu=P, batch=1, total=16):
    return getattr(B.lib(), fn)(None if c is None else C.byref(c), k, v, bt, pages, prefix, new, cu, batch, total, None)


def resume(c, q=P, out=P, bt=P, pages=4, prefix=P, new=P, cu=P, batch=1, total=16, max_new=16, max_ctx=16, hq=4, scale=0.1):
    return B.lib().ag_attn_resume_q8(None if c is None else C.byref(c), q, out, bt, pages, prefix, new, cu, batch, total, max_new, max_ctx, hq, scale, None)


def prefill(c, q=P, out=P, bt=P, pages=4, new=P, cu=P, batch=1, total=16, max_new=16, hq=4, scale=0.1):
    return B.lib().ag_attn_prefill_q8(None if c is None else C.byref(c), q, out, bt, pages, new, cu, batch, total, max_new, hq, scale, None)


def decode(c, q=P, out=P, bt=P, pages=4, ctx=P, batch=1, max_ctx=64, hq=4, scale=0.1, ws=P, nbytes=1 << 24):
    return B.lib().ag_attn_decode_q8(None if c is None else C.byref(c), q, out, bt, pages, ctx, batch, max_ctx, hq, scale, ws, nbytes, None)


CALLS = [lambda c, **m: rows("ag_kv_append_q8", c, **m), lambda c, **m: rows("ag_kv_read_q8", c, **m), resume, prefill, decode]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("field,value,want", [
    ("dtype", 2, B.AG_ERR_UNSUPPORTED), ("head_dim", 8, B.AG_ERR_UNSUPPORTED), ("head_dim", 100, B.AG_ERR_UNSUPPORTED), ("head_dim", 272, B.AG_ERR_UNSUPPORTED),
    ("head_dim", 0, B.AG_ERR_UNSUPPORTED), ("page_size", 8, B.AG_ERR_UNSUPPORTED), ("page_size", 24, B.AG_ERR_UNSUPPORTED), ("page_size", 512, B.AG_ERR_UNSUPPORTED),
    ("page_size", 0, B.AG_ERR_UNSUPPORTED), ("num_pages", 0, B.AG_ERR_INVALID_ARG), ("num_kv_heads", 0, B.AG_ERR_INVALID_ARG), ("k_pool", 0, B.AG_ERR_INVALID_ARG),
    ("v_pool", 0, B.AG_ERR_INVALID_ARG), ("exps", 0, B.AG_ERR_INVALID_ARG), ("k_pool", P + 8, B.AG_ERR_INVALID_ARG), ("exps", P + 4, B.AG_ERR_INVALID_ARG)])
def test_caches(call, field, value, want):
    assert call(cache(**{field: value})) == want
    assert call(None) == B.AG_ERR_INVALID_ARG and B.lib().ag_last_error()


@pytest.mark.parametrize("call,bad", [
    *((c, [dict(k=0), dict(v=0), dict(bt=0), dict(prefix=0), dict(new=0), dict(cu=0), dict(k=P + 2), dict(v=P + 8), dict(batch=0), dict(pages=0), dict(total=-1)])
      for c in CALLS[:2]),
    (resume, [dict(q=0), dict(out=0), dict(bt=0), dict(prefix=0), dict(new=0), dict(cu=0), dict(q=P + 2), dict(out=P + 8), dict(batch=0), dict(pages=0), dict(hq=3), dict(hq=0),
              dict(scale=0.0), dict(scale=float("nan")), dict(max_new=17), dict(max_ctx=15), dict(max_ctx=65), dict(total=-1), dict(max_new=-1)]),
    (prefill, [dict(q=0), dict(new=0), dict(out=P + 4), dict(hq=5), dict(scale=-1.0), dict(max_new=17), dict(pages=0), dict(total=80, max_new=65)]),
    (decode, [dict(q=0), dict(ctx=0), dict(q=P + 2), dict(hq=7), dict(scale=float("inf")), dict(max_ctx=65), dict(max_ctx=-1), dict(batch=0), dict(ws=P + 8)])])
def test_arguments(call, bad):
    for more in bad:
        assert call(cache(), **more) == B.AG_ERR_INVALID_ARG, more
        assert B.lib().ag_last_error()


def test_decode_workspace():
    need = B.ag_attn_decode_q8_workspace_bytes(1, 4, 128, 64)
    assert need > 0 and decode(cache(), nbytes=need - 1) == B.AG_ERR_WORKSPACE and decode(cache(), ws=None) == B.AG_ERR_WORKSPACE
    assert B.ag_attn_decode_q8_workspace_bytes(0, 4, 128, 64) == 0 and B.ag_attn_decode_q8_workspace_bytes(1, 4, 128, -1) == 0
    assert decode(cache(num_kv_heads=8), hq=8, batch=1 << 24, pages=1 << 20, max_ctx=1 << 20, nbytes=1 << 62) == B.AG_ERR_INVALID_ARG


def test_contexts_past_32_bits():
    most = (1 << 31) - 1025
    assert resume(cache(), pages=1 << 27, max_ctx=most + 1) == B.AG_ERR_INVALID_ARG and b"max_ctx" in B.lib().ag_last_error()
    assert prefill(cache(), pages=1 << 27, total=most + 1, max_new=most + 1) == B.AG_ERR_INVALID_ARG
    assert decode(cache(), pages=1 << 27, max_ctx=most + 1, nbytes=1 << 62) == B.AG_ERR_INVALID_ARG
    assert B.ag_attn_decode_q8_workspace_bytes(1, 4, 128, most + 1) == 0 and B.ag_attn_decode_q8_workspace_bytes(1, 4, 128, most) > 0


def test_nothing_to_do_reaches_no_device():
    for call in CALLS[:2]:
        assert call(cache(), total=0) == B.AG_OK
    assert resume(cache(), total=0, max_new=0, max_ctx=0) == B.AG_OK and prefill(cache(), total=0, max_new=0) == B.AG_OK


def test_the_binding_refuses_what_is_no_device_memory_and_shapes_that_no_cache_has():
    for args in [(4, 16, 2, 24), (4, 8, 2, 64), (4, 16, 2, 0)]:
        with pytest.raises(ValueError, match="multiples of 16"):
            B.KVCacheQ8(*args, B.AG_BF16, "cpu")
    c = B.KVCacheQ8(4, 32, 2, 64, B.AG_BF16, "cpu", fill=0x7F)
    assert c.k_pool.dtype == torch.float8_e4m3fn and c.k_pool.shape == (4, 2, 8, 4, 4, 16) and c.v_pool.shape == (4, 2, 2, 64, 16) and c.exps.shape == (4, 2, 2, 32)
    assert bool(torch.isnan(c.k_pool.float()).all())
    x, i = torch.zeros(1, 2, 64, dtype=torch.bfloat16), lambda *v: torch.tensor(v, dtype=torch.int32)
    bt = i(0, 1).view(1, 2)
    for call in (lambda: B.ag_kv_append_q8(c, x, x, bt, i(0), i(1), i(0, 1), 1), lambda: B.ag_kv_read_q8(c, x, x, bt, i(0), i(1), i(0, 1), 1),
                 lambda: B.ag_attn_prefill_q8(c, x, x, bt, i(1), i(0, 1), 1, 1, 2, 0.1), lambda: B.ag_attn_resume_q8(c, x, x, bt, i(0), i(1), i(0, 1), 1, 1, 1, 2, 0.1),
                 lambda: B.ag_attn_decode_q8(c, x, x, bt, i(1), 1, 2, 0.1, x)):
        with pytest.raises(ValueError, match="contiguous CUDA"):
            call()
    other = B.KVCache(4, 16, 2, 64, B.AG_BF16, "cpu")
    assert B._calls().kv_append_q8(other, x, x, bt, i(0), i(1), i(0, 1), 1, None) is None


def test_token_major_views_follow_the_layout():
    c = B.KVCacheQ8(3, 32, 2, 48, B.AG_F32, "cpu", fill=0)
    kp, vp, e = c.k_pool.view(torch.uint8), c.v_pool.view(torch.uint8), c.exps
    for page, head, slot, ch in [(0, 0, 0, 0), (2, 1, 31, 47), (1, 0, 6, 17), (1, 1, 19, 33)]:
        kp[page, head, slot // 4, ch // 16, slot % 4, ch % 16] = 1 + slot
        vp[page, head, slot // 16, ch, slot % 16] = 100 + slot
        e[page, head, 0, slot // 16 * 16 + 4 * (slot % 4) + slot % 16 // 4] = 17 + slot
        e[page, head, 1, slot] = 80 + slot
        assert c.k_pool_token_major()[page, head, slot, ch] == 1 + slot and c.v_pool_token_major()[page, head, slot, ch] == 100 + slot
        ke, ve = c.exps_token_major()
        assert ke[page, head, slot] == 17 + slot and ve[page, head, slot] == 80 + slot
