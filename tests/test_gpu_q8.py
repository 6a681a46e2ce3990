"""The 8-bit cache on the GPU against the 64-bit oracle (q8_oracle.py): bytes exactly, attention within bounds that are derived here.

Bounds of an output o = sum p v, with size = sum p |v| (both in the oracle), elementwise:
  weights   bf16 activations round them to bf16, off by up to 2^-8 of themselves; the normaliser sums them rounded or not: 2 * 2^-8 size.
            fp32: three bf16 terms, 2^-24.
  scores    D products, each exact, are added up in fp32: D + 2 roundings of at most 2^-24 of sum |q| |k| scale = reach (taken twice: the factor
            scale * log2 e and its product round too); a weight is off by that, and so is the normaliser: 2 (D + 4) 2^-24 reach * size.
  sums      over n keys in fp32, and exp2: (n + 16) 2^-24 size, the normaliser's as much.
  output    rounded once: 2^-8 |o| in bf16, 2^-24 |o| in fp32.
Roundings are independent, so that the norm of all errors is far below: half of the elementwise bound for bf16 (2^-9 |o| and 2^-8 size / sqrt(keys)
are typical, with size about sqrt(keys) |o| in these inputs); fp32, 2^-24 * sqrt(D) of scores of size 3, in both of numerator and normaliser,
and as much for the sums: 4e-6 up to 128 channels, 6e-6 to 256."""
import numpy as np
import pytest
import torch

import q8_oracle as Q
from gpu_helpers import i32
from paper_2603_10342_amd import binding as B
from test_q8_dispatch import FOUR_LENS, SHARED_CTX, TILED

pytestmark = pytest.mark.gpu
DEV = "cuda"
TD = {"bf16": torch.bfloat16, "f32": torch.float32}
AG = {"bf16": B.AG_BF16, "f32": B.AG_F32}


class Side:
    """A cache on the GPU, poisoned, and what its sessions hold on the host: quantised rows."""

    def __init__(self, dtype, d, page, hkv, ctx, seed=1, fill=0xFF, spare=5, pages=None):
        self.rng = np.random.default_rng(seed)
        self.dtype, self.d, self.page, self.hkv = dtype, d, page, hkv
        need = [-(-c // page) for c in ctx]
        n = sum(need) + spare
        self.cache = B.KVCacheQ8(pages or n, page, hkv, d, AG[dtype], DEV, fill=fill)
        ids = self.rng.permutation(n)
        self.bt = np.zeros((len(ctx), max(max(need), 1)), np.int32)
        at = 0
        for s, k in enumerate(need):
            self.bt[s, :k] = ids[at:at + k]
            at += k
        self.bt_dev = i32(self.bt)
        self.k = [np.zeros((0, hkv, d)) for _ in ctx]
        self.v = [np.zeros((0, hkv, d)) for _ in ctx]

    def draw(self, *shape, sigma=1.0):
        x = (self.rng.standard_normal(shape) * sigma).astype(np.float32)
        return Q.bf16(x) if self.dtype == "bf16" else x

    def dev(self, x):
        return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(DEV).to(TD[self.dtype])

    def lens(self):
        return np.array([k.shape[0] for k in self.k])

    def append(self, new, k=None, v=None, bound=None, stream=None):
        """`new` tokens to every session; bound: total_new, more rows than there are."""
        new = np.asarray(new)
        t = int(new.sum())
        sizes = np.exp2(self.rng.integers(-2, 3, (t, self.hkv, 1)))
        k = self.draw(t, self.hkv, self.d) if k is None else k
        v = (self.draw(t, self.hkv, self.d) * sizes).astype(np.float32) if v is None else v
        extra = np.full(((bound or t) - t, self.hkv, self.d), 7.0)
        args = [self.dev(np.concatenate([x, extra])) for x in (k, v)] + [self.bt_dev, i32(self.lens()), i32(new), i32(np.concatenate([[0], np.cumsum(new)]))]
        torch.cuda.synchronize()
        B.ag_kv_append_q8(self.cache, *args, bound or t, stream)
        torch.cuda.synchronize()
        at = 0
        for s, n in enumerate(new):
            for mine, x in ((self.k, k), (self.v, v)):
                mine[s] = np.concatenate([mine[s], Q.values(*Q.quantise(x[at:at + n]))])
            at += n

    def stored(self, s):
        """Session s's rows as the pools hold them."""
        n, out = self.lens()[s], []
        pos = np.arange(n)
        pages, slots = torch.from_numpy(self.bt[s, pos // self.page].astype(np.int64)).to(DEV), torch.from_numpy(pos % self.page).to(DEV)
        for pool, e in zip((self.cache.k_pool_token_major(), self.cache.v_pool_token_major()), self.cache.exps_token_major()):
            out.append((pool[pages, :, slots].cpu().numpy(), e[pages, :, slots].cpu().numpy().astype(int) - 127))
        return out


def bounds(dtype, d, n, ref, size, reach):
    u, w = (2.0 ** -8, 2 * 2.0 ** -8) if dtype == "bf16" else (2.0 ** -24, 2 * 2.0 ** -24)
    return u * np.abs(ref) + size * (w + 2 * (d + 4) * 2.0 ** -24 * reach[..., None] + 2 * (n + 16) * 2.0 ** -24) + 1e-30


def check(dtype, got, q, k, v, prefix, scale, what=""):
    ref, size, reach = Q.attend(q, k, v, prefix, scale)
    d, n = q.shape[-1], k.shape[0]
    assert np.isfinite(got).all(), what
    err, most = np.abs(got - ref), bounds(dtype, d, n, ref, size, reach)
    assert (err <= most).all(), (what, float((err / most).max()))
    return err, ref, most


def check_norm(dtype, d, errs, refs, mosts, what=""):
    e, r, m = (np.concatenate([x.ravel() for x in y]) for y in (errs, refs, mosts))
    rel = np.linalg.norm(e) / max(np.linalg.norm(r), 1e-30)
    if dtype == "bf16":
        assert np.linalg.norm(e) <= 0.5 * np.linalg.norm(m), (what, rel)
    else:
        assert rel <= (4e-6 if d <= 128 else 6e-6), (what, rel)


def decode(side, q, hq, scale, ctx=None, max_ctx=None, ws_fill=float("nan"), stream=None):
    ctx = side.lens() if ctx is None else np.asarray(ctx)
    max_ctx = int(ctx.max()) if max_ctx is None else max_ctx
    nbytes = B.ag_attn_decode_q8_workspace_bytes(len(ctx), hq, side.d, max_ctx)
    ws = torch.full((nbytes // 4,), ws_fill, dtype=torch.float32, device=DEV)
    out = torch.full((len(ctx), hq, side.d), float("nan"), dtype=TD[side.dtype], device=DEV)
    args = side.dev(q), i32(ctx)
    pages = max(side.bt.shape[1], -(-max_ctx // side.page))          # a larger bound than there are tokens: pages that no session has
    bt = i32(np.pad(side.bt, ((0, 0), (0, pages - side.bt.shape[1]))))
    torch.cuda.synchronize()
    B.ag_attn_decode_q8(side.cache, args[0], out, bt, args[1], max_ctx, hq, scale, ws, stream)
    torch.cuda.synchronize()
    return out


def resume(side, q, new, hq, scale, cold=False, bound=None, stream=None):
    """The last new[s] tokens of every session attend."""
    new = np.asarray(new)
    t = int(new.sum())
    out = torch.full((bound or t, hq, side.d), 5.0, dtype=TD[side.dtype], device=DEV)
    qd = side.dev(np.concatenate([q, np.zeros(((bound or t) - t,) + q.shape[1:])]))
    lens, cu = i32(new), i32(np.concatenate([[0], np.cumsum(new)]))
    prefix, ctx = side.lens() - new, side.lens()
    prefix_dev = i32(prefix)
    torch.cuda.synchronize()
    if cold:
        assert not prefix.any()
        B.ag_attn_prefill_q8(side.cache, qd, out, side.bt_dev, lens, cu, bound or t, int(new.max()), hq, scale, stream)
    else:
        B.ag_attn_resume_q8(side.cache, qd, out, side.bt_dev, prefix_dev, lens, cu, bound or t, int(new.max()), int(ctx.max()), hq, scale, stream)
    torch.cuda.synchronize()
    assert bool((out[t:] == 5.0).all()), "rows of nobody"
    return out[:t]


def check_decode(side, q, out, scale, what, ctx=None):
    got = out.double().cpu().numpy()
    found = []
    for s, n in enumerate(side.lens() if ctx is None else ctx):
        if n == 0:
            assert not got[s].any(), what
        else:
            found.append(check(side.dtype, got[s:s + 1], q[s:s + 1], side.k[s][:n], side.v[s][:n], n - 1, scale, (what, s)))
    check_norm(side.dtype, side.d, *zip(*found), what)


def check_resume(side, q, out, new, scale, what):
    got, at, found = out.double().cpu().numpy(), 0, []
    for s, n in enumerate(new):
        if n:
            found.append(check(side.dtype, got[at:at + n], q[at:at + n], side.k[s], side.v[s], len(side.k[s]) - n, scale, (what, s)))
        at += n
    check_norm(side.dtype, side.d, *zip(*found), what)


GEOMETRIES = [(128, 16), (128, 64), (64, 16), (64, 32), (256, 16), (16, 16), (48, 128), (80, 64), (96, 32), (112, 16), (176, 32), (192, 16), (208, 256), (240, 16)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", GEOMETRIES)
def test_append_and_read_back_to_the_bit(dtype, d, page):
    """Ragged pieces that begin and end inside groups and pages, one after the other; every byte that is nobody's stays."""
    lens = [(0, 1, 15, 16, 17, 3), (1, 1, 1, 1, 1, 1), (31, 0, 130, 16, 32, 2), (0, 0, 0, 0, 0, 257)]
    side = Side(dtype, d, page, 3, np.sum(lens, 0), seed=d + page, fill=0xA5)
    for i, new in enumerate(lens):
        side.append(new, bound=int(np.sum(new)) + (0, 40, 1, 0)[i])
    mine = np.zeros((side.cache.num_pages, page), bool)
    for s in range(6):
        for (byte, e), want in zip(side.stored(s), (side.k[s], side.v[s])):
            assert np.array_equal(Q.values(byte, e), want), (s, d, page)
        pos = np.arange(side.lens()[s])
        mine[side.bt[s, pos // page], pos % page] = True
    for pool in (side.cache.k_pool_token_major(), side.cache.v_pool_token_major(), *side.cache.exps_token_major()):
        assert bool((pool.cpu().numpy().swapaxes(1, 2)[~mine] == 0xA5).all())
    # back as rows, all of it and pieces of it, with a bound that is more than there is
    for first, n in [(np.zeros(6, int), side.lens()), (side.lens() // 3, side.lens() // 2), (side.lens() - np.minimum(side.lens(), 1), np.minimum(side.lens(), 1))]:
        t = int(n.sum())
        out = [torch.full((t + 3, 3, d), 9.0, dtype=TD[dtype], device=DEV) for _ in range(2)]
        B.ag_kv_read_q8(side.cache, *out, side.bt_dev, i32(first), i32(n), i32(np.concatenate([[0], np.cumsum(n)])), t + 3)
        torch.cuda.synchronize()
        for got, want in zip(out, (side.k, side.v)):
            assert np.array_equal(got[:t].double().cpu().numpy(), np.concatenate([w[f:f + c] for w, f, c in zip(want, first, n)]))
            assert bool((got[t:] == 9.0).all())


@pytest.mark.parametrize("dtype,d,hkv", [("bf16", 64, 8), ("bf16", 128, 6), ("f32", 48, 4), ("f32", 128, 2)])
def test_many_groups_take_several_heads_a_workgroup(dtype, d, hkv):
    """Past 8192 (group, head) pairs (test_q8_dispatch.py has the line): bytes as before, appended and read back, ragged."""
    new = [40] * (8192 // (4 * hkv) + 60) + [1, 17, 33]
    side = Side(dtype, d, 32, hkv, new, seed=d, fill=0xA5)
    side.append(new)
    n, t = np.array(new), sum(new)
    out = [torch.full((t + 1, hkv, d), 9.0, dtype=TD[dtype], device=DEV) for _ in range(2)]
    B.ag_kv_read_q8(side.cache, *out, side.bt_dev, i32(np.zeros(len(new))), i32(n), i32(np.concatenate([[0], np.cumsum(n)])), t + 1)
    torch.cuda.synchronize()
    for got, want in zip(out, (side.k, side.v)):
        assert np.array_equal(got[:t].double().cpu().numpy(), np.concatenate(want)) and bool((got[t:] == 9.0).all())
    mine = np.zeros((side.cache.num_pages, 32), bool)
    for s in range(len(new)):
        pos = np.arange(new[s])
        mine[side.bt[s, pos // 32], pos % 32] = True
    for pool in (side.cache.k_pool_token_major(), side.cache.v_pool_token_major(), *side.cache.exps_token_major()):
        assert bool((pool.cpu().numpy().swapaxes(1, 2)[~mine] == 0xA5).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_of_every_kind_of_number(dtype):
    """Rows of zeros, infinities, NaN, denormal and the largest numbers, ties, sizes at both sides of a power's end."""
    d = 64
    side = Side(dtype, d, 16, 2, [64])
    x = side.draw(48, 2, d) * np.exp2(side.rng.integers(-140, 125, (48, 2, 1))).astype(np.float64)
    x = x.astype(np.float32)
    x[0] = 0
    x[1, :, 1:] = 0
    x[2, 0, 3], x[2, 0, 4], x[2, 1, 5] = np.inf, -np.inf, np.nan
    x[3] = np.nan
    x[4, :, 0] = np.float32(3.3e38)
    x[5] = np.float32(1e-40)
    for i, v in enumerate((448.0, 449.0, 450.0, 447.0, 224.0, 225.0, 1.75, 1.7578125)):
        x[6 + i] = np.sign(x[6 + i]) * np.minimum(np.abs(x[6 + i]), 1)
        x[6 + i, :, 7] = v
        x[6 + i, :, 8:40] = (2 * np.arange(32) + 1) * 2.0 ** -10          # ties of the subnormals
        x[6 + i, :, 40:60] = 16 + np.arange(20) * 0.5                     # ... and of larger ones
        x[6 + i] = np.minimum(x[6 + i], v)
    x = Q.bf16(x) if dtype == "bf16" else x
    x[3] = np.nan
    x[2, 0, 3], x[2, 0, 4], x[2, 1, 5] = np.inf, -np.inf, np.nan
    side.append([48], k=x, v=x[::-1].copy())
    for (byte, e), rows in zip(side.stored(0), (x, x[::-1])):
        want = Q.quantise(rows)
        assert np.array_equal(e, want[1]) and np.array_equal(Q.values(byte, e), Q.values(*want), equal_nan=True)



@pytest.fixture(scope="module")
def few_cus():
    """A stream of eight CUs, on which small batches are many workgroups."""
    stream = B.ag_stream_create_cumask(B.ag_cumask_build(256, 8, 0, 1))
    yield stream
    torch.cuda.synchronize()
    B.ag_stream_destroy(stream)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", GEOMETRIES)
def test_decode(few_cus, dtype, d, page):
    """Contexts of none, one and every few tokens around the ends of groups, pages, steps and shares; stale slots are NaN under infinite powers.
    One workgroup a pair, and with a larger bound shares (test_q8_dispatch.py), also on few CUs, where they are longer."""
    ctx = [0, 1, 15, 16, 17, 63, 64, 65, 0, 127, 200, 513, 1100]
    side = Side(dtype, d, page, 2, ctx, seed=d)
    side.append(ctx)
    hq = 8
    q = side.draw(len(ctx), hq, d)
    for max_ctx, stream in ((None, None), (SHARED_CTX, None), (SHARED_CTX, few_cus)):
        check_decode(side, q, decode(side, q, hq, d ** -0.5, max_ctx=max_ctx, stream=stream), d ** -0.5, (dtype, d, page))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (6, 2), (3, 3), (16, 1), (24, 1), (40, 2), (17, 1), (32, 8)])
def test_decode_groups(few_cus, dtype, hq, hkv):
    ctx = [5, 700, 64, 129] + [1] * 6
    side = Side(dtype, 128, 16, hkv, ctx, seed=hq)
    side.append(ctx)
    q = side.draw(len(ctx), hq, 128)
    for max_ctx, stream in ((None, None), (SHARED_CTX, None), (SHARED_CTX, few_cus)):
        check_decode(side, q, decode(side, q, hq, 0.11, max_ctx=max_ctx, stream=stream), 0.11, (hq, hkv))


def test_decode_of_many_sessions_and_of_a_long_one():
    """More sessions than a wave scans at once, most of them empty; then one context over many shares, and the same bits again."""
    ctx = [(7 * s) % 90 if s % 3 else 0 for s in range(150)]
    side = Side("bf16", 64, 16, 1, ctx)
    side.append(ctx)
    q = side.draw(len(ctx), 4, 64)
    for max_ctx in (None, SHARED_CTX):                            # one workgroup a pair, and shares
        check_decode(side, q, decode(side, q, 4, 0.125, max_ctx=max_ctx), 0.125, "many")
    side = Side("bf16", 128, 16, 2, [20000])
    side.append([20000])
    q = side.draw(1, 8, 128)
    out = decode(side, q, 8, 0.09)
    check_decode(side, q, out, 0.09, "long")
    again = decode(side, q, 8, 0.09, ws_fill=3.0)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))
    # the context counts what is attended, not what is there
    q2 = side.draw(1, 8, 128)
    check_decode(side, q2, decode(side, q2, 8, 0.09, ctx=[4097], max_ctx=20000), 0.09, "shorter", ctx=[4097])


NEW = {"short": ([0, 3, 40, 100, 17], [1, 2, 7, 0, 33]), "prompts": ([0] * 5, [1, 64, 130, 0, 70]), "long": ([700, 64, 1000], [150, 64, 9])}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", GEOMETRIES)
@pytest.mark.parametrize("lens", list(NEW))
def test_prefill_and_resume(dtype, d, page, lens):
    prefix, new = (np.array(x) for x in NEW[lens])
    hq, hkv = {"short": (6, 2), "prompts": (4, 4), "long": (16, 2)}[lens]
    side = Side(dtype, d, page, hkv, prefix + new, seed=d)
    if prefix.any():
        side.append(prefix)
    side.append(new)
    q = side.draw(int(new.sum()), hq, d)
    out = resume(side, q, new, hq, d ** -0.5, bound=int(new.sum()) + 2)
    check_resume(side, q, out, new, d ** -0.5, (lens, d, page))
    if not prefix.any():
        cold = resume(side, q, new, hq, d ** -0.5, cold=True)
        assert torch.equal(cold.view(torch.uint8), out.view(torch.uint8))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", GEOMETRIES)
@pytest.mark.parametrize("lens", list(TILED))
def test_whole_tiles(few_cus, dtype, d, page, lens):
    prefix, new = (np.array(x) for x in TILED[lens])
    hq, hkv = 16, 2
    side = Side(dtype, d, page, hkv, prefix + new, seed=d)
    if prefix.any():
        side.append(prefix)
    side.append(new)
    q = side.draw(int(new.sum()), hq, d)
    out = resume(side, q, new, hq, d ** -0.5, bound=int(new.sum()) + 2, stream=few_cus)
    check_resume(side, q, out, new, d ** -0.5, (lens, d, page))
    if not prefix.any():
        cold = resume(side, q, new, hq, d ** -0.5, cold=True, stream=few_cus)
        assert torch.equal(cold.view(torch.uint8), out.view(torch.uint8))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(128, 16), (64, 32), (96, 16), (48, 128)])
def test_few_rows_by_four_waves(few_cus, dtype, d, page):
    prefix, new = (np.array(x) for x in FOUR_LENS)
    side = Side(dtype, d, page, 2, prefix + new, seed=d)
    side.append(prefix)
    side.append(new)
    q = side.draw(int(new.sum()), 16, d)
    check_resume(side, q, resume(side, q, new, 16, d ** -0.5, stream=few_cus), new, d ** -0.5, (d, page))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,prefix,new", [(32, 8, [300, 900], [300, 41]), (24, 1, [50], [90]), (1, 1, [2000], [5]), (8, 2, [0] * 70, list(range(70))),
                                               (16, 1, [1500, 0, 20], [260, 515, 1])])
def test_resume_groups_and_batches(dtype, hq, hkv, prefix, new):
    prefix, new = np.array(prefix), np.array(new)
    side = Side(dtype, 128, 16, hkv, prefix + new, seed=hq)
    if prefix.any():
        side.append(prefix)
    side.append(new)
    q = side.draw(int(new.sum()), hq, 128)
    check_resume(side, q, resume(side, q, new, hq, 0.09), new, 0.09, (hq, hkv))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sharp_scores_and_rising_ones(few_cus, dtype):
    """Logits of standard deviation 20: nearly one key a row; and keys whose scores rise along the context, so that every tile moves the maximum."""
    d, hkv, hq = 128, 2, 8
    new = [190]
    side = Side(dtype, d, 16, hkv, [190 + 300])
    k = side.draw(300, hkv, d)
    ramp = np.linspace(0, 8, 300)[:, None, None] * np.ones((1, hkv, d))
    side.append([300], k=(k + ramp).astype(np.float32) if dtype == "f32" else Q.bf16(k + ramp), v=side.draw(300, hkv, d))
    side.append(new)
    q = side.draw(190, hq, d)
    q[::2] = np.abs(q[::2])                                       # (against the ramp: up to 8 * 128 * 0.8 * scale = 70)
    scale = 0.09 * 2
    for stream in (None, few_cus):
        got = resume(side, q, new, hq, scale, stream=stream).double().cpu().numpy()
        check(dtype, got, q, side.k[0], side.v[0], 300, scale, "resume")
    check(dtype, decode(side, q[-1:], hq, scale).double().cpu().numpy(), q[-1:], side.k[0], side.v[0], 489, scale, "decode")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_and_infinities_stay_with_the_rows_that_see_them(few_cus, dtype):
    """A NaN key reaches the rows at and behind it; a session beside it, and decode before it, do not notice."""
    side = Side(dtype, 64, 16, 1, [80, 80])
    k, v = side.draw(160, 1, 64), side.draw(160, 1, 64)
    k[40, 0, 3] = np.inf
    side.append([80, 80], k=k, v=v)
    q = side.draw(160, 2, 64)
    for stream in (None, few_cus):
        out = resume(side, q, [80, 80], 2, 0.125, stream=stream).double().cpu().numpy()
        assert np.isnan(out[40:80]).all() and np.isfinite(out[:40]).all() and np.isfinite(out[80:]).all()
        check(dtype, out[80:], q[80:], side.k[1], side.v[1], 0, 0.125)
    got = decode(side, q[:2], 2, 0.125, ctx=[40, 80]).double().cpu().numpy()
    check(dtype, got[:1], q[:1], side.k[0][:40], side.v[0][:40], 39, 0.125)
    check(dtype, got[1:], q[1:2], side.k[1], side.v[1], 79, 0.125)


def seeing(side, s, prefix, n, hq):
    """[n][hq][d]: outputs that a value of session s that is not finite reaches."""
    bad = ~np.isfinite(side.v[s])                                 # [context][hkv][d]
    seen = np.cumsum(bad, 0)[prefix:prefix + n] > 0
    return np.repeat(seen, hq // side.hkv, axis=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", GEOMETRIES)
@pytest.mark.parametrize("lens,few,hq,hkv", [*((n, True, 16, 2) for n in TILED), *((n, False, 16, 2) for n in NEW), ("four", True, 16, 2), ("ragged", True, 3, 3),
                                             ("long", True, 2, 2), ("ragged", True, 48, 1)])
def test_values_that_are_not_finite_stay_with_the_rows_that_see_them(few_cus, dtype, d, page, lens, few, hq, hkv):
    """In prefixes, at the first, the last and other new tokens, in one channel each; by whole tiles and by few rows (test_q8_dispatch.py)."""
    prefix, new = (np.array(x) for x in {**NEW, **TILED, "four": FOUR_LENS}[lens])
    side = Side(dtype, d, page, hkv, prefix + new, seed=d + hq)
    if prefix.any():
        side.append(prefix)
    t, scale = int(new.sum()), d ** -0.5
    v, at = side.draw(t, hkv, d), 0
    for s, n in enumerate(new):
        for i, x in ((0, np.inf), (n // 3, np.nan), (n // 2 + 1, -np.inf), (n - 1, np.inf)):
            if 0 <= i < n and (s + i) % 3:
                v[at + i, i % hkv, (5 * i + 11 * s + 3) % d] = x
        at += n
    side.append(new, v=v)
    q = side.draw(t, hq, d)
    got, at = resume(side, q, new, hq, scale, stream=few_cus if few else None).double().cpu().numpy(), 0
    clean = [np.where(np.isfinite(x), x, 0) for x in side.v]
    for s, n in enumerate(new):
        if n:
            o, p = got[at:at + n], int(prefix[s])
            seen = seeing(side, s, p, n, hq)
            assert np.array_equal(np.isnan(o), seen), (s, np.argwhere(np.isnan(o) != seen)[:5])
            ref = Q.attend(q[at:at + n], side.k[s], clean[s], p, scale)[0]
            check(dtype, np.where(seen, ref, o), q[at:at + n], side.k[s], clean[s], p, scale, (lens, s))
        at += n
    ctx = prefix + np.where(new > 0, new // 2 + 1, 0)
    q1 = side.draw(len(new), hq, d)
    for bound in (None, SHARED_CTX):
        got = decode(side, q1, hq, scale, ctx=ctx, max_ctx=bound).double().cpu().numpy()
        for s, n in enumerate(ctx):
            if n:
                assert np.array_equal(np.isnan(got[s]), seeing(side, s, n - 1, 1, hq)[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_powers_of_two_change_no_bit(few_cus, dtype, d):
    """Keys and queries by opposite powers, values by any in the documented range: every rounding is relative, so that the outputs are the
    same but for the power (scores are small: no weight below 2^-20)."""
    lens, new, hq, hkv, scale = [300, 77], [120, 77], 8, 2, d ** -0.5 / 4
    outs = []
    for kq, pv in ((0, 0), (40, 60), (-40, -60)):
        side = Side(dtype, d, 16, hkv, lens, seed=3)
        old = [n - m for n, m in zip(lens, new)]
        for n in (old, new):
            k, v = (side.draw(sum(n), hkv, d) for _ in range(2))
            side.append(n, k=np.ldexp(k, kq).astype(np.float32), v=np.ldexp(v, pv).astype(np.float32))
        q = np.ldexp(side.draw(sum(new), hq, d), -kq)
        got = [resume(side, q, new, hq, scale), resume(side, q, new, hq, scale, stream=few_cus)]
        got += [decode(side, q[:2], hq, scale), decode(side, q[:2], hq, scale, max_ctx=SHARED_CTX)]
        outs.append([np.ldexp(x.double().cpu().numpy(), -pv) for x in got])
    for other in outs[1:]:
        for x, y in zip(outs[0], other):
            assert np.array_equal(x, y)


def test_a_session_from_prompt_to_decode():
    """The operators together: prompt appended and attended, a tool's output behind it, then decode steps; read back and appended elsewhere,
    the same outputs to the bit."""
    for dtype, d, page in (("bf16", 128, 16), ("f32", 64, 32)):
        hq, hkv, scale = 8, 2, d ** -0.5
        side = Side(dtype, d, page, hkv, [400, 333, 90])
        for new, cold in (([150, 80, 0], True), ([37, 100, 61], False), ([200, 1, 5], False)):
            side.append(new)
            q = side.draw(int(np.sum(new)), hq, d)
            if cold:
                check_resume(side, q, resume(side, q, new, hq, scale, cold=True), new, scale, "cold")
            else:
                check_resume(side, q, resume(side, q, new, hq, scale), new, scale, "resume")
        for step in range(4):
            side.append([1, 1, 1 if step else 0])
            q = side.draw(3, hq, d)
            out = decode(side, q, hq, scale)
            check_decode(side, q, out, scale, step)
        n = side.lens()
        rows = [torch.empty((int(n.sum()), hkv, d), dtype=TD[dtype], device=DEV) for _ in range(2)]
        prefix, new, cu = i32(np.zeros(3)), i32(n), i32(np.concatenate([[0], np.cumsum(n)]))
        B.ag_kv_read_q8(side.cache, *rows, side.bt_dev, prefix, new, cu, int(n.sum()))
        other = B.KVCacheQ8(side.cache.num_pages, page, hkv, d, AG[dtype], DEV, fill=0x7F)
        B.ag_kv_append_q8(other, *rows, side.bt_dev, prefix, new, cu, int(n.sum()))
        side.cache = other
        assert torch.equal(decode(side, q, hq, scale).view(torch.uint8), out.view(torch.uint8))


def test_pools_past_four_gigabytes():
    """Pages whose offsets do not fit 32 bits, in every operator."""
    pages = (5 << 30) // (16 * 8 * 128)
    ctx = [100, 33]
    side = Side("bf16", 128, 16, 8, ctx, fill=0, pages=pages)
    side.bt[:] = pages - 1 - side.bt
    side.bt_dev = i32(side.bt)
    side.append([60, 33])
    side.append([40, 0])
    for s in range(2):
        n = side.lens()[s]
        out = [torch.empty((n, 8, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        B.ag_kv_read_q8(side.cache, *out, side.bt_dev[s:s + 1].contiguous(), i32([0]), i32([n]), i32([0, n]), int(n))
        torch.cuda.synchronize()
        assert np.array_equal(out[0].double().cpu().numpy(), side.k[s]) and np.array_equal(out[1].double().cpu().numpy(), side.v[s])
    q = side.draw(2, 16, 128)
    check_decode(side, q, decode(side, q, 16, 0.09), 0.09, "decode")
    q = side.draw(40, 16, 128)
    out = resume(side, q, [40, 0], 16, 0.09)
    check_resume(side, q, out, [40, 0], 0.09, "resume")


def test_calls_on_two_streams_and_in_graphs():
    """Two decode steps and a resume side by side on their own streams, and a whole step - append, decode, resume - captured and replayed
    with eager work between."""
    side = Side("bf16", 128, 16, 2, [700, 300, 64], seed=9)
    side.append([640, 290, 60])
    side.append([1, 1, 1])
    hq, scale = 8, 0.09
    qs = [side.draw(3, hq, 128) for _ in range(3)]
    ctx, max_ctx = i32(side.lens()), int(side.lens().max())
    want = [decode(side, q, hq, scale) for q in qs[:2]]
    rq, new = side.dev(qs[2]), i32([1, 1, 1])
    cu, prefix = i32([0, 1, 2, 3]), i32(side.lens() - 1)
    want.append(torch.empty_like(rq))
    B.ag_attn_resume_q8(side.cache, rq, want[2], side.bt_dev, prefix, new, cu, 3, 1, max_ctx, hq, scale)
    nbytes = B.ag_attn_decode_q8_workspace_bytes(3, hq, 128, max_ctx)
    ws = [torch.empty(nbytes, dtype=torch.uint8, device=DEV) for _ in range(2)]
    qd = [side.dev(q) for q in qs]
    got = [torch.zeros_like(x) for x in want]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(5):
        B.ag_attn_decode_q8(side.cache, qd[0], got[0], side.bt_dev, ctx, max_ctx, hq, scale, ws[0], streams[0])
        B.ag_attn_decode_q8(side.cache, qd[1], got[1], side.bt_dev, ctx, max_ctx, hq, scale, ws[1], streams[1].cuda_stream)
        B.ag_attn_resume_q8(side.cache, rq, got[2], side.bt_dev, prefix, new, cu, 3, 1, max_ctx, hq, scale, streams[2])
        torch.cuda.synchronize()
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(got, want))

    k, v = (side.dev(side.draw(3, 2, 128)) for _ in range(2))
    back = [torch.empty_like(k) for _ in range(2)]

    def step():
        B.ag_kv_append_q8(side.cache, k, v, side.bt_dev, prefix, new, cu, 3)
        B.ag_attn_decode_q8(side.cache, qd[0], got[0], side.bt_dev, ctx, max_ctx, hq, scale, ws[0])
        B.ag_attn_resume_q8(side.cache, rq, got[2], side.bt_dev, prefix, new, cu, 3, 1, max_ctx, hq, scale)
        B.ag_kv_read_q8(side.cache, *back, side.bt_dev, prefix, new, cu, 3)

    step()
    torch.cuda.synchronize()
    eager = [x.clone() for x in (got[0], got[2], *back)]
    spare = int(np.setdiff1d(np.arange(side.cache.num_pages), side.bt.ravel())[0])
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=other):
        step()
    for r in range(4):
        for x in (got[0], got[2], *back):
            x.fill_(float("nan"))
        ws[0].random_()
        side.cache.k_pool.view(torch.uint8)[spare] = r
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip((got[0], got[2], *back), eager)), r


@pytest.mark.parametrize("dtype,d,hq,new", [("bf16", 128, 16, [130, 40, 1]), ("f32", 96, 6, [9, 140, 33]), ("bf16", 192, 4, [64, 1, 200])])
def test_replays_of_every_kernel(few_cus, dtype, d, hq, new):
    """Decode in shares with its merge, prefill by few rows and, on few CUs, by whole tiles: captured, and replayed over dirty workspaces."""
    side = Side(dtype, d, 16, 2, [700, 300, 260], seed=9)
    old = [n - m for n, m in zip([700, 300, 260], new)]
    side.append(old)
    side.append(new)
    t, scale, s = sum(new), d ** -0.5, torch.cuda.ExternalStream(few_cus)
    lens, cu, prefix, ctx = i32(new), i32(np.concatenate([[0], np.cumsum(new)])), i32(old), i32(side.lens())
    bt = i32(np.pad(side.bt, ((0, 0), (0, SHARED_CTX // 16 - side.bt.shape[1]))))
    q, q1 = side.dev(side.draw(t, hq, d)), side.dev(side.draw(3, hq, d))
    ws = torch.empty(B.ag_attn_decode_q8_workspace_bytes(3, hq, d, SHARED_CTX), dtype=torch.uint8, device=DEV)
    got = [torch.empty_like(q), torch.empty_like(q1)]

    def step():
        B.ag_attn_resume_q8(side.cache, q, got[0], bt, prefix, lens, cu, t, max(new), 700, hq, scale)
        B.ag_attn_decode_q8(side.cache, q1, got[1], bt, ctx, SHARED_CTX, hq, scale, ws)

    for stream in (torch.cuda.Stream(), s):
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            step()
        torch.cuda.synchronize()
        eager = [x.clone() for x in got]
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
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, eager)), r


def test_plain_calls_and_those_through_ctypes_are_the_same(monkeypatch):
    outs = []
    for calls in (B._calls(), B._NoCalls()):
        monkeypatch.setattr(B, "_native", calls)
        side = Side("bf16", 64, 32, 2, [90, 40], seed=3, fill=0)
        side.append([80, 40])
        side.append([10, 0])
        q = side.draw(10, 4, 64)
        rows = [torch.empty((10, 2, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        B.ag_kv_read_q8(side.cache, *rows, side.bt_dev, i32([80, 40]), i32([10, 0]), i32([0, 10, 10]), total_new=10, stream=None)
        outs.append([side.cache.k_pool, side.cache.v_pool, side.cache.exps, resume(side, q, [10, 0], 4, 0.1), decode(side, q[:2], 4, 0.1), *rows])
    assert all(torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)) for a, b in zip(*outs))
