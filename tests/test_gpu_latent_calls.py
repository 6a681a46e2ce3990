"""The rotating append and the latent cache as a serving loop uses them, and calls that their headers allow beside the usual ones: whole steps, replayed graphs, masked and
side streams, workspaces of the exact size, both ways into the library, batches drawn at random."""
import numpy as np
import pytest
import torch

import latent_oracle as O
from gpu_helpers import i32
from paper_2603_10342_amd import binding as B
from test_gpu_latent import DEV, Side, check_decode, check_resume, decode, resume
from test_gpu_rope import make_rope, same_bits

pytestmark = pytest.mark.gpu


def guarded(nbytes):
    """A workspace of exactly nbytes, and what stands behind it."""
    whole = torch.full((nbytes + 256,), 0x5A, dtype=torch.uint8, device=DEV)
    return whole[:nbytes], whole[nbytes:]


# ---- steps ----

@pytest.mark.parametrize("heads", [16, 128])
def test_a_serving_loop_over_latent_rows(heads):
    """Prompts appended with their rotation, a chunk attending, then steps: the step's rows appended, its queries' rotary slices rotated into place, attention - against
    rotations and attention in 64 bits of the rows that went in."""
    lat, rd, page, scale = 512, 64, 32, 0.05
    rope, t = make_rope(rd, "pairs", 1.1)
    rng = np.random.default_rng(2)
    lens = np.array([70, 33, 128])
    room, batch = 160, 3
    cache = B.LatentCache(batch * room // page, page, lat, rd, DEV, fill=float("nan"))
    bt = i32(rng.permutation(batch * room // page).reshape(batch, -1))
    keys = [np.zeros((0, lat + rd)) for _ in range(batch)]

    def rows(n):
        x = torch.randn(n, lat + rd, device=DEV).bfloat16()
        return x, x.double().cpu().numpy()

    def attend(new, prefix):
        """Appends new[s] rows and queries them; checks every output."""
        total, cu = int(new.sum()), np.concatenate([[0], np.cumsum(new)])
        x, x64 = rows(total)
        at = i32(prefix), i32(new), i32(cu)
        B.ag_kv_append_latent(cache, rope, x[:, :lat], x[:, lat:], bt, *at, total)
        q_nope, q_rot = torch.randn(total, heads, lat, device=DEV).bfloat16(), torch.randn(total, heads, 192, device=DEV).bfloat16()
        q = torch.empty(total, heads, lat + rd, dtype=torch.bfloat16, device=DEV)
        q[..., :lat] = q_nope
        B.ag_rope_rows(rope, q_rot[..., 128:], q[..., lat:], *at, total)
        out = torch.empty(total, heads, lat, dtype=torch.bfloat16, device=DEV)
        max_ctx = int((prefix + new).max())
        if (new == 1).all():
            ws, behind = guarded(B.ag_attn_decode_latent_workspace_bytes(batch, heads, lat, max_ctx))
            B.ag_attn_decode_latent(cache, q, out, bt, i32(prefix + new), max_ctx, heads, scale, ws)
        else:
            ws, behind = guarded(B.ag_attn_resume_latent_workspace_bytes(batch, total, heads, lat, max_ctx))
            B.ag_attn_resume_latent(cache, q, out, bt, *at, total, int(new.max()), max_ctx, heads, scale, ws)
        torch.cuda.synchronize()
        assert bool((behind == 0x5A).all())
        for s in range(batch):
            r = slice(cu[s], cu[s + 1])
            pos = prefix[s] + np.arange(new[s])
            turned, _ = O.rotate(x64[r, lat:], pos, t, "pairs", 1.1)
            keys[s] = np.concatenate([keys[s], np.concatenate([x64[r, :lat], turned], 1)])
            qr, _ = O.rotate(q_rot[r, :, 128:].double().cpu().numpy(), pos, t, "pairs", 1.1)
            o, size, spread, reach = O.attend(np.concatenate([q_nope[r].double().cpu().numpy(), qr], -1), keys[s], lat, prefix[s], scale)
            # queries' and keys' rotated channels are rounded to bf16, 2^-8 each: a score is off by up to 2 * 2^-8 of its rotary part, |q_r| |r| scale <= reach here
            most = O.elementwise(o, size, reach, lat + rd, len(keys[s])) + 2 * 2 * O.HALF_STEP * reach[..., None] * size
            assert (np.abs(out[r].double().cpu().numpy() - o) <= most).all()

    attend(lens, np.zeros(batch, int))                                          # whole prompts
    attend(np.array([5, 20, 1]), lens)                                          # chunks on them
    lens = lens + [5, 20, 1]
    for _ in range(3):
        attend(np.ones(batch, int), lens)
        lens = lens + 1


def test_a_serving_loop_with_the_rotating_append():
    """ag_kv_append_rope and decode over a paged cache against attention in 64 bits."""
    hq, hkv, d, page, scale = 8, 2, 128, 16, 0.09
    rope, t = make_rope(64, "halves")
    cache, bt, keys, values = B.KVCache(8, page, hkv, d, B.AG_BF16, DEV, fill=float("nan")), i32([[5, 2, 7, 0]]), [], []
    at = 0
    for n in (40, 1, 1):
        q, k, v = (torch.randn(n, h, d, device=DEV).bfloat16() for h in (hq, hkv, hkv))
        out = torch.empty_like(q)
        B.ag_kv_append_rope(cache, rope, q, q, k_new := k, v, bt, i32([at]), i32([n]), i32([0, n]), n)
        keys.append(O.rotate(k_new.double().cpu().numpy(), at + np.arange(n), t, "halves")[0])
        values.append(v.double().cpu().numpy())
        if n == 1:
            ws = torch.empty(B.ag_attn_decode_workspace_bytes(1, hq, d, at + 1), dtype=torch.uint8, device=DEV)
            B.ag_attn_decode(cache, q, out, bt, i32([at + 1]), at + 1, hq, scale, ws)
        else:
            B.ag_attn_prefill(cache, q, out, bt, i32([n]), i32([0, n]), n, n, hq, scale)
        kk, vv, qq = np.concatenate(keys), np.concatenate(values), q.double().cpu().numpy()
        for h in range(hq):
            s = scale * qq[:, h] @ kk[:, h // 4].T
            s[np.arange(at + n)[None] > at + np.arange(n)[:, None]] = -np.inf
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            size = p @ np.abs(vv[:, h // 4])
            # keys of the cache are rounded, 2^-8 of |q| |k| scale of a score; weights and output 2^-8 each, as bounded in latent_oracle.py
            reach = (scale * np.abs(qq[:, h]) @ np.abs(kk[:, h // 4]).T).max(-1, keepdims=True)
            assert (np.abs(out[:, h].double().cpu().numpy() - p @ vv[:, h // 4]) <= O.HALF_STEP * (np.abs(p @ vv[:, h // 4]) + (2 + 2 * reach) * size) + 1e-5).all()
        at += n


# ---- graphs and streams ----

@pytest.mark.parametrize("heads", [8, 40, 128])
def test_a_replayed_step(heads):
    """Append, rotation of the queries and decode in one graph, replayed over new rows and longer contexts with eager work between; a second graph shares its workspace."""
    lat, rd, batch, max_ctx = 256, 32, 4, 400
    rope, _ = make_rope(rd, "halves")
    cache, eager = (B.LatentCache(batch * 25, 16, lat, rd, DEV, fill=0.5) for _ in range(2))
    bt = i32(np.random.default_rng(3).permutation(batch * 25).reshape(batch, 25))
    x, raw = torch.empty(batch, lat + rd, dtype=torch.bfloat16, device=DEV), torch.empty(batch, heads, lat + rd, dtype=torch.bfloat16, device=DEV)
    prefix, new, cu, ctx = i32([3, 100, 390, 31]), i32([1] * batch), i32(range(batch + 1)), i32([4, 101, 391, 32])
    q, out, want = torch.empty_like(raw), torch.empty(batch, heads, lat, dtype=torch.bfloat16, device=DEV), torch.empty(batch, heads, lat, dtype=torch.bfloat16, device=DEV)
    n = B.ag_attn_decode_latent_workspace_bytes(batch, heads, lat, max_ctx)
    ws, ws2 = torch.empty(n, dtype=torch.uint8, device=DEV), torch.empty(n, dtype=torch.uint8, device=DEV)

    def step(c, o, w):
        B.ag_kv_append_latent(c, rope, x[:, :lat], x[:, lat:], bt, prefix, new, cu, batch)
        q.copy_(raw)
        B.ag_rope_rows(rope, q[..., lat:], q[..., lat:], prefix, new, cu, batch)
        B.ag_attn_decode_latent(c, q, o, bt, ctx, max_ctx, heads, 0.06, w)

    for y in (x, raw):
        y.copy_(torch.randn_like(y))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cache, out, ws)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(cache, out, ws)
        graphs.append(g)
    for i in range(5):
        for y in (x, raw):
            y.copy_(torch.randn_like(y))
        out.fill_(float("nan"))
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        got = out.clone()
        step(eager, want, ws2)
        assert same_bits(got, want), i
        prefix.add_(1)
        ctx.add_(1)


def test_streams_with_few_cus_and_two_at_once():
    """Shares as a masked stream's CUs hold them (32, and 24 that no XCD count divides evenly); two calls at once on streams of their own."""
    info = B.ag_device_info()
    total, n_xcd = info["num_cus"], info["num_xcd"] or 8
    ctx, new = np.array([900, 20, 0, 333, 2000]), [3, 1, 0, 30, 5]
    side = Side(512, 64, 16, ctx)
    side.append(ctx)
    q, chunk = side.draw(5, 128, side.w), side.draw(sum(new), 48, side.w)
    streams = [B.ag_stream_create_cumask(B.ag_cumask_build(total, n_xcd, first, n)) for first, n in ((0, 4), (8, 3), (16, 8))]
    try:
        for s in streams:
            check_decode(side, q, 0.04, decode(side, q, 0.04, stream=s))
        outs = [torch.full((5, 128, 512), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in streams]
        spaces = [torch.empty(B.ag_attn_decode_latent_workspace_bytes(5, 128, 512, 2000), dtype=torch.uint8, device=DEV) for _ in streams]
        qd, bt, cd = side.dev(q), side.table(2000), i32(ctx)
        torch.cuda.synchronize()
        for _ in range(3):
            for s, o, w in zip(streams, outs, spaces):
                B.ag_attn_decode_latent(side.cache, qd, o, bt, cd, 2000, 128, 0.04, w, s)
        torch.cuda.synchronize()
        for o in outs:
            check_decode(side, q, 0.04, o.double().cpu().numpy())
    finally:
        for s in streams:
            B.ag_stream_destroy(s)
    check_resume(side, chunk, new, 0.04, resume(side, chunk, new, 0.04))


def test_both_ways_into_the_library(monkeypatch):
    """The calling module and ctypes: same bits."""
    rope, _ = make_rope(64, "pairs")

    def run():
        torch.manual_seed(5)
        cache, kv = B.LatentCache(8, 16, 512, 64, DEV, fill=0.0), B.KVCache(8, 16, 2, 64, B.AG_BF16, DEV, fill=0.0)
        x, q = torch.randn(20, 576, device=DEV).bfloat16(), torch.randn(20, 4, 576, device=DEV).bfloat16()
        bt, lens, out, one = i32([[3, 1, 6, 0]]), (i32([7]), i32([20]), i32([0, 20])), torch.empty(20, 4, 512, dtype=torch.bfloat16, device=DEV), torch.empty(1, 4, 512, dtype=torch.bfloat16, device=DEV)
        B.ag_kv_append_latent(cache, rope, x[:, :512], x[:, 512:], bt, *lens, 20)
        B.ag_rope_rows(rope, q[..., 512:], q[..., 512:], *lens, 20, True)
        ws = torch.empty(max(B.ag_attn_resume_latent_workspace_bytes(1, 20, 4, 512, 27), B.ag_attn_decode_latent_workspace_bytes(1, 4, 512, 27)), dtype=torch.uint8, device=DEV)
        B.ag_attn_resume_latent(cache, q, out, bt, *lens, 20, 20, 27, 4, 0.05, ws)
        B.ag_attn_decode_latent(cache, q[:1].contiguous(), one, bt, i32([27]), 27, 4, 0.05, ws)
        k, v, qq = (torch.randn(20, h, 64, device=DEV).bfloat16() for h in (2, 2, 4))
        B.ag_kv_append_rope(kv, rope, qq, qq, k, v, bt, *lens, 20)
        B.ag_kv_append_rope(kv, rope, None, None, k, v, bt, *lens, 20)
        return cache.pool, q, out, one, kv.k_pool, kv.v_pool, qq

    assert not isinstance(B._calls(), B._NoCalls)
    a = run()
    monkeypatch.setattr(B, "_native", B._NoCalls())
    assert all(same_bits(x, y) for x, y in zip(a, run()))


def test_what_python_refuses_before_the_library(monkeypatch):
    rope, _ = make_rope(64, "pairs")
    cache = B.LatentCache(2, 16, 512, 64, DEV, fill=2.0)
    x, bt, lens = torch.zeros(4, 576, dtype=torch.bfloat16, device=DEV), i32([[0, 1]]), (i32([0]), i32([4]), i32([0, 4]))
    for _ in range(2):
        for rows, what, error in ((x, 5, ValueError), (x.float(), 4, TypeError), (x.t().contiguous().t(), 4, ValueError), (x[:, 8:], 4, ValueError), (x.cpu(), 4, ValueError)):
            with pytest.raises(error):
                B.ag_kv_append_latent(cache, rope, rows[:, :512], rows[:, 512:], bt, *lens, what)
        q = x.view(4, 1, 576)[..., 512:]
        for rows, what, error in ((q, 5, ValueError), (q.half(), 4, TypeError), (q[:, 0], 4, ValueError)):
            with pytest.raises(error):
                B.ag_rope_rows(rope, rows, rows, *lens, what)
        torch.cuda.synchronize()
        assert bool((cache.pool == 2).all()) and bool((x == 0).all())
        monkeypatch.setattr(B, "_native", B._NoCalls())


# ---- batches drawn at random ----

@pytest.mark.parametrize("seed", range(24))
def test_random_batches(seed):
    rng = np.random.default_rng(100 + seed)
    lat, rd = [(512, 64), (512, 32), (256, 64), (256, 32), (128, 64), (128, 32)][rng.integers(6)]
    page, heads, batch = int(2 ** rng.integers(4, 9)), int(rng.choice([1, 2, 7, 16, 24, 32, 48, 64, 96, 128, 130])), int(rng.integers(1, 20))
    ctx = rng.integers(0, int(2 ** rng.integers(4, 11)), batch)
    side = Side(lat, rd, page, ctx, seed=seed)
    side.append(ctx)
    scale = float(rng.uniform(0.5, 1.5)) * side.w ** -0.5
    loose = int(ctx.max()) + int(rng.integers(0, 5000))
    q = side.draw(batch, heads, side.w)
    if ctx.max() > 0:
        check_decode(side, q, scale, decode(side, q, scale, max_ctx=loose))
    new = np.minimum(ctx, rng.integers(0, int(2 ** rng.integers(1, 7)), batch))
    if new.sum():
        q = side.draw(int(new.sum()), heads, side.w)
        check_resume(side, q, new, scale, resume(side, q, new, scale, bound=int(new.sum()) + int(rng.integers(0, 9)), max_ctx=max(loose, 1), max_new=int(new.max())))


@pytest.mark.parametrize("heads", [3, 60, 128])
def test_scores_far_from_zero(heads):
    """All scores of a row shifted by one large number, either way, and first tiles that weigh nothing beside later ones."""
    ctx, new = [700], [40]
    side = Side(512, 64, 16, ctx)
    rows = side.draw(700, side.w)
    rows[:, 512] = 16.0
    rows[:640, 513] = 0.0
    rows[640:, 513] = 8.0
    side.append(ctx, rows)
    q = side.draw(40, heads, side.w)
    q[..., 512] = np.where(np.arange(40)[:, None] % 2 == 0, 64.0, -64.0)        # +-41 or so at this scale
    q[..., 513] = np.where(np.arange(40)[:, None] % 3 == 0, 256.0, 0.0)         # 82 more for the last keys: the first tile's reference is left behind
    check_resume(side, q, new, 0.04, resume(side, q, new, 0.04))


def test_an_empty_batch_of_contexts():
    side = Side(128, 64, 16, [5, 3])
    side.append([5, 3])
    q = side.draw(2, 16, side.w)
    assert (decode(side, q, 0.1, ctx=[0, 0], max_ctx=40) == 0).all()
    got = decode(side, q, 0.1, ctx=[0, 3], max_ctx=3)
    check_decode(side, q, 0.1, got, [0, 3])
