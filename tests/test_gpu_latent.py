"""The latent cache on the GPU against the 64-bit oracle (latent_oracle.py): rows as they are appended, attention within bounds derived there."""
import numpy as np
import pytest
import torch

import latent_oracle as O
from gpu_helpers import i32
from paper_2603_10342_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
WIDTHS = [(512, 64), (512, 32), (256, 64), (256, 32), (128, 64), (128, 32)]


class Side:
    """A cache on the GPU, poisoned, and its sessions' rows on the host."""

    def __init__(self, lat, rd, page, ctx, seed=1, fill=float("nan"), spare=5, pages=None):
        self.rng = np.random.default_rng(seed)
        self.lat, self.rd, self.page, self.w = lat, rd, page, lat + rd
        need = [-(-c // page) for c in ctx]
        n = sum(need) + spare
        self.cache = B.LatentCache(pages or n, page, lat, rd, DEV, fill=fill)
        ids = self.rng.permutation(n)
        self.bt = np.full((len(ctx), max(max(need), 1)), 1 << 30, np.int32)      # entries that no token uses are not followed
        at = 0
        for s, k in enumerate(need):
            self.bt[s, :k] = ids[at:at + k]
            at += k
        self.bt_dev = i32(self.bt)
        self.rows = [np.zeros((0, self.w)) for _ in ctx]

    def draw(self, *shape, sigma=1.0):
        return O.bf16((self.rng.standard_normal(shape) * sigma).astype(np.float32))

    def dev(self, x):
        return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(DEV).bfloat16()

    def lens(self):
        return np.array([len(r) for r in self.rows])

    def append(self, new, rows=None, bound=None):
        """`new` tokens to every session, whose rotary part is rotated already."""
        new = np.asarray(new)
        t = int(new.sum())
        rows = self.draw(t, self.w) if rows is None else rows
        extra = np.full(((bound or t) - t, self.w), 7.0)
        x = self.dev(np.concatenate([rows, extra]))
        B.ag_kv_append_latent(self.cache, None, x[:, :self.lat], x[:, self.lat:], self.bt_dev, i32(self.lens()), i32(new), i32(np.concatenate([[0], np.cumsum(new)])), bound or t)
        torch.cuda.synchronize()
        at = 0
        for s, n in enumerate(new):
            self.rows[s] = np.concatenate([self.rows[s], rows[at:at + n]])
            at += n

    def stored(self, s):
        pos = np.arange(len(self.rows[s]))
        return self.cache.pool[torch.from_numpy(self.bt[s, pos // self.page].astype(np.int64)).to(DEV), torch.from_numpy(pos % self.page).to(DEV)].float().cpu().numpy()

    def table(self, max_ctx):
        pages = max(self.bt.shape[1], -(-max_ctx // self.page))
        return i32(np.pad(self.bt, ((0, 0), (0, pages - self.bt.shape[1]))))


def decode(side, q, scale, ctx=None, max_ctx=None, ws_fill=float("nan"), stream=None):
    ctx = side.lens() if ctx is None else np.asarray(ctx)
    max_ctx = int(ctx.max()) if max_ctx is None else max_ctx
    heads = q.shape[1]
    ws = torch.full((B.ag_attn_decode_latent_workspace_bytes(len(ctx), heads, side.lat, max_ctx) // 4,), ws_fill, dtype=torch.float32, device=DEV)
    out = torch.full((len(ctx), heads, side.lat), float("nan"), dtype=torch.bfloat16, device=DEV)
    args = side.dev(q), side.table(max_ctx), i32(ctx)
    torch.cuda.synchronize()
    B.ag_attn_decode_latent(side.cache, args[0], out, args[1], args[2], max_ctx, heads, scale, ws, stream)
    torch.cuda.synchronize()
    return out.double().cpu().numpy()


def resume(side, q, new, scale, bound=None, max_ctx=None, max_new=None):
    """Chunks of new[s] rows at the end of every session."""
    new = np.asarray(new)
    t, heads, lens = int(new.sum()), q.shape[1], side.lens()
    bound, max_ctx, max_new = bound or t, max_ctx or int(lens.max()), max_new or int(new.max())
    ws = torch.full((B.ag_attn_resume_latent_workspace_bytes(len(new), bound, heads, side.lat, max_ctx) // 4,), float("nan"), dtype=torch.float32, device=DEV)
    q = side.dev(np.concatenate([q, np.full((bound - t, *q.shape[1:]), np.nan)]))
    out = torch.full((bound, heads, side.lat), 7.0, dtype=torch.bfloat16, device=DEV)
    B.ag_attn_resume_latent(side.cache, q, out, side.table(max_ctx), i32(lens - new), i32(new), i32(np.concatenate([[0], np.cumsum(new)])), bound, max_new, max_ctx, heads, scale, ws)
    torch.cuda.synchronize()
    assert bool((out[t:] == 7).all()), "rows behind the last session's"
    return out[:t].double().cpu().numpy()


def check(got, parts):
    """parts: (got rows, oracle's four, width, keys) of each session."""
    errs, refs, spreads = [], [], []
    for g, (o, size, spread, reach), w, n in parts:
        assert np.isfinite(g).all()
        err, most = np.abs(g - o), O.elementwise(o, size, reach, w, n)
        assert (err <= most).all(), float((err / most).max())
        errs.append(err.ravel()); refs.append(o.ravel()); spreads.append(spread.ravel())
    e, o, s = (np.concatenate(x) for x in (errs, refs, spreads))
    if e.size >= 4096:                                             # the norm's bound is one of an average
        assert np.linalg.norm(e) <= O.norm_allowed(o, s), float(np.linalg.norm(e) / O.norm_allowed(o, s))


def check_decode(side, q, scale, got, ctx=None):
    ctx = side.lens() if ctx is None else ctx
    check(got, [(got[s:s + 1], O.attend(q[s:s + 1].astype(float), side.rows[s][:c], side.lat, c - 1, scale), side.w, c) for s, c in enumerate(ctx) if c])
    assert all((got[s] == 0).all() for s, c in enumerate(ctx) if c == 0)


def check_resume(side, q, new, scale, got):
    at, parts = 0, []
    for s, n in enumerate(new):
        if n:
            parts.append((got[at:at + n], O.attend(q[at:at + n].astype(float), side.rows[s], side.lat, len(side.rows[s]) - n, scale), side.w, len(side.rows[s])))
        at += n
    check(got, parts)


# ---- append ----

@pytest.mark.parametrize("lat,rd", WIDTHS)
@pytest.mark.parametrize("layout", ["halves", "pairs"])
def test_append_rotates_on_the_way(lat, rd, layout):
    from test_gpu_rope import make_rope
    rope, t = make_rope(rd, layout, 1.25)
    prefix, new, page = np.array([0, 31, 5, 700]), np.array([1, 40, 0, 2]), 32
    side = Side(lat, rd, page, prefix + new, fill=9.0)
    total, wide = int(new.sum()), torch.randn(int(new.sum()) + 3, lat + rd, device=DEV).bfloat16()
    cu = np.concatenate([[0], np.cumsum(new)])
    B.ag_kv_append_latent(side.cache, rope, wide[:, :lat], wide[:, lat:], side.bt_dev, i32(prefix), i32(new), i32(cu), total + 3)
    pool, touched = side.cache.pool, torch.zeros(side.cache.pool.shape[:2], dtype=torch.bool, device=DEV)
    for s, n in enumerate(new):
        pos = prefix[s] + np.arange(n)
        page_of, slot = torch.from_numpy(side.bt[s, pos // page].astype(np.int64)).to(DEV), torch.from_numpy(pos % page).to(DEV)
        rows, x = pool[page_of, slot].double().cpu().numpy(), wide[cu[s]:cu[s + 1]].double().cpu().numpy()
        assert (rows[:, :lat] == x[:, :lat]).all() and (rows[:, lat + rd:] == 9).all()
        y, size = O.rotate(x[:, lat:], pos, t, layout, 1.25)
        assert (np.abs(rows[:, lat:lat + rd] - y) <= O.rotation_allowed(y, size, "bf16", 1.25)).all()
        touched[page_of, slot] = True
    assert bool((pool[~touched] == 9).all()), "other slots stay as they were"


@pytest.mark.parametrize("new", [[1] * 200, [5000, 0, 1, 130], [3] * 2000])
def test_append_of_many_rows(new):
    side = Side(128, 32, 16, new, fill=9.0)
    side.append(new, bound=sum(new) + 2)
    for s in list(range(min(len(new), 5))) + [len(new) - 1]:
        assert (side.stored(s)[:, :side.w] == side.rows[s]).all()
    used = sum(-(-n // 16) for n in new)
    assert int((side.cache.pool[..., 0] == 9).sum()) == (used + 5) * 16 - sum(new)


def test_append_is_the_rotation_of_rows():
    """The pool's rotary part is what ag_rope_rows gives, bit by bit."""
    from test_gpu_rope import make_rope, same_bits
    rope, _ = make_rope(64, "pairs")
    side = Side(256, 64, 16, [90])
    x = torch.randn(90, 320, device=DEV).bfloat16()
    lens = i32([0]), i32([90]), i32([0, 90])
    B.ag_kv_append_latent(side.cache, rope, x[:, :256], x[:, 256:], side.bt_dev, *lens, 90)
    y = torch.empty(90, 1, 64, dtype=torch.bfloat16, device=DEV)
    B.ag_rope_rows(rope, x[:, 256:].unflatten(1, (1, 64)), y, *lens, 90)
    rows = side.cache.pool[side.bt_dev[0].long()].flatten(0, 1)[:90]
    assert same_bits(rows[:, 256:320], y[:, 0]) and same_bits(rows[:, :256], x[:, :256])


# ---- attention ----

HEADS = [1, 3, 16, 31, 32, 33, 64, 65, 100, 128, 129, 200]


@pytest.mark.parametrize("lat,rd", WIDTHS)
@pytest.mark.parametrize("heads", [5, 40, 128])
def test_decode_widths(lat, rd, heads):
    ctx = [1, 16, 31, 32, 33, 200, 64, 777]
    side = Side(lat, rd, 16, ctx)
    side.append(ctx)
    q = side.draw(len(ctx), heads, side.w)
    scale = side.w ** -0.5
    check_decode(side, q, scale, decode(side, q, scale))


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("page", [16, 64, 256])
def test_decode_heads(heads, page):
    ctx = [2, 300, 0, 47, 1024]
    side = Side(512, 64, page, ctx)
    side.append(ctx)
    q = side.draw(len(ctx), heads, side.w)
    check_decode(side, q, 0.04, decode(side, q, 0.04))


@pytest.mark.parametrize("lat,rd", WIDTHS)
@pytest.mark.parametrize("heads", [2, 24, 128])
def test_resume_widths(lat, rd, heads):
    ctx, new = [1, 33, 200, 64, 130], [1, 33, 17, 2, 30]
    side = Side(lat, rd, 16, ctx)
    side.append(ctx)
    q = side.draw(sum(new), heads, side.w)
    scale = side.w ** -0.5
    check_resume(side, q, new, scale, resume(side, q, new, scale))


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("page", [16, 128])
def test_resume_heads(heads, page):
    ctx, new = [40, 5, 600, 90], [7, 5, 13, 0]
    side = Side(512, 64, page, ctx)
    side.append(ctx)
    q = side.draw(sum(new), heads, side.w)
    check_resume(side, q, new, 0.04, resume(side, q, new, 0.04, bound=sum(new) + 3, max_ctx=700, max_new=20))


@pytest.mark.parametrize("heads,new", [(1, [700]), (16, [257, 1, 64]), (128, [40])])
def test_whole_prompts(heads, new):
    side = Side(512, 64, 16, new)
    side.append(new)
    q = side.draw(sum(new), heads, side.w)
    check_resume(side, q, new, 0.04, resume(side, q, new, 0.04))


@pytest.mark.parametrize("batch,heads", [(70, 16), (130, 64), (300, 3)])
def test_many_sessions(batch, heads):
    ctx = np.random.default_rng(9).integers(0, 150, batch)
    side = Side(128, 64, 16, ctx)
    side.append(ctx)
    q = side.draw(batch, heads, side.w)
    check_decode(side, q, 0.07, decode(side, q, 0.07))
    new = np.minimum(ctx, np.random.default_rng(10).integers(0, 4, batch))
    q = side.draw(int(new.sum()), heads, side.w)
    check_resume(side, q, new, 0.07, resume(side, q, new, 0.07))


@pytest.mark.parametrize("heads", [16, 128])
def test_long_contexts(heads):
    ctx = [9001, 20000]
    side = Side(512, 64, 64, ctx)
    side.append(ctx)
    q = side.draw(2, heads, side.w)
    check_decode(side, q, 0.05, decode(side, q, 0.05))


def test_scores_that_grow_and_shrink():
    """Maxima that rise by more than the slack late, and fall, in one context: O is rescaled, weights far below the largest vanish."""
    side = Side(512, 64, 16, [1500])
    rows = side.draw(1500, side.w) * np.linspace(0.01, 1.0, 1500)[:, None]
    rows[700] *= 20
    side.append([1500], O.bf16(rows.astype(np.float32)))
    q = side.draw(6, 40, side.w, sigma=2.0)
    check_resume(side, q, [6], 0.3, resume(side, q, [6], 0.3))
    check_decode(side, q[:1], 0.3, decode(side, q[:1], 0.3))


def test_decode_is_the_last_row_of_resume():
    side = Side(256, 64, 32, [333])
    side.append([333])
    q = side.draw(1, 64, side.w)
    a, b = decode(side, q, 0.06), resume(side, q, [1], 0.06)
    assert np.abs(a - b).max() <= 2.0 ** -7 * np.abs(b).max()


# ---- what is not finite, stale slots, sharing ----

@pytest.mark.parametrize("heads", [1, 16, 60, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_is_not_finite_reaches_those_that_see_it(heads, bad):
    n, new = 300, 70
    side = Side(512, 64, 16, [n, 50])
    rows = side.draw(n + 50, side.w)
    at, ch = n - 30, 77
    rows[at, ch] = bad
    side.append([n, 50], rows)
    q = side.draw(new + 5, heads, side.w)
    got = resume(side, q, [new, 5], 0.04)
    sees = np.arange(new) + n - new >= at
    assert np.isnan(got[:new][sees][..., ch]).all()
    clean = Side(512, 64, 16, [n, 50], seed=1)
    rows[at] = 1.0
    clean.append([n, 50], rows)
    want = resume(clean, q, [new, 5], 0.04)
    assert (got[:new][~sees] == want[:new][~sees]).all() and (got[new:] == want[new:]).all()
    if np.isnan(bad):
        assert np.isnan(got[:new][sees]).all()
    else:                                          # a score of -inf is a weight of zero, and only the channel itself is lost
        s = side.rows[0][at, ch] * q[:new, :, ch].astype(float)
        low, other = (s < 0) & sees[:, None], np.arange(512) != ch
        assert np.isnan(got[:new][(s > 0) & sees[:, None]]).all()
        assert np.isfinite(got[:new][low][:, other]).all()


@pytest.mark.parametrize("fill", [float("inf"), 1e38])
def test_stale_slots_do_not_matter(fill):
    ctx = [1, 17, 40, 100]
    a, b = (Side(512, 64, 64, ctx, fill=f) for f in (fill, 0.0))
    for x in (a, b):
        x.append(ctx)
    q = a.draw(4, 24, a.w)
    assert (decode(a, q, 0.04) == decode(b, q, 0.04)).all()
    q = a.draw(8, 24, a.w)
    assert (resume(a, q, [1, 3, 2, 2], 0.04) == resume(b, q, [1, 3, 2, 2], 0.04)).all()


def test_same_bits_again_and_whatever_the_workspace_holds():
    ctx = np.random.default_rng(4).integers(1, 3000, 20)
    side = Side(512, 64, 16, ctx)
    side.append(ctx)
    q = side.draw(20, 128, side.w)
    a = decode(side, q, 0.04)
    assert (decode(side, q, 0.04, ws_fill=3.0) == a).all()
    assert np.abs(decode(side, q, 0.04, max_ctx=9000) - a).max() <= 2.0 ** -6 * np.abs(a).max()


def test_shared_pages():
    """Two sessions on one prefix."""
    side = Side(512, 64, 16, [160, 160])
    side.append([160, 0])
    side.bt[1] = side.bt[0]
    side.bt_dev = i32(side.bt)
    side.rows[1] = side.rows[0][:130]
    q = side.draw(2, 16, side.w)
    check_decode(side, q, 0.04, decode(side, q, 0.04, max_ctx=160))


def test_places_past_32_bits():
    """Pages beyond 4 GiB and 2^31 numbers of the pool."""
    side = Side(512, 64, 256, [600], spare=0, pages=16000)          # 4.7 GB
    side.bt[0, :3] = [15999, 7300, 14564]
    side.bt_dev = i32(side.bt)
    side.append([600])
    assert (side.stored(0)[:, :side.w] == side.rows[0]).all()
    q = side.draw(4, 16, side.w)
    check_resume(side, q, [4], 0.04, resume(side, q, [4], 0.04))
    check_decode(side, q[:1], 0.04, decode(side, q[:1], 0.04))
