"""Rotary positions, the append that rotates on its way into the cache, and attention over a cache of latent vectors.

Rotation: channel pairs of the first `rot` channels of a row at position p turn by 2 pi p turns[i], i < rot / 2:
    a' = m (a cos - b sin),  b' = m (b cos + a sin)      (transposed: sin with the other sign)
where (a, b) are channels i and i + rot / 2 ("halves") or 2 i and 2 i + 1 ("pairs"), and m is a magnitude; other channels stay as they are.
turns[i] = base^(-2 i / rot) / (2 pi), as 64-bit numbers, here with positions that are stretched over a longer context in part of the cases.

Paged cache of keys and values: keys [page][KV head][channel / 8][slot][channel % 8], values [page][KV head][chunk][channel][8 keys], where chunk 2 g + h
of a group g of 16 slots holds slots h * 4 + {0..3} and 8 + h * 4 + {0..3}.

Latent cache: one row a token that all heads share, [page][slot][row], a row being `lat` latent channels and `rd` rotary ones, padded to a multiple of 64.
Keys are whole rows, values their latent part:
    S[t, h, j] = scale * q[t, h] . row[j],   O[t, h] = softmax_j(S) . row[j, :lat],   j <= position of t.

A case is a dict of plain values.  `kind` says which operator a pass runs:
  rope           rows of ragged sessions are rotated
  append         new tokens of ragged sessions go into a paged cache, their keys and queries rotated
  latent_append  latent rows of ragged sessions go into a latent cache, their rotary part rotated
  latent_decode  one query per session and head over all of its latent rows
  latent_resume  causal attention of chunks behind cached prefixes over latent rows
Sizes: `batch` sessions with `p_lo`..`p_hi` cached tokens and `n_lo`..`n_hi` new ones (decode: its context is p), drawn from `lens`.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"


def _case(name, kind, dtype="bf16", hq=32, hkv=8, d=128, rot=128, layout="halves", stretch=1.0, transposed=False, lat=512, rd=64, page=16, batch=1,
          p=(0, 0), n=(1, 1), lens=1):
    c = {"kind": kind, "dtype": dtype, "hq": hq, "page": page, "batch": batch, "p_lo": p[0], "p_hi": p[1], "n_lo": n[0], "n_hi": n[1], "lens": lens}
    if kind in ("rope", "append"):
        c.update(d=d, rot=rot, layout=layout, stretch=stretch)
        c.update({"transposed": transposed} if kind == "rope" else {"hkv": hkv})
    else:
        c.update(lat=lat, rd=rd)
        if kind == "latent_append":
            c.update(rot=rd, layout=layout, stretch=stretch)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the queries of a decode step of 64 sessions, the benchmark's geometry: all latency
        _case("rope_64", "rope", batch=64, p=(1023, 4095), lens=2),
        # queries of the benchmark's cold prompts where half of a head turns, interleaved, on positions stretched fourfold: a stream through
        _case("rope_8x4096", "rope", rot=64, layout="pairs", stretch=4.0, batch=8, n=(4096, 4096), lens=3),
        # a decode step's tokens of 64 sessions
        _case("append_64", "append", batch=64, p=(1023, 4095), lens=2),
        # the benchmark's cold prompts, 8 of 4096 tokens
        _case("append_8x4096", "append", batch=8, n=(4096, 4096), lens=3),
        # tool outputs of a few agents, half-width heads of which half turn, larger pages, fp32
        _case("append_5_f32", "append", dtype="f32", hq=4, hkv=2, d=64, rot=32, layout="pairs", page=32, batch=5, p=(0, 900), n=(3, 300), lens=4),
        # a decode step's latent rows of 64 sessions
        _case("latent_append_64", "latent_append", layout="pairs", batch=64, p=(1023, 4095), lens=2),
        # whole prompts into a latent cache
        _case("latent_append_8x4096", "latent_append", layout="pairs", batch=8, n=(4096, 4096), lens=3),
        # one agent decoding alone
        _case("latent_decode_1", "latent_decode", hq=32, batch=1, p=(1000, 1000)),
        # the benchmark's decode contexts with many heads over each row
        _case("latent_decode_64", "latent_decode", hq=128, batch=64, p=(1024, 4096), lens=2),
        # few heads a device, as where heads are dealt to eight of them, long contexts on large pages
        _case("latent_decode_long", "latent_decode", hq=16, page=64, batch=4, p=(20000, 32768), lens=5),
        # one agent's tool output comes back: one ragged chunk on a long prefix
        _case("latent_resume_1", "latent_resume", hq=32, batch=1, p=(6007, 6007), n=(211, 211)),
        # chunks of several agents on long prefixes, many heads: the matrix units' work
        _case("latent_resume_8", "latent_resume", hq=128, batch=8, p=(2048, 8192), n=(32, 256), lens=6),
    ]


# ---- sizes ----

def lengths(case):
    """(cached, new) tokens of every session, as int64 arrays."""
    rng = np.random.default_rng(case["lens"])
    p = rng.integers(case["p_lo"], case["p_hi"] + 1, size=case["batch"])
    n = rng.integers(case["n_lo"], case["n_hi"] + 1, size=case["batch"])
    if case["kind"] == "latent_decode":
        n = np.ones_like(p)
        p = p - 1
    return p.astype(np.int64), n.astype(np.int64)


def _pages(p, n, page):
    """Pages that hold tokens p .. p + n - 1, of all sessions."""
    return int(((p + n - 1) // page - p // page + 1).sum())


def work(case):
    p, n = lengths(case)
    el, t, kind, page = 4 if case["dtype"] == "f32" else 2, int(n.sum()), case["kind"], case["page"]
    if kind == "rope":
        return {"bytes": 2 * t * case["hq"] * case["d"] * el, "flops": 3 * t * case["hq"] * case["rot"]}
    if kind == "append":
        return {"bytes": t * (2 * case["hq"] + 4 * case["hkv"]) * case["d"] * el + 4 * _pages(p, n, page), "flops": 3 * t * (case["hq"] + case["hkv"]) * case["rot"]}
    lat, row = case["lat"], case["lat"] + case["rd"]
    if kind == "latent_append":
        return {"bytes": 2 * t * row * el + 4 * _pages(p, n, page), "flops": 3 * t * case["rd"]}
    pairs = int((n * p + n * (n + 1) // 2).sum())
    return {"bytes": int((p + n).sum()) * row * el + t * case["hq"] * (row + lat) * el + 4 * _pages(0 * p, p + n, page), "flops": 2 * case["hq"] * pairs * (row + lat)}


MOST_TOKENS = 1 << 18           # of all contexts of a drawn decode
MOST_BYTES = 3 << 28            # of rows read and written by a drawn rotation or append
MOST_FLOPS = 1.2e12
MOST_SCORES = 2 << 30           # scores of a drawn chunk attention with every session as long as the longest


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rope", "append", "append", "latent_append", "latent_decode", "latent_decode", "latent_decode", "latent_resume", "latent_resume"])
    page = rng.choice([16, 16, 16, 32, 64, 128, 256])
    lens = rng.randrange(1, 1 << 30)
    layout, stretch = rng.choice(["halves", "pairs"]), rng.choice([1.0, 1.0, 4.0, 40.0])
    if kind in ("rope", "append", "latent_append"):
        n_lo = log(1, 2048)
        n_hi = log(n_lo, 4096)
        p_hi = log(1, 8192 if kind != "rope" else 1 << 20)
        sizes = dict(page=page, batch=log(1, 128), p=(rng.randrange(0, p_hi), p_hi), n=(n_lo, n_hi), lens=lens, layout=layout, stretch=stretch)
        if kind == "latent_append":
            lat, rd = rng.choice([(512, 64), (512, 64), (256, 32), (256, 64), (128, 64)])
            c = _case(None, kind, lat=lat, rd=rd, **sizes)
        else:
            d, rot = rng.choice([(128, 128), (128, 128), (128, 64), (64, 64), (64, 32), (256, 64), (256, 256), (96, 48), (80, 32), (48, 16)])
            hq, hkv = rng.choice([(32, 8), (32, 8), (8, 2), (16, 2), (4, 4), (6, 2), (16, 1), (24, 1), (7, 7)])
            c = _case(None, kind, dtype=rng.choice(["bf16", "bf16", "f32"]), hq=hq, hkv=hkv, d=d, rot=rot, transposed=rng.random() < 0.3, **sizes)
        while c["batch"] > 1 and (work(c)["bytes"] > MOST_BYTES or c["batch"] * (c["p_hi"] + c["n_hi"]) > (1 << 20 if kind != "rope" else 1 << 30)):
            c["batch"] //= 2
        return c
    lat, rd = rng.choice([(512, 64)] * 5 + [(256, 32), (256, 64), (128, 64)])
    hq = rng.choice([1, 5, 8, 16, 16, 24, 32, 32, 40, 64, 100, 128, 128])
    if kind == "latent_decode":
        lo = log(1, 2048)
        hi = log(lo, 32768)
        return _case(None, kind, hq=hq, lat=lat, rd=rd, page=page, batch=min(log(1, 128), max(1, MOST_TOKENS // hi)), p=(lo, hi), lens=lens)
    p_lo, n_lo = log(1, 2048), log(1, 128)
    c = _case(None, kind, hq=hq, lat=lat, rd=rd, page=page, batch=log(1, 32), p=(rng.choice([0, p_lo]), log(p_lo, 8192)), n=(n_lo, log(n_lo, 1024)), lens=lens)
    while c["batch"] > 1 and (work(c)["flops"] > MOST_FLOPS or c["batch"] * hq * c["n_hi"] * (c["p_hi"] + c["n_hi"]) > MOST_SCORES):
        c["batch"] //= 2
    while c["n_hi"] > 1 and (work(c)["flops"] > MOST_FLOPS or hq * c["n_hi"] * (c["p_hi"] + c["n_hi"]) > MOST_SCORES):
        c["n_hi"] //= 2
        c["n_lo"] = min(c["n_lo"], c["n_hi"])
    return c


# ---- what a program has in hand ----

def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _row(case):
    """Channels of a latent cache's row, its padding included."""
    return (case["lat"] + case["rd"] + 63) // 64 * 64


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    dt, hq, ps, kind = _dtype(case), case["hq"], case["page"], case["kind"]
    p, n = lengths(case)
    t = int(n.sum())

    def randn(*shape, size=1.0):
        return (torch.randn(shape, device=DEV, generator=gen) * size).to(dt)

    def pool(*shape):
        x = torch.empty(shape, dtype=dt, device=DEV)
        flat = x.view(-1)
        for i in range(0, flat.numel(), 1 << 28):
            flat[i:i + (1 << 28)] = torch.randn(min(1 << 28, flat.numel() - i), device=DEV, generator=gen).to(dt)
        return x

    state = {"kind": kind, "dtype": dt, "hq": hq, "ps": ps, "prefix": _i32(p), "new": _i32(n), "ctx": _i32(p + n), "cu": _i32(np.concatenate([[0], np.cumsum(n)])),
             "total": t, "max_new": int(n.max()), "max_ctx": int((p + n).max())}
    if "rot" in case:
        rot = case["rot"]
        i = torch.arange(rot // 2, dtype=torch.float64, device=DEV)
        state["turns"] = torch.pow(10000.0, -2.0 * i / rot) / (2 * math.pi * case["stretch"])
        state["pairs"], state["magnitude"] = case["layout"] == "pairs", 1.0 + 0.1 * math.log(case["stretch"])
    if kind == "rope":
        state["x"] = randn(t, hq, case["d"])
        state["y"], state["transposed"] = torch.empty_like(state["x"]), case["transposed"]
        return state
    need = (p + n + ps - 1) // ps
    pages = int(need.sum()) + 16
    perm = np.random.default_rng(int(seed)).permutation(pages)
    bt = np.zeros((len(need), int(need.max())), np.int32)                      # unused entries name a valid page, as stale rows do
    at = 0
    for s, k in enumerate(need):
        bt[s, :k] = perm[at:at + k]
        at += k
    state.update(bt=_i32(bt), pages=pages)
    if kind == "append":
        hkv, d = case["hkv"], case["d"]
        state.update(k_pool=pool(pages, hkv, d // 8, ps, 8), v_pool=pool(pages, hkv, ps // 8, d, 8), q=randn(t, hq, d), k=randn(t, hkv, d), v=randn(t, hkv, d))
        state["q_out"] = torch.empty_like(state["q"])
        return state
    lat, rd = case["lat"], case["rd"]
    state.update(lat=lat, rd=rd, pool=pool(pages, ps, _row(case)), scale=1.0 / math.sqrt(lat + rd))
    if kind == "latent_append":
        state["latent"] = randn(t, lat)
        state["rotary"] = randn(t, lat + rd)[:, lat:]                           # a slice of the projection that makes both
    else:
        state["q"] = randn(t, hq, lat + rd)
        state["out"] = torch.empty((t, hq, lat), dtype=dt, device=DEV)
    return state


# ---- the plain form ----

def _sessions(state):
    """Session and position of every row."""
    t = torch.arange(state["total"], device=DEV)
    s = torch.searchsorted(state["cu"][1:].contiguous(), t, right=True)
    return s, state["prefix"].long()[s] + t - state["cu"].long()[s]


def _rotate(state, x, pos, transposed=False):
    """Rows [T][...][d] at positions [T], in fp32."""
    angle = pos.double()[:, None] * state["turns"]
    angle = (angle - angle.round()) * (2 * math.pi)
    m = state["magnitude"]
    shape = (len(pos),) + (1,) * (x.dim() - 2) + (-1,)
    cos, sin = (angle.cos() * m).float().view(shape), (angle.sin() * (-m if transposed else m)).float().view(shape)
    rot, y = 2 * angle.shape[1], x.float().clone()
    a, b = (x[..., 0:rot:2].float(), x[..., 1:rot:2].float()) if state["pairs"] else (x[..., :rot // 2].float(), x[..., rot // 2:rot].float())
    u, v = a * cos - b * sin, b * cos + a * sin
    if state["pairs"]:
        y[..., 0:rot:2], y[..., 1:rot:2] = u, v
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = u, v
    return y


def _plain_append(state):
    s, pos = _sessions(state)
    page, slot = state["bt"].long()[s, pos // state["ps"]], pos % state["ps"]
    dt = state["dtype"]
    t, hkv, d = state["k"].shape
    state["k_pool"][page, :, :, slot, :] = _rotate(state, state["k"], pos).to(dt).view(t, hkv, d // 8, 8)
    state["v_pool"][page, :, slot // 16 * 2 + slot // 4 % 2, :, slot % 4 + slot // 8 % 2 * 4] = state["v"]
    return {"q": _rotate(state, state["q"], pos).to(dt), "k_pool": state["k_pool"], "v_pool": state["v_pool"]}


def _plain_latent_append(state):
    s, pos = _sessions(state)
    page, slot = state["bt"].long()[s, pos // state["ps"]], pos % state["ps"]
    lat, rd = state["lat"], state["rd"]
    state["pool"][page, slot, :lat] = state["latent"]
    state["pool"][page, slot, lat:lat + rd] = _rotate(state, state["rotary"], pos).to(state["dtype"])
    return {"pool": state["pool"]}


def _plain_attention(state):
    hq, lat, w, m, ps = state["hq"], state["lat"], state["lat"] + state["rd"], state["max_new"], state["ps"]
    table = state["bt"].long()
    b = table.shape[0]
    rows = state["pool"][table].view(b, table.shape[1] * ps, -1)[:, :state["max_ctx"], :w].float()
    cu = state["cu"].long()
    row = torch.arange(m, device=DEV)
    q = state["q"][(cu[:-1, None] + row).clamp(max=state["total"] - 1)].float().view(b, m * hq, w)
    x = torch.bmm(q, rows.transpose(1, 2).contiguous()).view(b, m, hq, -1)
    hidden = torch.arange(x.shape[-1], device=DEV) > (state["prefix"].long()[:, None] + row)[..., None]
    x.mul_(state["scale"]).masked_fill_(hidden[:, :, None, :], -math.inf)
    x.sub_(x.amax(-1, keepdim=True)).exp_()
    o = torch.bmm(x.view(b, m * hq, -1), rows[..., :lat].contiguous()).view(b, m, hq, lat) / x.sum(-1, keepdim=True)
    t = torch.arange(state["total"], device=DEV)
    s = torch.searchsorted(state["cu"][1:].contiguous(), t, right=True)
    return {"out": o[s, t - cu[s]].to(state["dtype"])}


# ---- the framework's calls ----

def _own(state):
    from paper_2603_10342_amd import binding as B
    x, kind = state, state["kind"]
    if "turns" in x and "rope" not in x:                                        # handles, which a program keeps
        x["rope"] = B.Rope(x["turns"], B.AG_ROPE_PAIRS if x["pairs"] else B.AG_ROPE_HALVES, x["magnitude"])
    if kind == "rope":
        B.ag_rope_rows(x["rope"], x["x"], x["y"], x["prefix"], x["new"], x["cu"], x["total"], x["transposed"])
        return {"y": x["y"]}
    if "cache" not in x:
        if kind == "append":
            c = B.KVCache(1, x["ps"], x["k"].shape[1], x["k"].shape[2], B.AG_F32 if x["dtype"] == torch.float32 else B.AG_BF16, DEV)
            c.num_pages, c.k_pool, c.v_pool = x["pages"], x["k_pool"], x["v_pool"]
        else:
            c = B.LatentCache(1, x["ps"], x["lat"], x["rd"], DEV)
            c.num_pages, c.pool = x["pages"], x["pool"]
        x["cache"] = c
    c = x["cache"]
    if kind == "append":
        B.ag_kv_append_rope(c, x["rope"], x["q"], x["q_out"], x["k"], x["v"], x["bt"], x["prefix"], x["new"], x["cu"], x["total"])
        return {"q": x["q_out"], "k_pool": x["k_pool"], "v_pool": x["v_pool"]}
    if kind == "latent_append":
        B.ag_kv_append_latent(c, x["rope"], x["latent"], x["rotary"], x["bt"], x["prefix"], x["new"], x["cu"], x["total"])
        return {"pool": x["pool"]}
    if kind == "latent_decode":
        if "ws" not in x:                                                       # kept by a program from step to step
            x["ws"] = torch.empty(B.ag_attn_decode_latent_workspace_bytes(len(x["ctx"]), x["hq"], x["lat"], x["max_ctx"]), dtype=torch.uint8, device=DEV)
        B.ag_attn_decode_latent(c, x["q"], x["out"], x["bt"], x["ctx"], x["max_ctx"], x["hq"], x["scale"], x["ws"])
    else:
        if "ws" not in x:
            x["ws"] = torch.empty(B.ag_attn_resume_latent_workspace_bytes(len(x["ctx"]), x["total"], x["hq"], x["lat"], x["max_ctx"]), dtype=torch.uint8, device=DEV)
        B.ag_attn_resume_latent(c, x["q"], x["out"], x["bt"], x["prefix"], x["new"], x["cu"], x["total"], x["max_new"], x["max_ctx"], x["hq"], x["scale"], x["ws"])
    return {"out": x["out"]}


def run(state):
    if own:
        return _own(state)
    kind = state["kind"]
    if kind == "rope":
        _, pos = _sessions(state)
        return {"y": _rotate(state, state["x"], pos, state["transposed"]).to(state["dtype"])}
    if kind == "append":
        return _plain_append(state)
    return _plain_latent_append(state) if kind == "latent_append" else _plain_attention(state)


# ---- the same in 64 bits ----

def _exact_rotation(state, case, x, first, transposed=False):
    """Rows [N][...][d] at positions first, first + 1, ..: as complex numbers times e^(i theta)."""
    x = x.double()
    rot = case["rot"]
    theta = torch.outer(torch.arange(first, first + x.shape[0], dtype=torch.float64, device=DEV), state["turns"])
    theta = 2 * math.pi * torch.frac(theta) * (-1 if transposed else 1)
    turn = torch.polar(torch.full_like(theta, state["magnitude"]), theta)
    turn = turn.view(x.shape[0], *[1] * (x.dim() - 2), rot // 2)
    part = x[..., :rot]
    z = torch.view_as_complex(part.unflatten(-1, (-1, 2)).contiguous()) if case["layout"] == "pairs" else torch.complex(*part.chunk(2, -1))
    z = z * turn
    part = torch.view_as_real(z).flatten(-2) if case["layout"] == "pairs" else torch.cat([z.real, z.imag], -1)
    return torch.cat([part, x[..., rot:]], -1)


def exact(case, seed):
    state = prepare(case, seed)
    kind, ps, hq = case["kind"], case["page"], case["hq"]
    p, n = lengths(case)
    row_of = np.concatenate([[0], np.cumsum(n)])
    rows = [slice(int(a), int(b)) for a, b in zip(row_of[:-1], row_of[1:])]
    if kind == "rope":
        return {"y": torch.cat([_exact_rotation(state, case, state["x"][r], int(p[s]), case["transposed"]) for s, r in enumerate(rows)])}
    bt = state["bt"].cpu().numpy().astype(np.int64)

    def places(s, first, last):
        pos = np.arange(first, last)
        return torch.from_numpy(bt[s, pos // ps]).to(DEV), torch.from_numpy(pos % ps).to(DEV)

    if kind == "append":
        hkv, d = case["hkv"], case["d"]
        kp, vp, q = state["k_pool"].double(), state["v_pool"].double(), []
        chunk = np.array([x // 16 * 2 + (x % 8 >= 4) for x in range(ps)])
        eighth = np.array([x % 4 + 4 * (x % 16 >= 8) for x in range(ps)])
        for s, r in enumerate(rows):
            page, slot = places(s, p[s], p[s] + n[s])
            at = slot.cpu().numpy()
            kp[page, :, :, slot, :] = _exact_rotation(state, case, state["k"][r], int(p[s])).view(-1, hkv, d // 8, 8)
            vp[page, :, torch.from_numpy(chunk[at]).to(DEV), :, torch.from_numpy(eighth[at]).to(DEV)] = state["v"][r].double()
            q.append(_exact_rotation(state, case, state["q"][r], int(p[s])))
        return {"q": torch.cat(q), "k_pool": kp, "v_pool": vp}
    lat, w = case["lat"], case["lat"] + case["rd"]
    if kind == "latent_append":
        pool = state["pool"].double()
        for s, r in enumerate(rows):
            page, slot = places(s, p[s], p[s] + n[s])
            pool[page, slot, :w] = torch.cat([state["latent"][r].double(), _exact_rotation(state, case, state["rotary"][r], int(p[s]))], -1)
        return {"pool": pool}
    outs = []
    for s, r in enumerate(rows):
        page, slot = places(s, 0, p[s] + n[s])
        keys = state["pool"][page, slot, :w].double()
        kt, values = keys.t().contiguous(), keys[:, :lat].contiguous()
        out = torch.empty((int(n[s]), hq, lat), dtype=torch.float64, device=DEV)
        step = max(1, (1 << 27) // (hq * len(keys)))                            # rows at once: scores of a gigabyte
        for i in range(0, int(n[s]), step):
            q = state["q"][r][i:i + step].double()
            x = (q.reshape(-1, w) @ kt).view(-1, hq, len(keys)) * state["scale"]
            last = int(p[s]) + i + torch.arange(len(q), device=DEV)
            x.masked_fill_(torch.arange(len(keys), device=DEV) > last[:, None, None], -math.inf)
            out[i:i + step] = (torch.softmax(x, -1).view(-1, len(keys)) @ values).view(-1, hq, lat)
        outs.append(out)
    return {"out": torch.cat(outs)}
