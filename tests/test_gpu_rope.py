"""Rotary positions on the GPU against the 64-bit oracle (latent_oracle.py), and the rotating append against its two parts bit by bit."""
import numpy as np
import pytest
import torch

import latent_oracle as O
from gpu_helpers import i32
from paper_2603_10342_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
TD = {"bf16": torch.bfloat16, "f32": torch.float32}
AG = {"bf16": B.AG_BF16, "f32": B.AG_F32}
LAYOUT = {"halves": B.AG_ROPE_HALVES, "pairs": B.AG_ROPE_PAIRS}


def make_rope(rot, layout, magnitude=1.0, t=None):
    t = O.turns(rot) if t is None else t
    return B.Rope(torch.from_numpy(t).to(DEV), LAYOUT[layout], magnitude), t


def ragged(prefix, new):
    """(prefix, new, cu) on the GPU, rows, position of every row."""
    cu = np.concatenate([[0], np.cumsum(new)])
    pos = np.concatenate([p + np.arange(n) for p, n in zip(prefix, new)]) if len(new) else np.zeros(0, int)
    return (i32(prefix), i32(new), i32(cu)), int(cu[-1]), pos


def same_bits(a, b):
    v = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
    return torch.equal(a.contiguous().view(v), b.contiguous().view(v))


def close(got, x, pos, t, layout, dtype, magnitude=1.0, transposed=False):
    y, size = O.rotate(x.double().cpu().numpy(), pos, t, layout, magnitude, transposed)
    err = np.abs(got.double().cpu().numpy() - y)
    assert (err <= O.rotation_allowed(y, size, dtype, magnitude)).all(), float(err.max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("heads,d,rot", [(1, 16, 16), (3, 24, 16), (5, 128, 128), (32, 128, 64), (7, 80, 32), (2, 256, 256), (4, 96, 48), (1, 72, 64), (130, 64, 64)])
def test_rows(dtype, layout, heads, d, rot):
    rope, t = make_rope(rot, layout, 1.25)
    lens, total, pos = ragged([0, 7, 100, 4095, 0], [1, 0, 9, 3, 5])
    x = torch.randn(total, heads, d, device=DEV).to(TD[dtype])
    y = torch.full_like(x, float("nan"))
    B.ag_rope_rows(rope, x, y, *lens, total)
    close(y, x, pos, t, layout, dtype, 1.25)
    z = torch.full_like(x, float("nan"))
    B.ag_rope_rows(rope, x, z, *lens, total, True)
    close(z, x, pos, t, layout, dtype, 1.25, True)
    B.ag_rope_rows(rope, x, x, *lens, total)                                   # where they stand
    assert same_bits(x, y)


@pytest.mark.parametrize("layout", ["halves", "pairs"])
def test_far_positions_keep_their_angles(layout):
    rope, t = make_rope(64, layout)
    lens, total, pos = ragged([(1 << 31) - 1100, 1 << 24, 999999], [3, 2, 2])
    x = torch.randn(total, 2, 64, device=DEV)
    y = torch.empty_like(x)
    B.ag_rope_rows(rope, x, y, *lens, total)
    close(y, x, pos, t, layout, "f32")


@pytest.mark.parametrize("dtype,new", [("bf16", [1] * 70), ("f32", [3, 0, 800, 1, 64, 0, 1300, 2]), ("bf16", [2500])])
def test_many_rows_and_rows_behind_the_last_session(dtype, new):
    rope, t = make_rope(32, "halves")
    lens, total, pos = ragged([11 * i for i in range(len(new))], new)
    more = total + 5
    x = torch.randn(more, 3, 40, device=DEV).to(TD[dtype])
    y = torch.full_like(x, 7.0)
    B.ag_rope_rows(rope, x, y, *lens, more)
    assert bool((y[total:] == 7).all())
    keep = np.unique(np.concatenate([np.arange(0, total, 37), [0, total - 1]]))
    close(y[keep], x[keep], pos[keep], t, "halves", dtype)
    other = torch.empty_like(x)                                                # every row, against rows one by one
    B.ag_rope_rows(rope, x, other, i32(pos), i32(np.ones(total)), i32(np.arange(total + 1)), total)
    assert same_bits(y[:total], other[:total])


def test_slices_of_wider_rows():
    rope, t = make_rope(64, "pairs")
    lens, total, pos = ragged([5, 90], [4, 3])
    wide = torch.randn(total, 6, 192, device=DEV).bfloat16()
    before, q = wide.clone(), torch.full((total, 6, 576), 3.0, dtype=torch.bfloat16, device=DEV)
    B.ag_rope_rows(rope, wide[..., 128:], q[..., 512:], *lens, total)
    close(q[..., 512:], before[..., 128:], pos, t, "pairs", "bf16")
    assert bool((q[..., :512] == 3).all()) and same_bits(wide, before)
    B.ag_rope_rows(rope, wide[..., 128:], wide[..., 128:], *lens, total)
    assert same_bits(wide[..., 128:], q[..., 512:]) and same_bits(wide[..., :128], before[..., :128])
    heads_first = before[..., 128:].transpose(0, 1).contiguous().transpose(0, 1)
    y = torch.empty_like(heads_first)
    B.ag_rope_rows(rope, heads_first, y, *lens, total)
    assert same_bits(y, q[..., 512:])


def test_the_transposed_rotation_is_the_gradient():
    """d/dx of g . rotate(x) is rotate_transposed(g): exactly, as sums, since rotation is linear."""
    rope, t = make_rope(48, "halves", 1.5)
    lens, total, pos = ragged([3, 1000], [6, 2])
    x, g = (torch.randn(total, 4, 64, device=DEV) for _ in range(2))
    y, back = torch.empty_like(x), torch.empty_like(x)
    B.ag_rope_rows(rope, x, y, *lens, total)
    B.ag_rope_rows(rope, g, back, *lens, total, True)
    lhs, rhs = (g.double() * y.double()).sum(-1), (back.double() * x.double()).sum(-1)
    # either side's numbers are off by 3.01 * 2^-24 * 1.5 (|a| + |b|), a row's sum by that times |g| or |x|: at most 4 |g| |x| of a row, by Cauchy and Schwarz
    most = 2 * 3.01 * 2.0 ** -24 * 1.5 * 2 * g.double().norm(dim=-1) * x.double().norm(dim=-1)
    assert bool(((lhs - rhs).abs() <= most).all())
    rope.magnitude = 1.0
    B.ag_rope_rows(rope, x, y, *lens, total)
    B.ag_rope_rows(rope, y, back, *lens, total, True)
    assert float((back - x).abs().max()) <= 2 * 3.01 * 2.0 ** -24 * 2 * float(x.abs().max()) * 1.5


def split_append(cache, rope, q, k, v, bt, lens, total):
    """What ag_kv_append_rope does, by its parts."""
    kr, qr = torch.empty_like(k), torch.empty_like(q)
    B.ag_rope_rows(rope, k, kr, *lens, total)
    B.ag_rope_rows(rope, q, qr, *lens, total)
    B.ag_kv_append(cache, kr, v, bt, *lens, total)
    return qr


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("hq,hkv,d,rot,page", [(32, 8, 128, 128, 16), (4, 2, 64, 32, 32), (6, 2, 256, 256, 16), (1, 1, 16, 16, 256), (9, 3, 72, 48, 64), (40, 1, 128, 64, 128)])
def test_append_is_rotation_and_append(dtype, layout, hq, hkv, d, rot, page):
    rope, _ = make_rope(rot, layout, 0.75)
    prefix, new = np.array([0, 15, 33, 200, 16, 5]), np.array([1, 1, 40, 0, 16, 3])
    lens, total, _ = ragged(prefix, new)
    need = -(-(prefix + new) // page)
    ids = np.random.default_rng(3).permutation(int(need.sum()) + 4)
    bt = np.zeros((len(new), int(need.max())), np.int32)
    at = 0
    for s, n in enumerate(need):
        bt[s, :n] = ids[at:at + n]
        at += n
    bt = i32(bt)
    more = total + 3                                                           # a bound, and rows behind it
    q, k, v = (torch.randn(more, h, d, device=DEV).to(TD[dtype]) for h in (hq, hkv, hkv))
    one, two = (B.KVCache(len(ids), page, hkv, d, AG[dtype], DEV, fill=9.0) for _ in range(2))
    want = split_append(one, rope, q, k, v, bt, lens, total)
    q_out, kept = torch.full_like(q, 7.0), k.clone()
    B.ag_kv_append_rope(two, rope, q, q_out, k, v, bt, *lens, more)
    assert same_bits(one.k_pool, two.k_pool) and same_bits(one.v_pool, two.v_pool) and same_bits(q_out[:total], want[:total])
    assert bool((q_out[total:] == 7).all()) and same_bits(k, kept)
    three = B.KVCache(len(ids), page, hkv, d, AG[dtype], DEV, fill=9.0)
    tail = q[total:].clone()
    B.ag_kv_append_rope(three, rope, q, q, k, v, bt, *lens, more)              # queries where they stand
    assert same_bits(three.k_pool, two.k_pool) and same_bits(q[:total], want[:total]) and same_bits(q[total:], tail)
    four = B.KVCache(len(ids), page, hkv, d, AG[dtype], DEV, fill=9.0)
    B.ag_kv_append_rope(four, rope, None, None, k, v, bt, *lens, more)
    assert same_bits(four.k_pool, two.k_pool) and same_bits(four.v_pool, two.v_pool)


def test_what_is_not_finite_stays_in_its_pair():
    rope, _ = make_rope(32, "pairs")
    lens, total, _ = ragged([5], [2])
    x = torch.randn(2, 1, 48, device=DEV)
    x[0, 0, 6], x[1, 0, 40] = float("inf"), float("nan")
    y = torch.empty_like(x)
    B.ag_rope_rows(rope, x, y, *lens, total)
    bad = ~torch.isfinite(y)
    assert bad.nonzero().tolist() == [[0, 0, 6], [0, 0, 7], [1, 0, 40]]


def test_another_stream_and_a_replayed_step():
    """A step's rotation and append in a graph, replayed over new rows, with eager work between."""
    rope, _ = make_rope(64, "halves")
    lens, total, _ = ragged([30, 4], [1, 1])
    bt = i32([[0, 1, 2], [5, 4, 3]])
    q, k, v = (torch.randn(2, h, 64, device=DEV).bfloat16() for h in (8, 2, 2))
    cache, eager = (B.KVCache(6, 16, 2, 64, B.AG_BF16, DEV, fill=0.0) for _ in range(2))
    q_out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.ag_kv_append_rope(cache, rope, q, q_out, k, v, bt, *lens, total)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.ag_kv_append_rope(cache, rope, q, q_out, k, v, bt, *lens, total)
    for i in range(4):
        for x in (q, k, v):
            x.copy_(torch.randn_like(x))
        lens[0].add_(1)
        g.replay()
        torch.cuda.synchronize()
        want = split_append(eager, rope, q, k, v, bt, lens, total)
        assert same_bits(q_out, want)
        for s, pos in enumerate(lens[0].tolist()):
            page, slot = bt[s, pos // 16], pos % 16
            assert same_bits(cache.k_pool_token_major()[page, :, slot], eager.k_pool_token_major()[page, :, slot])
            assert same_bits(cache.v_pool_token_major()[page, :, slot], eager.v_pool_token_major()[page, :, slot])
