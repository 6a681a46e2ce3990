"""Which kernel a call over an 8-bit cache takes, at batches where both sides of a line were measured and differ (the figures stand at
the lines in the sources), and on which the GPU tests rely: seen on the CPU, through a HIP runtime that logs launches."""
import pytest

from q8_launches import launched


@pytest.fixture(scope="module")
def tmp(tmp_path_factory):
    return tmp_path_factory.mktemp("launches")


def kernels(tmp, *calls):
    return [[l.split(" ")[0].replace("q8::", "") for l in r] for r in launched(calls, tmp)]


SPLIT, TILES, WIDE = "prefill_q8_split_kernel<", "prefill_q8_kernel<4,", "prefill_q8_kernel<8,128,true>"


@pytest.mark.parametrize("want,batches", [
    (SPLIT, [dict(batch=1, prefix=6007, new=211), dict(batch=1, prefix=6007, new=600), dict(batch=1, prefix=2000, new=211), dict(batch=16, prefix=600, new=30),
             dict(batch=1, prefix=6007, new=211, dtype="f32"), dict(batch=6, total=784, max_new=300, max_ctx=2300, d=64, page=32, dtype="f32"),
             dict(batch=4, prefix=2000, new=16, hq=24, hkv=1), dict(batch=8, new=1500, dtype="f32"), dict(batch=8, total=1300, max_new=300, max_ctx=4300, d=64), dict(batch=4, total=690, max_new=300, max_ctx=4300, d=256),
             dict(batch=2, new=700, d=96), dict(batch=1, prefix=2000, new=1000, d=192)]),
    (TILES, [dict(batch=1, prefix=2000, new=1000), dict(batch=16, new=50), dict(batch=1, new=1000), dict(batch=8, new=512), dict(batch=64, new=600), dict(batch=1, new=2048), dict(batch=16, total=1200, max_new=100, max_ctx=400), dict(batch=16, total=6500, max_new=600, max_ctx=600, d=64),
             dict(batch=16, total=6500, max_new=600, max_ctx=600, d=256), dict(batch=16, total=6500, max_new=600, max_ctx=600, d=96), dict(batch=2, new=700, d=192)]),
    (WIDE, [dict(batch=8, new=4096), dict(batch=2, prefix=2000, new=1000), dict(batch=32, prefix=3000, new=200)]),
])
def test_prefill(tmp, want, batches):
    for b, k in zip(batches, kernels(tmp, *(dict(call="resume", **b) for b in batches))):
        assert len(k) == 1 and k[0].startswith(want), (b, k)


# sessions of the GPU tests of whole tiles, on streams of eight CUs: prefix, new
TILED = {"ragged": ([130, 0, 64, 700, 33], [70, 90, 0, 130, 1]), "prompts": ([0, 0, 0], [200, 333, 64]), "long": ([1700, 1500], [300, 120])}


def tiled(name, **more):
    prefix, new = TILED[name]
    return dict(call="resume", batch=len(new), total=sum(new), max_new=max(new), max_ctx=max(p + n for p, n in zip(prefix, new)), cus=8, **more)


def test_waves_of_a_split_workgroup(tmp):
    """Eight up to one workgroup a CU and past 256 tokens, where two waves a SIMD fit; the last is the GPU test's."""
    for b, w in [(dict(batch=1, prefix=6007, new=211), 8), (dict(batch=1, prefix=6007, new=400), 4), (dict(batch=8, prefix=100, new=30), 4), (dict(batch=8, prefix=300, new=30), 8),
                 (dict(batch=11, total=1100, max_new=286, max_ctx=7400, hq=6, hkv=2), 8), (dict(batch=1, prefix=2000, new=300), 4),
                 (dict(batch=1, prefix=6007, new=211, d=256), 4), (dict(batch=1, prefix=6007, new=211, dtype="f32"), 8), (dict(batch=1, prefix=6007, new=211, dtype="f32", d=64), 8),
                 (dict(FOUR, d=128), 4), (dict(FOUR, d=64, dtype="f32"), 4)]:
        (k,) = kernels(tmp, dict(call="resume", **b))
        assert k[0].startswith(SPLIT) and k[0].endswith(",%d>" % w), (b, k)


FOUR_LENS = ([900, 17], [20, 5])                                  # prefix, new; on eight CUs at 16 / 2 heads
FOUR = dict(batch=2, total=25, max_new=20, max_ctx=920, hq=16, hkv=2, cus=8)


@pytest.mark.parametrize("d,page", [(128, 16), (128, 64), (64, 32), (256, 16), (48, 128), (96, 32), (208, 256)])
def test_tiles_of_the_gpu_tests(tmp, d, page):
    for name, k in zip(TILED, kernels(tmp, *(tiled(name, d=d, page=page, hq=16, hkv=2) for name in TILED))):
        assert k[0].startswith("prefill_q8_kernel<"), (name, k)
        if d == 128 and name == "long":
            assert k[0] == WIDE, k


SHARED_CTX = 6400                                                 # the bound on contexts at which the GPU tests' decodes take shares, whatever their geometry


@pytest.mark.parametrize("alone,batches", [
    (True, [dict(batch=1, new=1000), dict(batch=17, new=2000), dict(batch=64, new=2000), dict(batch=256, new=512), dict(batch=1, new=900, dtype="f32"), dict(batch=1, new=1900, d=64),
            dict(batch=64, new=1250, d=256), dict(batch=13, new=1100, hq=8, hkv=2), dict(batch=10, new=704, hq=40, hkv=2), dict(batch=150, new=90, d=64, hq=4, hkv=1)]),
    (False, [dict(batch=1, new=1600), dict(batch=17, new=2400), dict(batch=64, new=4096), dict(batch=1, new=1000, dtype="f32"), dict(batch=16, new=2400, dtype="f32"), dict(batch=1, new=2400, d=64),
             dict(batch=1, new=900, d=256), dict(batch=13, new=SHARED_CTX, hq=8, hkv=2), dict(batch=10, new=SHARED_CTX, hq=1, hkv=1), dict(batch=150, new=SHARED_CTX, d=64, hq=4, hkv=1),
             *(dict(batch=13, new=SHARED_CTX, hq=8, hkv=2, d=d) for d in (16, 48, 64, 96, 112, 208, 240, 256))]),
])
def test_decode(tmp, alone, batches):
    for b, k in zip(batches, kernels(tmp, *(dict(call="decode", **b) for b in batches))):
        assert [x.split("<")[0] for x in k] == (["decode_q8_direct_kernel"] if alone else ["decode_q8_split_kernel", "decode_q8_merge_kernel"]), (b, k)


def test_heads_of_an_append_workgroup(tmp):
    few, many = dict(batch=64, total=704, max_ctx=200), dict(batch=100, total=150000, max_ctx=2000)
    calls = [(dict(few), 1), (dict(many, d=64), 4), (dict(many), 2), (dict(many, d=256), 1), (dict(many, hkv=6, d=64), 2), (dict(many, hkv=3, d=64), 1), (dict(many, d=64, dtype="f32"), 4)]
    # ... and those of the GPU test
    for dtype, d, hkv, heads in [("bf16", 64, 8, 4), ("bf16", 128, 6, 2), ("f32", 48, 4, 4), ("f32", 128, 2, 2)]:
        n = 8192 // (4 * hkv) + 60
        calls.append((dict(batch=n + 3, total=40 * n + 52, max_ctx=40, page=32, dtype=dtype, d=d, hkv=hkv), heads))
    for name in ("append", "read"):
        for (c, heads), k in zip(calls, kernels(tmp, *(dict(call=name, **c) for c, _ in calls))):
            assert k == ["%s_q8_kernel<%s,%d>" % (name, "float" if c.get("dtype") == "f32" else "__bf16", heads)], (c, k)


def test_rows_past_a_launch_are_refused(tmp):
    call = dict(call="resume", batch=1 << 20, total=0x7fffffff, max_new=2048, max_ctx=2048, hq=8, hkv=1)
    (k,) = launched([call], tmp)
    assert k[0].startswith("refused -1"), k
