"""Which kernel a rotary or latent-cache call takes, at batches where both sides of a line were measured and differ (the figures stand at the lines in
the sources), and on which the GPU tests rely: seen on the CPU, through a HIP runtime that logs launches."""
import pytest

import test_gpu_latent_columns as G
from latent_launches import launched


@pytest.fixture(scope="module")
def tmp(tmp_path_factory):
    return tmp_path_factory.mktemp("launches")


def logs(tmp, *calls):
    return [[l.replace("latent::", "").replace("rope::", "").split(" ") for l in r] for r in launched(calls, tmp)]


def columns(log):
    """Columns of a call's workgroups: 128 over the waves that share one."""
    assert log[0][0].startswith("latent_kernel<"), log
    return 128 // int(log[0][0].split(",")[2])


@pytest.mark.parametrize("cols,batches", [
    (128, [dict(batch=64, max_ctx=4096), dict(batch=256, max_ctx=128), dict(batch=64, max_ctx=4096, heads=65), dict(batch=70, max_ctx=4096, heads=200)]),
    (64, [dict(batch=128, max_ctx=300), dict(batch=32, max_ctx=800), dict(batch=64, max_ctx=4096, heads=64), dict(batch=256, max_ctx=32, heads=33)]),
    (32, [dict(batch=2, max_ctx=5687), dict(batch=1, max_ctx=3000), dict(batch=1, max_ctx=30), dict(batch=4, max_ctx=32768, heads=16), dict(batch=1, max_ctx=1000, heads=32),
          dict(batch=256, max_ctx=2048, heads=32), dict(batch=1000, max_ctx=1, heads=1)]),
])
def test_columns_of_a_decode(tmp, cols, batches):
    for b, l in zip(batches, logs(tmp, *(dict(call="decode", **b) for b in batches))):
        assert columns(l) == cols and l[0][0].endswith(",true>"), (b, l)


@pytest.mark.parametrize("cols,batches", [
    (128, [dict(batch=8, total=1100, max_new=256, max_ctx=8300), dict(batch=1, prefix=6007, new=211, heads=32), dict(batch=4, total=2400, max_new=700, max_ctx=700)]),
    (64, [dict(batch=1, prefix=500, new=32), dict(batch=32, prefix=4096, new=4, heads=16)]),
    (32, [dict(batch=1, new=40, heads=16), dict(batch=1, prefix=4000, new=8, heads=16), dict(batch=300, prefix=50, new=1, heads=3)]),
])
def test_columns_of_chunks(tmp, cols, batches):
    for b, l in zip(batches, logs(tmp, *(dict(call="resume", **b) for b in batches))):
        assert columns(l) == cols and l[0][0].endswith(",false>"), (b, l)


def test_a_stream_with_few_cus_takes_wide_columns(tmp):
    whole, few = logs(tmp, dict(call="decode", batch=5, max_ctx=2000), dict(call="decode", batch=5, max_ctx=2000, cus=24))
    assert columns(whole) == 32 and columns(few) == 128 and few[0][1] == "24"


def test_merges(tmp):
    none, small, wide = logs(tmp, dict(call="decode", batch=256, max_ctx=128), dict(call="decode", batch=4, max_ctx=32768, heads=16), dict(call="decode", batch=64, max_ctx=4096))
    assert len(none) == 1                                              # nothing that a share could cut
    assert small[1][0] == "latent_merge_kernel<1>" and wide[1][0] == "latent_merge_kernel<4>"


def test_short_contexts_stay_whole(tmp):
    """... and launch no merge, where there are units for an eighth of the CUs."""
    whole = [dict(batch=128, max_ctx=300), dict(batch=64, max_ctx=512, heads=32), dict(batch=16, max_ctx=500), dict(call="resume", batch=1, prefix=300, new=60, heads=100)]
    cut = [dict(batch=4, max_ctx=400, heads=32), dict(batch=64, max_ctx=513, heads=32), dict(call="resume", batch=2, prefix=400, new=8, heads=16)]
    got = logs(tmp, *({"call": "decode", **b} for b in whole + cut))
    assert [len(l) for l in got] == [1] * len(whole) + [2] * len(cut), got


@pytest.mark.parametrize("heads", G.HEADS)
def test_the_gpu_tests_of_whole_columns_reach_them(tmp, heads):
    decode, resume = logs(tmp, dict(call="decode", batch=len(G.CTX), max_ctx=G.LOOSE, heads=heads),
                          dict(call="resume", batch=len(G.CTX), total=sum(G.NEW), max_new=max(G.NEW), max_ctx=G.LOOSE, heads=heads))
    assert columns(decode) == (32 if heads <= 32 else 64 if heads <= 64 else 128)
    assert columns(resume) == (32 if max(G.NEW) * heads <= 32 else 64 if max(G.NEW) * heads <= 64 else 128)


def test_tokens_of_a_rotation(tmp):
    few, many = logs(tmp, dict(call="rows", batch=64, heads=32), dict(call="rows", batch=8, new=4096, heads=32))
    assert few == [["rope_rows_kernel<__bf16,false,1>", "64"]] and many == [["rope_rows_kernel<__bf16,false,4>", "8192"]]


def test_appends(tmp):
    step, prompt, f32 = logs(tmp, dict(call="append_rope", batch=64, heads=32), dict(call="append_rope", batch=8, new=4096, heads=32),
                             dict(call="append_rope", batch=5, new=40, heads=32, dtype="f32", layout=1))
    assert step[0][0] == "append_rope_kernel<__bf16,false,false>" and prompt[0][0] == "append_rope_kernel<__bf16,false,true>" and f32[0][0] == "append_rope_kernel<float,true,false>"
    got = logs(tmp, *(dict(call="append", batch=8, new=n, lat=lat, rd=rd) for lat, rd, n in ((512, 64, 100), (256, 32, 100), (128, 64, 101))))
    assert got == [[["append_latent_kernel<64,32>", "200"]], [["append_latent_kernel<32,16>", "100"]], [["append_latent_kernel<16,32>", "101"]]]


MOST = 0xFFFFFFFF // 256                       # workgroups of 256 threads that a launch holds


@pytest.mark.parametrize("call,most", [(dict(call="rows", heads=32), 4 * MOST), (dict(call="append"), 4 * MOST), (dict(call="append", lat=128, rd=32), 4 * MOST),
                                       (dict(call="append_rope", heads=32), 16 * (MOST - 2) + 15)])
def test_what_one_launch_holds(tmp, call, most):
    at, past = logs(tmp, *(dict(batch=1, max_ctx=16, total=n, **call) for n in (most, most + 1)))
    assert len(at) == 1 and int(at[0][1]) <= MOST, at
    assert past[0][0] == "refused" and past[0][1] == "-1", past
