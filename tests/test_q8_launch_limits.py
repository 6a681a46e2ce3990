"""Calls over an 8-bit cache at the ends of what one launch holds: HIP refuses 2^32 threads along a dimension of the grid, and a call beyond is
refused with a message, or takes another kernel, before any launch.  Seen on the CPU, through a HIP runtime that logs launches."""
import pytest

from q8_launches import launched

THREADS = {"decode_q8_direct_kernel": 256, "decode_q8_split_kernel": 256, "decode_q8_merge_kernel": 256, "append_q8_kernel": 256, "read_q8_kernel": 256,
           "prefill_q8_kernel<4": 256, "prefill_q8_kernel<8": 512, "prefill_q8_split_kernel": 256}
ONE = dict(hq=1, hkv=1, d=64)


@pytest.fixture(scope="module")
def tmp(tmp_path_factory):
    return tmp_path_factory.mktemp("launches")


def rows(n):
    return dict(batch=1, total=n, max_ctx=n, **ONE)


@pytest.mark.parametrize("fits,beyond,kernel", [
    (dict(call="decode", batch=(1 << 24) - 1, new=64, **ONE), dict(batch=1 << 24), "decode_q8_direct_kernel"),
    (dict(call="decode", batch=1 << 21, new=64, hq=32, hkv=8), None, "decode_q8_split_kernel"),
    (dict(call="decode", batch=(1 << 26) - 4, new=64, hq=1, hkv=1, d=256), dict(batch=(1 << 26) - 3), "decode_q8_split_kernel"),
    (dict(call="append", **rows(16 * ((1 << 24) - 3))), rows(16 * ((1 << 24) - 2)), "append_q8_kernel"),
    (dict(call="read", **rows(16 * ((1 << 24) - 3))), rows(16 * ((1 << 24) - 2)), "read_q8_kernel"),
    (dict(call="resume", batch=1 << 17, new=128 * 127, **ONE), dict(new=128 * 128 - 1), "prefill_q8_kernel<4"),
    (dict(call="resume", batch=1 << 16, new=256 * 127, hq=1, hkv=1), dict(new=256 * 128 - 1), "prefill_q8_kernel<8"),
    (dict(call="resume", batch=1 << 17, new=32 * 127, dtype="f32", **ONE), dict(new=32 * 128), "prefill_q8_split_kernel"),
])
def test_a_call_is_within_a_launch_or_refused(tmp, fits, beyond, kernel):
    inside, outside = launched([fits, {**fits, **(beyond or {})}], tmp)
    assert inside[0].split("q8::")[1].startswith(kernel), inside
    for line in inside + (outside if not outside[0].startswith("refused") else []):
        name, n = line.split("q8::")[1].rsplit(" ", 1)
        threads = next(t for k, t in THREADS.items() if name.startswith(k))
        assert 0 < int(n) * threads < 1 << 32, line
    if kernel == "decode_q8_direct_kernel":                       # one workgroup a pair no longer fits: shares
        assert outside[0].split("q8::")[1].startswith("decode_q8_split_kernel")
    elif beyond:
        assert outside[0].startswith("refused -1") and "launch" in outside[0], outside
