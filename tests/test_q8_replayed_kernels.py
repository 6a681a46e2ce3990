"""The kernels that the batches of test_gpu_q8_replays.py take, on the whole device and on a stream of eight CUs."""
import pytest

from q8_launches import launched
from test_q8_dispatch import SHARED_CTX

# activations, channels, query heads (2 KV heads, pages of 16), prefixes, new tokens, prefill kernel: all CUs, eight CUs
REPLAYS = [
    ("bf16", 128, 16, [570, 260, 259], [130, 40, 1], "prefill_q8_split_kernel<__bf16,128,true,8>", "prefill_q8_kernel<4,128,true>"),
    ("bf16", 128, 16, [1700, 1500], [300, 120], "prefill_q8_split_kernel<__bf16,128,true,8>", "prefill_q8_kernel<8,128,true>"),
    ("bf16", 64, 16, [130, 0, 64, 700, 33], [70, 90, 0, 130, 1], "prefill_q8_split_kernel<__bf16,64,true,8>", "prefill_q8_kernel<4,64,true>"),
    ("bf16", 80, 16, [130, 0, 64, 700, 33], [70, 90, 0, 130, 1], "prefill_q8_split_kernel<__bf16,96,false,8>", "prefill_q8_kernel<4,128,false>"),
    ("bf16", 192, 16, [0, 0, 0], [200, 333, 64], "prefill_q8_split_kernel<__bf16,192,true,4>", "prefill_q8_kernel<4,256,false>"),
    ("bf16", 256, 16, [130, 0, 64, 700, 33], [70, 90, 0, 130, 1], "prefill_q8_split_kernel<__bf16,256,true,4>", "prefill_q8_kernel<4,256,true>"),
    ("f32", 96, 6, [691, 160, 227], [9, 140, 33], "prefill_q8_split_kernel<float,96,true,8>", "prefill_q8_split_kernel<float,96,true,4>"),
]


@pytest.mark.parametrize("dtype,d,hq,prefix,new,all_cus,eight", REPLAYS)
def test_kernels(tmp_path, dtype, d, hq, prefix, new, all_cus, eight):
    shape = dict(dtype=dtype, d=d, hq=hq, hkv=2, batch=len(new))
    resume = dict(call="resume", total=sum(new), max_new=max(new), max_ctx=max(p + n for p, n in zip(prefix, new)), **shape)
    calls = [dict(resume), dict(resume, cus=8), dict(call="decode", max_ctx=SHARED_CTX, **shape), dict(call="decode", max_ctx=SHARED_CTX, cus=8, **shape)]
    got = [[x.replace("q8::", "").rsplit(" ", 1)[0] for x in k] for k in launched(calls, tmp_path)]
    assert got[0] == [all_cus] and got[1] == [eight]
    for k in got[2:]:
        assert [x.split("<")[0] for x in k] == ["decode_q8_split_kernel", "decode_q8_merge_kernel"]
