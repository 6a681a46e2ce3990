"""Which kernels a call over an 8-bit cache launches, seen without a GPU, as launches.py sees it for the other caches."""
import json
import os
import subprocess
import sys

from launches import LIB, ROOT

SHAPE = dict(dtype="bf16", d=128, page=16, hq=32, hkv=8, cus=256, prefix=0)


def launched(calls, tmp):
    """calls: dicts with call = resume | decode | append | read, the shape (SHAPE where left out), and either batch, prefix and new (equal
    sessions) or total, batch, max_new and max_ctx."""
    so = os.path.join(str(tmp), "launch_log.so")
    if not os.path.exists(so):
        subprocess.run(["g++", "-shared", "-fPIC", "-O1", "-std=c++17", os.path.join(ROOT, "tests", "hostbuild", "launch_log.cpp"), "-o", so],
                       check=True, capture_output=True)
    r = subprocess.run([sys.executable, os.path.abspath(__file__), so, LIB], input=json.dumps([{**SHAPE, **c} for c in calls]),
                       capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    return json.loads(r.stdout)


def _main(log_so, lib_so):
    import ctypes as C
    log = C.CDLL(log_so, mode=C.RTLD_GLOBAL)
    log.launch_log_take.restype = C.c_char_p
    lib = C.CDLL(lib_so)
    lib.ag_last_error.restype = C.c_char_p
    lib.ag_attn_decode_q8_workspace_bytes.restype = C.c_size_t

    class Cache(C.Structure):
        _fields_ = [(n, C.c_void_p) for n in ("k_pool", "v_pool", "exps")] + [(n, C.c_int32) for n in ("num_pages", "page_size", "num_kv_heads", "head_dim", "dtype")]

    p, f = C.c_void_p, C.c_float
    any_ = p(1 << 20)                                                  # an aligned address that nothing reads
    results = []
    for c in json.loads(sys.stdin.read()):
        batch, new = c["batch"], c.get("new", 1)
        total, max_new, max_ctx = c.get("total", batch * new), c.get("max_new", new), c.get("max_ctx", c["prefix"] + new)
        cache = Cache(any_, any_, any_, 1 << 20, c["page"], c["hkv"], c["d"], 1 if c["dtype"] == "bf16" else 0)
        pages = -(-max_ctx // c["page"])
        stream = p(c["cus"] if c["cus"] != 256 else 0)
        log.launch_log_take()
        if c["call"] == "resume":
            st = lib.ag_attn_resume_q8(C.byref(cache), any_, any_, any_, pages, any_, any_, any_, batch, total, max_new, max_ctx, c["hq"], f(0.1), stream)
        elif c["call"] == "decode":
            n = lib.ag_attn_decode_q8_workspace_bytes(batch, c["hq"], c["d"], max_ctx)
            st = lib.ag_attn_decode_q8(C.byref(cache), any_, any_, any_, pages, any_, batch, max_ctx, c["hq"], f(0.1), any_, C.c_size_t(n), stream)
        else:
            call = lib.ag_kv_append_q8 if c["call"] == "append" else lib.ag_kv_read_q8
            st = call(C.byref(cache), any_, any_, any_, pages, any_, any_, any_, batch, total, stream)
        if st:
            results.append(["refused %d %s" % (st, lib.ag_last_error().decode())])
        else:
            results.append(log.launch_log_take().decode().split("\n")[:-1])
    print(json.dumps(results))


if __name__ == "__main__":
    _main(*sys.argv[1:])
