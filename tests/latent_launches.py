"""Which kernels rotary and latent-cache calls launch, seen without a GPU, as launches.py sees it for the other caches."""
import json
import os
import subprocess
import sys

from launches import LIB, ROOT

SHAPE = dict(lat=512, rd=64, page=16, heads=128, d=128, hkv=8, dtype="bf16", layout=0, cus=256, prefix=0)


def launched(calls, tmp):
    """calls: dicts with call = decode | resume | append | rows | append_rope, the shape (SHAPE where left out), and either batch, prefix and new
    (equal sessions) or total, batch, max_new and max_ctx."""
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
    for n in ("decode", "resume"):
        getattr(lib, "ag_attn_%s_latent_workspace_bytes" % n).restype = C.c_size_t

    def struct(*fields):
        return type("S", (C.Structure,), {"_fields_": list(fields)})

    i32, p, i64, f = C.c_int32, C.c_void_p, C.c_int64, C.c_float
    ints = lambda *names: [(n, i32) for n in names]
    Latent = struct(("pool", p), *ints("num_pages", "page_size", "latent_dim", "rope_dim"))
    Cache = struct(("k_pool", p), ("v_pool", p), *ints("num_pages", "page_size", "num_kv_heads", "head_dim", "dtype"))
    Rope = struct(("turns", p), *ints("rot_dim", "layout"), ("magnitude", f))
    any_ = p(1 << 20)                                                  # an aligned address that nothing reads
    results = []
    for c in json.loads(sys.stdin.read()):
        batch, new, heads, lat, rd, d = c["batch"], c.get("new", 1), c["heads"], c["lat"], c["rd"], c["d"]
        total, max_new, max_ctx = c.get("total", batch * new), c.get("max_new", new), c.get("max_ctx", c["prefix"] + new)
        dtype, pages = (1 if c["dtype"] == "bf16" else 0), -(-max_ctx // c["page"])
        stream = p(c["cus"] if c["cus"] != 256 else 0)
        cache, lens = Latent(any_, 1 << 20, c["page"], lat, rd), (any_, any_, any_)
        rope = lambda rot: C.byref(Rope(any_, rot, c["layout"], f(1.0)))
        log.launch_log_take()
        if c["call"] == "decode":
            n = lib.ag_attn_decode_latent_workspace_bytes(batch, heads, lat, max_ctx)
            st = lib.ag_attn_decode_latent(C.byref(cache), any_, any_, any_, pages, any_, batch, max_ctx, heads, f(0.1), any_, C.c_size_t(n), stream)
        elif c["call"] == "resume":
            n = lib.ag_attn_resume_latent_workspace_bytes(batch, total, heads, lat, max_ctx)
            st = lib.ag_attn_resume_latent(C.byref(cache), any_, any_, any_, pages, *lens, batch, total, max_new, max_ctx, heads, f(0.1), any_, C.c_size_t(n), stream)
        elif c["call"] == "append":
            st = lib.ag_kv_append_latent(C.byref(cache), rope(rd), any_, i64(lat), any_, i64(rd), any_, pages, *lens, batch, total, stream)
        elif c["call"] == "rows":
            st = lib.ag_rope_rows(rope(d), dtype, any_, i64(heads * d), i64(d), any_, i64(heads * d), i64(d), heads, d, *lens, batch, total, 0, stream)
        else:
            kv = Cache(any_, any_, 1 << 20, c["page"], c["hkv"], d, dtype)
            st = lib.ag_kv_append_rope(C.byref(kv), rope(d), any_, any_, heads, any_, any_, any_, pages, *lens, batch, total, stream)
        if st:
            results.append(["refused %d %s" % (st, lib.ag_last_error().decode())])
        else:
            results.append(log.launch_log_take().decode().split("\n")[:-1])
    print(json.dumps(results))


if __name__ == "__main__":
    _main(*sys.argv[1:])
