"""Which kernels the attention calls launch, how a call is cut into workgroups, and that the workspace bound holds: the library's host side on the CPU
over a HIP runtime that only writes launches down (tests/san/fake_hip.cpp).  As a script, in a process of its own: `python
test_host_attention.py FAKE LIB` with a JSON list of calls on stdin, results on stdout."""
import json
import os
import random
import shutil
import subprocess
import sys

if __name__ != "__main__":
    import pytest

    from fake_hip import build_runtime

    pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no g++")

    @pytest.fixture(scope="module")
    def fake(tmp_path_factory):
        return build_runtime(tmp_path_factory.mktemp("fake_hip"))

    def run(fake, calls):
        import paper_2502_19078_amd as pkg
        if not os.path.exists(pkg.lib_path()):
            from paper_2502_19078_amd import build
            build.build()
        r = subprocess.run([sys.executable, os.path.abspath(__file__), fake, pkg.lib_path()], input=json.dumps(calls), capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stderr[-2000:]
        return json.loads(r.stdout)

    def _kernels(result):
        assert result["status"] == 0, result
        short = lambda n: next(k for k in ("rows", "tiles", "prefix", "join", "qk_rope") if "k_attn_" + k in n or "k_" + k in n)
        return [(short(n), grid) for n, grid in result["launches"]]

    @pytest.mark.parametrize("call,want", [
        # 256 compute units: a step of few rows takes a workgroup for each, tiles two; a split has 128 keys at least
        (dict(do="window", B=1, T=1, Hq=32, H=8, D=128, cap=131072), [("rows", 8 * 32), ("join", 32)]),
        (dict(do="window", B=8, T=1, Hq=32, H=8, D=128, cap=16384, window=4096, sinks=4), [("rows", 64 * 4), ("join", 256)]),
        (dict(do="window", B=1, T=1, Hq=8, H=1, D=256, cap=128), [("rows", 1)]),
        (dict(do="window", B=1, T=1, Hq=40, H=1, D=256, cap=128), [("rows", 3)]),                   # a head group in tiles of 16
        (dict(do="window", B=64, T=1, Hq=32, H=8, D=128, cap=4096), [("rows", 512)]),
        (dict(do="window", B=2, T=4, Hq=4, H=1, D=64, cap=100), [("rows", 2)]),                     # 16 rows
        (dict(do="window", B=2, T=5, Hq=4, H=1, D=64, cap=100), [("tiles", 2)]),                    # 20
        (dict(do="window", B=1, T=8192, Hq=32, H=8, D=128, cap=8192, window=4096), [("tiles", 2048)]),
        (dict(do="window", B=1, T=100, Hq=4, H=4, D=80, cap=32768, dtype=0), [("tiles", 4 * 128), ("join", 400)]),
        (dict(do="prefix", B=4, Hq=8, H=2, D=64, cap=64, P=1000), [("rows", 2 * 8 + 4 * 2), ("join", 32)]),
        (dict(do="prefix", B=16, Hq=32, H=8, D=128, cap=512, P=8192), [("prefix", 8 * 32 + 128 * 2), ("join", 512)]),
        (dict(do="prefix", B=64, Hq=32, H=8, D=128, cap=64, P=100, dtype=0), [("prefix", 8 * 2 + 512), ("join", 2048 // 8)]),
        (dict(do="rope", B=1, T=1, Hq=32, H=8, D=128), [("qk_rope", 2)]),
        (dict(do="rope", B=1, T=4096, Hq=32, H=8, D=128), [("qk_rope", 4096 * 12 * 8 // 256)]),
        (dict(do="rope", B=2, T=300, Hq=5, H=1, D=256, dtype=0), [("qk_rope", 600 * 7 * 32 // 256)]),
    ])
    def test_kernels_and_workgroups(fake, call, want):
        assert _kernels(run(fake, [call])[0]) == want

    def test_the_workspace_bound_is_enough_for_every_call(fake):
        rng = random.Random(1)
        calls = []
        for _ in range(400):
            G, H = rng.choice([1, 2, 3, 7, 8, 20, 64]), rng.choice([1, 2, 5, 8, 16])
            c = dict(B=rng.choice([1, 2, 5, 17, 64, 300]), Hq=G * H, H=H, D=rng.choice([8, 64, 80, 96, 128, 200, 256]), dtype=rng.randint(0, 1),
                     cap=int(2 ** rng.uniform(0, 18)))
            if rng.random() < 0.6:
                calls.append(dict(c, do="window", T=rng.choice([1, 1, 2, 5, 16, 17, 100, 1000]), window=rng.choice([0, 0, 1, 100, 5000])))
            else:
                calls.append(dict(c, do="prefix", T=1, P=int(2 ** rng.uniform(0, 18))))
        assert [c for c, r in zip(calls, run(fake, calls)) if r["status"] != 0] == []

    def test_a_smaller_workspace_is_refused_and_a_refused_launch_reported(fake):
        c = dict(do="window", B=1, T=1, Hq=32, H=8, D=128, cap=131072)
        small, whole, fails = run(fake, [dict(c, bytes=256), c, dict(c, fail=1)])
        assert small["status"] == 5 and small["launches"] == []
        assert whole["status"] == 0 and len(whole["launches"]) == 2
        assert fails["status"] == 7 and len(fails["launches"]) == 1


def _main(fake_path, lib_path):
    import ctypes as C
    fake = C.CDLL(fake_path, mode=C.RTLD_GLOBAL)
    lib = C.CDLL(lib_path)
    fake.fake_take_log.restype = C.c_char_p
    lib.clada_attn_workspace_bytes.restype = C.c_size_t
    vp, i32, f32 = C.c_void_p, C.c_int32, C.c_float

    class Heads(C.Structure):
        _fields_ = [("data", vp), ("stride_b", C.c_int64), ("stride_t", C.c_int64), ("stride_h", C.c_int64)]

    class Kv(C.Structure):
        _fields_ = [("k", vp), ("v", vp), ("stride_b", C.c_int64), ("stride_h", C.c_int64), ("stride_n", C.c_int64)] + \
                   [(n, i32) for n in ("batch", "heads", "d", "capacity", "dtype", "n_sink", "ring")]

    class Rope(C.Structure):
        _fields_ = [("turns", vp), ("rotary_dim", i32), ("layout", i32), ("magnitude", f32)]

    buf = C.create_string_buffer(1 << 16)
    p = (C.addressof(buf) + 255) // 256 * 256               # stands for every device pointer; nothing reads it
    out = []
    for c in json.load(sys.stdin):
        B, T, Hq, H, D = c["B"], c.get("T", 1), c["Hq"], c["H"], c["D"]
        dt, cap = c.get("dtype", 1), c.get("cap", T)
        heads = C.byref(Heads(p, T * Hq * D, Hq * D, D))
        kv = lambda batch, rows: C.byref(Kv(p, p, H * rows * D, rows * D, D, batch, H, D, rows, dt, 0, 0))
        n = c.get("bytes") or lib.clada_attn_workspace_bytes(B, T, Hq, D)
        ctx = vp()
        assert lib.clada_create(C.byref(ctx), 0, C.c_size_t(n)) == 0
        if "fail" in c:
            fake.fake_fail_launch(C.c_long(c["fail"]))
        if c["do"] == "window":
            st = lib.clada_window_attn(ctx, heads, kv(B, cap), vp(p), None, B, T, Hq, c.get("window", 0), c.get("sinks", 0), f32(1.0), heads, vp(p), None)
        elif c["do"] == "prefix":
            st = lib.clada_shared_prefix_attn(ctx, heads, kv(1, c["P"]), c["P"], kv(B, cap), vp(p), B, Hq, f32(1.0), heads, vp(p), None)
        else:
            st = lib.clada_qk_rope(ctx, C.byref(Rope(p, D, 0, 1.0)), None, B, T, Hq, heads, heads, heads, vp(p), None, heads, kv(B, cap), None)
        rows = [r.split() for r in fake.fake_take_log().decode().splitlines()]
        out.append({"status": st, "launches": [[r[0], int(r[1])] for r in rows]})
        lib.clada_destroy(ctx)
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    _main(*sys.argv[1:3])
