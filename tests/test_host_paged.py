"""Which kernels the paged cache's calls launch, how a call is cut into workgroups, and that the workspace bound holds: the library's host side on the CPU
over a HIP runtime that only writes launches down (tests/san/fake_hip.cpp).  As a script, in a process of its own: `python
test_host_paged.py FAKE LIB` with a JSON list of calls on stdin, results on stdout."""
import json
import os
import random
import shutil
import subprocess
import sys

F32, BF16, MX4 = 0, 1, 2

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
        short = lambda n: next(k for k in ("paged_rows", "paged_tiles", "paged_read", "attn_join", "qk_rope") if "k_" + k in n)
        return [(short(n), grid) for n, grid in result["launches"]]

    @pytest.mark.parametrize("call,want", [
        # 256 compute units: a workgroup for each where rows are long (128 values) or eight waves share a tile, two where they are short; a split has 128 keys
        # at least, and is joined in the same launch
        (dict(do="attn", type=BF16, B=1, T=1, Hq=32, H=8, D=128, cap=131072), [("paged_rows", 8 * 32)]),
        (dict(do="attn", type=MX4, B=1, T=1, Hq=32, H=8, D=128, cap=131072), [("paged_rows", 8 * 32)]),
        (dict(do="attn", type=MX4, B=1, T=1, Hq=8, H=8, D=64, cap=131072), [("paged_rows", 8 * 32)]),
        (dict(do="attn", type=BF16, B=8, T=1, Hq=8, H=4, D=64, cap=16384), [("paged_rows", 32 * 16)]),
        (dict(do="attn", type=BF16, B=1, T=1, Hq=32, H=8, D=128, cap=131072, max_len=200), [("paged_rows", 8 * 2)]),
        (dict(do="attn", type=F32, B=1, T=1, Hq=8, H=8, D=128, cap=131072, window=256), [("paged_rows", 8 * 3)]),
        (dict(do="attn", type=F32, B=1, T=1, Hq=8, H=8, D=128, cap=131072, window=256, prefix=True), [("paged_rows", 8 * 32)]),
        (dict(do="attn", type=MX4, B=300, T=1, Hq=32, H=16, D=128, cap=131072), [("paged_rows", 4800)]),
        (dict(do="attn", type=BF16, B=1, T=1, Hq=40, H=1, D=256, cap=128), [("paged_rows", 3)]),               # a head group in tiles of 16
        (dict(do="attn", type=F32, B=2, T=2, Hq=8, H=1, D=64, cap=100), [("paged_rows", 2)]),                  # 16 rows
        (dict(do="attn", type=BF16, B=2, T=2, Hq=4, H=1, D=64, cap=100), [("paged_rows", 2)]),                 # 8
        (dict(do="attn", type=MX4, B=2, T=5, Hq=4, H=1, D=64, cap=100), [("paged_tiles", 2)]),                 # 20
        (dict(do="attn", type=BF16, B=1, T=8192, Hq=32, H=8, D=128, cap=8192, window=4096), [("paged_tiles", 2048)]),
        (dict(do="attn", type=F32, B=1, T=100, Hq=4, H=4, D=80, cap=32768), [("paged_tiles", 4 * 128), ("attn_join", 400)]),
        (dict(do="read", type=MX4, B=4, T=1001, Hq=8, H=8, D=128, cap=1024), [("paged_read", 1001)]),
        (dict(do="read", type=F32, B=1, T=1, Hq=1, H=1, D=8, cap=16), [("paged_read", 1)]),
        (dict(do="append", type=BF16, B=1, T=1, Hq=32, H=8, D=128, cap=1024), [("qk_rope", 2)]),
        (dict(do="append", type=MX4, B=2, T=2048, Hq=32, H=8, D=128, cap=4096), [("qk_rope", 4096 * 12 * 8 // 256)]),
    ])
    def test_kernels_and_workgroups(fake, call, want):
        assert _kernels(run(fake, [call])[0]) == want

    def test_the_workspace_bound_is_enough_for_every_call(fake):
        rng = random.Random(2)
        calls = []
        for _ in range(500):
            t, G, H = rng.randint(0, 2), rng.choice([1, 2, 3, 7, 8, 20, 64]), rng.choice([1, 2, 5, 8, 16])
            calls.append(dict(do="attn", type=t, B=rng.choice([1, 2, 5, 17, 64, 300]), Hq=G * H, H=H, D=rng.choice([32, 64, 96, 128, 256] if t == MX4 else [8, 64, 80, 128, 200]),
                              cap=16 * int(2 ** rng.uniform(0, 14)), T=rng.choice([1, 1, 2, 5, 16, 17, 100, 1000]), window=rng.choice([0, 0, 1, 100, 5000])))
        assert [c for c, r in zip(calls, run(fake, calls)) if r["status"] != 0] == []

    def test_a_smaller_workspace_is_refused_and_a_refused_launch_reported(fake):
        c = dict(do="attn", type=MX4, B=1, T=1, Hq=32, H=8, D=128, cap=131072)
        small, whole, fails = run(fake, [dict(c, bytes=256), c, dict(c, fail=0)])
        assert small["status"] == 5 and small["launches"] == []
        assert whole["status"] == 0 and len(whole["launches"]) == 1
        assert fails["status"] == 7 and fails["launches"] == []


def _main(fake_path, lib_path):
    import ctypes as C
    fake = C.CDLL(fake_path, mode=C.RTLD_GLOBAL)
    lib = C.CDLL(lib_path)
    fake.fake_take_log.restype = C.c_char_p
    lib.clada_attn_workspace_bytes.restype = C.c_size_t
    vp, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float

    class Heads(C.Structure):
        _fields_ = [("data", vp), ("stride_b", i64), ("stride_t", i64), ("stride_h", i64)]

    class Cache(C.Structure):
        _fields_ = [(n, vp) for n in ("k", "v", "k_scales", "v_scales")] + [(n, i64) for n in ("stride_p", "stride_h", "stride_n")] + [("table", vp), ("table_stride", i64)] + \
                   [(n, i32) for n in ("pages", "heads", "page_size", "d", "batch", "max_pages", "type")]

    class Scores(C.Structure):
        _fields_ = [("scale", f32), ("cap", f32), ("slopes", vp), ("prefix_lens", vp), ("first", vp), ("window", i32)]

    class Rope(C.Structure):
        _fields_ = [("turns", vp), ("rotary_dim", i32), ("layout", i32), ("magnitude", f32)]

    buf = C.create_string_buffer(1 << 16)
    p = (C.addressof(buf) + 255) // 256 * 256               # stands for every device pointer; nothing reads it
    out = []
    for c in json.load(sys.stdin):
        B, T, Hq, H, D = c["B"], c["T"], c["Hq"], c["H"], c["D"]
        heads = C.byref(Heads(p, T * Hq * D, Hq * D, D))
        cache = C.byref(Cache(p, p, p, p, 16 * H * D, 16 * D, D, p, c["cap"] // 16, 1000, H, 16, D, B, c["cap"] // 16, c["type"]))
        n = c.get("bytes") or lib.clada_attn_workspace_bytes(B, T, Hq, D)
        ctx = vp()
        assert lib.clada_create(C.byref(ctx), 0, C.c_size_t(n)) == 0
        if "fail" in c:
            fake.fake_fail_launch(C.c_long(c["fail"]))
        if c["do"] == "attn":
            scores = C.byref(Scores(1.0, 0.0, None, p if c.get("prefix") else None, None, c.get("window", 0)))
            st = lib.clada_paged_attn(ctx, heads, cache, vp(p), None, B, T, Hq, c.get("max_len", 0), scores, heads, vp(p), None)
        elif c["do"] == "read":
            st = lib.clada_paged_read(ctx, cache, vp(p), B, T, heads, heads, None)
        else:
            st = lib.clada_paged_rope(ctx, C.byref(Rope(p, D, 0, 1.0)), None, B, T, Hq, heads, heads, heads, vp(p), heads, cache, None)
        rows = [r.split() for r in fake.fake_take_log().decode().splitlines()]
        out.append({"status": st, "launches": [[r[0], int(r[1])] for r in rows]})
        lib.clada_destroy(ctx)
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    _main(*sys.argv[1:3])
