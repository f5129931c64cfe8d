"""The host code of the paged 4-bit cache, of the heads and of the scaled tables under the address and undefined-behaviour sanitizers, and the argument marshalling in C
under the latter, as tests/test_sanitizers.py does for the other calls."""
import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_sanitizers import ROOT, SAN, run

SOURCES = ["api.hip", "attn_paged4.hip", "attn_paged.hip", "paged4_append.hip", "heads.hip", "rope_scaled.hip"]      # with launches that are cut on the host


def test_paged4_host_code_under_address_and_undefined_sanitizers(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    from paper_2311_02103_amd import build as b
    objs = {s: os.path.join(b.OBJ, s[:-4] + ".o") for s in b.sources()}
    if not all(os.path.exists(o) for o in objs.values()):
        b.build(verbose=False)
    made = {s: str(tmp_path / (s[:-4] + "_san.o")) for s in SOURCES}

    def compile_(s):
        run([hipcc] + b.FLAGS + [f for x in SAN[:2] for f in ("-Xarch_host", x)] + ["-Xarch_host", "-fno-omit-frame-pointer", "-c", os.path.join(b.CSRC, s), "-o", made[s]], timeout=900)
    with ThreadPoolExecutor(max_workers=6) as pool:
        list(pool.map(compile_, SOURCES))
    lib, exe = str(tmp_path / "librelax_san.so"), str(tmp_path / "paged4_san")
    run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-fsanitize=address,undefined", "-fno-gpu-sanitize", "-o", lib] + [made.get(s, o) for s, o in objs.items()], timeout=600)
    run(["/opt/rocm/lib/llvm/bin/clang", "-std=c11", "-O1"] + SAN + ["-I" + os.path.join(ROOT, "include"), "-o", exe, os.path.join(ROOT, "tests", "sanitize", "paged4_driver.c"),
         lib, "-lm", "-Wl,-rpath," + str(tmp_path), "-Wl,-rpath,/opt/rocm/lib"], timeout=300)
    res = run([exe], leaks=False)
    assert "paged4 driver ok" in res.stdout and "runtime error" not in res.stderr and "AddressSanitizer" not in res.stderr


MARSHAL = r'''
import ctypes as C, importlib.util, sys
spec = importlib.util.spec_from_file_location("_marshal", sys.argv[1])
m = importlib.util.module_from_spec(spec)
spec.loader.exec_module(m)
got = []
f = C.CFUNCTYPE(C.c_int32, *[C.c_int64] * 6)(lambda *a: got.append(a) or -1)
call = m.Call(C.cast(f, C.c_void_p).value, "pirsip")
m.slow_stream(lambda s: 0x50 if s is None else 1 << 63)
class At:
    _at = 0xffffffffffff
class Stream:
    cuda_stream = 0x7fffffff0000
for q, kv, slots in ([[1], [1], None], [[2 ** 31 - 1] * 3, [5, 6, 7], [0, 2, 1]], [list(range(1, 3000)), list(range(1, 3000)), list(range(2999))]):
    for table in (None, 0x7fffffffffff):
        s = m.Seqs(q, kv, slots, table)
        assert call(2 ** 64 - 1, -2 ** 63, s, Stream(), 2 ** 63 - 1, None) == -1
for args in (("x", 1, None, None, 1, 1), (1, 2 ** 63, None, None, 1, 1), (-1, 1, None, None, 1, 1), (1,), (1, 1, object(), None, 1, 1)):
    try:
        call(*args)
    except (TypeError, OverflowError, ValueError, AttributeError):
        pass
for bad in (([1], [], None, None), ([1, 1], [1, 1], [1], None), (["x"], [1], None, None), ([None], [1], None, None), (1, [1], None, None), ([1], [1], 7, None)):
    try:
        m.Seqs(*bad)
    except (TypeError, OverflowError, ValueError):
        continue
    raise SystemExit("accepted %r" % (bad,))
assert call(0, 0, At(), None, 0, 0) == -1
print("marshal ok", len(got))
'''


def test_marshalling_under_the_undefined_behaviour_sanitizer(tmp_path):
    from paper_2311_02103_amd import build as b
    lib = str(tmp_path / "_marshal.so")
    run(["gcc", "-O1", "-g", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-shared", "-fPIC", "-I" + sysconfig.get_paths()["include"],
         "-I" + os.path.join(ROOT, "include"), "-o", lib, os.path.join(b.CSRC, "marshal.c")])
    res = subprocess.run([sys.executable, "-c", MARSHAL, lib], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and "marshal ok" in res.stdout and "runtime error" not in res.stderr, res.stdout + res.stderr
