"""The host code of the paged cache calls and of relax_token_logprobs under the address and undefined-behaviour sanitizers, as
tests/test_sanitizers.py does for the other calls."""
import os

import pytest

from test_sanitizers import ROOT, SAN, run


def test_paged_host_code_under_address_and_undefined_sanitizers(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    from paper_2311_02103_amd import build as b
    objs = {s: os.path.join(b.OBJ, s[:-4] + ".o") for s in b.sources()}
    if not all(os.path.exists(o) for o in objs.values()):
        b.build(verbose=False)
    api_o, lib, exe = (str(tmp_path / name) for name in ("api_san.o", "librelax_san.so", "paged_san"))
    run([hipcc] + b.FLAGS + [f for s in SAN[:2] for f in ("-Xarch_host", s)] + ["-Xarch_host", "-fno-omit-frame-pointer", "-c", os.path.join(b.CSRC, "api.hip"), "-o", api_o],
        timeout=900)
    run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-fsanitize=address,undefined", "-fno-gpu-sanitize", "-o", lib, api_o] +
        [o for s, o in objs.items() if s != "api.hip"], timeout=600)
    run(["/opt/rocm/lib/llvm/bin/clang", "-std=c11", "-O1"] + SAN + ["-I" + os.path.join(ROOT, "include"), "-o", exe, os.path.join(ROOT, "tests", "sanitize", "paged_driver.c"),
         lib, "-Wl,-rpath," + str(tmp_path), "-Wl,-rpath,/opt/rocm/lib"], timeout=300)
    res = run([exe], leaks=False)
    assert "paged driver ok" in res.stdout and "runtime error" not in res.stderr and "AddressSanitizer" not in res.stderr
