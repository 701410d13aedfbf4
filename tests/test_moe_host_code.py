"""The operators' host code without the optimiser, which may drop a faulty operation whose result is unused.  No GPU needed."""
import os
import subprocess
import sys

import pytest

from paper_2411_02581_b200 import build as build_mod

ASK = """
import ctypes, sys
L, n = ctypes.CDLL(sys.argv[1]), ctypes.c_size_t(77)
i64 = ctypes.c_int64
for f in (L.tuna_moe_order_workspace_bytes, L.tuna_moe_route_workspace_bytes):
    for ranks in (1, 4, 4096):
        assert f(i64(0), 64, 2, ranks, ctypes.byref(n)) == 0 and n.value == 0, (f, ranks, n.value)
    assert f(i64(4096), 64, 2, 4, ctypes.byref(n)) == 0 and n.value > 0
print("asked")
"""


@pytest.fixture(scope="module")
def plain_library(tmp_path_factory):
    """tuna_route.cu with its host code at -O0 (and its kernels left as PTX: they are not run)."""
    out = str(tmp_path_factory.mktemp("plain") / "route.so")
    subprocess.check_call([build_mod._nvcc(), "-gencode", "arch=compute_100a,code=compute_100a", "-std=c++20", "-O0", "-Xcompiler", "-O0,-fPIC", "-shared",
                           "-cudart", "static", "-I", os.path.join(build_mod.ROOT, "include"), "-I", build_mod.CSRC,
                           os.path.join(build_mod.CSRC, "tuna_route.cu"), "-o", out])
    return out


def test_workspace_sizes_of_no_tokens(plain_library):
    r = subprocess.run([sys.executable, "-c", ASK, plain_library], capture_output=True, text=True)
    assert r.returncode == 0 and "asked" in r.stdout, (r.returncode, r.stderr)
