"""A torch without the types of 4-bit operands: everything else is there."""
import subprocess
import sys
import sysconfig

from paper_2411_02581_b200 import build as build_mod


def test_the_operators_import_without_the_types():
    code = ("import torch\n"
            "del torch.float4_e2m1fn_x2, torch.float8_e8m0fnu\n"
            "from paper_2411_02581_b200 import moe\n"
            "assert moe.FP4 is None and moe.POWER is None and callable(moe.route) and callable(moe.fp8_matmul)\n")
    subprocess.run([sys.executable, "-c", code], check=True, cwd=build_mod.ROOT)


def test_the_marshalling_compiles_without_the_types():
    import os

    import torch
    base = os.path.dirname(torch.__file__)
    subprocess.run(["g++", "-fsyntax-only", "-std=c++20", "-DTUNA_TORCH_FP4=0", "-I", os.path.join(build_mod.ROOT, "include"), "-isystem", os.path.join(base, "include"),
                    "-isystem", os.path.join(base, "include", "torch", "csrc", "api", "include"), "-isystem", sysconfig.get_paths()["include"],
                    "-isystem", "/usr/local/cuda/include", build_mod.TORCH_SOURCE], check=True)
    named = [line for line in open(build_mod.TORCH_SOURCE) if "ScalarType::Float4_e2m1fn_x2" in line or "ScalarType::Float8_e8m0fnu" in line]
    assert len(named) == 1      # behind the switch
