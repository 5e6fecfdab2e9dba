"""The 8-bit products' index and dispatch rules on the CPU: a host program
(gemm_q8_host.cpp) against the library's own headers and host code."""
import os
import subprocess

import pytest

from paper_2606_28516_amd import build as hb
from tests import test_gpu_q8_operands as operands
from tests import test_gpu_q8_range as scales

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if not os.path.exists(hb.HIPCC) or not os.path.exists(hb.LIB):
        pytest.skip("needs hipcc and the built library")
    out = str(tmp_path_factory.mktemp("gemm_host") / "gemm_q8_host")
    subprocess.check_call([hb.HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", f"-I{hb.INCLUDE}",
                           f"-I{hb.CSRC}", os.path.join(HERE, "gemm_q8_host.cpp"), "-o", out,
                           f"-L{hb.HERE}", "-l:" + os.path.basename(hb.LIB), f"-Wl,-rpath,{hb.HERE}"])
    return out


@pytest.mark.parametrize("check", ["row_tiles", "launch"])
def test_host_rules(program, check):
    r = subprocess.run([program, check], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr


OUT = {"float32": 0, "bfloat16": 1, "float8_e4m3fn": 2, "float8_e5m2": 3}
ALL = {"float32": {"rows", "small", "large"}, "bfloat16": {"rows", "small", "middle", "large"},
       "float8_e4m3fn": {"small", "large"}, "float8_e5m2": {"small", "large"}}


def _kernels(program, products):
    args = [str(v) for p in products for v in p]
    return subprocess.run([program, "kernels", *args], capture_output=True, text=True, check=True,
                          timeout=60).stdout.splitlines()


@pytest.mark.parametrize("out", OUT)
def test_gpu_sizes_cover_every_kernel(program, out):
    """What the GPU tests say about their sizes."""
    assert set(_kernels(program, [(M, N, 0, OUT[out]) for M, N, _ in scales.SIZES])) == ALL[out]
    mine = [(M, N, 0, OUT[out]) for M, N, _, o in operands.PRODUCTS if str(o) == f"torch.{out}"]
    if mine:
        assert set(_kernels(program, mine)) == ALL[out]
    # results stored in whole 16-byte pieces, and element by element
    for wide in (False, True):
        some = [p for p in mine if (p[1] % 8 == 0) == wide]
        assert not mine or out.startswith("float8") or set(_kernels(program, some)) >= ALL[out] - {"rows"}
