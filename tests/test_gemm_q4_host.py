"""The 4-bit products' dispatch rules on the CPU: a host program
(gemm_q4_host.cpp) against the library's own headers and host code."""
import os
import subprocess

import pytest

from paper_2606_28516_amd import build as hb
from tests import test_gpu_q4 as gpu
from tests.q8_util import up

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if not os.path.exists(hb.HIPCC) or not os.path.exists(hb.LIB):
        pytest.skip("needs hipcc and the built library")
    out = str(tmp_path_factory.mktemp("gemm_host") / "gemm_q4_host")
    subprocess.check_call([hb.HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", f"-I{hb.INCLUDE}",
                           f"-I{hb.CSRC}", os.path.join(HERE, "gemm_q4_host.cpp"), "-o", out,
                           f"-L{hb.HERE}", "-l:" + os.path.basename(hb.LIB), f"-Wl,-rpath,{hb.HERE}"])
    return out


@pytest.mark.parametrize("what", ["launch", "rounds"])
def test_launch(program, what):
    r = subprocess.run([program, what], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr


OUT = {gpu.F32: 0, gpu.BF16: 1, gpu.E4M3: 2, gpu.E2M1: 4}
ALL = {(gpu.E2M1, gpu.F32): {"rows", "small", "split", "wide", "middle", "deep"},
       (gpu.E2M1, gpu.BF16): {"rows", "small", "split", "wide", "middle", "deep", "large"},
       (gpu.E2M1, gpu.E4M3): {"wide", "middle", "deep", "large"},
       (gpu.E2M1, gpu.E2M1): {"small", "split", "wide", "middle", "deep", "large"},
       (gpu.E4M3, gpu.F32): {"rows", "small", "split", "wide", "middle"},
       (gpu.E4M3, gpu.BF16): {"rows", "small", "split", "wide", "middle", "large"},
       (gpu.E4M3, gpu.E4M3): {"wide", "middle", "large"},
       (gpu.E4M3, gpu.E2M1): {"small", "split", "wide", "middle", "large"}}


@pytest.mark.parametrize("fa,out", ALL)
def test_gpu_sizes_cover_every_kernel(program, fa, out):
    sizes = [(M, N, K, 0) for M, N, K in gpu.SIZES + gpu.MORE]
    sizes += [(M, N, K, len(o) - 1 if o else 0) for M, N, K, o, a, c in gpu.MANY if (a, c) == (fa, out)]
    unit = 32 if fa == gpu.E2M1 else 16
    args = [str(v) for M, N, K, E in sizes for v in (M, N, up(K, unit), E, 4 if fa == gpu.E2M1 else 0, OUT[out])]
    names = subprocess.run([program, "kernels", *args], capture_output=True, text=True, check=True,
                           timeout=60).stdout.split()
    assert set(names) == ALL[fa, out]


def test_gpu_sizes_of_two_launches(program):
    args = [str(v) for M, N, K, _ in gpu.ROUNDS for v in (M, N, K)]
    rows = subprocess.run([program, "whole", *args], capture_output=True, text=True, check=True, timeout=60).stdout.split()
    assert [int(r) for r in rows] == [w for *_, w in gpu.ROUNDS]
