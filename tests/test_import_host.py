"""The binding on a torch that lacks the 4-bit and the scales' type (on the
CPU: no call reaches the GPU)."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import torch
for name in {missing}:
    delattr(torch, name)
from paper_2606_28516_amd import clearmoe as cm

assert cm.workspace_bytes(cm.make_shape(300, 128, 4, 2, cm.BF16, H=256, r=64, q=16)) > 0
x, w = torch.zeros(4, 128), torch.zeros(256, 128)

def refused(f, *a, **kw):
    try:
        f(*a, **kw)
    except cm.ClearMoEError:
        return True
    return False

# (tensors of the CPU)
assert refused(cm.dense_ffn_forward, x, w, torch.zeros(256), w.T, torch.zeros(128))
assert refused(cm.rms_norm, x) and refused(cm.quantize, x)
assert cm._format(torch.float8_e4m3fn) == 2 and refused(cm._format, torch.float32)
assert refused(cm._format, "float4_e2m1fn_x2")
assert (cm._value_cols(40), cm._scale_cols(40)) == (48, 4)
if hasattr(torch, "float4_e2m1fn_x2"):
    assert cm._format(torch.float4_e2m1fn_x2) == 5
"""


def _run(missing):
    r = subprocess.run([sys.executable, "-c", PROGRAM.format(missing=missing)], cwd=ROOT, capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


def test_without_the_4bit_type():
    _run(["float4_e2m1fn_x2"])


def test_without_the_scales_type():
    _run(["float8_e8m0fnu"])


def test_with_both():
    _run([])
