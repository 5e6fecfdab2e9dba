"""The GELU's polynomials as they stand in the source (csrc/q8_tile.h),
evaluated in float32 on the CPU: the errors that its comments state."""
import math
import os
import re

import numpy as np
import pytest
import torch

from paper_2606_28516_amd import build as hb
from tests.test_gpu_q4_gelu import OWN


def coefficients(name):
    with open(os.path.join(hb.CSRC, "q8_tile.h")) as f:
        body = re.search(r"constexpr float %s\[\d+\] = \{(.*?)\};" % name, f.read(), re.S).group(1)
    return [np.float32(c.strip().rstrip("f")) for c in body.split(",")]


def evaluate(c, x):
    """The polynomial in x by fused multiply-adds in float32 (a product of two
    float32 is exact in float64, and so is all but the last bits of the sum)."""
    p = np.full(x.shape, c[-1], np.float32)
    for k in c[-2::-1]:
        p = (x.astype(np.float64) * p.astype(np.float64) + np.float64(k)).astype(np.float32)
    return p


def log2_phi(a):
    return (torch.special.log_ndtr(torch.from_numpy(-a.astype(np.float64))) / math.log(2.0)).numpy()


def tail(a):
    """|v| Phi(-|v|) far out, as the kernels have it."""
    s = a * a
    t = evaluate(coefficients("kQ4GeluTail"), np.float32(1) / s)
    return t * np.exp2(s * np.float32(-0.72134752044448170368))


def test_4bit_products():
    c = coefficients("kQ4Gelu")
    assert c[0] == -1.0
    lo = 0.0
    for hi, own in OWN:
        a = np.linspace(lo, hi, 400001).astype(np.float32)
        if lo < 5.0:
            off = np.abs(np.exp2(evaluate(c, a).astype(np.float64) - log2_phi(a)) - 1)
        else:
            off = np.abs(tail(a).astype(np.float64) / (a * np.exp2(log2_phi(a))) - 1)
        assert off.max() <= own, (hi, off.max())
        lo = hi
    # further out: nothing
    far = np.concatenate([np.linspace(13.25, 100, 20001), np.logspace(2, 18, 2001)]).astype(np.float32)
    assert (tail(far) < 2.0 ** -126).all()
    # the halves of small values are exact
    small = np.float32(2.0) ** -np.arange(27, 149, dtype=np.float32)
    assert (evaluate(c, small) == -1).all()


@pytest.mark.parametrize("name,most", [("kQ8Gelu", 3.5e-6)])
def test_8bit_products(name, most):
    """Up to |v| = 6: the polynomial's own error (5.0e-6 of the exponent)."""
    c = [np.float64(k) for k in coefficients(name)]
    a = np.linspace(0, 6, 400001)
    off = np.abs(np.polyval(c[::-1], a) - log2_phi(a))
    assert off.max() <= 5.05e-6 and off.max() * math.log(2.0) <= most
