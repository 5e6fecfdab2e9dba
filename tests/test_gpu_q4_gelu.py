"""GELU of the 4-bit products, from its middle to where it leaves float32's
range, at sizes that reach every kernel: the sums are the bias, so that all of
the error is the GELU's."""
import math

import pytest
import torch

from paper_2606_28516_amd import clearmoe as cm
from tests.q4_util import E2M1, dequantize4, exponent4
from tests.q8_util import HALF, TINY, dequantize, scale_exponent
from tests.test_gpu_q8 import _gelu

pytestmark = pytest.mark.gpu

E4M3, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
BF16, F32 = torch.bfloat16, torch.float32

# |v| up to .. and what |v| Phi(-|v|) is off by there, of itself
OWN = [(1.0, 3e-7), (2.0, 5.6e-7), (4.0, 1.6e-6), (5.0, 3.8e-6), (13.2, 8e-6)]


def _bound(v):
    """Before the result's rounding: that, and the last bits of the power of two
    and of the reciprocal (2^-23 of themselves each); below 2^-126 nothing may
    be left."""
    a = v.abs()
    own = torch.zeros_like(v)
    for most, e in reversed(OWN):
        own = torch.where(a <= most, e, own)
    h = 0.5 * a * torch.special.erfc(a / math.sqrt(2.0))
    return (own + 2.0 ** -22) * h + 2.0 ** -126


def _values(n, g):
    """In order, so that blocks of small results have no large one beside them."""
    v = [torch.linspace(-13.5, -6, n // 3), torch.linspace(-6, 6, n // 4), torch.linspace(6, 40, n // 20),
         torch.ldexp(torch.randn(n // 8, generator=g), torch.randint(-60, -1, (n // 8,), generator=g))]
    v = torch.cat(v)
    return torch.cat([v, 6 * torch.randn(n - v.shape[0], generator=g)]).float()


# rows; 64 x 64; 64 x 128; two groups along k; 128 x 128 of both stages, the largest
SIZES = [(5, 1990, 64), (90, 2000, 64), (2000, 2000, 96), (700, 1990, 2112), (3000, 2100, 528), (4300, 2100, 800),
         (12000, 2100, 96), (16000, 2000, 544)]


@pytest.mark.parametrize("out", [BF16, F32, E4M3, E2M1])
@pytest.mark.parametrize("fa", [E4M3, E2M1])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_gelu(M, N, K, fa, out):
    g = torch.Generator().manual_seed(M)
    v = _values(N, g)
    a, sa = cm.quantize(torch.zeros(M, K, device="cuda"), fa)
    b, sb = cm.quantize(torch.zeros(N, K, device="cuda"), E2M1)
    c = cm.quantized_gemm(a, sa, b, sb, bias=v.cuda(), gelu=True, out_dtype=out)
    first = [t.view(torch.uint8)[:1] for t in (c if isinstance(c, tuple) else (c,))]
    for t, f in zip(c if isinstance(c, tuple) else (c,), first):
        assert (t.view(torch.uint8) == f).all()                          # (all rows alike)
    ref = _gelu(v.double())
    _check(first, ref, _bound(v.double()), out)


def _check(c, ref, d, out):
    N = ref.shape[0]
    if out in (BF16, F32):
        got = c[0].view(out).cpu().double()[0]
        half = torch.finfo(out).eps / 2
        bad = (got - ref).abs() > half * ref.abs() + (1 + half) * d
        assert not bad.any(), (bad.nonzero()[:4].tolist(), int(bad.sum()))
        return
    width = 32 if out == E2M1 else 128
    full = (dequantize4(c[0], c[1]) if out == E2M1 else dequantize(c[0].view(E4M3), c[1], 1))[0, :N]
    nb = -(-N // width)
    e = c[1].cpu()[0, :nb].int() - 127
    pad = torch.nn.functional.pad
    block = lambda t: pad(t, (0, nb * width - N)).reshape(nb, width)
    at = (lambda t: exponent4(t)) if out == E2M1 else (lambda t: scale_exponent(t, E4M3))
    most = block(ref.abs()).amax(1)
    off = torch.gather(block(d), 1, block(ref.abs()).argmax(1, keepdim=True))[:, 0]
    assert ((e >= at((most - off).clamp(min=0))) & (e <= at(most + off)) | (most <= off)).all()
    step = torch.ldexp(torch.ones(nb, dtype=torch.float64), e).repeat_interleave(width)[:N]
    if out == E2M1:
        size = (ref.abs() + d) / step
        bound = torch.where(size < 2, 0.25, torch.where(size < 4, 0.5, 1.0)) * step + d
    else:
        bound = HALF[E4M3] * (ref.abs() + d) + TINY[E4M3] * step + d
    bad = (full - ref).abs() > bound
    assert not bad.any(), (bad.nonzero()[:4].tolist(), int(bad.sum()))


@pytest.mark.parametrize("act", [E4M3, E2M1])
@pytest.mark.parametrize("T", [1, 16, 17, 700])
def test_hidden_values_of_an_ffn(T, act):
    """Each output is one hidden value as it was rounded."""
    n = 640
    g = torch.Generator().manual_seed(T)
    v = _values(n, g)
    w1, s1 = cm.quantize(torch.zeros(n, n, device="cuda"), E2M1)
    w2, s2 = cm.quantize(torch.eye(n, device="cuda"), E2M1)
    x = torch.randn(T, n, generator=g).cuda()
    y = cm.quantized_ffn_forward(x, w1, s1, v.cuda(), w2, s2, None, activations=act)
    assert (y == y[:1]).all()
    # the same rounding by the quantiser, of values that are off by the bound at most
    ref, d = _gelu(v.double()), _bound(v.double())
    y = y[0].cpu().double()
    near = [cm.quantize(t.float()[None].cuda(), act) for t in (ref - d, ref + d)]
    lo, hi = [cm.dequantize(*q, n, dtype=F32)[0].cpu().double() for q in near]
    bad = (y < lo) | (y > hi)
    assert not bad.any(), (bad.nonzero()[:4].tolist(), int(bad.sum()))
