"""The 8-bit products and the FFN made of them far from one: scales near both
ends of their range, at sizes that reach every kernel."""
import math

import pytest
import torch

from paper_2606_28516_amd import clearmoe as cm
from tests.q8_util import HALF, TINY, dequantize, quantize_ref
from tests.test_gpu_q8 import CUT, FLIPS, _ffn_inputs, _ffn_reference, _sum_bound

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
DENORMAL = 2.0 ** -149        # the smallest step of a float32


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _operand(g, rows, K, fmt, block_rows, exponents, tiny=False):
    """Random bytes with the scales 2^exponents[block] and up to eight times
    more or less; tiny: only the format's smallest values."""
    v, s = quantize_ref(torch.randn(1, rows, K, generator=g), fmt, block_rows)
    v, s = v[0].contiguous(), s[0]
    if tiny:
        v = torch.randint(0, 4, v.shape, generator=g).to(torch.uint8)
    nk = len(exponents)
    s[:, :nk] = (127 + exponents + torch.randint(-3, 4, (s.shape[0], nk), generator=g)).to(torch.uint8)
    s = s.contiguous()
    return v.view(fmt).cuda(), s.view(torch.float8_e8m0fnu).cuda(), dequantize(v.view(fmt), s, block_rows)


# rows, columns, k: 16 x 16 tiles, the small and the large tiles of each result
# type (128 x 128 for bfloat16 alone), edge tiles in all of them
SIZES = [(5, 40, 400), (300, 1550, 400), (2000, 1550, 272), (4200, 1550, 400), (9000, 1550, 144)]


def _check(M, N, K, out, ea, eb, fa=E4M3, fb=E4M3, tiny=False):
    g = _gen(M + K)
    nk = -(-K // 128)
    a, sa, a64 = _operand(g, M, K, fa, 1, ea[:nk], tiny)
    b, sb, b64 = _operand(g, N, K, fb, 128, eb[:nk], tiny)
    ref, mass = a64 @ b64.T, a64.abs() @ b64.abs().T
    # every product, block sum and addition may end among the denormals
    d = _sum_bound(K, mass, out == F32) + (K + nk) * DENORMAL
    c = cm.quantized_gemm(a, sa, b, sb, out_dtype=out)
    if out in HALF:
        v, s = c
        step = torch.ldexp(torch.ones(s.shape, dtype=torch.float64), s.cpu().view(torch.uint8).int() - 127)
        c = dequantize(v, s, 1)[:, :N]
        bound = HALF[out] * ref.abs() + TINY[out] * step.repeat_interleave(128, dim=1)[:, :N] + 1.2 * d
    else:
        c = c.cpu().double()
        half = torch.finfo(out).eps / 2
        # (bfloat16 denormals have steps of 2^-133)
        bound = half * ref.abs() + (1 + half) * d + (2.0 ** -134 if out == BF16 else DENORMAL)
    bad = ~((c - ref).abs() <= bound)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist())


@pytest.mark.parametrize("out", [F32, BF16, E4M3, E5M2])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_opposite_scales(M, N, K, out):
    """The two operands' scales of a block are up to 2^113 and 2^-113: a sum
    times one of them alone would leave float32's range."""
    e = torch.tensor([110, -110, 60, -100])
    _check(M, N, K, out, e, -e)


@pytest.mark.parametrize("fa,fb", [(E4M3, E5M2), (E5M2, E4M3), (E5M2, E5M2)])
@pytest.mark.parametrize("M,N,K", [(5, 40, 400), (300, 1550, 400)])
def test_opposite_scales_of_other_formats(M, N, K, fa, fb):
    e = torch.tensor([-100, 100, -60, 90])
    _check(M, N, K, F32, e, -e, fa, fb)


@pytest.mark.parametrize("M,N,K", SIZES)
def test_scales_whose_product_is_no_normal_number(M, N, K):
    """2^-135 and 2^127 together (up to 2^6 more or less), and sums that bring the
    results back."""
    _check(M, N, K, F32, torch.tensor([-120] * 4), torch.tensor([-15] * 4))
    _check(M, N, K, F32, torch.tensor([110] * 4), torch.tensor([17] * 4), tiny=True)


@pytest.mark.parametrize("M,N,K", [(5, 40, 400), (300, 1550, 400), (4200, 1550, 400)])
def test_nan_scales_spoil_their_rows_alone(M, N, K):
    g = _gen(4)
    e = torch.zeros(4, dtype=torch.int32)
    a, sa, _ = _operand(g, M, K, E4M3, 1, e)
    b, sb, _ = _operand(g, N, K, E4M3, 128, e)
    want = cm.quantized_gemm(a, sa, b, sb, out_dtype=F32)
    sa.view(torch.uint8)[3, 1] = 255
    got = cm.quantized_gemm(a, sa, b, sb, out_dtype=F32)
    keep = [i for i in range(M) if i != 3]
    assert got[3].isnan().all() and torch.equal(got[keep], want[keep])
    sb.view(torch.uint8)[0, 2] = 255
    got = cm.quantized_gemm(a, sa, b, sb, out_dtype=F32)
    assert got[:, :128].isnan().all() and torch.equal(got[keep, 128:], want[keep, 128:])


@pytest.mark.parametrize("M,N,K", [(5, 40, 400), (300, 1550, 400), (4200, 1550, 400)])
def test_rows_do_not_depend_on_the_rows_beside_them(M, N, K):
    """Extreme scales of some rows leave the others' results as they were."""
    g = _gen(6)
    e = torch.zeros(4, dtype=torch.int32)
    a, sa, _ = _operand(g, M, K, E4M3, 1, e)
    b, sb, _ = _operand(g, N, K, E4M3, 128, e)
    want = cm.quantized_gemm(a, sa, b, sb, out_dtype=F32)
    odd = torch.zeros(M, dtype=torch.bool)
    odd[1::3] = True
    sa.view(torch.uint8)[1::6] = 1
    sa.view(torch.uint8)[4::6] = 254
    got = cm.quantized_gemm(a, sa, b, sb, out_dtype=F32)
    assert torch.equal(got[~odd], want[~odd])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("power", [118, -118])
@pytest.mark.parametrize("T", [1, 16, 17, 300])
def test_ffn_of_large_and_small_rows(T, power, dtype):
    D, H = 200, 392
    x, W1, b1, W2, b2 = _ffn_inputs(T, D, H, 0, dtype, T)
    x = x * 2.0 ** power
    b1, b2 = torch.zeros_like(b1), torch.zeros_like(b2)
    w1, s1 = cm.quantize(W1.cuda(), block_rows=128)
    w2, s2 = cm.quantize(W2.cuda(), block_rows=128)
    y = cm.quantized_ffn_forward(x.cuda(), w1, s1, b1.cuda(), w2, s2, b2.cuda()).cpu().double()
    half = torch.finfo(dtype).eps / 2
    ref, coarse, fine = _ffn_reference(x, dequantize(w1, s1, 128), b1.double(), dequantize(w2, s2, 128), b2.double(),
                                       D, H, half)
    assert y.isfinite().all()
    assert ((y - ref).abs() <= coarse).all()
    assert (y - fine).norm() <= (half + CUT + FLIPS) * fine.norm()
