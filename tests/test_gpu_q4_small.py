"""The 4-bit FFN where a bound that counts absolute errors says nothing: rows
far below one value by value, few rows by expert; and what a NaN scale leaves of
8-bit results beside it."""
import pytest
import torch

from paper_2606_28516_amd import clearmoe as cm
from tests.q4_util import E2M1
from tests.q8_util import HALF, TINY, dequantize, scale_exponent
from tests.test_gpu_q4 import _ffn_weights, _operand4, _rounded, _rows
from tests.test_gpu_q4_gelu import _bound
from tests.test_gpu_q8 import _ffn_inputs, _gelu, _gen, _sum_bound

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("act", [E4M3, E2M1])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("power", [-118, -40, -3])
@pytest.mark.parametrize("T", [1, 16, 17, 300])
def test_ffn_of_small_rows(T, power, dtype, act):
    """Each value against the definition with z exact and any rounding of it to
    the grid around it: a bound that is as small as the rows are."""
    D, H = 200, 392
    x, W1, b1, W2, b2 = _ffn_inputs(T, D, H, 0, dtype, T)
    x = x * 2.0 ** power
    w1, s1, w2, s2, d1, d2 = _ffn_weights(W1, W2)
    y = cm.quantized_ffn_forward(x.cuda(), w1, s1, None, w2, s2, None, activations=act).cpu().double()
    half = torch.finfo(dtype).eps / 2
    xq = _rounded(x.double(), act)[0]
    pre, mass = xq @ d1.T, xq.abs() @ d1.abs().T
    z = _gelu(pre)
    # GELU's slope is at most 1.13
    dz = 1.13 * _sum_bound(D, mass, True) + _bound(pre) - 2.0 ** -126 + 2.0 ** -149
    _, s = _rounded(z.abs() + dz, act)
    off = 1.0 * s + 1.2 * dz if act == E2M1 else HALF[E4M3] * z.abs() + TINY[E4M3] * s + 1.2 * dz
    ref, ym = z @ d2.T, (z.abs() + off) @ d2.abs().T
    bound = off @ d2.abs().T + _sum_bound(H, ym, True) + half * ym + 2.0 ** -134
    assert ((y - ref).abs() <= bound).all()
    assert y.norm() > 0.7 * ref.norm()


@pytest.mark.parametrize("act", [E4M3, E2M1])
@pytest.mark.parametrize("T,D,H,offsets", [(7, 64, 256, [0, 1, 1, 7]), (12, 72, 264, [2, 5, 9]), (16, 384, 1536, [0, 3, 4, 15]),
                                           (16, 130, 516, [1, 16])])
def test_few_rows_by_expert_as_by_themselves(T, D, H, offsets, act):
    E = len(offsets) - 1
    x, W1, b1, W2, b2 = _ffn_inputs(T, D, H, E, BF16, T)
    w1, s1, w2, s2, _, _ = _ffn_weights(W1, W2)
    x, b1, b2 = x.cuda(), b1.cuda(), b2.cuda()
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    y = cm.quantized_ffn_forward(x, w1, s1, b1, w2, s2, b2, offsets=off, activations=act)
    for e, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        if hi > lo:
            one = [t[e].contiguous() for t in (w1, s1, b1, w2, s2, b2)]
            assert torch.equal(y[lo:hi], cm.quantized_ffn_forward(x[lo:hi].contiguous(), *one, activations=act))


@pytest.mark.parametrize("fa", [E4M3, E2M1])
@pytest.mark.parametrize("M,N", [(12, 100), (40, 300), (3000, 300), (9000, 1500)])
def test_8bit_results_beside_a_nan_column(M, N, fa):
    """A NaN scale of B makes one column NaN; the others of its block are rounded
    under the scale of the finite ones."""
    K = 288
    g = _gen(12)
    a, sa, a64 = _rows(g, fa, (M, K))
    b, sb, b64 = _operand4(g, (N, K))
    sb.view(torch.uint8)[70, 8] = 255
    v, s = cm.quantized_gemm(a, sa, b, sb, out_dtype=E4M3)
    got = dequantize(v, s, 1)[:, :N]
    rest = [n for n in range(N) if n != 70]
    assert got[:, 70].isnan().all() and got[:, rest].isfinite().all()
    ref = a64 @ b64.T
    d = _sum_bound(K, a64.abs() @ b64.abs().T, True)
    ref[:, 70], d[:, 70] = 0.0, 0.0
    e = s.cpu().view(torch.uint8).int() - 127
    step = torch.ldexp(torch.ones(e.shape, dtype=torch.float64), e).repeat_interleave(128, dim=1)[:, :N]
    bad = (got - ref).abs() > HALF[E4M3] * ref.abs() + TINY[E4M3] * step + 1.2 * d
    assert not bad[:, rest].any()
    for i in range(-(-N // 128)):
        blk = slice(128 * i, 128 * i + 128)
        lo, hi = (ref[:, blk].abs() - d[:, blk]).clamp(min=0).amax(1), (ref[:, blk].abs() + d[:, blk]).amax(1)
        assert ((e[:, i] >= scale_exponent(lo, E4M3)) & (e[:, i] <= scale_exponent(hi, E4M3))).all()
