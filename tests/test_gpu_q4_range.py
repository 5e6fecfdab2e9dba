"""The 4-bit products and the FFN made of them far from one: scales near both
ends of their range, rows that are no numbers, as many rows as a launch holds;
at sizes that reach every kernel."""
import pytest
import torch

from paper_2606_28516_amd import clearmoe as cm
from tests.q4_util import E2M1, dequantize4, exponent4, quantize4_ref
from tests.q8_util import HALF, TINY, dequantize, quantize_ref, up
from tests.test_gpu_q4 import FLIPS4, _ffn_reference, _ffn_weights
from tests.test_gpu_q8 import CUT, FLIPS, _ffn_inputs, _gen, _sum_bound

pytestmark = pytest.mark.gpu

F32, BF16, E4M3, E8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn, torch.float8_e8m0fnu
DENORMAL = 2.0 ** -149        # the smallest step of a float32
ROWS = [E4M3, E2M1]


def _operand(g, rows, K, fmt, exponents, tiny=False):
    """Random values with the scales 2^exponents[k / 128] and up to eight times
    more or less; tiny: only the format's smallest values."""
    x = torch.randn(1, rows, K, generator=g)
    v, s = quantize4_ref(x) if fmt == E2M1 else quantize_ref(x, E4M3, 1)
    v, s = v[0].contiguous(), s[0]
    if tiny:
        v = torch.randint(0, 4, v.shape, generator=g).to(torch.uint8)
        v = v % 2 + 16 * (v // 2) if fmt == E2M1 else v
    per = 32 if fmt == E2M1 else 128
    n = -(-K // per)
    e = exponents.repeat_interleave(128 // per)[:n]
    s[:, :n] = (127 + e + torch.randint(-3, 4, (rows, n), generator=g)).to(torch.uint8)
    s = s.contiguous()
    f64 = dequantize4(v, s) if fmt == E2M1 else dequantize(v.view(E4M3), s, 1)
    return v.cuda().view(fmt), s.cuda().view(E8), f64[:, :K]


# 16 x 16 tiles, 64 x 64, 64 x 128, two groups along k, 128 x 128 of both
# stages, the largest
SIZES = [(5, 40, 400), (300, 390, 400), (300, 1550, 400), (1000, 1030, 2112), (4200, 1550, 400), (3000, 1300, 640),
         (6600, 1990, 672)]


def _check(M, N, K, fa, out, ea, eb, tiny=False):
    g = _gen(M + K)
    nk = -(-K // 128)
    a, sa, a64 = _operand(g, M, K, fa, ea.repeat(8)[:nk], tiny)
    b, sb, b64 = _operand(g, N, K, E2M1, eb.repeat(8)[:nk], tiny)
    ref, mass = a64 @ b64.T, a64.abs() @ b64.abs().T
    # every product, block sum and addition may end among the denormals
    d = _sum_bound(K, mass, out == F32 or fa == E2M1) + (K + 4 * nk) * DENORMAL
    c = cm.quantized_gemm(a, sa, b, sb, out_dtype=out)
    if out in (E4M3, E2M1):
        v, s = c
        width = 32 if out == E2M1 else 128
        step = torch.ldexp(torch.ones(s.shape, dtype=torch.float64), s.cpu().view(torch.uint8).int() - 127)
        step = step.repeat_interleave(width, dim=1)[:, :N]
        c = (dequantize4(v, s) if out == E2M1 else dequantize(v, s, 1))[:, :N]
        if out == E2M1:
            at = (ref.abs() + d) / step
            bound = torch.where(at < 2, 0.25, torch.where(at < 4, 0.5, 1.0)) * step + 1.0001 * d
        else:
            bound = HALF[out] * ref.abs() + TINY[out] * step + 1.2 * d
    else:
        c = c.cpu().double()
        half = torch.finfo(out).eps / 2
        # (bfloat16 denormals have steps of 2^-133)
        bound = half * ref.abs() + (1 + half) * d + (2.0 ** -134 if out == BF16 else DENORMAL)
    bad = ~((c - ref).abs() <= bound)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist())


@pytest.mark.parametrize("out", [F32, BF16, E4M3, E2M1])
@pytest.mark.parametrize("fa", ROWS)
@pytest.mark.parametrize("M,N,K", SIZES[:-1])
def test_opposite_scales(M, N, K, fa, out):
    """The two operands' scales of a block are up to 2^113 and 2^-113: a sum
    times one of them alone would leave float32's range."""
    e = torch.tensor([110, -110, 60, -100])
    _check(M, N, K, fa, out, e, -e)


@pytest.mark.parametrize("fa,out", [(E2M1, BF16), (E4M3, BF16), (E4M3, E2M1)])
def test_opposite_scales_of_the_largest_tiles(fa, out):
    e = torch.tensor([110, -110, 60, -100])
    _check(*SIZES[-1], fa, out, e, -e)


@pytest.mark.parametrize("fa", ROWS)
@pytest.mark.parametrize("M,N,K", SIZES[:-1])
def test_scales_whose_product_is_no_normal_number(M, N, K, fa):
    """2^-135 and 2^127 together (up to 2^6 more or less), and sums that bring the
    results back."""
    _check(M, N, K, fa, F32, torch.tensor([-120] * 4), torch.tensor([-15] * 4))
    if fa == E4M3:                                # (e2m1 has no value small enough)
        _check(M, N, K, fa, F32, torch.tensor([110] * 4), torch.tensor([11] * 4), tiny=True)


@pytest.mark.parametrize("fa", ROWS)
@pytest.mark.parametrize("M,N,K", SIZES[:-1])
def test_rows_do_not_depend_on_the_rows_beside_them(M, N, K, fa):
    """Extreme scales of some rows leave the others' results as they were."""
    g = _gen(6)
    e = torch.zeros(40, dtype=torch.int32)
    a, sa, _ = _operand(g, M, K, fa, e)
    b, sb, _ = _operand(g, N, K, E2M1, e)
    want = cm.quantized_gemm(a, sa, b, sb, out_dtype=F32)
    odd = torch.zeros(M, dtype=torch.bool)
    odd[1::3] = True
    sa.view(torch.uint8)[1::9] = 1
    sa.view(torch.uint8)[4::9] = 254
    sa.view(torch.uint8)[7::9] = 255
    got = cm.quantized_gemm(a, sa, b, sb, out_dtype=F32)
    assert torch.equal(got[~odd], want[~odd]) and got[7::9].isnan().all()


@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("out", [E4M3, E2M1])
@pytest.mark.parametrize("M,N,K", [(20, 390, 272), (20, 1, 64), (9000, 390, 272), (9000, 1030, 64), (300, 65, 96)])
def test_bytes_past_the_columns_are_zero(M, N, K, out, gelu):
    """Also in rows that hold NaN, or whose scale is NaN; scales past the last
    block are 1."""
    g = _gen(N)
    e = torch.zeros(40, dtype=torch.int32)
    a, sa, _ = _operand(g, M, K, E4M3, e)
    b, sb, _ = _operand(g, N, K, E2M1, e)
    cols = up(N, 32) // 2 if out == E2M1 else up(N, 16)
    fill = lambda: torch.full((M, cols), 0x3c, dtype=torch.uint8, device="cuda").view(out)
    want, ws = cm.quantized_gemm(a, sa, b, sb, gelu=gelu, out_dtype=out, out=fill())
    a.view(torch.uint8)[2, 5] = 0x7f
    sa.view(torch.uint8)[7, 0] = 255
    got, gs = cm.quantized_gemm(a, sa, b, sb, gelu=gelu, out_dtype=out, out=fill())
    keep = [i for i in range(M) if i not in (2, 7)]
    v, s = got.view(torch.uint8), gs.view(torch.uint8)
    if out == E2M1:
        if N % 32:
            assert (v[:, N // 2 + N % 2:] == 0).all() and (N % 2 == 0 or (v[:, N // 2] < 16).all())
        assert (s[[2, 7], :-(-N // 32)] == 255).all() and (s[:, -(-N // 32):] == 127).all()
    else:
        assert (v[:, N:] == 0).all() and got.float()[[2, 7], :N].isnan().all()
        assert (s[:, -(-N // 128):] == 127).all()
    assert torch.equal(v[keep], want.view(torch.uint8)[keep]) and torch.equal(s[keep], ws.view(torch.uint8)[keep])


@pytest.mark.parametrize("act", ROWS)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("power", [118, -118])
@pytest.mark.parametrize("T", [1, 16, 17, 300])
def test_ffn_of_large_and_small_rows(T, power, dtype, act):
    D, H = 200, 392
    x, W1, b1, W2, b2 = _ffn_inputs(T, D, H, 0, dtype, T)
    x = x * 2.0 ** power
    b1, b2 = torch.zeros_like(b1), torch.zeros_like(b2)
    w1, s1, w2, s2, d1, d2 = _ffn_weights(W1, W2)
    y = cm.quantized_ffn_forward(x.cuda(), w1, s1, b1.cuda(), w2, s2, b2.cuda(), activations=act).cpu().double()
    half = torch.finfo(dtype).eps / 2
    ref, coarse, fine = _ffn_reference(x, d1, b1.double(), d2, b2.double(), act, half)
    assert y.isfinite().all()
    assert ((y - ref).abs() <= coarse).all()
    assert (y - fine).norm() <= (half + (FLIPS4 if act == E2M1 else CUT + FLIPS)) * fine.norm()


def test_the_largest_scales_of_a_result():
    """Results whose block's scale is the largest and the smallest that there
    are (one block's sum is exact); a block with a value past float32's range,
    2^128 (1 - 2^-25) and more, is no number."""
    M, N, K = 40, 64, 32
    g = _gen(8)
    for e in (60, -63):
        a, sa, a64 = _operand(g, M, K, E2M1, torch.tensor([e]))
        b, sb, b64 = _operand(g, N, K, E2M1, torch.tensor([e]))
        v, s = cm.quantized_gemm(a, sa, b, sb, out_dtype=E2M1)
        ref = a64 @ b64.T
        most = ref.reshape(M, 2, 32).abs().amax(2)
        want = torch.where(most >= 2.0 ** 128 * (1 - 2.0 ** -25), 255, exponent4(most) + 127)
        got = s.cpu().view(torch.uint8)[:, :2].int()
        assert torch.equal(got, want.int())


@pytest.mark.parametrize("fa,last", [(E4M3, 0), (E2M1, 100)])
def test_as_many_rows_as_a_launch_holds(fa, last):
    E = 2 if last else 0
    M, N, K = (2 ** 24 - 32 - 2 * E) * 128, 1, 32 if fa == E2M1 else 16
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB of device memory")
    one = 0x22 if fa == E2M1 else 0x38
    a = torch.full((M, 16), one, dtype=torch.uint8, device="cuda").view(fa)
    sa = torch.full((M, 4), 127, dtype=torch.uint8, device="cuda").view(E8)
    lead = (E,) if E else ()
    b = torch.full((*lead, N, 16), 0x22, dtype=torch.uint8, device="cuda").view(E2M1)
    sb = torch.full((*lead, N, 4), 127, dtype=torch.uint8, device="cuda")
    if last:
        sb[-1] += 1                                                      # the last expert's: twos
    off = torch.tensor([0, M - last, M], dtype=torch.int32, device="cuda") if E else None
    out = torch.full((M, N), 7.5, dtype=BF16, device="cuda")
    cm.quantized_gemm(a, sa, b, sb.view(E8), offsets=off, out=out)
    right = int((out[:M - last] == K).sum()), int((out[M - last:] == 2 * K).sum())
    del a, sa, out
    torch.cuda.empty_cache()
    assert right == (M - last, last)


def test_quantisers_and_norm_of_more_rows_than_a_launch_holds():
    """Pieces around the borders against the same pieces by themselves: 2^28
    units a launch of the quantiser, 2^24 workgroups of the norm and the way
    back."""
    g = torch.Generator(device="cuda").manual_seed(1)
    n = 2 ** 28 + 1000
    x = torch.randn(n, 1, device="cuda", generator=g, dtype=BF16)
    v, s = cm.quantize(x, E2M1)
    y = cm.dequantize(v, s, 1)
    h = cm.rms_norm(x)
    for at in (300, 2 ** 26, 2 ** 28 - 16, 2 ** 28, n - 300):
        lo, hi = at - 300, min(n, at + 300)
        w, t = cm.quantize(x[lo:hi].contiguous(), E2M1)
        assert torch.equal(v[lo:hi].view(torch.uint8), w.view(torch.uint8)) and torch.equal(s[lo:hi].view(torch.uint8), t.view(torch.uint8))
        assert torch.equal(y[lo:hi], cm.dequantize(w, t, 1))
        assert torch.equal(h[lo:hi], cm.rms_norm(x[lo:hi].contiguous()))
    del x, v, s, y, h
    torch.cuda.empty_cache()
