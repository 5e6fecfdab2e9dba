"""rms_norm against the formula in 64 bits: widths around every variant's
border, strides, aliases, values at the ends of the range."""
import math

import pytest
import torch

from paper_2606_28516_amd import clearmoe as cm
from tests.q8_util import HALF, TINY, dequantize, quantize_ref, scale_exponent, up
from tests.test_gpu_q8 import _gen

pytestmark = pytest.mark.gpu

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-6
# y = h * inv * w before it is rounded: inv is the hardware's root (1 ulp,
# 2^-23) of a mean in double rounded to float32 (half of 2^-24 after the root)
# and two products are rounded (2^-24 each)
FLOAT = 2.0 ** -23 + 2.0 ** -25 + 2 * 2.0 ** -24


def _formula(x, residual, weight, eps=EPS):
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    f = h.double()
    y = f / (f.square().mean(dim=1, keepdim=True) + eps).sqrt()
    return (y if weight is None else y * weight.double()), h


def _check(x, residual, weight, out, **kw):
    ref, h = _formula(x, residual, weight)
    cuda = lambda t: None if t is None else t.cuda()
    r = cm.rms_norm(cuda(x), cuda(weight), residual=cuda(residual), eps=EPS, out_dtype=out, **kw)
    r = r if isinstance(r, tuple) else (r,)
    if residual is not None:
        assert torch.equal(r[-1].cpu(), h)
    if out in (E4M3, E5M2):
        v, s = r[:2]
        n, nb = x.shape[1], -(-x.shape[1] // 128)
        assert v.dtype == out and tuple(v.shape) == (x.shape[0], up(n, 16)) and tuple(s.shape) == (x.shape[0], up(nb, 4))
        full, sb = dequantize(v, s, 1), s.cpu().view(torch.uint8)
        assert (full[:, n:] == 0).all() and (sb[:, nb:] == 127).all()
        cols = torch.ldexp(torch.ones(sb.shape, dtype=torch.float64), sb.int() - 127).repeat_interleave(128, 1)[:, :n]
        assert ((full[:, :n] - ref).abs() <= HALF[out] * ref.abs() + TINY[out] * cols + 1.2 * FLOAT * ref.abs()).all()
        for i in range(nb):
            m = ref[:, 128 * i:128 * i + 128].abs().amax(1)
            e = sb[:, i].int() - 127
            assert ((e >= scale_exponent(m * (1 - FLOAT), out)) & (e <= scale_exponent(m * (1 + FLOAT), out))).all()
    else:
        half = torch.finfo(out).eps / 2
        assert r[0].dtype == out
        assert ((r[0].cpu().double() - ref).abs() <= (half + FLOAT) * ref.abs() + 2.0 ** -149).all()


def _inputs(rows, cols, dtype, seed):
    g = _gen(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-3, 4, (rows, 1), generator=g).float())
    return x.to(dtype), torch.randn(rows, cols, generator=g).to(dtype), 1 + 0.3 * torch.randn(cols, generator=g)


WIDTHS = [(1, 1), (3, 7), (5, 8), (2, 16), (9, 127), (4, 128), (130, 129), (1, 768), (257, 384), (64, 511), (6, 512),
          (7, 513), (33, 1000), (5, 1024), (5, 1025), (3, 2048), (3, 2049), (4, 4096), (2, 4099), (3, 8192), (2, 8200),
          (2, 16384), (2, 16400), (1, 32768), (2, 33001), (1, 65536), (2, 65535), (1030, 700), (1030, 1000), (1025, 8000), (1027, 4100)]


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (F32, F32), (BF16, E4M3), (F32, E4M3), (BF16, E5M2), (F32, E5M2)])
@pytest.mark.parametrize("rows,cols", WIDTHS)
def test_widths(rows, cols, dtype, out):
    x, r, w = _inputs(rows, cols, dtype, rows + cols)
    _check(x, r, w, out)
    _check(x, None, w if cols % 2 else None, out)


@pytest.mark.parametrize("out", [None, E4M3])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strided_rows(dtype, out):
    """Rows of x, residual, sum and y inside wider arrays, at odd elements."""
    g = _gen(3)
    for rows, cols in ((9, 75), (40, 384), (3, 1500)):
        wide = [torch.randn(rows, cols + 40, generator=g).to(dtype).cuda() for _ in range(3)]
        x, r = wide[0][:, 3:cols + 3], wide[1][:, 11:cols + 11]
        w = torch.randn(cols + 1, generator=g).cuda()[1:]
        want = cm.rms_norm(x.contiguous(), w.clone(), residual=r.contiguous(), out_dtype=out)
        before = wide[2].clone()
        kw = {}
        if out is None:
            y = torch.full((rows, cols + 9), 7.5, dtype=dtype, device="cuda")
            kw["out"] = y[:, 5:cols + 5]
        else:
            y = torch.full((rows, up(cols, 16) + 32), 0x55, dtype=torch.uint8, device="cuda").view(out)
            kw["out"] = y[:, 16:up(cols, 16) + 16]
        got = cm.rms_norm(x, w, residual=r, out_dtype=out, sum_out=wide[2][:, 1:cols + 1], **kw)
        for a, b in zip(got, want):
            assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
        assert torch.equal(wide[2][:, :1], before[:, :1]) and torch.equal(wide[2][:, cols + 1:], before[:, cols + 1:])
        if out is None:
            assert (y[:, :5] == 7.5).all() and (y[:, cols + 5:] == 7.5).all()
        else:
            u = y.view(torch.uint8)
            assert (u[:, :16] == 0x55).all() and (u[:, up(cols, 16) + 16:] == 0x55).all()


@pytest.mark.parametrize("cols", [100, 768, 3000, 9000])
def test_the_stream_in_place(cols):
    """sum_out may be x or the residual, and the result x, too."""
    x, r, w = (t.cuda() for t in _inputs(37, cols, BF16, 5))
    y, h = cm.rms_norm(x, w, residual=r)
    for at in (0, 1):
        a, b = x.clone(), r.clone()
        got, total = cm.rms_norm(a, w, residual=b, sum_out=(a, b)[at])
        assert torch.equal(got, y) and torch.equal(total, h) and torch.equal((a, b)[at], h)
    a = x.clone()
    got, total = cm.rms_norm(a, w, residual=r, out=a)
    assert got is a and torch.equal(a, y) and torch.equal(total, h)
    a, b = x.clone(), r.clone()
    cm.rms_norm(a, w, residual=b, out=a, sum_out=b)
    assert torch.equal(a, y) and torch.equal(b, h)
    assert torch.equal(cm.rms_norm(x, w, sum_out=torch.empty_like(x))[1], x)


@pytest.mark.parametrize("cols", [7, 768, 1500, 20000])
def test_values_at_the_ends_of_the_range(cols):
    """Rows whose squares leave float32's range on either side, zeros, one
    value alone."""
    g = _gen(6)
    base = torch.randn(1, cols, generator=g)
    for dtype in (F32, BF16):
        x = torch.cat([base * 1e30, base * 2e37, base * 1e-30, base * 1e-37, torch.zeros(1, cols), base]).to(dtype)
        x[5, 1:] = 0
        _check(x, None, None, dtype)
        _check(x[:1], None, None, E4M3)
        y = cm.rms_norm(x[2:5].cuda(), eps=1.2e-38)
        ref, _ = _formula(x[2:5], None, None, 1.2e-38)
        half = torch.finfo(dtype).eps / 2
        assert ((y.cpu().double() - ref).abs() <= (half + FLOAT) * ref.abs() + 2.0 ** -149).all()
        assert (y[2] == 0).all()


@pytest.mark.parametrize("out", [BF16, E4M3, E5M2])
def test_nan_and_infinity_stay_in_their_row(out):
    x, r, w = _inputs(9, 390, BF16, 7)
    clean = cm.rms_norm(x.cuda(), w.cuda(), residual=r.cuda(), out_dtype=out)
    x[2, 5], x[4, 389], r[6, 0] = math.nan, math.inf, -math.inf
    got = cm.rms_norm(x.cuda(), w.cuda(), residual=r.cuda(), out_dtype=out)
    rows = [0, 1, 3, 5, 7, 8]
    f = (got[0].float() if out == BF16 else dequantize(got[0], got[1], 1)[:, :390]).cpu()
    assert f[2].isnan().all()
    for i, at in ((4, 389), (6, 0)):
        assert f[i, at].isnan() and (f[i, [c for c in range(390) if c != at]] == 0).all()
    if out != BF16:
        assert (got[0].view(torch.uint8)[:, 390:] == 0).all()
    for a, b in zip(got[:-1], clean[:-1]):
        assert torch.equal(a[rows].view(torch.uint8), b[rows].view(torch.uint8))


def test_many_rows():
    """More rows than one workgroup's share, the last ones alone in theirs."""
    for rows, cols in ((70001, 40), (1, 40), (4097, 600)):
        x, r, w = _inputs(rows, cols, BF16, 9)
        _check(x, r, w, BF16)


def test_no_rows():
    y, h = cm.rms_norm(torch.empty(0, 64, device="cuda"), residual=torch.empty(0, 64, device="cuda"))
    assert y.shape == h.shape == (0, 64)


def test_refusals():
    x = torch.randn(6, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    for args, kw in (((x[0], w), {}), ((x.half(), w), {}), ((x, w[:63]), {}), ((x, w.bfloat16()), {}),
                     ((x, w), dict(residual=x[:5])), ((x, w), dict(residual=x.bfloat16())),
                     ((x, w), dict(out_dtype=BF16)), ((x, w), dict(out_dtype=torch.float4_e2m1fn_x2)),
                     ((x, w), dict(eps=0.0)), ((x, w), dict(eps=-1.0)), ((x, w), dict(eps=math.nan)),
                     ((x, w), dict(eps=1e-39)), ((x, w), dict(eps=math.inf)),
                     ((x[:, ::2], w[:32]), {}), ((x[:1].expand(6, 64), w), {}),
                     ((x, w), dict(residual=x[:1].expand(6, 64))), ((x, w), dict(out=torch.empty(6, 65, device="cuda"))),
                     ((x, w), dict(sum_out=torch.empty(6, 64, device="cuda", dtype=BF16))),
                     ((x, w), dict(sum_out=torch.empty(64, 6, device="cuda").T)),
                     ((x.cpu(), w), {}), ((x, w.cpu()), {}), ((x, w), dict(residual=x.cpu()))):
        with pytest.raises(cm.ClearMoEError):
            cm.rms_norm(*args, **kw)
