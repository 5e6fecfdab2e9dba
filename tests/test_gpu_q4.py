"""The 4-bit operators (quantize and dequantize, quantized_gemm and
quantized_ffn_forward with 4-bit weights) against plain 64-bit forms, at the
sizes and values where they can go wrong."""
import ctypes
import math

import pytest
import torch

from paper_2606_28516_amd import clearmoe as cm
from tests.q4_util import E2M1, HALF4, dequantize4, exponent4, quantize4_ref, scales4, values4
from tests.q8_util import HALF, TINY, dequantize, quantize_ref, scale_exponent, up
from tests.test_gpu_q8 import CUT, FLIPS, GROUPS, SIZES, _ffn_inputs, _gelu, _gelu_bound, _gen, _reference, _sum_bound

pytestmark = pytest.mark.gpu

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
E8 = torch.float8_e8m0fnu
BF16, F32 = torch.bfloat16, torch.float32


def bytes_of(t):
    return t.cpu().view(torch.uint8)


# ---------------------------------------------------------------------------
# quantize and dequantize: bit for bit
# ---------------------------------------------------------------------------
def _check_quantize(x):
    v, s = cm.quantize(x.cuda(), E2M1)
    x3 = x if x.dim() == 3 else x[None]
    rv, rs = quantize4_ref(x3)
    assert v.dtype == E2M1 and s.dtype == E8
    assert tuple(v.shape) == (*x.shape[:-1], rv.shape[-1]) and tuple(s.shape) == (*x.shape[:-1], rs.shape[-1])
    assert torch.equal(bytes_of(s).reshape(rs.shape), rs)
    assert torch.equal(bytes_of(v).reshape(rv.shape), rv)
    for dtype in (F32, BF16):
        y = cm.dequantize(v, s, x.shape[-1], dtype=dtype)
        want = dequantize4(rv, rs)[..., :x.shape[-1]].reshape(x.shape).float().to(dtype)
        assert y.shape == x.shape and torch.equal(y.cpu().isnan(), want.isnan())
        assert torch.equal(y.cpu()[~want.isnan()], want[~want.isnan()])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(1, 1), (3, 7), (1, 32), (5, 33), (17, 128), (130, 129), (257, 384), (64, 700),
                                   (2, 65536), (3, 200, 390), (2, 1, 16), (300, 8), (9, 95)])
def test_quantize(shape, dtype):
    g = _gen(sum(shape))
    x = torch.randn(*shape, generator=g) * torch.exp2(torch.randint(-20, 20, shape[:-1] + (1,), generator=g).float())
    _check_quantize(x.to(dtype))


def test_quantize_special_values():
    """Blocks of zeros, the range's border on both sides, the smallest and
    largest floats, all ties, infinities and NaN."""
    inf, nan = math.inf, math.nan
    nxt = torch.nextafter(torch.tensor(6.0), torch.tensor(inf)).item()
    firsts = [0.0, -0.0, 6.0, nxt, -6.0, -nxt, 12.0, 6 / 2 ** 20, nxt / 2 ** 20, 1e-45, 1.2e-38, 3e-38, 8e-38, 3.4e38,
              inf, -inf, nan]
    x = torch.zeros(len(firsts), 100)
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    for i, f in enumerate(firsts):
        x[i, 3] = f
        k = f if math.isfinite(f) and f != 0 else 6.0
        scale = 2.0 ** int(exponent4(torch.tensor(abs(k))))
        x[i, 4:11], x[i, 11:18] = ties * scale, -ties * scale
        x[i, 18:25] = torch.nextafter(ties, torch.tensor(0.0)) * scale
        x[i, 25:32] = torch.nextafter(ties, torch.tensor(9.0)) * scale
        x[i, 40] = 1.0
        x[i, 99] = f
    _check_quantize(x)
    _check_quantize(-x[None].repeat(2, 1, 1))
    _check_quantize(x.to(BF16))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_quantize_strided_rows(dtype):
    g = _gen(2)
    wide = torch.randn(30, 211, generator=g).to(dtype).cuda()
    for x in (wide[:, 3:100], wide[::2, 1:2], wide[:1, 5:70], wide.reshape(2, 15, 211)[:, :, 100:200]):
        v, s = cm.quantize(x, E2M1)
        w, t = cm.quantize(x.contiguous(), E2M1)
        assert torch.equal(bytes_of(v), bytes_of(w)) and torch.equal(bytes_of(s), bytes_of(t))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("fmt", [E4M3, E5M2])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("shape", [(1, 1), (5, 127), (130, 129), (3, 200, 390)])
def test_dequantize_8bit(shape, block_rows, fmt, dtype):
    g = _gen(sum(shape))
    x = torch.randn(*shape, generator=g) * torch.exp2(torch.randint(-3, 3, shape[:-1] + (1,), generator=g).float())
    v, s = cm.quantize(x.cuda(), fmt, block_rows=block_rows)
    y = cm.dequantize(v, s, shape[-1], dtype=dtype, block_rows=block_rows)
    want = dequantize(v, s, block_rows)[..., :shape[-1]]
    assert torch.equal(y.cpu(), want.float().to(dtype))


def test_dequantize_every_byte_and_scale():
    for fmt in (E4M3, E5M2):
        v = torch.arange(256, dtype=torch.uint8).reshape(1, 256).repeat(256, 1).cuda().view(fmt)
        s = torch.arange(256, dtype=torch.uint8).reshape(256, 1).repeat(1, 4).cuda().view(E8)
        for dtype in (F32, BF16):
            y = cm.dequantize(v, s, dtype=dtype).cpu()
            e = torch.ldexp(torch.ones(256, 1, dtype=torch.float64), torch.arange(256).reshape(256, 1) - 127)
            e[255] = math.nan
            want = (v.cpu().double() * e).float().to(dtype)
            assert torch.equal(y.isnan(), want.isnan()) and torch.equal(y[~want.isnan()], want[~want.isnan()])


def test_dequantize_into_strided_rows():
    g = _gen(4)
    x = torch.randn(37, 75, generator=g).cuda()
    v, s = cm.quantize(x, E2M1)
    out = torch.full((37, 100), 7.5, device="cuda", dtype=BF16)
    y = cm.dequantize(v, s, 75, out=out[:, 10:85])
    assert torch.equal(y, cm.dequantize(v, s, 75))
    assert (out[:, :10] == 7.5).all() and (out[:, 85:] == 7.5).all()


# ---------------------------------------------------------------------------
# quantized_gemm
# ---------------------------------------------------------------------------
def _operand4(g, shape):
    """A 4-bit operand made on the CPU, and its values in 64 bits."""
    x = torch.randn(*shape, generator=g) * torch.exp2(torch.randint(-4, 5, shape[:-1] + (1,), generator=g).float())
    v, s = quantize4_ref(x if x.dim() == 3 else x[None])
    if x.dim() == 2:
        v, s = v[0], s[0]
    return v.contiguous().cuda().view(E2M1), s.contiguous().cuda().view(E8), dequantize4(v, s)[..., :shape[-1]]


def _operand8(g, shape):
    x = torch.randn(*shape, generator=g) * torch.exp2(torch.randint(-4, 5, shape[:-1] + (1,), generator=g).float())
    v, s = quantize_ref(x[None], E4M3, 1)
    return v[0].contiguous().cuda().view(E4M3), s[0].contiguous().cuda().view(E8), dequantize(v[0].view(E4M3), s[0], 1)[:, :shape[-1]]


def _rows(g, fa, shape):
    return _operand4(g, shape) if fa == E2M1 else _operand8(g, shape)


def _check_product(M, N, K, E=0, offsets=None, fa=E4M3, out=BF16, bias=True, gelu=False, seed=0):
    g = _gen(seed + M * 7 + N * 3 + K)
    a, sa, fa64 = _rows(g, fa, (M, K))
    b, sb, fb64 = _operand4(g, (E, N, K) if E else (N, K))
    bi = torch.randn(*((E, N) if E else (N,)), generator=g).cuda() if bias else None
    off = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda")
    # (products with float32 results, and all of 4-bit rows, are not cut; the
    # GELU is the more exact one for float32 results alone)
    wide = out == F32 or fa == E2M1
    ref, d, mean, live = _reference(fa64, fb64, bi, offsets, False, wide)
    if gelu:
        ref, d, mean = _gelu(ref), _gelu_bound(ref, d, out == F32), _gelu_bound(ref, mean, out == F32)
    if out in (E4M3, E2M1):
        c, cs = cm.quantized_gemm(a, sa, b, sb, bias=bi, gelu=gelu, offsets=off, out_dtype=out)
        width = 32 if out == E2M1 else 128
        nb = -(-N // width)
        full = dequantize4(c, cs) if out == E2M1 else dequantize(c, cs, 1)
        sbytes = bytes_of(cs)
        assert full.shape[1] == (up(N, 32) if out == E2M1 else up(N, 16))
        assert (full[live][:, N:] == 0).all() and (sbytes[live][:, nb:] == 127).all()
        s = torch.ldexp(torch.ones(sbytes.shape, dtype=torch.float64), sbytes.int() - 127)
        cols = s.repeat_interleave(width, dim=1)[:, :N]
        err = (full[:, :N] - ref).abs()
        if out == E2M1:       # steps of the grid: 0.5, from 2 on 1, from 4 on 2 (a value and its sum's error: either side)
            a_ = (ref.abs() + d) / cols
            half = torch.where(a_ < 2, 0.25, torch.where(a_ < 4, 0.5, 1.0)) * cols
            bound = half + 1.0001 * d
        else:
            bound = HALF[out] * ref.abs() + TINY[out] * cols + 1.2 * d
        assert (err <= bound)[live].all(), (err - bound)[live].max()
        for i in range(nb):                       # the scale is that of the block's largest value
            blk = slice(width * i, width * i + width)
            lo, hi = (ref[:, blk].abs() - d[:, blk]).clamp(min=0).amax(1), (ref[:, blk].abs() + d[:, blk]).amax(1)
            e = torch.log2(s[:, i])
            at = (lambda v: exponent4(v)) if out == E2M1 else (lambda v: scale_exponent(v, out))
            assert ((e >= at(lo)) & (e <= at(hi)) | (lo == 0))[live].all()
        return
    sentinel = torch.full((M, N), 7.5, dtype=out, device="cuda")
    c = cm.quantized_gemm(a, sa, b, sb, bias=bi, gelu=gelu, offsets=off, out_dtype=out, out=sentinel)
    c = c.cpu().double()
    half = torch.finfo(out).eps / 2
    err = (c - ref).abs()
    bad = (err > half * ref.abs() + (1 + half) * d + 1e-38) & live[:, None]
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), float(err.max()))
    assert (c[~live] == 7.5).all()
    if live.any():
        assert err[live].norm() <= half * ref[live].norm() + mean[live].norm() + 1e-30


ROWS = [E4M3, E2M1]
MORE = [(1, 1, 32), (64, 128, 512), (65, 129, 544), (70, 64, 1024), (300, 200, 1056), (20, 500, 4128), (1, 8, 65536),
        (1000, 1540, 1200), (1000, 1030, 2112), (1000, 1030, 176)]


@pytest.mark.parametrize("out", [BF16, F32, E4M3, E2M1])
@pytest.mark.parametrize("fa", ROWS)
@pytest.mark.parametrize("M,N,K", SIZES + MORE)
def test_product(M, N, K, fa, out):
    _check_product(M, N, K - 3 if K % 96 == 0 else K, fa=fa, out=out, gelu=(M + N) % 2 == 0, bias=K % 32 == 0)


@pytest.mark.parametrize("out", [BF16, F32, E4M3, E2M1])
@pytest.mark.parametrize("fa", ROWS)
@pytest.mark.parametrize("M,N,K,offsets", GROUPS)
def test_product_groups(M, N, K, offsets, fa, out):
    _check_product(M, N, K, E=len(offsets) - 1, offsets=offsets, fa=fa, out=out, gelu=N % 16 == 0)


MANY = [
    (8200, 1990, 544, None, E2M1, BF16), (6500, 1830, 576, None, E2M1, E2M1), (6500, 1830, 576, None, E2M1, E4M3),
    (3000, 1300, 640, None, E2M1, F32), (3000, 1300, 640, None, E2M1, BF16), (3000, 1300, 640, None, E2M1, E2M1),
    (3000, 1300, 640, None, E2M1, E4M3), (6500, 1830, 160, None, E4M3, BF16), (6500, 1830, 160, None, E4M3, E4M3),
    (6500, 1830, 160, None, E4M3, E2M1), (9000, 1900, 544, [0, 5, 4000, 4001, 9000], E2M1, BF16),
    (7000, 1900, 544, [9, 3000, 3000, 6995], E2M1, E2M1), (7000, 1900, 160, [9, 3000, 3000, 6995], E4M3, E4M3),
    (3000, 1300, 640, [7, 1000, 1000, 2900], E2M1, F32), (6600, 1990, 672, None, E2M1, BF16),
    (6400, 1900, 672, [0, 5, 4000, 4001, 6400], E2M1, BF16), (9000, 1500, 544, None, E2M1, E2M1),
    (9000, 1500, 544, None, E2M1, E4M3)]


@pytest.mark.parametrize("M,N,K,offsets,fa,out", MANY)
def test_product_of_many_rows(M, N, K, offsets, fa, out):
    """The largest tiles, and those for a long k."""
    _check_product(M, N, K, E=len(offsets) - 1 if offsets else 0, offsets=offsets, fa=fa, out=out, gelu=N % 20 == 0)


@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("fa", ROWS)
@pytest.mark.parametrize("M", [3, 40, 300, 3000])
def test_product_scales_reach_their_blocks(fa, out, M):
    """Every scale of A and B is a different power of two and the values are
    one: each block's share of the sum is its scales' product, exactly."""
    N, K = 300, 1120
    nk = K // 32
    g = _gen(11)
    a = (torch.ones(M, K).to(E4M3) if fa == E4M3 else torch.full((M, K // 2), 0x22, dtype=torch.uint8).view(E2M1)).cuda()
    b = torch.full((N, K // 2), 0x22, dtype=torch.uint8).view(E2M1).cuda()
    wa = 128 if fa == E4M3 else 32
    na = -(-K // wa)
    sa = torch.full((M, up(na, 4)), 255, dtype=torch.uint8)              # what lies past the blocks does not count
    sb = torch.full((N, up(nk, 4)), 255, dtype=torch.uint8)
    sa[:, :na] = torch.randint(122, 132, (M, na), generator=g).to(torch.uint8)
    sb[:, :nk] = torch.randint(122, 132, (N, nk), generator=g).to(torch.uint8)
    c = cm.quantized_gemm(a, sa.cuda().view(E8), b, sb.cuda().view(E8), out_dtype=out)
    xa = torch.exp2(sa.double() - 127)[:, :na].repeat_interleave(wa, dim=1)[:, :K]
    xb = torch.exp2(sb.double() - 127)[:, :nk].repeat_interleave(32, dim=1)
    assert torch.equal(c.cpu(), (xa @ xb.T).to(out))


@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("fa", ROWS)
@pytest.mark.parametrize("M", [5, 300, 3000])
def test_product_scales_far_apart(fa, out, M):
    """One scale alone leaves float32's range, the two together do not."""
    N, K = 130, 256
    g = _gen(17)
    a, sa, a64 = _rows(g, fa, (M, K))
    b, sb, b64 = _operand4(g, (N, K))
    want = cm.quantized_gemm(a, sa, b, sb, out_dtype=out)
    for up_ in (100, -100, 118, -110):
        ta = (sa.view(torch.uint8).int() + up_).to(torch.uint8).view(E8)
        tb = (sb.view(torch.uint8).int() - up_).to(torch.uint8).view(E8)
        assert torch.equal(cm.quantized_gemm(a, ta, b, tb, out_dtype=out), want), up_


@pytest.mark.parametrize("out", [F32, BF16, E4M3, E2M1])
@pytest.mark.parametrize("fa", ROWS)
@pytest.mark.parametrize("M", [12, 40, 3000])
def test_product_nan_stays_in_its_row(M, fa, out):
    """NaN in a row of A (a byte, or a scale), or a scale of B: that row or that
    column is NaN, everything else as before (4-bit results: the blocks that hold
    one)."""
    N, K = 100, 288
    g = _gen(12)
    a, sa, _ = _rows(g, fa, (M, K))
    b, sb, _ = _operand4(g, (N, K))
    call = lambda: cm.quantized_gemm(a, sa, b, sb, out_dtype=out)
    flat = lambda r: r if torch.is_tensor(r) else (dequantize4(*r) if out == E2M1 else dequantize(*r, 1))[:, :N]
    want = flat(call()).cpu()
    if fa == E4M3:
        a.view(torch.uint8)[3, 17] = 0x7f
    else:
        sa.view(torch.uint8)[3, 1] = 255
    sa.view(torch.uint8)[9, sa.shape[1] - 2 if fa == E2M1 else 2] = 255 if fa == E4M3 else 127  # (4 bits: past the blocks)
    got = flat(call()).cpu()
    rows = [3] + [9] * (fa == E4M3)
    keep = [i for i in range(M) if i not in rows]
    assert got[rows].isnan().all() and torch.equal(got[keep], want[keep])
    sb.view(torch.uint8)[70, 8] = 255
    got = flat(call()).cpu()
    cols = [70] if out != E2M1 else list(range(64, 96))
    rest = [n for n in range(N) if n not in cols]
    assert got[:, cols].isnan().all()
    if out == E4M3:          # (the block's scale is that of the finite ones)
        rest = [n for n in rest if n >= 0]
        assert got[keep][:, rest].isfinite().all()
    else:
        assert torch.equal(got[keep][:, rest], want[keep][:, rest])


@pytest.mark.parametrize("M", [20, 9000])
def test_product_to_4_bits_with_infinities(M):
    """An infinite or NaN result marks its block of 32, and no other."""
    N, K = 200, 64
    g = _gen(14)
    a, sa, _ = _operand8(g, (M, K))
    b, sb, _ = _operand4(g, (N, K))
    bias = torch.zeros(N, device="cuda")
    want, ws = cm.quantized_gemm(a, sa, b, sb, bias=bias, out_dtype=E2M1)
    bias[7], bias[70], bias[199] = math.inf, -math.inf, math.nan
    got, gs = cm.quantized_gemm(a, sa, b, sb, bias=bias, out_dtype=E2M1)
    s = bytes_of(gs)
    assert (s[:, [0, 2, 6]] == 255).all() and (values4(got)[:, :32] == 0).all()
    keep = [1, 3, 4, 5, 7]
    assert torch.equal(s[:, keep], bytes_of(ws)[:, keep])
    assert torch.equal(values4(got)[:, 96:192], values4(want)[:, 96:192])


@pytest.mark.parametrize("out", [BF16, E2M1])
@pytest.mark.parametrize("fa", ROWS)
@pytest.mark.parametrize("M", [11, 300])
def test_product_row_strides(M, fa, out):
    """lda and ldc through the C ABI: rows inside wider arrays, whose other
    bytes stay as they were."""
    N, K = 50, 96
    g = _gen(13)
    a, sa, _ = _rows(g, fa, (M, K))
    b, sb, _ = _operand4(g, (N, K))
    want = cm.quantized_gemm(a, sa, b, sb, out_dtype=out)
    per = 2 if fa == E2M1 else 1
    wide = torch.full((M, 256 // per), 0x7e, dtype=torch.uint8, device="cuda")
    wide[:, :K // per] = a.view(torch.uint8)
    ptr = lambda t: ctypes.c_void_p(t.data_ptr())
    if out == BF16:
        c, cs = torch.full((M, 61), 7.5, dtype=out, device="cuda"), None
        p = cm.Product(M, N, K, 0, cm._OUTS[fa], 5, cm.BF16, 0, 0, 256, 61)
    else:
        c = torch.full((M, 64), 0x99, dtype=torch.uint8, device="cuda")
        cs = torch.empty(M, 4, dtype=torch.uint8, device="cuda")
        p = cm.Product(M, N, K, 0, cm._OUTS[fa], 5, 5, 0, 0, 256, 128)
    rc = cm.lib().clearmoe_quantized_gemm(ctypes.byref(p), ptr(wide), ptr(sa), ptr(b), ptr(sb), None, None, ptr(c),
                                          None if cs is None else ptr(cs), cm._stream(None))
    assert rc == 0
    if out == BF16:
        assert torch.equal(c[:, :N], want) and (c[:, N:] == 7.5).all()
    else:
        assert torch.equal(c[:, :32], want[0].view(torch.uint8)) and (c[:, 32:] == 0x99).all()
        assert torch.equal(cs, want[1].view(torch.uint8))


# (M, N, K) whose rows after the first `whole` are a launch of their own
ROUNDS = [(13100, 1270, 2080, 13056), (16500, 2000, 1024, 16384), (600, 21800, 2080, 512), (17000, 1024, 2048, 16384),
          (20480, 1024, 2048, 16384)]


@pytest.mark.parametrize("M,N,K,whole", ROUNDS)
def test_product_of_a_few_more_rows_than_whole_rounds(M, N, K, whole):
    """Rows inside wider arrays, results that begin at any element: as the two
    parts' own products; bytes around them stay as they were."""
    g = torch.Generator(device="cuda").manual_seed(19)
    a, sa = cm.quantize(torch.randn(M, K, device="cuda", generator=g), E2M1)
    b, sb = cm.quantize(torch.randn(N, K, device="cuda", generator=g), E2M1)
    bias = torch.randn(N, device="cuda", generator=g)
    ptr = lambda t: ctypes.c_void_p(t.data_ptr())
    wide = torch.full((M, K // 2 + 48), 0x7e, dtype=torch.uint8, device="cuda")
    wide[:, :K // 2] = a.view(torch.uint8)
    parts = [cm.quantized_gemm(a[lo:hi].contiguous(), sa[lo:hi].contiguous(), b, sb, bias=bias, gelu=True, out_dtype=BF16)
             for lo, hi in ((0, whole), (whole, M))]
    for at, ldc in ((0, N), (1, N + 9), (8, (N + 7) // 8 * 8 + 16)):
        flat = torch.full((at + M * ldc + 8,), 7.5, dtype=BF16, device="cuda")
        p = cm.Product(M, N, K, 0, 5, 5, cm.BF16, 1, 0, K + 96, ldc)
        rc = cm.lib().clearmoe_quantized_gemm(ctypes.byref(p), ptr(wide), ptr(sa), ptr(b), ptr(sb), ptr(bias), None,
                                              ptr(flat[at:]), None, cm._stream(None))
        assert rc == 0
        c = flat[at:at + M * ldc].view(M, ldc)
        assert torch.equal(c[:whole, :N], parts[0]) and torch.equal(c[whole:, :N], parts[1])
        assert (c[:, N:] == 7.5).all() and (flat[:at] == 7.5).all() and (flat[at + M * ldc:] == 7.5).all()


def test_product_unaligned_results():
    """Float results at any element, of any width."""
    g = _gen(18)
    for M, N, K in ((7, 51, 64), (300, 77, 160)):
        a, sa, _ = _operand8(g, (M, K))
        b, sb, _ = _operand4(g, (N, K))
        for out in (BF16, F32):
            want = cm.quantized_gemm(a, sa, b, sb, out_dtype=out)
            flat = torch.full((M * N + 2,), 7.5, dtype=out, device="cuda")
            c = flat[1:M * N + 1].view(M, N)
            cm.quantized_gemm(a, sa, b, sb, out_dtype=out, out=c)
            assert torch.equal(c, want) and flat[0] == 7.5 and flat[-1] == 7.5


def test_mismatched_tensors_are_refused():
    g = _gen(15)
    a, sa, _ = _operand8(g, (6, 64))
    a4, sa4, _ = _operand4(g, (6, 64))
    b, sb, _ = _operand4(g, (40, 64))
    b8, sb8 = cm.quantize(torch.randn(40, 64, generator=g).cuda(), block_rows=128)
    cm.quantized_gemm(a, sa, b, sb)
    cm.quantized_gemm(a4, sa4, b, sb)
    e5, se5 = cm.quantize(torch.randn(6, 64, generator=g).cuda(), E5M2)
    for args, kw in (((a, sa[:5], b, sb), {}), ((a, sa, b, sb[:39]), {}), ((a, sa, b, sb8), {}), ((a4, sa, b, sb[:, :3]), {}),
                     ((a, sa, b[:, :16].contiguous(), sb), {}), ((a4, sa4, b8, sb8), {}), ((e5, se5, b, sb), {}),
                     ((a, sa, b, sb), dict(out_dtype=E5M2)), ((a, sa, b8, sb8), dict(out_dtype=E2M1)),
                     ((a, sa, b.view(torch.uint8), sb), {}),
                     ((a, sa, b, sb), dict(out=torch.empty(6, 41, dtype=BF16, device="cuda")))):
        with pytest.raises(cm.ClearMoEError):
            cm.quantized_gemm(*args, **kw)
    for args, kw in (((a.float(), E2M1), dict(block_rows=128)), ((a, E2M1), {}), ((torch.zeros(3, 4).cuda(), torch.uint8), {})):
        with pytest.raises(cm.ClearMoEError):
            cm.quantize(*args, **kw)
    for args, kw in (((b, sb, 65), {}), ((b, sb, 32), {}), ((b, sb8, 64), {}), ((b, sb, 64), dict(block_rows=128)),
                     ((b, sb, 64), dict(dtype=torch.float16)), ((b.view(torch.uint8), sb, 64), {}),
                     ((b, sb, 64), dict(out=torch.empty(40, 63, dtype=BF16, device="cuda")))):
        with pytest.raises(cm.ClearMoEError):
            cm.dequantize(*args, **kw)


# ---------------------------------------------------------------------------
# quantized_ffn_forward
# ---------------------------------------------------------------------------
def _rounded(x, act):
    """x [T, n] float64 as its 8- or 4-bit form has it, and the scale of each value."""
    n = x.shape[1]
    if act == E2M1:
        v, s = quantize4_ref(x[None])
        return dequantize4(v[0], s[0])[:, :n], scales4(s[0], -(-n // 32))[:, :n]
    v, s = quantize_ref(x[None], E4M3, 1)
    f = torch.ldexp(torch.ones(s[0].shape, dtype=torch.float64), s[0].int() - 127).repeat_interleave(128, dim=1)[:, :n]
    return dequantize(v[0].contiguous().view(E4M3), s[0], 1)[:, :n], f


def _ffn_reference(x, w1, b1, w2, b2, act, half):
    """One group's FFN in 64 bits from the weights' values, z exact, and a bound
    that allows any rounding of z to the grid around it; and with z rounded as
    the definition says."""
    D, H = w1.shape[1], w1.shape[0]
    xq, _ = _rounded(x.double(), act)
    pre = xq @ w1.T + b1
    mass = xq.abs() @ w1.abs().T + b1.abs()
    z = _gelu(pre)
    dz = _gelu_bound(pre, _sum_bound(D, mass, act == E2M1), False)
    _, s = _rounded(z.abs() + dz, act)            # (the largest scale that z may get)
    if act == E2M1:
        off = 1.0 * s + 1.2 * dz                  # half the widest step
    else:
        off = HALF[E4M3] * z.abs() + TINY[E4M3] * s + 1.2 * dz
    y = z @ w2.T + b2
    ym = (z.abs() + off) @ w2.abs().T + b2.abs()
    coarse = off @ w2.abs().T + _sum_bound(H, ym, half < 1e-6 or act == E2M1) + half * ym
    fine = _rounded(z, act)[0] @ w2.T + b2
    return y, coarse, fine


# 4 bits: z is off by at most 1e-5 of itself on average (the GELU's polynomial;
# its sums are exact to 2^-23) before it is rounded; steps of e2m1 are at least
# 2^-2 of a value of 2 or more and lie 0.5 apart below, so at most 2e-5 / 2^-3 of
# the values fall on the other side of a tie, which moves them by a third of
# themselves at most (3 to 2 or 4, 6 to 4).
FLIPS4 = math.sqrt(2e-5 / 2.0 ** -3) / 3 + 1e-3
FFN = [(1, 8, 8), (1, 768, 1536), (3, 100, 390), (16, 384, 1536), (17, 130, 516), (40, 390, 1550), (300, 192, 768),
       (515, 256, 1030), (1000, 384, 512), (2500, 144, 2000)]


def _ffn_weights(W1, W2):
    w1, s1 = cm.quantize(W1.cuda(), E2M1)
    w2, s2 = cm.quantize(W2.cuda(), E2M1)
    return w1, s1, w2, s2, dequantize4(w1, s1)[..., :W1.shape[-1]], dequantize4(w2, s2)[..., :W2.shape[-1]]


@pytest.mark.parametrize("act", ROWS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,D,H", FFN)
def test_ffn(T, D, H, dtype, act):
    x, W1, b1, W2, b2 = _ffn_inputs(T, D, H, 0, dtype, T + D)
    w1, s1, w2, s2, d1, d2 = _ffn_weights(W1, W2)
    y = cm.quantized_ffn_forward(x.cuda(), w1, s1, b1.cuda(), w2, s2, b2.cuda(), activations=act).cpu().double()
    half = torch.finfo(dtype).eps / 2
    ref, coarse, fine = _ffn_reference(x, d1, b1.double(), d2, b2.double(), act, half)
    assert ((y - ref).abs() <= coarse).all()
    flips = FLIPS4 if act == E2M1 else CUT + FLIPS
    assert (y - fine).norm() <= (half + flips) * fine.norm()


@pytest.mark.parametrize("act", ROWS)
@pytest.mark.parametrize("T,D,H,offsets", [
    (7, 64, 256, [0, 1, 1, 7]), (12, 72, 264, [2, 5, 9]), (40, 100, 390, [2, 20, 30]), (700, 192, 512, [0, 300, 301, 301, 650]),
    (1000, 256, 1030, [0, 250, 480, 770, 1000])])
def test_ffn_groups(T, D, H, offsets, act):
    E = len(offsets) - 1
    x, W1, b1, W2, b2 = _ffn_inputs(T, D, H, E, BF16, T)
    w1, s1, w2, s2, d1, d2 = _ffn_weights(W1, W2)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    out = torch.full((T, D), 7.5, dtype=BF16, device="cuda")
    y = cm.quantized_ffn_forward(x.cuda(), w1, s1, b1.cuda(), w2, s2, b2.cuda(), offsets=off, out=out,
                                 activations=act).cpu().double()
    flips = FLIPS4 if act == E2M1 else CUT + FLIPS
    for e, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        if hi > lo:
            ref, coarse, fine = _ffn_reference(x[lo:hi], d1[e], b1[e].double(), d2[e], b2[e].double(), act, 2.0 ** -8)
            assert ((y[lo:hi] - ref).abs() <= coarse).all()
            if act == E4M3 or hi - lo > 20:       # (a single flip in a single row is more than its share)
                assert (y[lo:hi] - fine).norm() <= (2.0 ** -8 + flips) * fine.norm()
    assert (y[:offsets[0]] == 7.5).all() and (y[offsets[-1]:] == 7.5).all()


@pytest.mark.parametrize("act", ROWS)
def test_workspace_of_more_rows_holds_fewer(act):
    """And what lies behind its bytes is not touched."""
    D, H = 72, 1000
    x, W1, b1, W2, b2 = _ffn_inputs(40, D, H, 0, BF16, 3)
    w1, s1, w2, s2, _, _ = _ffn_weights(W1, W2)
    n = cm.quantized_workspace_bytes(cm.make_shape(17, D, 1, 1, cm.BF16, H=H))
    mem = torch.full((n + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    for T in (1, 9, 16, 17):
        xt = x[:T].contiguous().cuda()
        call = lambda **kw: cm.quantized_ffn_forward(xt, w1, s1, b1.cuda(), w2, s2, b2.cuda(), activations=act, **kw)
        assert torch.equal(call(ws=mem[:n]), call())
    assert (mem[n:] == 0x5a).all()


@pytest.mark.parametrize("act", ROWS)
def test_same_result_every_time(act):
    x, W1, b1, W2, b2 = _ffn_inputs(333, 384, 1536, 0, BF16, 5)
    w1, s1, w2, s2, _, _ = _ffn_weights(W1, W2)
    for T in (1, 20, 333):
        xt = x[:T].contiguous().cuda()
        call = lambda: cm.quantized_ffn_forward(xt, w1, s1, b1.cuda(), w2, s2, b2.cuda(), activations=act)
        first = call()
        for _ in range(5):
            assert torch.equal(call(), first)


def test_8bit_weights_take_8bit_activations_only():
    x, W1, b1, W2, b2 = _ffn_inputs(3, 64, 128, 0, BF16, 5)
    w1, s1 = cm.quantize(W1.cuda(), block_rows=128)
    w2, s2 = cm.quantize(W2.cuda(), block_rows=128)
    with pytest.raises(cm.ClearMoEError):
        cm.quantized_ffn_forward(x.cuda(), w1, s1, b1.cuda(), w2, s2, b2.cuda(), activations=E2M1)


# ---------------------------------------------------------------------------
# Used together
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("T", [200, 7])
def test_experts_between_dispatch_and_combine(T):
    """Norm, route, dispatch with rows, the experts' 4-bit FFN, combine, and the
    next norm with the residual's addition to 8 bits for the product that
    follows: eager, and as a captured graph on another stream, replayed with
    other inputs and eager calls in between."""
    D, H, E, k = 128, 320, 5, 2
    x, W1, b1, W2, b2 = _ffn_inputs(T, D, H, E, BF16, 21)
    g = _gen(22)
    Wg, bg = torch.randn(E, D, generator=g).bfloat16().cuda(), 0.1 * torch.randn(E, generator=g).cuda()
    nw = (1 + 0.1 * torch.randn(D, generator=g)).cuda()
    x, b1, b2 = x.cuda(), b1.cuda(), b2.cuda()
    w1, s1, w2, s2, _, _ = _ffn_weights(W1, W2)
    w3, s3 = cm.quantize(torch.randn(96, D, generator=g).cuda(), E2M1)
    ws = cm.alloc_workspace(cm.make_shape(T, D, E, k, cm.BF16))
    wq = cm.alloc_quantized_workspace(cm.make_shape(T * k, D, E, 1, cm.BF16, H=H))

    def block(x):
        h = cm.rms_norm(x, nw)
        idx, gate = cm.route(h, Wg, bg, k, ws=ws)
        _, offsets, _, inv, xperm = cm.dispatch(idx, E, ws=ws, x=h, hist_in_ws=True)
        ye = cm.quantized_ffn_forward(xperm, w1, s1, b1, w2, s2, b2, offsets=offsets, ws=wq)
        y = cm.combine(ye, inv, gate)
        v, s, total = cm.rms_norm(y, nw, residual=x, out_dtype=E4M3)
        return cm.quantized_gemm(v, s, w3, s3), total

    out, total = block(x)
    f = total.double().cpu()
    n = f / (f.square().mean(1, keepdim=True) + 1e-6).sqrt() * nw.double().cpu()
    want = _rounded(n, E4M3)[0] @ dequantize4(w3, s3).T
    assert (out.cpu().double() - want).norm() <= (2.0 ** -8 + CUT + FLIPS) * want.norm()

    stream, graph, xs = torch.cuda.Stream(), torch.cuda.CUDAGraph(), x.clone()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        block(xs)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        og, tg = block(xs)
    for i in range(4):
        xi = torch.randn(T, D, generator=g).bfloat16().cuda()
        want, total = block(xi)
        torch.cuda.synchronize()
        xs.copy_(xi)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(og, want) and torch.equal(tg, total), i


@pytest.mark.parametrize("T", [5, 700])
def test_calls_on_a_busy_stream(T):
    x, W1, b1, W2, b2 = _ffn_inputs(T, 192, 768, 0, BF16, 3)
    w1, s1, w2, s2, _, _ = _ffn_weights(W1, W2)
    x, b1, b2 = x.cuda(), b1.cuda(), b2.cuda()
    a, sa = cm.quantize(x, E2M1)
    calls = [lambda **kw: cm.quantized_ffn_forward(x, w1, s1, b1, w2, s2, b2, activations=E2M1, **kw),
             lambda **kw: cm.quantized_gemm(a, sa, w1, s1, **kw), lambda **kw: cm.dequantize(a, sa, **kw),
             lambda **kw: cm.quantize(x, E2M1, **kw)[0].view(torch.uint8),
             lambda **kw: cm.rms_norm(x, None, residual=x, **kw)[0]]
    work = torch.randn(4096, 4096, device="cuda")
    side = torch.cuda.Stream()
    for call in calls:
        want = call()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(8):
                busy = work @ work
        y = call(stream=side)
        other = [torch.full((T * 400,), 0xff, dtype=torch.uint8, device="cuda") for _ in range(20)]
        other += [torch.full_like(want, 77) for _ in range(20)]
        side.synchronize()
        assert torch.equal(y, want)
        torch.cuda.synchronize()
        del y, other, busy
