"""The 8-bit operators (quantize, quantized_gemm, quantized_ffn_forward) against
plain 64-bit forms, at the sizes and values where they can go wrong."""
import math

import pytest
import torch

from paper_2606_28516_amd import clearmoe as cm
from tests.q8_util import HALF, TINY, dequantize, quantize_ref, scale_exponent, up

pytestmark = pytest.mark.gpu

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
FMTS = [E4M3, E5M2]


def _gen(seed):
    return torch.Generator().manual_seed(seed)


# ---------------------------------------------------------------------------
# quantize: bit for bit
# ---------------------------------------------------------------------------
def _check_quantize(x, fmt, block_rows):
    v, s = cm.quantize(x.cuda(), fmt, block_rows=block_rows)
    x3 = x if x.dim() == 3 else x[None]
    rv, rs = quantize_ref(x3, fmt, block_rows)
    assert v.dtype == fmt and s.dtype == torch.float8_e8m0fnu
    assert tuple(v.shape[-2:]) == tuple(rv.shape[-2:]) and tuple(s.shape[-2:]) == tuple(rs.shape[-2:])
    assert torch.equal(s.cpu().view(torch.uint8).reshape(rs.shape), rs)
    got = v.cpu().view(torch.uint8).reshape(rv.shape)
    nan = v.cpu().float().reshape(rv.shape).isnan()
    assert torch.equal(nan, rv.view(fmt).float().isnan())
    assert torch.equal(got[~nan], rv[~nan])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (1, 16), (5, 127), (17, 128), (130, 129), (257, 384), (64, 700),
                                       (2, 65536)])
def test_quantize_rows(rows, cols, dtype, fmt):
    g = _gen(rows * 31 + cols)
    x = torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-20, 20, (rows, 1), generator=g).float())
    _check_quantize(x.to(dtype), fmt, 1)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(1, 1), (127, 130), (128, 128), (129, 257), (3, 200, 390), (2, 1, 16), (300, 8)])
def test_quantize_square(shape, dtype, fmt):
    g = _gen(sum(shape))
    x = torch.randn(*shape, generator=g) * torch.exp2(torch.randint(-3, 3, shape[:-1] + (1,), generator=g).float())
    _check_quantize(x.to(dtype), fmt, 128)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_special_values(fmt, block_rows):
    """Blocks of zeros, the range's border on both sides, the smallest and
    largest floats, ties, infinities and NaN."""
    inf, nan = math.inf, math.nan
    top = 448.0 if fmt == E4M3 else 57344.0
    nxt = torch.nextafter(torch.tensor(top), torch.tensor(inf)).item()
    firsts = [0.0, -0.0, top, nxt, -top, 2 * top, top / 2 ** 20, nxt / 2 ** 20, 1e-45, 1.2e-38, 3.4e38, inf, -inf, nan]
    x = torch.zeros(len(firsts), 256)
    for i, f in enumerate(firsts):
        x[i, 3] = f
        # ties and values around them under the scale of the block
        x[i, 10:42] = torch.arange(32) * (top / 512) if math.isfinite(f) and abs(f) >= 1 else f
        x[i, 200] = 1.0
    if block_rows == 1:
        _check_quantize(x, fmt, 1)
        x3 = x[None].repeat(2, 1, 1)
        x3[1] *= -1
        _check_quantize(x3, fmt, 1)
    else:
        for i in range(len(firsts)):
            _check_quantize(x[i:i + 1], fmt, 128)
        _check_quantize(x, fmt, 128)


def test_quantize_strided_rows_and_empty():
    g = _gen(5)
    big = torch.randn(40, 600, generator=g).cuda()
    for sl in (big[:, 8:208], big[:, 3:203], big[::2, :130], big.bfloat16()[:, 1:300]):
        v, s = cm.quantize(sl)
        w, t = cm.quantize(sl.contiguous())
        assert torch.equal(v.view(torch.uint8), w.view(torch.uint8))
        assert torch.equal(s.view(torch.uint8), t.view(torch.uint8))
    v, s = cm.quantize(big[:0])
    assert v.shape == (0, 608) and s.shape == (0, 8)
    with pytest.raises(cm.ClearMoEError):
        cm.quantize(big.T)
    with pytest.raises(cm.ClearMoEError):
        cm.quantize(big.half())
    with pytest.raises(cm.ClearMoEError):
        cm.quantize(big, torch.float16)
    with pytest.raises(cm.ClearMoEError):
        cm.quantize(big, block_rows=64)


# ---------------------------------------------------------------------------
# quantized_gemm
# ---------------------------------------------------------------------------
def _operand(g, shape, fmt, block_rows):
    """A quantised operand made on the CPU, and its values in 64 bits."""
    x = torch.randn(*shape, generator=g) * torch.exp2(torch.randint(-4, 5, shape[:-1] + (1,), generator=g).float())
    x3 = x if x.dim() == 3 else x[None]
    v, s = quantize_ref(x3, fmt, block_rows)
    if x.dim() == 2:
        v, s = v[0], s[0]
    v = v.contiguous().view(fmt)
    return v.cuda(), s.contiguous().view(torch.float8_e8m0fnu).cuda(), dequantize(v, s, block_rows)


def _gelu(v):
    return 0.5 * v * torch.special.erfc(-v / math.sqrt(2.0))


def _sum_bound(K, mass, wide):
    """K products and their sum in float32, in any order: every addition is off
    by at most 2^-24 of the sum of magnitudes (2^-23 where an instruction
    truncates what it aligns).  The 8-bit instructions (not used for float32
    results: wide) also cut every product up to 14 bits below the largest of
    the eight it is added with: seven of them by 2^-13 of the eighth at most,
    7 * 2^-13 < 2^-10 of the sum of magnitudes."""
    return ((K + 8) * 2.0 ** -23 + (0.0 if wide else 2.0 ** -10)) * mass


def _gelu_bound(v, d, wide):
    """Error of the GELU of a sum v that is off by d: slope at most 1.13, and
    its own error: the erf's 1.5e-7 and a few roundings for float32 results;
    otherwise that of a polynomial for log2 Phi(-|v|), 4.7e-6 ln 2 = 3.3e-6 of
    |v| Phi(-|v|) up to |v| = 6 (further out that is below 6e-9), and the
    roundings of the exponent, seven terms below 64: 7 * 64 * 2^-24 ln 2 of
    |v| Phi(-|v|) <= |v| / 2, less than 1e-5 |v|."""
    return 1.13 * d + (4e-7 * v.abs() if wide else 1.4e-5 * v.abs() + 1e-8)


# The share of _sum_bound that seven cut products in eight leave on average:
# each off by at most 2^-13 of the largest (root mean square 2^-13 / sqrt 3),
# seven of them by 1.53 * 2^-13, the eights independent of each other, so
# 1.6 * 2^-13 of the root of the sum of squared products.
CUT = 1.6 * 2.0 ** -13


def _reference(a, b, bias, offsets, gelu, wide):
    """(values, bound before the last rounding, its size on average, rows that
    are written)."""
    M, K = a.shape
    b = b if b.dim() == 3 else b[None]
    o = [0, M] if offsets is None else offsets
    y = torch.zeros(M, b.shape[1], dtype=torch.float64)
    mass, live, sq = torch.zeros_like(y), torch.zeros(M, dtype=torch.bool), torch.zeros_like(y)
    for e, (lo, hi) in enumerate(zip(o, o[1:])):
        y[lo:hi] = a[lo:hi] @ b[e].T
        sq[lo:hi] = (a[lo:hi] ** 2 @ (b[e] ** 2).T).sqrt()
        mass[lo:hi] = a[lo:hi].abs() @ b[e].abs().T
        live[lo:hi] = True
        if bias is not None:
            w = bias.cpu().double().reshape(b.shape[0], -1)[e]
            y[lo:hi] += w
            mass[lo:hi] += w.abs()
    d = _sum_bound(K, mass, wide)
    mean = (math.sqrt(K) + 8) * 2.0 ** -23 * mass + (0.0 if wide else CUT) * sq
    if gelu:
        return _gelu(y), _gelu_bound(y, d, wide), _gelu_bound(y, mean, wide), live
    return y, d, mean, live


def _check_product(M, N, K, E=0, offsets=None, fa=E4M3, fb=E4M3, out=torch.bfloat16, bias=True, gelu=False, seed=0):
    g = _gen(seed + M * 7 + N * 3 + K)
    a, sa, fa64 = _operand(g, (M, K), fa, 1)
    b, sb, fb64 = _operand(g, (E, N, K) if E else (N, K), fb, 128)
    bi = torch.randn(*((E, N) if E else (N,)), generator=g).cuda() if bias else None
    off = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda")
    ref, d, mean, live = _reference(fa64, fb64, bi, offsets, gelu, out == torch.float32)
    if out in HALF:
        c, cs = cm.quantized_gemm(a, sa, b, sb, bias=bi, gelu=gelu, offsets=off, out_dtype=out)
        s = torch.ldexp(torch.ones(cs.shape, dtype=torch.float64), cs.cpu().view(torch.uint8).int() - 127)
        nb = -(-N // 128)
        full = dequantize(c, cs, 1)
        assert (full[live][:, N:] == 0).all() and (s[live][:, nb:] == 1).all()
        cols = s.repeat_interleave(128, dim=1)[:, :N]
        err = (full[:, :N] - ref).abs()
        assert (err <= HALF[out] * ref.abs() + TINY[out] * cols + 1.2 * d)[live].all()
        for i in range(nb):                       # the scale is that of the block's largest value
            lo = (ref[:, 128 * i:128 * i + 128].abs() - d[:, 128 * i:128 * i + 128]).clamp(min=0).amax(1)
            hi = (ref[:, 128 * i:128 * i + 128].abs() + d[:, 128 * i:128 * i + 128]).amax(1)
            e = torch.log2(s[:, i])
            zero = lo == 0                        # a block that may be zero has scale 1
            assert ((e >= scale_exponent(lo, out)) & (e <= scale_exponent(hi, out)) | zero)[live].all()
        return
    sentinel = torch.full((M, N), 7.5, dtype=out, device="cuda")
    c = cm.quantized_gemm(a, sa, b, sb, bias=bi, gelu=gelu, offsets=off, out_dtype=out, out=sentinel)
    c = c.cpu().double()
    half = torch.finfo(out).eps / 2
    err = (c - ref).abs()
    bad = (err > half * ref.abs() + (1 + half) * d + 1e-38) & live[:, None]
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), float(err.max()))
    assert (c[~live] == 7.5).all()
    # over the whole result the errors stay near the rounding of the output
    # and the average error of the sum
    if live.any():
        assert err[live].norm() <= half * ref[live].norm() + mean[live].norm() + 1e-30


SIZES = [
    (1, 1, 16), (1, 16, 128), (1, 1536, 384), (2, 17, 144), (16, 128, 112), (17, 130, 400), (33, 200, 1040),
    (100, 384, 1536), (129, 257, 272), (300, 1550, 400), (256, 256, 128), (257, 300, 640), (1003, 520, 1200),
    (512, 512, 2064), (2000, 72, 784), (700, 1032, 128), (4100, 1550, 208), (3000, 1300, 144), (8200, 776, 336),
]


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32, E4M3, E5M2])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_product(M, N, K, out):
    _check_product(M, N, K, out=out, gelu=(M + N) % 2 == 0, bias=K % 32 == 0)


@pytest.mark.parametrize("out", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("M,N,K", [(5, 40, 144), (300, 300, 400), (700, 300, 400), (3000, 1300, 144), (4200, 1550, 144)])
@pytest.mark.parametrize("fa", FMTS)
@pytest.mark.parametrize("fb", FMTS)
def test_product_formats(fa, fb, M, N, K, out):
    _check_product(M, N, K, fa=fa, fb=fb, out=out)


GROUPS = [
    (40, 48, 160, [0, 40]), (40, 48, 160, [0, 0, 40, 40]), (40, 200, 160, [3, 9, 9, 30]),
    (900, 130, 272, [0, 1, 300, 300, 557, 813, 900]), (900, 264, 144, [100, 400, 656, 880]),
    (1200, 384, 400, [0, 37, 150, 300, 600, 601, 890, 1100, 1200]),
    (64, 32, 48, list(range(65))), (5, 24, 32, [0, 0, 0, 0]),
    (4000, 700, 144, [0, 1000, 1001, 2500, 4000]), (6000, 1160, 144, [0, 5, 5, 1700, 3333, 6000]), (7000, 900, 272, [64, 100, 3000, 6900]),
]


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32, E4M3])
@pytest.mark.parametrize("M,N,K,offsets", GROUPS)
def test_product_groups(M, N, K, offsets, out):
    _check_product(M, N, K, E=len(offsets) - 1, offsets=offsets, out=out, gelu=N % 16 == 0)


def test_product_offsets_outside_the_rows_are_clamped():
    """Bad offsets reach no memory outside the arrays: they are clamped to the
    rows, and a group whose end lies before its start is empty."""
    M, N, K, E = 70, 40, 64, 4
    g = _gen(3)
    a, sa, a64 = _operand(g, (M, K), E4M3, 1)
    b, sb, b64 = _operand(g, (E, N, K), E4M3, 128)
    off = torch.tensor([-5, 20, 10, 50, 1000000], dtype=torch.int32, device="cuda")
    out = torch.full((M, N), 7.5, dtype=torch.float32, device="cuda")
    cm.quantized_gemm(a, sa, b, sb, offsets=off, out_dtype=torch.float32, out=out)
    c = out.cpu().double()
    for e, (lo, hi) in enumerate([(0, 20), (20, 20), (10, 50), (50, 70)]):
        if e == 0:
            hi = 10                               # rows 10 .. 19 belong to two groups
        ref = a64[lo:hi] @ b64[e].T
        mass = a64[lo:hi].abs() @ b64[e].abs().T
        if e == 2:
            ref, mass, lo = ref[10:], mass[10:], 20
        assert ((c[lo:hi] - ref).abs() <= _sum_bound(K, mass, True) + 2.0 ** -24 * ref.abs()).all()


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_product_scales_reach_their_blocks(out):
    """Every scale of A and B is a different power of two and the values are
    one: each block's share of the sum is its scales' product, exactly."""
    M, N, K = 300, 300, 1152
    nk = K // 128
    g = _gen(11)
    a = torch.ones(M, K).to(E4M3).cuda()
    b = torch.ones(N, K).to(E4M3).cuda()
    sa = torch.full((M, up(nk, 4)), 127, dtype=torch.uint8)
    sb = torch.full((3, up(nk, 4)), 127, dtype=torch.uint8)
    sa[:, :nk] = torch.randint(122, 132, (M, nk), generator=g).to(torch.uint8)
    sb[:, :nk] = torch.randint(122, 132, (3, nk), generator=g).to(torch.uint8)
    c = cm.quantized_gemm(a, sa.view(torch.float8_e8m0fnu).cuda(), b, sb.view(torch.float8_e8m0fnu).cuda(),
                          out_dtype=out)
    fa, fb = torch.exp2(sa.double() - 127)[:, :nk], torch.exp2(sb.double() - 127)[:, :nk]
    ref = 128 * fa @ fb.repeat_interleave(128, dim=0)[:N].T
    assert torch.equal(c.cpu(), ref.to(out))


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_product_nan_and_infinity_stay_in_their_row(out):
    M, N, K = 40, 96, 256
    g = _gen(12)
    a, sa, _ = _operand(g, (M, K), E5M2, 1)
    b, sb, _ = _operand(g, (N, K), E4M3, 128)
    want = cm.quantized_gemm(a, sa, b, sb, out_dtype=out)
    bytes_ = a.view(torch.uint8)
    bytes_[3, 17] = 0x7f                          # NaN
    bytes_[20, 200] = 0x7c                        # infinity
    c = cm.quantized_gemm(a, sa, b, sb, out_dtype=out)
    assert c[3].isnan().all()
    assert (~c[20].isfinite()).all()
    keep = [i for i in range(M) if i not in (3, 20)]
    assert torch.equal(c[keep], want[keep])


@pytest.mark.parametrize("M", [20, 9000])
@pytest.mark.parametrize("out", FMTS)
def test_product_to_bytes_with_infinities(out, M):
    """Infinite and NaN results: NaN in e4m3, infinity kept in e5m2; the block's
    scale is that of the finite ones."""
    N, K = 400, 64
    g = _gen(14)
    a, sa, _ = _operand(g, (M, K), E4M3, 1)
    b, sb, _ = _operand(g, (N, K), E4M3, 128)
    bias = torch.zeros(N, device="cuda")
    want, ws = cm.quantized_gemm(a, sa, b, sb, bias=bias, out_dtype=out)
    bias[7], bias[200], bias[399] = math.inf, -math.inf, math.nan
    got, gs = cm.quantized_gemm(a, sa, b, sb, bias=bias, out_dtype=out)
    f = got.float()
    assert f[:, 399].isnan().all()
    if out == E4M3:
        assert f[:, 7].isnan().all() and f[:, 200].isnan().all()
    else:
        assert (f[:, 7] == math.inf).all() and (f[:, 200] == -math.inf).all()
    keep = [n for n in range(N) if n not in (7, 200, 399)]
    assert f[:, keep].isfinite().all()
    same = (gs.view(torch.uint8) == ws.view(torch.uint8))[:, :4]
    assert same.float().mean() > 0.9              # the largest of a block was rarely one of the three
    for i in range(4):
        cols = [n for n in keep if n // 128 == i]
        rows = same[:, i]
        assert torch.equal(f[rows][:, cols], want.float()[rows][:, cols])


def test_workspace_of_more_rows_holds_fewer():
    D, H = 72, 1000
    x, W1, b1, W2, b2 = _ffn_inputs(40, D, H, 0, torch.bfloat16, 3)
    w1, s1 = cm.quantize(W1.cuda(), block_rows=128)
    w2, s2 = cm.quantize(W2.cuda(), block_rows=128)
    last = 0
    for T in range(1, 41):
        n = cm.quantized_workspace_bytes(cm.make_shape(T, D, 1, 1, cm.BF16, H=H))
        assert n >= last
        last = n
    ws = cm.alloc_quantized_workspace(cm.make_shape(17, D, 1, 1, cm.BF16, H=H))
    for T in (1, 9, 16, 17):
        xt = x[:T].contiguous().cuda()
        y = cm.quantized_ffn_forward(xt, w1, s1, b1.cuda(), w2, s2, b2.cuda(), ws=ws)
        assert torch.equal(y, cm.quantized_ffn_forward(xt, w1, s1, b1.cuda(), w2, s2, b2.cuda()))


def test_mismatched_tensors_are_refused():
    g = _gen(15)
    a, sa, _ = _operand(g, (6, 64), E4M3, 1)
    b, sb, _ = _operand(g, (40, 64), E4M3, 128)
    ok = dict(bias=torch.zeros(40, device="cuda"))
    cm.quantized_gemm(a, sa, b, sb, **ok)
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    for args, kw in (((a, sa[:5], b, sb), {}), ((a, sa, b, sb.repeat(2, 1)), {}), ((a, sa, b[:, :48].contiguous(), sb), {}),
                     ((a, sa, b, sb), dict(bias=torch.zeros(39, device="cuda"))),
                     ((a, sa, b, sb), dict(bias=torch.zeros(40, device="cuda").double())),
                     ((a, sa, b, sb), dict(offsets=off)),
                     ((a, sa, b[None], sb[None]), dict(offsets=off)),
                     ((a, sa.view(torch.uint8), b, sb), {}), ((a.float(), sa, b, sb), {}),
                     ((a, sa, b, sb), dict(out=torch.empty(6, 41, dtype=torch.bfloat16, device="cuda"))),
                     ((a, sa, b, sb), dict(out_dtype=torch.float16))):
        with pytest.raises(cm.ClearMoEError):
            cm.quantized_gemm(*args, **kw)


def test_product_row_strides():
    """lda and ldc through the C ABI: rows inside wider arrays, whose other
    bytes stay as they were."""
    import ctypes
    M, N, K = 37, 50, 80
    g = _gen(13)
    a, sa, _ = _operand(g, (M, K), E4M3, 1)
    b, sb, _ = _operand(g, (N, K), E4M3, 128)
    want = cm.quantized_gemm(a, sa, b, sb)
    wide = torch.zeros(M, 128, dtype=torch.uint8, device="cuda").view(E4M3)
    wide.view(torch.uint8)[:, :K] = a.view(torch.uint8)
    wide.view(torch.uint8)[:, K:] = 0x7e
    out = torch.full((M, 61), 7.5, dtype=torch.bfloat16, device="cuda")
    p = cm.Product(M, N, K, 0, 2, 2, cm.BF16, 0, 0, 128, 61)
    ptr = lambda t: ctypes.c_void_p(t.data_ptr())
    rc = cm.lib().clearmoe_quantized_gemm(ctypes.byref(p), ptr(wide), ptr(sa), ptr(b), ptr(sb), None, None, ptr(out),
                                          None, cm._stream(None))
    assert rc == 0
    assert torch.equal(out[:, :N], want) and (out[:, N:] == 7.5).all()


# ---------------------------------------------------------------------------
# quantized_ffn_forward
# ---------------------------------------------------------------------------
def _ffn_inputs(T, D, H, E, dtype, seed):
    g = _gen(seed)
    lead = (E,) if E else ()
    x = torch.randn(T, D, generator=g).to(dtype)
    W1 = torch.randn(*lead, H, D, generator=g) / math.sqrt(D)
    W2 = torch.randn(*lead, D, H, generator=g) / math.sqrt(H)
    b1, b2 = 0.1 * torch.randn(*lead, H, generator=g), 0.1 * torch.randn(*lead, D, generator=g)
    return x, W1, b1, W2, b2


def _ffn_reference(x, w1, b1, w2, b2, D, H, half):
    """One group's FFN in 64 bits from the weights' 8-bit values, z exact, and
    a bound that allows any rounding of z to the 8-bit grid around it."""
    T = x.shape[0]
    xv, xs = quantize_ref(x[None], E4M3, 1)
    xq = dequantize(xv[0].contiguous().view(E4M3), xs[0], 1)
    pre = xq @ w1.T + b1
    mass = xq.abs() @ w1.abs().T + b1.abs()
    z = _gelu(pre)
    dz = _gelu_bound(pre, _sum_bound(D, mass, False), False)
    zp = torch.zeros(T, up(H, 128), dtype=torch.float64)
    zp[:, :H] = z.abs() + dz
    zs = torch.ldexp(torch.ones(T, zp.shape[1] // 128, dtype=torch.float64),
                     scale_exponent(zp.reshape(T, -1, 128).amax(2), E4M3)).repeat_interleave(128, dim=1)[:, :H]
    off = HALF[E4M3] * z.abs() + TINY[E4M3] * zs + 1.2 * dz
    y = z @ w2[:, :H].T + b2
    ym = (z.abs() + off) @ w2[:, :H].abs().T + b2.abs()
    coarse = off @ w2[:, :H].abs().T + _sum_bound(H, ym, half < 1e-6) + half * ym
    # and with z rounded as the definition says: only values next to a tie may
    # fall on its other side
    zv, zz = quantize_ref(z[None], E4M3, 1)
    fine = dequantize(zv[0].contiguous().view(E4M3), zz[0], 1)[:, :H] @ w2[:, :H].T + b2
    return y, coarse, fine


# z is off by CUT of itself on average before it is rounded; steps of e4m3 are
# at least 2^-4 of a value, so at most 2 CUT / 2^-4 of the values round to the
# other side of a tie, which is 2^-3 of them at most.
FLIPS = 2.0 ** -3 * math.sqrt(2 * CUT / 2.0 ** -4)

FFN = [(1, 8, 8), (1, 768, 1536), (3, 100, 390), (16, 384, 1536), (17, 130, 516), (40, 390, 1550), (300, 192, 768),
       (515, 256, 1030), (1000, 384, 512), (2500, 144, 2000)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,D,H", FFN)
def test_ffn(T, D, H, dtype):
    x, W1, b1, W2, b2 = _ffn_inputs(T, D, H, 0, dtype, T + D)
    w1, s1 = cm.quantize(W1.cuda(), block_rows=128)
    w2, s2 = cm.quantize(W2.cuda(), block_rows=128)
    y = cm.quantized_ffn_forward(x.cuda(), w1, s1, b1.cuda(), w2, s2, b2.cuda()).cpu().double()
    half = torch.finfo(dtype).eps / 2
    ref, coarse, fine = _ffn_reference(x, dequantize(w1, s1, 128), b1.double(), dequantize(w2, s2, 128), b2.double(),
                                       D, H, half)
    assert ((y - ref).abs() <= coarse).all()
    assert (y - fine).norm() <= (half + CUT + FLIPS) * fine.norm()


@pytest.mark.parametrize("T,D,H,offsets", [
    (7, 64, 256, [0, 1, 1, 7]), (12, 72, 264, [2, 5, 9]), (40, 100, 390, [2, 20, 30]), (700, 192, 512, [0, 300, 301, 301, 650]),
    (1000, 256, 1030, [0, 250, 480, 770, 1000])])
def test_ffn_groups(T, D, H, offsets):
    E = len(offsets) - 1
    x, W1, b1, W2, b2 = _ffn_inputs(T, D, H, E, torch.bfloat16, T)
    w1, s1 = cm.quantize(W1.cuda(), block_rows=128)
    w2, s2 = cm.quantize(W2.cuda(), block_rows=128)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    out = torch.full((T, D), 7.5, dtype=torch.bfloat16, device="cuda")
    y = cm.quantized_ffn_forward(x.cuda(), w1, s1, b1.cuda(), w2, s2, b2.cuda(), offsets=off, out=out).cpu().double()
    d1, d2 = dequantize(w1, s1, 128), dequantize(w2, s2, 128)
    for e, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        if hi > lo:
            ref, coarse, fine = _ffn_reference(x[lo:hi], d1[e], b1[e].double(), d2[e], b2[e].double(), D, H, 2.0 ** -8)
            assert ((y[lo:hi] - ref).abs() <= coarse).all()
            assert (y[lo:hi] - fine).norm() <= (2.0 ** -8 + CUT + FLIPS) * fine.norm()
    assert (y[:offsets[0]] == 7.5).all() and (y[offsets[-1]:] == 7.5).all()


@pytest.mark.parametrize("T", [200, 7])
def test_experts_between_dispatch_and_combine(T):
    """Route, dispatch with rows, the experts' 8-bit FFN, combine: the layer of
    a caller's own experts, eager and as a captured graph on another stream,
    replayed with other inputs and eager calls in between."""
    D, H, E, k = 128, 320, 5, 2
    x, W1, b1, W2, b2 = _ffn_inputs(T, D, H, E, torch.bfloat16, 21)
    g = _gen(22)
    Wg, bg = torch.randn(E, D, generator=g).bfloat16(), 0.1 * torch.randn(E, generator=g)
    d = dict(x=x.cuda(), Wg=Wg.cuda(), bg=bg.cuda(), b1=b1.cuda(), b2=b2.cuda())
    w1, s1 = cm.quantize(W1.cuda(), block_rows=128)
    w2, s2 = cm.quantize(W2.cuda(), block_rows=128)
    ws = cm.alloc_workspace(cm.make_shape(T, D, E, k, cm.BF16))
    wq = cm.alloc_quantized_workspace(cm.make_shape(T * k, D, E, 1, cm.BF16, H=H))

    def layer(x, wq):
        idx, gate = cm.route(x, d["Wg"], d["bg"], k, ws=ws)
        counts, offsets, perm, inv, xperm = cm.dispatch(idx, E, ws=ws, x=x, hist_in_ws=True)
        ye = cm.quantized_ffn_forward(xperm, w1, s1, d["b1"], w2, s2, d["b2"], offsets=offsets, ws=wq)
        return cm.combine(ye, inv, gate), idx, gate

    y, idx, gate = layer(d["x"], wq)
    d1, d2 = dequantize(w1, s1, 128), dequantize(w2, s2, 128)
    want, bound = torch.zeros(T, D, dtype=torch.float64), torch.zeros(T, D, dtype=torch.float64)
    for e in range(E):
        ref, coarse, _ = _ffn_reference(x, d1[e], b1[e].double(), d2[e], b2[e].double(), D, H, 2.0 ** -8)
        for j in range(k):
            w = (gate[:, j].cpu().double() * (idx[:, j].cpu() == e))[:, None]
            want += w * ref
            bound += w * coarse
    assert ((y.cpu().double() - want).abs() <= bound + 2.0 ** -8 * (want.abs() + bound)).all()

    stream = torch.cuda.Stream()
    xs = d["x"].clone()
    graph = torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        layer(xs, wq)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        yg, _, _ = layer(xs, wq)
    for i in range(4):
        xi = torch.randn(T, D, generator=g).bfloat16().cuda()
        want, _, _ = layer(xi, wq)
        torch.cuda.synchronize()
        xs.copy_(xi)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(yg, want), i


def test_same_result_every_time():
    """No result depends on the order in which workgroups finish."""
    x, W1, b1, W2, b2 = _ffn_inputs(333, 384, 1536, 0, torch.bfloat16, 5)
    w1, s1 = cm.quantize(W1.cuda(), block_rows=128)
    w2, s2 = cm.quantize(W2.cuda(), block_rows=128)
    for T in (1, 20, 333):
        xt = x[:T].contiguous().cuda()
        first = cm.quantized_ffn_forward(xt, w1, s1, b1.cuda(), w2, s2, b2.cuda())
        for _ in range(5):
            assert torch.equal(cm.quantized_ffn_forward(xt, w1, s1, b1.cuda(), w2, s2, b2.cuda()), first)
