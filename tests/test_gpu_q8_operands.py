"""The 8-bit products' operands and results in memory, at sizes that reach
every kernel: values that are no numbers, bytes past the columns, row strides."""

import ctypes

import pytest
import torch

from paper_2606_28516_amd import clearmoe as cm
from tests.q8_util import up
from tests.test_gpu_q8 import _operand

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2


def _gen(seed):
    return torch.Generator().manual_seed(seed)


# ---------------------------------------------------------------------------
# Bytes past the columns
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("out", [E4M3, E5M2])
@pytest.mark.parametrize("M,N,K", [(20, 390, 272), (20, 1, 64), (9000, 390, 272), (9000, 1030, 64)])
def test_bytes_past_the_columns_are_zero(M, N, K, out, gelu):
    """Also in rows that hold NaN or an infinity, or whose scale is NaN."""
    g = _gen(N)
    a, sa, _ = _operand(g, (M, K), E5M2, 1)
    b, sb, _ = _operand(g, (N, K), E4M3, 128)
    cols = up(N, 16)
    fill = lambda: torch.full((M, cols), 0x3c, dtype=torch.uint8, device="cuda").view(out)
    want, ws = cm.quantized_gemm(a, sa, b, sb, gelu=gelu, out_dtype=out, out=fill())
    bytes_ = a.view(torch.uint8)
    bytes_[2, 5], bytes_[M - 1, K - 1] = 0x7f, 0x7c         # NaN, infinity
    sa.view(torch.uint8)[7, 0] = 255
    got, gs = cm.quantized_gemm(a, sa, b, sb, gelu=gelu, out_dtype=out, out=fill())
    bad = [2, 7, M - 1]
    keep = [i for i in range(M) if i not in bad]
    assert (got.view(torch.uint8)[:, N:] == 0).all()
    assert (~got.float()[bad, :N].isfinite()).all()
    assert torch.equal(got.view(torch.uint8)[keep], want.view(torch.uint8)[keep])
    assert torch.equal(gs.view(torch.uint8)[keep], ws.view(torch.uint8)[keep])


# ---------------------------------------------------------------------------
# As many rows as a product may have
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("last", [0, 100])
def test_a_group_of_almost_2_31_rows(last):
    M, N, K = 2 ** 31 - 1, 1, 16
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB of device memory")
    E = 2 if last else 1
    a = torch.full((M, K), 0x38, dtype=torch.uint8, device="cuda").view(E4M3)            # ones
    sa = torch.full((M, 4), 127, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    b = torch.full((E, N, K), 0x38, dtype=torch.uint8, device="cuda").view(E4M3)
    sb = torch.full((E, 1, 4), 127, dtype=torch.uint8, device="cuda")
    sb[-1] += 1 if last else 0                                                           # the last expert's: twos
    out = torch.full((M, N), 7.5, dtype=BF16, device="cuda")
    off = torch.tensor([0, M - last, M][:E] + [M], dtype=torch.int32, device="cuda")
    cm.quantized_gemm(a, sa, b, sb.view(torch.float8_e8m0fnu), offsets=off, out=out)
    right = int((out[:M - last] == 16).sum()), int((out[M - last:] == 32).sum())
    del a, sa, out
    torch.cuda.empty_cache()
    assert right == (M - last, last)


def test_most_rows_of_a_float32_result():
    """The largest launch of the 512-thread tiles that is taken."""
    M, N, K = 2 ** 31 - 2048, 1, 16
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB of device memory")
    a = torch.full((M, K), 0x38, dtype=torch.uint8, device="cuda").view(E4M3)
    sa = torch.full((M, 4), 127, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    b, sb = a[:1].clone(), sa[:1].clone()
    out = torch.full((M, N), 7.5, dtype=torch.float32, device="cuda")
    cm.quantized_gemm(a, sa, b, sb, out_dtype=torch.float32, out=out)
    right = int((out == 16).sum())
    del a, sa, out
    torch.cuda.empty_cache()
    assert right == M


# ---------------------------------------------------------------------------
# Row strides and values that are no numbers, in every kernel
# ---------------------------------------------------------------------------
F32 = torch.float32
# M, N, K, result; k a multiple of 128 and not, columns in whole pieces and not
PRODUCTS = [(M, N, K, F32) for M, N, K in ((37, 50, 80), (40, 96, 256), (300, 1550, 400), (257, 1544, 256),
                                           (4200, 1550, 272), (4300, 1544, 128))]
PRODUCTS += [(M, N, K, BF16) for M, N, K in ((37, 50, 80), (40, 96, 256), (300, 1550, 400), (257, 1544, 256),
                                             (2001, 1550, 272), (2050, 1544, 384), (9000, 1550, 144), (9100, 1544, 256))]
PRODUCTS += [(M, N, K, out) for out in (E4M3, E5M2)
             for M, N, K in ((300, 390, 400), (37, 400, 256), (9000, 390, 144), (9100, 1544, 256))]


@pytest.mark.parametrize("M,N,K,out", PRODUCTS)
def test_row_strides(M, N, K, out):
    """Rows of A inside wider ones whose other bytes are NaN, rows of C inside
    wider ones whose other elements stay as they were."""
    g = _gen(M + N)
    a, sa, _ = _operand(g, (M, K), E4M3, 1)
    b, sb, _ = _operand(g, (N, K), E4M3, 128)
    want = cm.quantized_gemm(a, sa, b, sb, out_dtype=out)
    byte = out in (E4M3, E5M2)
    want, ws = want if byte else (want, None)
    wide = torch.full((M, K + 48), 0x7f, dtype=torch.uint8, device="cuda")
    wide[:, :K] = a.view(torch.uint8)
    cols = want.shape[1]
    for more in ((16, 48) if byte else (8, 11)):
        c = torch.full((M, cols + more), 0x4d, dtype=torch.uint8, device="cuda") if byte else \
            torch.full((M, cols + more), 7.5, dtype=out, device="cuda")
        before = c[0, -1].clone()
        cs = torch.empty_like(ws) if byte else None
        p = cm.Product(M, N, K, 0, 2, 2, cm._OUTS[out], 0, 0, K + 48, cols + more)
        ptr = lambda t: None if t is None else ctypes.c_void_p(t.data_ptr())
        rc = cm.lib().clearmoe_quantized_gemm(ctypes.byref(p), ptr(wide), ptr(sa), ptr(b), ptr(sb), None, None, ptr(c),
                                              ptr(cs), cm._stream(None))
        assert rc == 0
        same = want.view(torch.uint8) if byte else want
        assert torch.equal(c[:, :cols], same) and bool((c[:, cols:] == before).all())
        assert not byte or torch.equal(cs.view(torch.uint8), ws.view(torch.uint8))


@pytest.mark.parametrize("M,N,K,out", [p for p in PRODUCTS if p[3] in (F32, BF16)])
def test_nan_and_infinity_stay_in_their_rows(M, N, K, out):
    """Of A: NaN, infinities and a NaN scale in the first and last tile and
    block; the other rows' results are the same to the bit."""
    g = _gen(M + K)
    a, sa, _ = _operand(g, (M, K), E5M2, 1)
    b, sb, _ = _operand(g, (N, K), E4M3, 128)
    want = cm.quantized_gemm(a, sa, b, sb, out_dtype=out)
    v = a.view(torch.uint8)
    v[3, 17], v[20, K - 1], v[M - 2, 0], v[M - 1, K - 1] = 0x7f, 0x7c, 0xfc, 0x7e
    sa.view(torch.uint8)[9, (K - 1) // 128] = 255
    c = cm.quantized_gemm(a, sa, b, sb, out_dtype=out)
    bad = [3, 9, 20, M - 2, M - 1]
    assert c[[3, 9, M - 1]].isnan().all() and not c[bad].isfinite().any()
    keep = [i for i in range(M) if i not in bad]
    assert torch.equal(c[keep], want[keep])


@pytest.mark.parametrize("M,N,K,out", [p for p in PRODUCTS if p[3] in (F32, BF16)])
def test_nan_and_infinity_of_b_stay_in_their_columns(M, N, K, out):
    g = _gen(N + K)
    a, sa, _ = _operand(g, (M, K), E4M3, 1)
    b, sb, _ = _operand(g, (N, K), E5M2, 128)
    want = cm.quantized_gemm(a, sa, b, sb, out_dtype=out)
    v = b.view(torch.uint8)
    v[1, 2], v[30, K - 1], v[N - 1, K - 16] = 0x7f, 0x7c, 0x7e
    c = cm.quantized_gemm(a, sa, b, sb, out_dtype=out)
    assert c[:, [1, N - 1]].isnan().all() and not c[:, 30].isfinite().any()
    keep = [n for n in range(N) if n not in (1, 30, N - 1)]
    assert torch.equal(c[:, keep], want[:, keep])
