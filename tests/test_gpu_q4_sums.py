"""Sums of the 4-bit products hold every product, whatever their result: sums
whose large products cancel, exactly, at sizes that reach every kernel."""
import pytest
import torch

from paper_2606_28516_amd import clearmoe as cm
from tests.q4_util import E2M1, GRID, dequantize4, quantize4_ref
from tests.q8_util import dequantize, quantize_ref
from tests.test_gpu_q4 import MANY

pytestmark = pytest.mark.gpu

E4M3, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
BF16, F32 = torch.bfloat16, torch.float32

# M, N, K, offsets
SIZES = [(1, 40, 384, None), (16, 130, 1040, None), (40, 200, 272, None), (300, 390, 400, None), (300, 1550, 1200, None),
         (1000, 1030, 2112, None), (1000, 1540, 176, None), (4200, 1550, 400, None), (70, 300, 400, [2, 9, 9, 60]),
         (2500, 390, 1056, [0, 700, 701, 2500])] + [(M, N, K, o) for M, N, K, o, a, c in MANY if (a, c) == (E4M3, E2M1)]


def _cancelling(rows, K, g):
    """Magnitudes [rows, K] and where the signs differ: of every eight that
    follow each other two are the largest of their format and cancel, the
    others the smallest that it has."""
    pair = torch.rand(rows, -(-K // 8), 8, generator=g).argsort(dim=-1)
    big = (pair < 2).reshape(rows, -1)[:, :K]
    big[:, K // 8 * 8:] = False
    return big, (pair == 1).reshape(rows, -1)[:, :K]


@pytest.mark.parametrize("out", [BF16, F32, E4M3, E2M1])
@pytest.mark.parametrize("M,N,K,offsets", SIZES)
def test_sums_of_8bit_rows(M, N, K, offsets, out):
    """Pairs of 448 x 6 that cancel beside products from 2^-10 on: whole
    multiples of 2^-10 times the scales, which float32 holds."""
    g = torch.Generator().manual_seed(M + N + K)
    E = len(offsets) - 1 if offsets else 0
    big, minus = (t.expand(M, K) for t in _cancelling(1, K, g))
    small = torch.randint(1, 8, (M, K), generator=g).double() * 2.0 ** -9
    a = torch.where(big, torch.where(minus, -448.0, 448.0).double(), small)
    w = GRID[torch.randint(0, 8, (max(E, 1) * N, K), generator=g)] * (1 - 2 * torch.randint(0, 2, (max(E, 1) * N, K), generator=g))
    b = torch.where(big[:1], 6.0, w)
    v = a.float().to(E4M3)
    code = (b.abs()[..., None] == GRID).int().argmax(-1) + 8 * (b < 0)
    code = torch.nn.functional.pad(code, (0, -K % 32)).reshape(b.shape[0], -1, 2)
    vb = (code[..., 0] + 16 * code[..., 1]).to(torch.uint8)
    sa = torch.full((M, (K + 511) // 512 * 4), 255, dtype=torch.uint8)
    sb = torch.full((b.shape[0], (K + 127) // 128 * 4), 255, dtype=torch.uint8)
    ea, eb = torch.randint(-9, 10, (M, 1), generator=g), torch.randint(-9, 10, (b.shape[0], 1), generator=g)
    sa[:, :-(-K // 128)], sb[:, :-(-K // 32)] = 127 + ea, 127 + eb
    lead = (E, N) if E else (N,)
    vb, sb = vb.reshape(*lead, -1), sb.reshape(*lead, -1)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda") if E else None
    c = cm.quantized_gemm(v.cuda(), sa.cuda().view(E8), vb.cuda().view(E2M1), sb.cuda().view(E8), offsets=off, out_dtype=out)
    live = torch.zeros(M, dtype=torch.bool)
    want = torch.zeros(M, N, dtype=torch.float64)
    for e, (lo, hi) in enumerate(zip(offsets, offsets[1:]) if E else [(0, M)]):
        one = slice(e * N, e * N + N)
        want[lo:hi] = torch.ldexp((a[lo:hi] @ b[one].T), ea[lo:hi] + eb[one].T)
        live[lo:hi] = True
    if out in (BF16, F32):
        assert torch.equal(c.cpu()[live], want.float().to(out)[live])
        return
    rv, rs = quantize4_ref(want[None]) if out == E2M1 else quantize_ref(want[None], E4M3, 1)
    got = [t.cpu().view(torch.uint8)[live] for t in c]
    assert torch.equal(got[1], rs[0][live])
    full = (lambda v, s: dequantize4(v, s)) if out == E2M1 else (lambda v, s: dequantize(v.view(E4M3), s, 1))
    assert torch.equal(full(*got), full(rv[0][live], rs[0][live]))


@pytest.mark.parametrize("T", [1, 16, 40, 700])
def test_sums_of_an_ffn(T):
    """Hidden values that are the bias (large ones, which GELU leaves as they
    are): from the smallest e4m3 value of their block to the largest, which
    cancel."""
    D, H = 100, 400
    g = torch.Generator().manual_seed(T)
    big, minus = _cancelling(1, H, g)
    z = torch.where(big, 448.0, torch.randint(1, 8, (1, H), generator=g) * 2.0 ** -9) * 2.0 ** 13
    b = GRID[torch.randint(0, 8, (D, H), generator=g)] * (1 - 2 * torch.randint(0, 2, (D, H), generator=g))
    b = torch.where(big, torch.where(minus, -6.0, 6.0).double(), b)
    b[:, ::32] = torch.where(big[:, ::32], b[:, ::32], 6.0)              # (every block's scale is 1)
    w1, s1 = cm.quantize(torch.zeros(H, D).cuda(), E2M1)
    w2, s2 = cm.quantize(b.float().cuda(), E2M1)
    x = torch.randn(T, D, generator=g).bfloat16().cuda()
    y = cm.quantized_ffn_forward(x, w1, s1, z[0].float().cuda(), w2, s2, None)
    want = (z.double() @ b.T).float().bfloat16().expand(T, D)
    assert torch.equal(y.cpu(), want)
