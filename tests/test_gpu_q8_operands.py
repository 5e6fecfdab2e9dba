"""The 8-bit products' operands and results in memory, at sizes that reach
every kernel: values that are no numbers, bytes past the columns, row strides."""

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
