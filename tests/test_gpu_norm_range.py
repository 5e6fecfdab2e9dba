"""rms_norm of rows at the top of float32's range, where the reciprocal of
their size is no normal number."""
import pytest
import torch

from paper_2606_28516_amd import clearmoe as cm
from tests.test_gpu_norm import E4M3, BF16, F32, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF16, BF16), (F32, E4M3)])
@pytest.mark.parametrize("rows,cols", [(4000, 8), (1500, 40), (64, 768), (1500, 900), (40, 3000), (20, 7000), (1100, 7001),
                                       (9, 16000), (5, 33000)])
def test_the_largest_rows(rows, cols, dtype, out):
    g = torch.Generator().manual_seed(cols)
    size = torch.rand(rows, 1, generator=g) * 3 + 0.35
    x = (size + 0.04 * torch.rand(rows, cols, generator=g)).clamp(max=3.38) * 1e38
    x = (x * (1 - 2 * torch.randint(0, 2, x.shape, generator=g))).to(dtype)
    w = 1 + 0.3 * torch.randn(cols, generator=g)
    assert x.isfinite().all()
    _check(x, None, w if cols % 2 else None, out)
    # beside small values: a few of a row carry its size
    x[:, 1::2] *= 1e-3
    x[::2, 2::3] = 1e-30
    _check(x, None, None, out)


def test_the_largest_rows_and_their_residual():
    g = torch.Generator().manual_seed(1)
    x = (1.6 * torch.rand(300, 512, generator=g) * 1e38).to(BF16)
    r = (1.6 * torch.rand(300, 512, generator=g) * 1e38).to(BF16)
    _check(x, r, torch.randn(512, generator=g), BF16)
    _check(x.float(), r.float(), None, F32)
