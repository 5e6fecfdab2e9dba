"""quantize on more blocks than one launch holds."""
import pytest
import torch

from paper_2606_28516_amd import clearmoe as cm

pytestmark = pytest.mark.gpu


def _bytes(t):
    return t.view(torch.uint8)


def _check(x, block_rows, borders):
    """Pieces around the borders against the same pieces by themselves."""
    v, s = cm.quantize(x, block_rows=block_rows)
    for at in (0, *borders, x.shape[0]):
        lo, hi = max(0, at - 300), min(x.shape[0], at + 300)
        w, t = cm.quantize(x[lo:hi].contiguous(), block_rows=block_rows)
        assert torch.equal(_bytes(v[lo:hi]), _bytes(w)) and torch.equal(_bytes(s[lo:hi]), _bytes(t)), at


def test_rows():
    """2^28 blocks a launch, less a workgroup's: narrow rows past it."""
    g = torch.Generator(device="cuda").manual_seed(1)
    n = 2 ** 28 + 1000
    x = torch.randn(n, 1, device="cuda", generator=g, dtype=torch.bfloat16)
    _check(x, 1, (2 ** 28 - 16, 2 ** 28))
    del x
    torch.cuda.empty_cache()


def test_squares():
    """2^24 squares a launch, less one: many small matrices."""
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(2 ** 24 + 500, 1, 5, device="cuda", generator=g, dtype=torch.bfloat16)
    _check(x, 128, (2 ** 24 - 1, 2 ** 24))
    y = torch.randn(2 ** 23 + 100, 1, 130, device="cuda", generator=g, dtype=torch.bfloat16)
    _check(y, 128, (2 ** 23 - 1, 2 ** 23))
    del x, y
    torch.cuda.empty_cache()
