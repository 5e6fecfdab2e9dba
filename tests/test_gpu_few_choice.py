"""The few-token layer's experts where float32 logits say least: sums of
products below its range, operands below it, products above it.  Every
workgroup chooses for itself; the outputs have to be those of the routing that
is given out."""
import pytest
import torch

from paper_2606_28516_amd import clearmoe as cm
from tests.test_gpu_few import _few, _layer, _reference, _router

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _check(L, expert):
    L["b1"].normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    L["bg"].zero_()
    y, idx, gate = _few(L, _router(L))
    assert (idx == expert).all()
    ref, d = _reference(L, idx.cpu(), gate.cpu().double())
    half = torch.finfo(y.dtype).eps / 2
    assert ((y.cpu().double() - ref).abs() <= half * ref.abs() + (1 + half) * d).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,D,E", [(1, 64, 3), (16, 200, 3), (5, 99, 20)])
@pytest.mark.parametrize("one,many", [(-125, -129), (-126, -130), (-148, -151), (-149, -152)])
def test_sums_of_products_below_the_range(one, many, T, D, E, dtype):
    """Expert 0's logit is one product, expert 2's the sum of 60 smaller ones,
    which is larger."""
    L = _layer(T, D, 96, E, 1, 24, 8, dtype, 5)
    L["x"].fill_(2.0 ** -63)
    L["Wg"].fill_(-2.0 ** -40)
    L["Wg"][0], L["Wg"][2] = 0, 0
    L["Wg"][0, 7] = 2.0 ** (one + 63)
    L["Wg"][2, :60] = 2.0 ** (many + 63)
    _check(L, 2)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,D,E", [(1, 64, 3), (16, 200, 3), (5, 99, 20)])
def test_operands_below_the_range(T, D, E, dtype):
    """A denormal activation times a large weight decides."""
    L = _layer(T, D, 96, E, 1, 24, 8, dtype, 6)
    L["x"].fill_(0)
    L["x"][:, 3], L["x"][:, 5] = 2.0 ** -130, 1.0
    L["Wg"].fill_(-1)
    L["Wg"][0], L["Wg"][2] = 0, 0
    L["Wg"][0, 5] = 2.0 ** -4
    L["Wg"][2, 3] = 2.0 ** 127
    _check(L, 2)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,D,E", [(1, 64, 3), (16, 200, 3), (5, 99, 20)])
def test_products_above_the_range(T, D, E, dtype):
    """Products that leave float32's range and cancel (in double, exactly)."""
    L = _layer(T, D, 96, E, 1, 24, 8, dtype, 7)
    L["x"].fill_(0)
    L["x"][:, 3], L["x"][:, 40], L["x"][:, 5] = 2.0 ** 70, 2.0 ** 70, 1.0
    L["W1"][:, 3], L["W1"][:, 40] = 0, 0
    L["Wg"].fill_(-1)
    L["Wg"][0], L["Wg"][2] = 0, 0
    L["Wg"][0, 5] = 2.0 ** 100
    L["Wg"][2, 3], L["Wg"][2, 40], L["Wg"][2, 5] = 2.0 ** 70, -2.0 ** 70, 2.0 ** 101
    _check(L, 2)
