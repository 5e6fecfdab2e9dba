"""The few-token layer's experts where float32 logits say least: sums of
products below its range, operands below it, products above it, NaN.  Every
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


def _same(a, b, atol):
    return bool(((a - b).abs() <= atol).logical_or(a.isnan() & b.isnan()).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("adaptive,renorm", [(False, 0), (False, 1), (True, 0), (True, 1)])
@pytest.mark.parametrize("E,k,experts", [(6, 2, (0,)), (6, 2, (0, 1)), (6, 2, (1, 3, 5)), (6, 2, (2,)),
                                         (6, 2, (0, 1, 2, 3, 4, 5)), (20, 2, (0, 19)), (7, 2, (6,))])
def test_nan_logits_are_chosen_as_by_the_router(E, k, experts, adaptive, renorm, dtype):
    """NaN in some experts' router rows: route_ex's choice and gates."""
    L = _layer(16, 64, 96, E, k, 16, 8, dtype, 3)
    for e in experts:
        L["Wg"][e, 0] = float("nan")
    rt = _router(L, adaptive=adaptive, tau=0.6 if adaptive else 0.0)
    _, idx, gate = _few(L, rt, renorm)
    want, wgate = cm.route_ex(L["x"], rt, E, k, renorm=renorm)
    assert torch.equal(idx, want)
    assert _same(gate, wgate, 2e-5)       # route_ex's gates may come from float32 logits


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k", [1, 3, 6])
def test_nan_and_infinite_logits_of_some_tokens(k, dtype):
    """An infinite activation makes infinite logits, and NaN where the router's
    weight is zero; the other tokens stay as they were."""
    L = _layer(16, 64, 96, 6, k, 16, 8, dtype, 3)
    L["Wg"][0, 3] = L["Wg"][4, 3] = 0
    rt = _router(L)
    y0, i0, g0 = _few(L, rt)
    L["x"][2, 3], L["x"][3, 3], L["x"][9] = float("inf"), -float("inf"), float("nan")
    y, idx, gate = _few(L, rt)
    want, wgate = cm.route_ex(L["x"], rt, 6, k)
    assert torch.equal(idx, want) and _same(gate, wgate, 2e-5)
    keep = [t for t in range(16) if t not in (2, 3, 9)]
    assert torch.equal(y[keep], y0[keep]) and torch.equal(gate[keep], g0[keep])
