"""The serving calls at the sizes where their kernels change or end: the most
columns of the few-token layer's sums, the most that the FFN of few rows
quantises in each workgroup."""
import pytest
import torch

from paper_2606_28516_amd import clearmoe as cm
from tests.q8_util import dequantize
from tests.test_gpu_few import _check as _check_few
from tests.test_gpu_few import _layer, _router
from tests.test_gpu_q8 import CUT, FLIPS, _ffn_inputs, _ffn_reference

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,D,H,E,k,r,q", [(2, 4096, 4096, 3, 2, 4096, 4096), (3, 200, 264, 64, 64, 192, 189),
                                           (1, 40, 65536, 2, 1, 40, 8), (2, 65536, 40, 3, 2, 8, 8)])
def test_few_tokens(T, D, H, E, k, r, q, dtype):
    L = _layer(T, D, H, E, k, r, q, dtype, 2)
    _check_few(L, _router(L))


def test_few_tokens_past_the_limit():
    L = _layer(1, 4096, 4096, 4, 3, 8, 4096, BF16, 2)
    with pytest.raises(cm.ClearMoEError):
        cm.ffn_forward_few(L["x"], L["W1"], L["b1"], L["US"], L["Vt"], L["b2"], L["P"], L["Q"], _router(L), 3)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,D,H", [(16, 2944, 72), (16, 2945, 72), (1, 48768, 40), (1, 48769, 40), (2, 65536, 40),
                                   (1, 40, 48768), (3, 40, 65536)])
def test_ffn_of_few_rows(T, D, H, dtype):
    x, W1, b1, W2, b2 = _ffn_inputs(T, D, H, 0, dtype, T + D)
    w1, s1 = cm.quantize(W1.cuda(), block_rows=128)
    w2, s2 = cm.quantize(W2.cuda(), block_rows=128)
    y = cm.quantized_ffn_forward(x.cuda(), w1, s1, b1.cuda(), w2, s2, b2.cuda()).cpu().double()
    half = torch.finfo(dtype).eps / 2
    ref, coarse, fine = _ffn_reference(x, dequantize(w1, s1, 128), b1.double(), dequantize(w2, s2, 128), b2.double(),
                                       D, H, half)
    assert ((y - ref).abs() <= coarse).all()
    assert (y - fine).norm() <= (half + CUT + FLIPS) * fine.norm()
