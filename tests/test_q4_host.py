"""The 4-bit operators and the norm refuse bad arguments before anything is
launched (on the CPU: no call here reaches the GPU)."""
import ctypes
import math

import pytest
import torch

from paper_2606_28516_amd import clearmoe as cm
from tests.test_binding_devices import far  # noqa: F401 (a fixture)
from tests.test_serving_host import A, INVALID, OK, UNSUPPORTED, WORKSPACE, _shape, off

E4, E2, E8 = torch.float8_e4m3fn, torch.float4_e2m1fn_x2, torch.float8_e8m0fnu
FOUR = 5                                          # CLEARMOE_E2M1


def _quantize(dtype=cm.BF16, block_rows=1, batch=1, rows=10, cols=40, x=A, ldx=40, v=A, s=A):
    return cm.lib().clearmoe_quantize(dtype, FOUR, block_rows, batch, rows, cols, x, ldx, v, s, None)


def _dequantize(fmt=FOUR, block_rows=1, batch=1, rows=10, cols=40, v=A, s=A, dtype=cm.BF16, y=A, ldy=40):
    return cm.lib().clearmoe_dequantize(fmt, block_rows, batch, rows, cols, v, s, dtype, y, ldy, None)


def test_quantize_refusals():
    assert _quantize(block_rows=128) == INVALID and _quantize(block_rows=32) == INVALID
    assert _quantize(dtype=2) == UNSUPPORTED
    assert _quantize(cols=0) == INVALID and _quantize(cols=65537, ldx=65537) == INVALID and _quantize(ldx=39) == INVALID
    assert _quantize(x=None) == INVALID and _quantize(v=None) == INVALID and _quantize(s=None) == INVALID
    assert _quantize(x=off(1)) == INVALID and _quantize(v=off(8)) == INVALID and _quantize(s=off(2)) == INVALID
    # at most 2^31 blocks of 32
    assert _quantize(rows=(1 << 20) + 1, cols=65536, ldx=65536) == INVALID
    assert _quantize(rows=(1 << 31) - 1, batch=(1 << 31) - 1) == INVALID
    assert _quantize(rows=0, x=None, v=None, s=None) == OK and _quantize(batch=0, x=None) == OK


def test_dequantize_refusals():
    for fmt in (-1, 0, 1, 4, 6):
        assert _dequantize(fmt=fmt) == UNSUPPORTED, fmt
    assert _dequantize(dtype=2) == UNSUPPORTED and _dequantize(dtype=FOUR) == UNSUPPORTED
    assert _dequantize(block_rows=128) == INVALID and _dequantize(fmt=2, block_rows=64) == INVALID
    assert _dequantize(cols=0) == INVALID and _dequantize(cols=65537, ldy=65537) == INVALID and _dequantize(ldy=39) == INVALID
    assert _dequantize(rows=-1) == INVALID and _dequantize(batch=-1) == INVALID and _dequantize(ldy=1 << 41) == INVALID
    assert _dequantize(rows=(1 << 20) + 1, cols=65536, ldy=65536) == INVALID
    for name in ("v", "s", "y"):
        assert _dequantize(**{name: None}) == INVALID, name
    assert _dequantize(v=off(8)) == INVALID and _dequantize(s=off(2)) == INVALID and _dequantize(y=off(1)) == INVALID
    assert _dequantize(dtype=cm.F32, y=off(2)) == INVALID
    assert _dequantize(rows=0, v=None, s=None, y=None) == OK


def _product(a=A, sa=A, b=A, sb=A, bias=None, offsets=None, c=A, sc=None, **kw):
    d = dict(M=10, N=40, K=64, groups=0, a_format=2, b_format=FOUR, out=cm.BF16, gelu=0, reserved=0, lda=0, ldc=0)
    d.update(kw)
    p = cm.Product(*d.values())
    return cm.lib().clearmoe_quantized_gemm(ctypes.byref(p), a, sa, b, sb, bias, offsets, c, sc, None)


def test_product_refusals():
    for kw in (dict(M=-1), dict(M=1 << 31), dict(M=(1 << 28) + 1, N=65536), dict(N=0), dict(N=65537), dict(K=0), dict(K=8),
               dict(K=72), dict(K=65552), dict(a_format=FOUR, K=16), dict(a_format=FOUR, K=80), dict(a_format=FOUR, K=65568),
               dict(a_format=FOUR, lda=80), dict(groups=-1), dict(groups=65), dict(gelu=2), dict(reserved=1), dict(lda=48),
               dict(lda=72), dict(lda=(1 << 22) + 16), dict(ldc=39), dict(ldc=(1 << 22) + 1)):
        extra = dict(offsets=A) if kw.get("groups", 0) > 0 else {}
        assert _product(**kw, **extra) == INVALID, kw
    for kw in (dict(a_format=3), dict(a_format=0), dict(a_format=4), dict(out=3), dict(out=4), dict(out=-1),
               dict(a_format=FOUR, b_format=2), dict(a_format=FOUR, b_format=3), dict(b_format=2, out=FOUR)):
        assert _product(**kw) == UNSUPPORTED, kw
    for kw in (dict(a=None), dict(sa=None), dict(b=None), dict(sb=None), dict(c=None), dict(a=off(8)), dict(b=off(8)),
               dict(sa=off(2)), dict(sb=off(1)), dict(bias=off(2)), dict(c=off(1)), dict(out=cm.F32, c=off(2)),
               dict(groups=2), dict(offsets=A), dict(groups=2, offsets=off(2)), dict(out=2), dict(out=2, sc=off(2)),
               dict(out=2, sc=A, c=off(8)), dict(out=FOUR, sc=A, c=off(8)), dict(out=FOUR), dict(out=FOUR, sc=A, ldc=48)):
        assert _product(**kw) == INVALID, kw
    assert _product(M=0, a=None, sa=None, c=None) == OK


def _ffn(act=2, wt=FOUR, x=A, W1=A, s1=A, b1=None, W2=A, s2=A, b2=None, offsets=None, y=A, ws=A, n=1 << 40, **kw):
    s = _shape(k=1, r=0, q=0, **kw)
    return cm.lib().clearmoe_quantized_ffn_forward_ex(ctypes.byref(s), act, wt, x, W1, s1, b1, W2, s2, b2, offsets, y,
                                                      ws, n, None)


def test_ffn_refusals():
    for act, wt in ((3, FOUR), (2, 3), (FOUR, 2), (3, 2), (0, FOUR), (4, FOUR), (2, 4), (2, 0)):
        assert _ffn(act, wt) == UNSUPPORTED, (act, wt)
    for act in (2, FOUR):
        for name in ("x", "W1", "s1", "W2", "s2", "y"):
            assert _ffn(act, **{name: None}) == INVALID, name
        for name, n in (("x", 1), ("y", 1), ("W1", 8), ("W2", 8), ("s1", 2), ("s2", 2), ("b1", 2), ("b2", 2), ("offsets", 2)):
            assert _ffn(act, **{name: off(n)}) == INVALID, name
        assert _ffn(act, ws=None) == WORKSPACE and _ffn(act, ws=off(128)) == WORKSPACE and _ffn(act, n=64) == WORKSPACE
        assert _ffn(act, H=0) == INVALID and _ffn(act, E=65) == INVALID
        assert _ffn(act, T=0, x=None, y=None) == OK


def test_one_workspace_for_both_kinds_of_activations():
    """It holds 4-bit values and scales of any width, each part at its own 256
    bytes."""
    up = lambda n, m: -(-n // m) * m
    for T in (17, 100, 1001):
        for D, H in ((1, 1), (8, 8), (33, 65), (100, 390), (768, 1536), (8, 65536)):
            have = cm.quantized_workspace_bytes(cm.make_shape(T, D, 1, 1, cm.BF16, H=H))
            for width, per in ((32, 16), (128, 128)):
                parts = [n for w in (D, H) for n in (-(-w // 32) * 16 if width == 32 else up(w, 16), up(-(-w // width), 4))]
                assert have >= sum(up(T * n, 256) for n in parts), (T, D, H, width)


def _norm(x=A, residual=None, weight=None, y=A, ys=None, total=None, **kw):
    d = dict(rows=10, cols=40, dtype=cm.BF16, out=cm.BF16, eps=1e-6, ldx=0, ldr=0, lds=0, ldy=0)
    d.update(kw)
    p = cm.Norm(*d.values())
    return cm.lib().clearmoe_rms_norm(ctypes.byref(p), x, residual, weight, y, ys, total, None)


def test_norm_refusals():
    for kw in (dict(dtype=2), dict(dtype=-1), dict(out=cm.F32), dict(out=4), dict(out=FOUR), dict(dtype=cm.F32)):
        assert _norm(**kw) == UNSUPPORTED, kw
    for kw in (dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=65537), dict(eps=0.0), dict(eps=-1e-6),
               dict(eps=1e-39), dict(eps=math.nan), dict(eps=math.inf), dict(ldx=39), dict(ldr=39), dict(lds=39),
               dict(ldy=39), dict(ldx=(1 << 31) + 1), dict(ldy=(1 << 31) + 1), dict(ldx=-40), dict(out=2, ys=A, ldy=47),
               dict(out=2, ys=A, ldy=56), dict(x=None), dict(y=None), dict(out=2), dict(x=off(1)), dict(residual=off(1)),
               dict(total=off(1)), dict(y=off(1)), dict(weight=off(2)), dict(out=2, ys=off(2)),
               dict(out=2, ys=A, y=off(8)), dict(dtype=cm.F32, out=cm.F32, x=off(2))):
        assert _norm(**kw) == INVALID, kw
    assert cm.lib().clearmoe_rms_norm(None, A, None, None, A, None, None, None) == INVALID
    assert _norm(rows=0, x=None, y=None) == OK


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=torch.uint8).view(dtype) if dtype in (E4, E2, E8) else torch.zeros(*shape, dtype=dtype)


def test_binding_checks_before_the_call():
    """Mismatched tensors are refused, and host tensors never get past it."""
    v, s, w, t = _t(4, 64, dtype=E4), _t(4, 4, dtype=E8), _t(8, 32, dtype=E2), _t(8, 4, dtype=E8)
    v4, s4 = _t(4, 32, dtype=E2), _t(4, 4, dtype=E8)
    for a, sa in ((v, s), (v4, s4)):
        with pytest.raises(cm.ClearMoEError, match="not on the GPU"):
            cm.quantized_gemm(a, sa, w, t)
    with pytest.raises(cm.ClearMoEError, match="b must be"):
        cm.quantized_gemm(v, s, _t(8, 16, dtype=E2), t)
    with pytest.raises(cm.ClearMoEError, match="b must be"):
        cm.quantized_gemm(v4, s4, _t(8, 32, dtype=E4), t)
    with pytest.raises(cm.ClearMoEError):
        cm.quantized_gemm(v, s, w, _t(1, 4, dtype=E8))
    with pytest.raises(cm.ClearMoEError, match="weights"):
        cm.quantized_ffn_forward(torch.zeros(3, 48), w, t, None, w, t, None)
    for call in (lambda: cm.quantize(torch.zeros(3, 4), E2), lambda: cm.dequantize(v4, s4, 64), lambda: cm.rms_norm(torch.zeros(3, 4))):
        with pytest.raises(cm.ClearMoEError, match="not on the GPU"):
            call()
    for call in (lambda: cm.dequantize(v4[0], s4[0]), lambda: cm.dequantize(v4, s4, 63 + 32), lambda: cm.dequantize(v4, s4, 64, dtype=torch.half),
                 lambda: cm.dequantize(torch.zeros(4, 32), s4), lambda: cm.rms_norm(torch.zeros(3)), lambda: cm.rms_norm(torch.zeros(3, 4).half()),
                 lambda: cm.rms_norm(torch.zeros(3, 4), out_dtype=torch.bfloat16), lambda: cm.quantize(torch.zeros(3, 4), torch.int8)):
        with pytest.raises(cm.ClearMoEError):
            call()


T, D, H, E = 6, 32, 64, 4
CALLS = {
    "gemm": (lambda a, **kw: cm.quantized_gemm(a["a"], a["sa"], a["b"], a["sb"], bias=a["bias"], offsets=a["offsets"], out=a["out"], **kw),
             lambda: dict(a=_t(T, 16, dtype=E2), sa=_t(T, 4, dtype=E8), b=_t(E, 16, 16, dtype=E2), sb=_t(E, 16, 4, dtype=E8),
                          bias=_t(E, 16, dtype=torch.float32), offsets=_t(E + 1, dtype=torch.int32), out=_t(T, 16))),
    "ffn": (lambda a, **kw: cm.quantized_ffn_forward(a["x"], a["W1"], a["s1"], a["b1"], a["W2"], a["s2"], a["b2"], ws=a["ws"], out=a["out"],
                                                     activations=E2, **kw),
            lambda: dict(x=_t(T, D), W1=_t(H, 16, dtype=E2), s1=_t(H, 4, dtype=E8), b1=_t(H, dtype=torch.float32), W2=_t(D, 32, dtype=E2),
                         s2=_t(D, 4, dtype=E8), b2=_t(D, dtype=torch.float32), ws=_t(4096, dtype=torch.uint8), out=_t(T, D))),
    "dequantize": (lambda a, **kw: cm.dequantize(a["v"], a["s"], 32, out=a["out"], **kw),
                   lambda: dict(v=_t(T, 16, dtype=E2), s=_t(T, 4, dtype=E8), out=_t(T, 32))),
    "norm": (lambda a, **kw: cm.rms_norm(a["x"], a["w"], residual=a["r"], sum_out=a["sum"], out=a["out"], **kw),
             lambda: dict(x=_t(T, D), w=_t(D, dtype=torch.float32), r=_t(T, D), sum=_t(T, D), out=_t(T, D))),
}


@pytest.mark.parametrize("name", CALLS)
def test_tensors_and_streams_of_another_device_are_refused(name, far):  # noqa: F811
    import types
    call, make = CALLS[name]
    args = make()
    for n, t in args.items():
        far.clear()
        far.add(t.data_ptr())
        with pytest.raises(cm.ClearMoEError):
            call(args)
    far.clear()
    with pytest.raises(cm.ClearMoEError):
        call(args, stream=types.SimpleNamespace(device_index=1, cuda_stream=5))
    with pytest.raises(AssertionError, match="was called"):
        call(args)
