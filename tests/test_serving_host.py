"""Host-only checks of the serving entry points (the layer for a few tokens,
the 8-bit operators): workspace sizes, and bad arguments refused before any
HIP call (the pointers here are never dereferenced)."""
import ctypes

import pytest
import torch

from paper_2606_28516_amd import clearmoe as cm

A = ctypes.c_void_p(0x10000)          # aligned
OK, INVALID, UNSUPPORTED, WORKSPACE, TOO_LARGE = 0, 1, 2, 3, 5


def off(n):
    return ctypes.c_void_p(0x10000 + n)


def _shape(**kw):
    d = dict(T=4, D=64, H=128, E=4, k=2, r=16, q=8, dtype=cm.BF16, renorm=1)
    d.update(kw)
    return cm.make_shape(d["T"], d["D"], d["E"], d["k"], d["dtype"], H=d["H"], r=d["r"], q=d["q"], renorm=d["renorm"])


def _router(**kw):
    d = dict(Wg=0x10000, bg=None, Wh=None, bh=None, W2=None, hidden=0, adaptive=0, dense_stride=0, reserved=0, tau=0.5)
    d.update(kw)
    return cm.Router(*d.values())


def test_few_workspace():
    a = cm.few_workspace_bytes(_shape())
    assert 0 < a < cm.few_workspace_bytes(_shape(T=64)) and a % 256 == 0
    for bad in (dict(T=65), dict(T=-1), dict(D=0), dict(k=5), dict(r=65), dict(dtype=9), dict(renorm=2)):
        assert cm.few_workspace_bytes(_shape(**bad)) == 0, bad
    assert cm.few_workspace_bytes(_shape(D=63, H=101, r=13, q=5)) > 0
    # r + k q beyond the second kernel's LDS
    assert cm.few_workspace_bytes(_shape(D=4096, H=4096, E=8, k=8, q=2048)) == 0
    assert cm.few_workspace_bytes(_shape(D=4096, H=4096, E=8, k=5, q=2048, r=2048)) > 0


def _few(shape=None, router=None, x=A, W1=A, b1=None, US=A, Vt=A, b2=None, P=A, Q=A, y=A, idx=None, gate=None, ws=A,
         n=1 << 40):
    s, r = shape or _shape(), router or _router()
    return cm.lib().clearmoe_ffn_forward_few(ctypes.byref(s), ctypes.byref(r), x, W1, b1, US, Vt, b2, P, Q, y, idx,
                                             gate, ws, n, None)


def test_few_refusals():
    assert _few(x=None) == INVALID
    assert _few(y=None) == INVALID
    assert _few(W1=None) == INVALID
    assert _few(US=None) == INVALID and _few(Vt=None) == INVALID
    assert _few(P=None) == INVALID and _few(Q=None) == INVALID
    for name in ("x", "W1", "US", "Vt", "P", "Q", "y"):
        assert _few(**{name: off(1)}) == INVALID, name
    for name in ("b1", "b2", "idx", "gate"):
        assert _few(**{name: off(2)}) == INVALID, name
    assert _few(ws=None) == WORKSPACE and _few(ws=off(16)) == WORKSPACE and _few(n=100) == WORKSPACE
    assert _few(_shape(T=65)) == TOO_LARGE
    assert _few(_shape(D=4096, H=4096, E=8, k=8, q=2048)) == UNSUPPORTED
    assert _few(_shape(k=5)) == INVALID and _few(_shape(dtype=5)) == UNSUPPORTED
    assert _few(router=_router(Wg=None)) == INVALID
    assert _few(router=_router(Wg=0x10001)) == INVALID
    assert _few(router=_router(dense_stride=2, W2=0x10000)) == UNSUPPORTED
    assert _few(router=_router(dense_stride=-1)) == INVALID
    assert _few(router=_router(hidden=257, Wh=0x10000)) == INVALID
    assert _few(router=_router(hidden=16)) == INVALID                     # no Wh
    assert _few(router=_router(hidden=16, Wh=0x10002)) == INVALID
    assert _few(router=_router(adaptive=1, tau=float("nan"))) == INVALID
    assert _few(_shape(k=1), _router(adaptive=1)) == INVALID
    assert _few(router=_router(reserved=1)) == INVALID
    s = _shape()
    assert cm.lib().clearmoe_ffn_forward_few(ctypes.byref(s), None, A, A, None, A, A, None, A, A, A, None, None, A,
                                             1 << 40, None) == INVALID
    # an MLP router keeps the alignment of clearmoe_route_ex: x as well
    assert _few(router=_router(hidden=16, Wh=0x10000), x=off(2)) == INVALID
    # no tokens: nothing to do, and no token arrays needed
    assert _few(_shape(T=0), x=None, y=None) == OK


def _quantize(dtype=cm.BF16, fmt=2, block_rows=1, batch=1, rows=10, cols=40, x=A, ldx=40, v=A, s=A):
    return cm.lib().clearmoe_quantize(dtype, fmt, block_rows, batch, rows, cols, x, ldx, v, s, None)


def test_quantize_refusals():
    assert _quantize(dtype=2) == UNSUPPORTED and _quantize(fmt=1) == UNSUPPORTED and _quantize(fmt=4) == UNSUPPORTED
    assert _quantize(block_rows=2) == INVALID and _quantize(block_rows=0) == INVALID
    assert _quantize(cols=0) == INVALID and _quantize(cols=65537, ldx=65537) == INVALID
    assert _quantize(ldx=39) == INVALID and _quantize(rows=-1) == INVALID and _quantize(batch=-1) == INVALID
    assert _quantize(x=None) == INVALID and _quantize(v=None) == INVALID and _quantize(s=None) == INVALID
    assert _quantize(x=off(1)) == INVALID and _quantize(v=off(8)) == INVALID and _quantize(s=off(2)) == INVALID
    assert _quantize(dtype=cm.F32, x=off(2)) == INVALID
    # more blocks than a grid holds, without overflow on the way
    assert _quantize(rows=1 << 31) == INVALID and _quantize(rows=1 << 62) == INVALID
    assert _quantize(batch=1 << 62) == INVALID and _quantize(rows=(1 << 31) - 1, batch=(1 << 31) - 1) == INVALID
    assert _quantize(rows=1 << 30, cols=65536, ldx=65536) == INVALID
    assert _quantize(rows=0, x=None, v=None, s=None) == OK and _quantize(batch=0, x=None) == OK


def _product(a=A, sa=A, b=A, sb=A, bias=None, offsets=None, c=A, sc=None, **kw):
    d = dict(M=10, N=40, K=64, groups=0, a_format=2, b_format=3, out=cm.BF16, gelu=0, reserved=0, lda=0, ldc=0)
    d.update(kw)
    p = cm.Product(*d.values())
    return cm.lib().clearmoe_quantized_gemm(ctypes.byref(p), a, sa, b, sb, bias, offsets, c, sc, None)


def test_product_refusals():
    for kw in (dict(M=-1), dict(M=1 << 31), dict(M=(1 << 28) + 1, N=65536), dict(N=0), dict(N=65537), dict(K=0), dict(K=8), dict(K=72), dict(K=65552),
               dict(groups=-1), dict(groups=65), dict(gelu=2), dict(reserved=1), dict(lda=48), dict(lda=72),
               dict(lda=(1 << 22) + 16), dict(ldc=39), dict(ldc=(1 << 22) + 1)):
        extra = dict(offsets=A) if kw.get("groups", 0) > 0 else {}
        assert _product(**kw, **extra) == INVALID, kw
    for kw in (dict(a_format=0), dict(b_format=4), dict(out=4), dict(out=-1)):
        assert _product(**kw) == UNSUPPORTED, kw
    for kw in (dict(a=None), dict(sa=None), dict(b=None), dict(sb=None), dict(c=None), dict(a=off(8)), dict(b=off(8)),
               dict(sa=off(2)), dict(sb=off(1)), dict(bias=off(2)), dict(c=off(1)), dict(out=cm.F32, c=off(2)),
               dict(groups=2), dict(offsets=A), dict(groups=2, offsets=off(2)), dict(out=2), dict(out=2, sc=off(2)),
               dict(out=2, sc=A, c=off(8)), dict(out=3, sc=A, ldc=40)):
        assert _product(**kw) == INVALID, kw
    assert cm.lib().clearmoe_quantized_gemm(None, A, A, A, A, None, None, A, None, None) == INVALID
    assert _product(M=0, a=None, sa=None, c=None) == OK


def _ffn(shape=None, x=A, W1=A, s1=A, b1=None, W2=A, s2=A, b2=None, offsets=None, y=A, ws=A, n=1 << 40):
    s = shape or _shape(k=1, r=0, q=0)
    return cm.lib().clearmoe_quantized_ffn_forward(ctypes.byref(s), x, W1, s1, b1, W2, s2, b2, offsets, y, ws, n, None)


def test_quantized_ffn_refusals():
    for name in ("x", "W1", "s1", "W2", "s2", "y"):
        assert _ffn(**{name: None}) == INVALID, name
    for name, n in (("x", 1), ("y", 1), ("W1", 8), ("W2", 8), ("s1", 2), ("s2", 2), ("b1", 2), ("b2", 2),
                    ("offsets", 2)):
        assert _ffn(**{name: off(n)}) == INVALID, name
    assert _ffn(ws=None) == WORKSPACE and _ffn(ws=off(128)) == WORKSPACE and _ffn(n=64) == WORKSPACE
    assert _ffn(_shape(H=0, k=1, r=0, q=0)) == INVALID and _ffn(_shape(dtype=3, k=1)) == UNSUPPORTED
    assert _ffn(_shape(E=65, k=1)) == INVALID
    assert _ffn(_shape(T=0, k=1, r=0, q=0), x=None, y=None) == OK
    assert cm.quantized_workspace_bytes(_shape(H=0)) == 0
    a, b = (cm.quantized_workspace_bytes(_shape(T=t)) for t in (4, 400))
    assert 0 < a < b and a % 256 == 0


def test_binding_checks_before_the_call():
    """The binding refuses mismatched tensors (host tensors never get past it)."""
    e4, e8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    v, s = torch.zeros(4, 64, dtype=torch.uint8).view(e4), torch.zeros(4, 4, dtype=torch.uint8).view(e8)
    w, t = torch.zeros(8, 64, dtype=torch.uint8).view(e4), torch.zeros(1, 4, dtype=torch.uint8).view(e8)
    with pytest.raises(cm.ClearMoEError, match="not on the GPU"):
        cm.quantized_gemm(v, s, w, t)
    with pytest.raises(cm.ClearMoEError):
        cm.quantized_gemm(v, s, w[:, :32], t)
    with pytest.raises(cm.ClearMoEError):
        cm.quantized_gemm(v, s, w, t, bias=torch.zeros(7))
    with pytest.raises(cm.ClearMoEError):
        cm.quantized_gemm(v, s, w[None], t[None], offsets=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(cm.ClearMoEError, match="unsupported"):
        cm.quantized_gemm(v, s, w, t, out_dtype=torch.float16)
    with pytest.raises(cm.ClearMoEError):
        cm.quantize(torch.zeros(3, 4))
    with pytest.raises(cm.ClearMoEError):
        cm.quantize(torch.zeros(3))
    with pytest.raises(cm.ClearMoEError, match="weights"):
        cm.quantized_ffn_forward(torch.zeros(3, 48), w, t, None, w, t, None)
