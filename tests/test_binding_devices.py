"""The serving calls refuse tensors and streams of different devices before
anything is launched (on the CPU: host tensors taken for device tensors)."""
import types

import pytest
import torch

from paper_2606_28516_amd import clearmoe as cm

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
E4, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
T, D, H, E, K, R, Q = 6, 32, 64, 4, 2, 8, 8


@pytest.fixture
def far(monkeypatch):
    """Tensors whose addresses are in the set are on device 1, others on 0, the
    current one; a call that gets as far as the library fails the test."""
    on_1 = set()

    class Lib:
        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return lambda *a: 4096

            def called(*a):
                raise AssertionError(f"{name} was called")
            return called

    monkeypatch.setattr(cm, "lib", Lib)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0, raising=False)
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda self: True))
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 1 if self.data_ptr() in on_1 else 0)
    return on_1


def _t(*shape, dtype=BF16):
    return torch.zeros(*shape, dtype=torch.uint8).view(dtype) if dtype in (E4, E8) else torch.zeros(*shape, dtype=dtype)


def _few(a, **kw):
    return cm.ffn_forward_few(a["x"], a["W1"], a["b1"], a["US"], a["Vt"], a["b2"], a["P"], a["Q"], cm.Router(), K,
                              ws=a["ws"], out=a["out"], idx_out=a["idx"], gate_out=a["gate"], **kw)


def _gemm(a, **kw):
    return cm.quantized_gemm(a["a"], a["sa"], a["b"], a["sb"], bias=a["bias"], offsets=a["offsets"], out=a["out"], **kw)


def _ffn(a, **kw):
    return cm.quantized_ffn_forward(a["x"], a["W1"], a["s1"], a["b1"], a["W2"], a["s2"], a["b2"], offsets=a["offsets"],
                                    ws=a["ws"], out=a["out"], **kw)


CALLS = {
    "few": (_few, lambda: dict(x=_t(T, D), W1=_t(H, D), b1=_t(H, dtype=F32), US=_t(D, R), Vt=_t(R, H), b2=_t(D, dtype=F32),
                               P=_t(E, D, Q), Q=_t(E, Q, H), ws=_t(4096, dtype=torch.uint8), out=_t(T, D),
                               idx=_t(T, K, dtype=I32), gate=_t(T, K, dtype=F32))),
    "gemm": (_gemm, lambda: dict(a=_t(T, 32, dtype=E4), sa=_t(T, 4, dtype=E8), b=_t(E, 16, 32, dtype=E4),
                                 sb=_t(E, 1, 4, dtype=E8), bias=_t(E, 16, dtype=F32), offsets=_t(E + 1, dtype=I32),
                                 out=_t(T, 16))),
    "ffn": (_ffn, lambda: dict(x=_t(T, D), W1=_t(E, H, 32, dtype=E4), s1=_t(E, 1, 4, dtype=E8), b1=_t(E, H, dtype=F32),
                               W2=_t(E, D, 64, dtype=E4), s2=_t(E, 1, 4, dtype=E8), b2=_t(E, D, dtype=F32),
                               offsets=_t(E + 1, dtype=I32), ws=_t(4096, dtype=torch.uint8), out=_t(T, D))),
    "quantize": (lambda a, **kw: cm.quantize(a["x"], **kw), lambda: dict(x=_t(T, D))),
}


@pytest.mark.parametrize("name", CALLS)
def test_a_tensor_of_another_device(name, far):
    call, make = CALLS[name]
    for which in make():
        a = make()
        far.clear()
        far.add(a[which].data_ptr())
        with pytest.raises(cm.ClearMoEError, match="device"):
            call(a)


@pytest.mark.parametrize("name", CALLS)
def test_tensors_or_a_stream_of_another_device_than_the_current_one(name, far):
    call, make = CALLS[name]
    a = make()
    with pytest.raises(cm.ClearMoEError, match="stream"):
        call(a, stream=types.SimpleNamespace(cuda_stream=7, device_index=1))
    far.update(t.data_ptr() for t in a.values())
    with pytest.raises(cm.ClearMoEError, match="current device"):
        call(a)
