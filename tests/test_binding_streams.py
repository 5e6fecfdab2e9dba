"""Calls of the binding on a stream that is not the current one, on the CPU:
whatever a call allocates comes from the pool of the stream that it runs on,
and what it hands out is recorded on the current one."""
import contextlib
import types

import pytest
import torch

from paper_2606_28516_amd import clearmoe as cm

BF16 = torch.bfloat16
T, D, H, E, K, R, Q = 6, 32, 64, 4, 2, 8, 8
STREAM = types.SimpleNamespace(cuda_stream=7, device_index=0)


class _Lib:
    """The C entry points: sizes are 4096 bytes, calls succeed."""

    def __getattr__(self, name):
        return lambda *args: 4096 if name.endswith("_bytes") else 0


@pytest.fixture
def log(monkeypatch):
    """Host tensors taken for device tensors; every allocation is noted with
    the stream that was current, and every recorded stream."""
    state = types.SimpleNamespace(inside=False, made=[], recorded=[])

    @contextlib.contextmanager
    def stream(s):
        assert s is STREAM
        state.inside = True
        yield
        state.inside = False

    def noted(make):
        def f(*args, **kw):
            t = make(*args, **{k: v for k, v in kw.items() if k != "device"})
            state.made.append((t, state.inside))
            return t
        return f

    monkeypatch.setattr(cm, "lib", lambda: _Lib())
    monkeypatch.setattr(cm, "_queue", lambda x, s, *a: s.cuda_stream)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: "current")
    monkeypatch.setattr(torch.Tensor, "new_empty", noted(torch.Tensor.new_empty))
    monkeypatch.setattr(torch, "empty", noted(torch.empty))
    monkeypatch.setattr(torch, "empty_like", noted(torch.empty_like))
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda self: True))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, s: state.recorded.append((self.data_ptr(), s)))
    return state


def _z(*shape, dtype=BF16):
    return torch.zeros(*shape, dtype=dtype)


def _layer():
    return [_z(T, D), _z(H, D), None, _z(D, R), _z(R, H), None, _z(E, D, Q), _z(E, Q, H)]


def _bytes(*shape, dtype):
    return torch.zeros(*shape, dtype=torch.uint8).view(dtype)


E4, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
CALLS = {
    "route": lambda: cm.route(_z(T, D), _z(E, D), None, K, stream=STREAM),
    "route_ex": lambda: cm.route_ex(_z(T, D), cm.Router(), E, K, stream=STREAM),
    "dispatch": lambda: cm.dispatch(_z(T, K, dtype=torch.int32), E, x=_z(T, D), stream=STREAM),
    "combine": lambda: cm.combine(_z(T * K, D), _z(T * K, dtype=torch.int32), _z(T, K, dtype=torch.float32),
                                  stream=STREAM),
    "ffn_forward": lambda: cm.ffn_forward(*_layer(), _z(E, D), None, K, stream=STREAM),
    "ffn_forward_padded": lambda: cm.ffn_forward_padded(*_layer(), _z(E, D), None, K, stream=STREAM),
    "ffn_forward_noalloc": lambda: cm.ffn_forward_noalloc(*_layer(), _z(E, D), None, K, stream=STREAM),
    "ffn_forward_ex": lambda: cm.ffn_forward_ex(*_layer(), cm.Router(), K, stream=STREAM),
    "ffn_forward_few": lambda: cm.ffn_forward_few(*_layer(), cm.Router(), K, stream=STREAM),
    "dense_ffn_forward": lambda: cm.dense_ffn_forward(_z(T, D), _z(H, D), None, _z(D, H), None, stream=STREAM),
    "stack_forward": lambda: cm.stack_forward(_z(T, D), [cm.make_stack_layer(_z(H, D), None, None, W2=_z(D, H))], H, E,
                                              R, Q, stream=STREAM),
    "quantize": lambda: cm.quantize(_z(T, D), stream=STREAM),
    "quantized_gemm": lambda: cm.quantized_gemm(_bytes(T, 32, dtype=E4), _bytes(T, 4, dtype=E8),
                                                _bytes(16, 32, dtype=E4), _bytes(1, 4, dtype=E8), out_dtype=E4,
                                                stream=STREAM),
    "quantized_ffn_forward": lambda: cm.quantized_ffn_forward(
        _z(T, D), _bytes(H, 32, dtype=E4), _bytes(1, 4, dtype=E8), None, _bytes(D, 64, dtype=E4),
        _bytes(1, 4, dtype=E8), None, stream=STREAM),
}


@pytest.mark.parametrize("name", CALLS)
def test_memory_of_a_call_on_another_stream(name, log):
    got = CALLS[name]()
    outputs = {t.data_ptr() for t in (got if isinstance(got, tuple) else (got,)) if t is not None}
    made = {t.data_ptr() for t, _ in log.made}
    assert outputs and outputs <= made
    assert all(inside for _, inside in log.made)
    assert {p for p, _ in log.recorded} == outputs and all(s == "current" for _, s in log.recorded)
