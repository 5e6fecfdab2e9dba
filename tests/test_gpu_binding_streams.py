"""Calls on a stream that is not the current one and is busy, with workspaces
of their own: work that the current stream does meanwhile, in memory of the same
sizes, does not touch them."""
import pytest
import torch

from paper_2606_28516_amd import clearmoe as cm
from tests.test_gpu_few import _layer, _router
from tests.test_gpu_q8 import _ffn_inputs

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def _ffn(T):
    x, W1, b1, W2, b2 = _ffn_inputs(T, 192, 768, 0, BF16, 3)
    w1, s1 = cm.quantize(W1.cuda(), block_rows=128)
    w2, s2 = cm.quantize(W2.cuda(), block_rows=128)
    x, b1, b2 = x.cuda(), b1.cuda(), b2.cuda()
    n = cm.quantized_workspace_bytes(cm.make_shape(T, 192, 1, 1, cm.BF16, H=768))
    return lambda **kw: cm.quantized_ffn_forward(x, w1, s1, b1, w2, s2, b2, **kw), n


def _few(T):
    L = _layer(T, 192, 768, 8, 2, 64, 16, BF16, 4)
    rt = _router(L)
    n = cm.few_workspace_bytes(cm.make_shape(T, 192, 8, 2, cm.BF16, H=768, r=64, q=16))
    return lambda **kw: cm.ffn_forward_few(L["x"], L["W1"], L["b1"], L["US"], L["Vt"], L["b2"], L["P"], L["Q"], rt, 2,
                                           **kw), n


def _full(T):
    L = _layer(T, 192, 768, 8, 2, 64, 16, BF16, 4)
    rt = _router(L)
    n = cm.workspace_bytes(cm.make_shape(T, 192, 8, 2, cm.BF16, H=768, r=64, q=16))
    return lambda **kw: cm.ffn_forward_ex(L["x"], L["W1"], L["b1"], L["US"], L["Vt"], L["b2"], L["P"], L["Q"], rt, 2,
                                          **kw), n


def _product(T):
    g = torch.Generator().manual_seed(5)
    a, sa = cm.quantize(torch.randn(T, 384, generator=g).cuda())
    b, sb = cm.quantize(torch.randn(400, 384, generator=g).cuda(), block_rows=128)
    return lambda **kw: cm.quantized_gemm(a, sa, b, sb, **kw), T * 800


@pytest.mark.parametrize("make,T", [(_few, 1), (_few, 16), (_full, 300), (_ffn, 5), (_ffn, 700), (_product, 300)])
def test_a_call_on_a_busy_stream(make, T):
    call, n = make(T)
    want = call()
    side = torch.cuda.Stream()
    work = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(side):
            for _ in range(8):
                busy = work @ work
        y = call(stream=side)
        other = [torch.full((n,), 0xff, dtype=torch.uint8, device="cuda") for _ in range(20)]
        other += [torch.full_like(want, float("nan")) for _ in range(20)]
        side.synchronize()
        assert torch.equal(y, want)
        torch.cuda.synchronize()
        del y, other, busy


def test_a_forked_stream_of_a_capture():
    """Two calls side by side in one captured graph, one of them on a stream
    that joins the capture, without workspaces of the caller's."""
    x, W1, b1, W2, b2 = _ffn_inputs(40, 192, 768, 0, BF16, 3)
    w1, s1 = cm.quantize(W1.cuda(), block_rows=128)
    w2, s2 = cm.quantize(W2.cuda(), block_rows=128)
    x, b1, b2 = x.cuda(), b1.cuda(), b2.cuda()
    call = lambda **kw: cm.quantized_ffn_forward(x, w1, s1, b1, w2, s2, b2, **kw)
    side, stream, graph = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    call(), call(stream=side)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        side.wait_stream(stream)
        there, here = call(stream=side), call()
        values, _ = cm.quantize(x, stream=side)
        stream.wait_stream(side)
        both = there + here
    g = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(4):
        x.copy_(torch.randn(x.shape, device="cuda", generator=g))
        want, bytes_ = call(), cm.quantize(x)[0].view(torch.uint8)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(there, want) and torch.equal(here, want) and torch.equal(both, want + want)
        assert torch.equal(values.view(torch.uint8), bytes_)


def test_an_mlp_router_captured():
    L = _layer(9, 384, 520, 8, 2, 64, 16, BF16, 1, mlp=64)
    rt = _router(L)
    ws = cm.alloc_few_workspace(cm.make_shape(9, 384, 8, 2, cm.BF16, H=520, r=64, q=16))
    call = lambda: cm.ffn_forward_few(L["x"], L["W1"], L["b1"], L["US"], L["Vt"], L["b2"], L["P"], L["Q"], rt, 2, ws=ws)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    call()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        got = call()
    g = torch.Generator(device="cuda").manual_seed(2)
    for _ in range(4):
        L["x"].copy_(torch.randn(9, 384, device="cuda", generator=g))
        want = call()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
