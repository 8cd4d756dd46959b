"""The layer's backward pass and the calls around it do all of their work on the caller's stream: captured, each is a chain of
nodes, without a fork."""
import pytest
import torch
from cuda.bindings import runtime

import test_gpu_dropout as drop
import test_gpu_head as head
import test_gpu_layer_norm as norm
from paper_2605_08527_b200 import binding as B

pytestmark = pytest.mark.gpu


def assert_chain(call):
    """Captures the call, which is not replayed."""
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.stream(st), torch.cuda.graph(g, stream=st):
        call()
    raw = runtime.cudaGraph_t(g.raw_cuda_graph())
    err, _, nodes = runtime.cudaGraphGetNodes(raw)
    assert err == runtime.cudaError_t.cudaSuccess
    err, _, _, _, edges = runtime.cudaGraphGetEdges_v2(raw)
    assert err == runtime.cudaError_t.cudaSuccess
    err, begin, end, _, edges = runtime.cudaGraphGetEdges_v2(raw, edges)
    assert err == runtime.cudaError_t.cudaSuccess
    begin, end = ([int(n) for n in ns[:edges]] for ns in (begin, end))
    assert nodes > 1 and edges == nodes - 1
    assert len(set(begin)) == edges and len(set(end)) == edges


@pytest.mark.parametrize("saved", [True, False])
@pytest.mark.parametrize("T,parts", [(300, None), (1300, None), (1300, [512, 256])])
def test_backward(T, parts, saved):
    c = drop.Case(T, 256, sum(parts or [384]), [8, 16, 24], 9, 1, parts=parts)
    h = torch.empty((len(c.parts), T, c.pool.rank_stride), device="cuda")
    B.marlaas_lora_forward(c.pool, c.x, c.W, c.seg, h_save=h)
    dx, (dA, dB) = torch.empty_like(c.x), c.grads()
    B.marlaas_lora_backward(c.pool, c.x, c.W, c.dy, c.seg, dx=dx)         # (the first workspace is made outside)
    assert_chain(lambda: B.marlaas_lora_backward(c.pool, c.x, c.W, c.dy, c.seg, dx=dx, dA=dA, dB=dB, h_saved=h if saved else None))


@pytest.mark.parametrize("T,parts", [(300, None), (1300, None), (1300, [512, 256])])
def test_backward_with_dropout(T, parts):
    c = drop.Case(T, 256, sum(parts or [384]), [8, 16, 24], 9, 1, parts=parts)
    _, h = c.forward()
    c.backward(h)
    assert_chain(lambda: B.marlaas_lora_backward_dropout(c.pool, c.x, c.W, c.dy, c.seg, c.rates_dev, 1, dx=torch.empty_like(c.x), dA=c.grads()[0],
                                                         dB=c.grads()[1], h_saved=h))


def test_head_and_norm():
    pool = B.AdapterPool(64, 64, 8, head.CAP)
    x, W, tgt, w, off, slot = head.inputs(300, 256, 1000, 1)
    dx = torch.empty_like(x)
    seg = head.segments(off, slot)
    call = lambda: B.marlaas_head_cross_entropy(pool, x, W, tgt, seg, weight=w, dx=dx)         # noqa: E731
    call()
    assert_chain(call)
    pool = B.AdapterPool(64, 64, 8, norm.CAP)
    gain, bias = norm.params(256, 1)
    seg = norm.segments(off, slot)
    _, mean, rstd = B.marlaas_layer_norm(pool, x, seg, gain, bias)
    dgain = torch.empty_like(gain)
    call = lambda: B.marlaas_layer_norm_backward(pool, x, x, seg, gain, mean, rstd, dx=dx, dgain=dgain)         # noqa: E731
    call()
    assert_chain(call)
