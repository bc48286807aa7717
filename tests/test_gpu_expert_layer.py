"""The example's layer: forward and gradients against automatic differentiation
of the layer's definition in 64 bits, the 4-bit form against its own decoded
weights, and the command as a whole.

Tolerances, fixed before the first run.  FP32: every product is within 1e-5 of
its absolute sums; through two products, the activation and the sums over
experts a 2-norm error of 1e-5 of each result leaves room.  BF16: five
roundings to 8 bits on the longest way (2^-8 each, adding in the 2-norm at most
linearly): 2e-2."""
import importlib.util
import os

import pytest

import paper_2609_04663_gb300 as emu
from helpers import device

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "expert_layer.py")


@pytest.fixture(scope="module")
def ex():
    device()
    spec = importlib.util.spec_from_file_location("expert_layer", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def rel(a, b):
    return float((a.double() - b).norm() / b.norm())


@pytest.mark.parametrize("dtype,tol", [("float32", 1e-5), ("bfloat16", 2e-2)])
def test_layer_and_gradients(ex, dtype, tol):
    import torch
    dt = getattr(torch, dtype)
    layer = ex.ExpertLayer(72, 136, 6, 2, dt)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(50, 72, generator=g, device="cuda").to(dt)
    dout = torch.randn(50, 72, generator=g, device="cuda").to(dt)
    out = layer.forward(x)
    got = layer.backward(dout)
    chosen = layer.saved[2].experts.long()                      # a rounded logit must not change the choice
    X, R, W1, W2 = (t.double().requires_grad_() for t in (x, layer.router, layer.W1, layer.W2))
    w = torch.softmax((X @ R).gather(1, chosen), 1)
    h = torch.einsum("td,tkdh->tkh", X, W1[chosen])
    y = torch.einsum("tkh,tkhd->tkd", h * torch.sigmoid(h), W2[chosen])
    want = (w[..., None] * y).sum(1)
    want.backward(dout.double())
    assert out.dtype == dt and rel(out, want.detach()) <= tol
    for a, b in zip(got, (X.grad, R.grad, W1.grad, W2.grad)):
        assert rel(a, b) <= tol


def test_quantized_experts(ex):
    import torch
    layer = ex.ExpertLayer(128, 256, 5, 2, torch.float32)
    served = ex.QuantizedExperts(layer, group=64)
    g = torch.Generator(device="cuda").manual_seed(4)
    for tokens in (1, 3):
        x = torch.randn(tokens, 128, generator=g, device="cuda")
        out = served.forward(x)

        def decoded(q, s, z):
            c = torch.stack((q & 15, q >> 4), -1).flatten(-2).double().unflatten(-1, (-1, 64))
            return ((c - z.double()[..., None]) * s.double()[..., None]).flatten(-2).transpose(1, 2)
        W1, W2 = decoded(*served.first), decoded(*served.second)
        assert float((W1 - layer.W1.double()).abs().max()) <= float(served.first[1].max()) * 0.76
        logits, _ = emu.gemm_f32(x, layer.router)
        r, _ = emu.route(logits, 2)
        ch = r.experts.long()
        h = torch.einsum("td,tkdh->tkh", x.double(), W1[ch])
        want = (r.weights.double()[..., None] * torch.einsum("tkh,tkhd->tkd", h * torch.sigmoid(h), W2[ch])).sum(1)
        assert rel(out, want) <= 1e-5


@pytest.mark.parametrize("served", [False, True])
def test_in_a_cuda_graph(ex, served):
    """The layer captured once and replayed on other tokens: the call's own results, bit for bit."""
    import torch
    layer = ex.ExpertLayer(128, 256, 5, 2, torch.bfloat16)
    if served:
        layer = ex.QuantizedExperts(layer, group=64)
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(6, 128, generator=g, device="cuda").bfloat16()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        layer.forward(x)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer.forward(x)
    for _ in range(3):
        x.normal_(generator=g)
        graph.replay()
        got = out.clone()
        assert torch.equal(got, layer.forward(x)) and bool(got.any())


def test_command(ex):
    losses, off = ex.main(["--tokens", "256", "--width", "128", "--hidden", "256", "--experts", "4", "--steps", "8"])
    assert losses[-1] < losses[0] and max(off) < 0.5
