"""The example's layer with a balance loss against automatic differentiation in 64
bits, and its 8-bit form within what quantisation can do.

Tolerances, fixed before the first run.  The gradients: those of the layer without a
balance loss, whose products are within 1e-5 of their absolute sums (FP32) or go through five
roundings to 8 bits (BF16); the balance loss's own part is in FP32.  The 8-bit form: a
value is off by at most half its row's scale, so an answer by the products' sum of such
differences, computed below entry by entry; 1e-4 of the absolute sums is left for the roundings of FP32
and 2^-7 for two of BF16 results."""
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


@pytest.mark.parametrize("dtype,tol", [("float32", 1e-5), ("bfloat16", 2e-2)])
@pytest.mark.parametrize("masked", [False, True])
def test_gradients_with_a_balance_loss(ex, dtype, tol, masked):
    import torch
    dt = getattr(torch, dtype)
    layer = ex.ExpertLayer(72, 136, 6, 2, dt, balance=3.0)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(50, 72, generator=g, device="cuda").to(dt)
    dout = torch.randn(50, 72, generator=g, device="cuda").to(dt)
    mask = torch.rand(50, generator=g, device="cuda") < 0.7 if masked else None
    layer.forward(x, mask=mask)
    got = layer.backward(dout)
    chosen = layer.saved[2].experts.long()
    X, R, W1, W2 = (t.double().requires_grad_() for t in (x, layer.router, layer.W1, layer.W2))
    w = torch.softmax((X @ R).gather(1, chosen), 1)
    h = torch.einsum("td,tkdh->tkh", X, W1[chosen])
    y = torch.einsum("tkh,tkhd->tkd", h * torch.sigmoid(h), W2[chosen])
    on = torch.ones(50, dtype=torch.bool, device="cuda") if mask is None else mask
    n = int(on.sum())
    counts = torch.bincount(chosen[on].reshape(-1), minlength=6).double()
    loss = 3.0 * 6 / (n * 2) * (counts * torch.softmax(X @ R, 1)[on].mean(0)).sum()
    ((w[..., None] * y).sum(1) * dout.double()).sum().add(loss).backward()
    assert torch.equal(layer.load.counts.double(), counts)
    assert abs(float(layer.load.loss) - loss.item()) <= 1e-4 * loss.item()      # (the logits are within 1e-5 of their sums)
    for a, b in zip(got, (X.grad, R.grad, W1.grad, W2.grad)):
        assert float((a.double() - b).norm() / b.norm()) <= tol


@pytest.mark.parametrize("dtype,extra", [("float32", 1e-4), ("bfloat16", 2.0 ** -7)])
@pytest.mark.parametrize("tokens", [1, 5, 300])
def test_eight_bit_experts(ex, dtype, extra, tokens):
    import torch
    dt = getattr(torch, dtype)
    layer = ex.ExpertLayer(128, 272, 6, 2, dt)
    served = ex.EightBitExperts(layer)
    x = torch.randn(tokens, 128, generator=torch.Generator(device="cuda").manual_seed(tokens), device="cuda").to(dt)
    out = served.forward(x)
    assert out.dtype is dt and out.shape == x.shape
    logits, _ = emu.gemm_f32(x.float(), layer.router)
    r, _ = emu.route(logits, 2)
    ch, wt = r.experts.long(), r.weights.double()[..., None]

    def product(a, da, W, s):
        """(value, bound of the difference) of a W with a off by da at most, quantised on the way."""
        W, half = W.double()[ch], s.double()[ch][:, :, None] / 2           # [t, k, in, out], [t, k, 1, out]
        q = da + (a.abs() + da).amax(-1, keepdim=True) / 254
        v = torch.einsum("tki,tkio->tko", a, W)
        off = torch.einsum("tki,tkio->tko", q, W.abs() + half) + (a.abs().sum(-1, keepdim=True) * half[:, :, 0])
        return v, off + extra * torch.einsum("tki,tkio->tko", a.abs(), W.abs())
    a = x.double()[:, None].expand(-1, 2, -1)
    h, dh = product(a, torch.zeros_like(a), layer.W1, served.first.scales)
    act = h * torch.sigmoid(h)
    y, dy = product(act, 1.1 * dh + extra * act.abs(), layer.W2, served.second.scales)      # |silu'| < 1.1
    want, room = (wt * y).sum(1), (wt * dy).sum(1) + extra * (wt * y.abs()).sum(1)
    assert bool(((out.double() - want).abs() <= room).all())


def test_eight_bit_experts_in_a_graph(ex):
    import torch
    served = ex.EightBitExperts(ex.ExpertLayer(128, 256, 5, 2, torch.bfloat16))
    g = torch.Generator(device="cuda").manual_seed(5)
    for tokens in (4, 90):
        x = torch.randn(tokens, 128, generator=g, device="cuda").bfloat16()
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            served.forward(x)
        torch.cuda.current_stream().wait_stream(stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = served.forward(x)
        for _ in range(3):
            x.normal_(generator=g)
            graph.replay()
            got = out.clone()
            assert torch.equal(got, served.forward(x)) and bool(got.any())


def test_command(ex, capsys):
    losses, off = ex.main(["--tokens", "256", "--width", "128", "--hidden", "256", "--experts", "4", "--steps", "3", "--balance", "0.01"])
    said = capsys.readouterr().out
    assert len(losses) == 3 and "8-bit" in said and "balance loss" in said
