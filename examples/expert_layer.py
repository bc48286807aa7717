"""A mixture-of-experts layer on the package's expert-layer operators.

Training: ``ExpertLayer.forward`` and ``.backward`` route tokens to experts,
run both matrices of every expert on its tokens in one call each, and add the
answers up; the gradients come from the same operators.  Serving:
``QuantizedExperts`` holds the experts with 4-bit weights and answers a few
tokens, reading each chosen expert's weights once.

    python examples/expert_layer.py [--tokens 4096] [--dtype bf16|f32] [--steps 20]

fits a layer to a random target for a few steps, prints the loss, then decodes
single tokens with the 4-bit experts and prints how far they are from the
unquantised layer.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_04663_gb300 as emu  # noqa: E402


def silu(h):
    return h * torch.sigmoid(h)


def silu_grad(h):
    s = torch.sigmoid(h)
    return s * (1 + h * (1 - s))


class ExpertLayer:
    """out[t] = sum over t's k experts of weight * silu(x[t] W1_e) W2_e."""

    def __init__(self, width, hidden, experts, k, dtype=torch.bfloat16, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.k = k
        self.router = torch.randn(width, experts, generator=g, device=device) / width ** 0.5
        self.W1 = (torch.randn(experts, width, hidden, generator=g, device=device) / width ** 0.5).to(dtype)
        self.W2 = (torch.randn(experts, hidden, width, generator=g, device=device) / hidden ** 0.5).to(dtype)

    def forward(self, x):
        logits, _ = emu.gemm_f32(x.float(), self.router)
        r, _ = emu.route(logits, self.k)
        h, _ = emu.grouped_gemm(x, self.W1, r.ends, src=r.rows)      # each expert's tokens, gathered
        a = silu(h)
        y, _ = emu.grouped_gemm(a, self.W2, r.ends)
        self.saved = (x, logits, r, h, a, y)
        return emu.rows_combine(y, r.slots, r.weights)

    def backward(self, dout):
        """Gradients (dx, router, W1, W2) for the last forward."""
        x, logits, r, h, a, y = self.saved
        dy, dweights = emu.rows_combine_backward(dout, y, r.slots, r.weights)
        da, _ = emu.grouped_gemm(dy, self.W2, r.ends, opW=emu.OP_T)
        dW2, _ = emu.grouped_wgrad(a, dy, r.ends)
        dh = da * silu_grad(h)
        dxs, _ = emu.grouped_gemm(dh, self.W1, r.ends, opW=emu.OP_T)
        dW1, _ = emu.grouped_wgrad(x, dh, r.ends, srcA=r.rows)
        dlogits = emu.route_backward(logits, r.experts, dweights)
        drouter, _ = emu.gemm_ex(x.float(), dlogits, opA=emu.OP_T)
        dx = emu.rows_combine(dxs, r.slots)                          # every token's rows added up
        back, _ = emu.gemm_ex(dlogits, self.router, opB=emu.OP_T)
        return dx + back.to(dx.dtype), drouter, dW1, dW2


def quantize(W, group=128):
    """Weights [E, K, N] -> codes [E, N, K/2], scales and zero points [E, N, K/group]
    as w4_matvec takes them: the range of every group on 16 levels."""
    E, K, N = W.shape
    w = W.float().transpose(1, 2).reshape(E, N, K // group, group)
    lo, hi = w.amin(-1).clamp(max=0), w.amax(-1).clamp(min=0)
    scale = ((hi - lo) / 15).clamp(min=1e-8)
    zero = (-lo / scale).round().clamp(0, 15)
    q = ((w / scale[..., None]).round() + zero[..., None]).clamp(0, 15).to(torch.uint8).reshape(E, N, K)
    return (q[..., 0::2] | q[..., 1::2] << 4).contiguous(), scale.to(W.dtype).contiguous(), zero.to(torch.uint8).contiguous()


class QuantizedExperts:
    """The layer with 4-bit experts, for a few tokens at a time."""

    def __init__(self, layer, group=128):
        self.router, self.k = layer.router, layer.k
        self.first, self.second = quantize(layer.W1, group), quantize(layer.W2, group)

    def forward(self, x):
        logits, _ = emu.gemm_f32(x.float(), self.router)
        r, _ = emu.route(logits, self.k)
        h = emu.w4_matvec(x[r.rows.long()], *self.first, ends=r.ends)
        y = emu.w4_matvec(silu(h), *self.second, ends=r.ends)
        return emu.rows_combine(y, r.slots, r.weights)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--experts", type=int, default=16)
    ap.add_argument("--k", type=int, default=2)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    a = ap.parse_args(argv)
    dtype = torch.bfloat16 if a.dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(1)
    layer = ExpertLayer(a.width, a.hidden, a.experts, a.k, dtype)
    target = ExpertLayer(a.width, a.hidden, a.experts, a.k, dtype, seed=2)
    losses = []
    for step in range(a.steps):
        x = torch.randn(a.tokens, a.width, generator=g, device="cuda").to(dtype)
        diff = layer.forward(x).float() - target.forward(x).float()
        losses.append(float(diff.square().mean()))
        _, drouter, dW1, dW2 = layer.backward((diff * (2.0 / a.tokens)).to(dtype))
        for p, d in ((layer.router, drouter), (layer.W1, dW1), (layer.W2, dW2)):
            p.sub_((d.float() * 0.1).to(p.dtype))
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} in {a.steps} steps of {a.tokens} tokens")
    served, off = QuantizedExperts(layer), []
    for _ in range(4):
        x = torch.randn(1, a.width, generator=g, device="cuda").to(dtype)
        want = layer.forward(x).float()
        off.append(float((served.forward(x).float() - want).norm() / want.norm()))
    print("single tokens with 4-bit experts: relative distances " + " ".join(f"{v:.3f}" for v in off))
    return losses, off


if __name__ == "__main__":
    main()
