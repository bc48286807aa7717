"""The README's lines for the expert layers run as they stand, one block after the other, and
give what the calls give by themselves."""
import os
import re

import pytest

import paper_2609_04663_gb300 as emu
from helpers import device

pytestmark = pytest.mark.gpu
README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


@pytest.mark.parametrize("T", [2, 37])
def test_expert_layer_blocks(T):
    import torch
    dev = device()
    blocks = [b for b in re.findall(r"```python\n(.*?)```", open(README).read(), flags=re.S) if "emu.route" in b]
    assert len(blocks) == 2 and "emu.i8_gemm" in blocks[1]
    g = torch.Generator(device=dev).manual_seed(T)
    rand = lambda *shape: torch.randn(*shape, generator=g, device=dev)
    names = dict(emu=emu, act=torch.relu, logits=rand(T, 6), x=rand(T, 48).bfloat16(), W1=rand(6, 48, 80).bfloat16(),
                 W2=rand(6, 80, 48).bfloat16(), W=rand(6, 80, 48).bfloat16(), dlogits=rand(T, 6), dloss=torch.tensor(2.0, device=dev))
    before = names["dlogits"].clone()
    exec(blocks[0], names)
    assert names["out"].shape == (T, 48)
    exec(blocks[1], names)
    r, logits = names["r"], names["logits"]
    b, _ = emu.route_balance(logits, r.experts, coef=0.01)
    assert torch.equal(names["b"].loss, b.loss)
    assert torch.equal(names["dlogits"], emu.route_balance_backward(logits, b, names["dloss"], 0.01, add=before))
    w, v = emu.i8_quantize(names["W"])
    y, _ = emu.i8_gemm(emu.i8_quantize(names["x"]), (w, v), r.ends, src=r.rows)
    assert y.shape == (2 * T, 80) and torch.equal(names["y"], y)
