"""grouped_workspace(train=True) is a workspace for the product, both gradients
and the splits of the same operands, from tensors as from plane sets."""
import pytest

import paper_2609_04663_gb300 as emu
from helpers import device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("trans", [False, True])
@pytest.mark.parametrize("rows,K,N,gather", [(60, 24, 200, False), (60, 200, 24, True), (5000, 40, 72, False), (3, 8, 8, True)])
def test_one_workspace_for_a_training_step(dtype, trans, rows, K, N, gather):
    import torch
    dev = device()
    g = torch.Generator(device=dev).manual_seed(1)
    dt = getattr(torch, dtype)
    T = rows // 3 if gather else rows
    X, W, dY = (torch.randn(s, generator=g, device=dev).to(dt) for s in ((T, K), (3, N, K) if trans else (3, K, N), (rows, N)))
    src = torch.randint(0, T, (rows,), generator=g, device=dev, dtype=torch.int32) if gather else None
    ends = torch.tensor([rows // 2, rows // 2, rows], dtype=torch.int32, device=dev)
    op, back = (emu.OP_T, emu.OP_N) if trans else (emu.OP_N, emu.OP_T)
    ws = emu.grouped_workspace(X, W, ends, op, src, train=True)
    size = ws.numel()
    want = (emu.grouped_gemm(X, W, ends, opW=op, src=src)[0], emu.grouped_gemm(dY, W, ends, opW=back)[0],
            emu.grouped_wgrad(X, dY, ends, srcA=src)[0])
    got = (emu.grouped_gemm(X, W, ends, opW=op, src=src, ws=ws)[0], emu.grouped_gemm(dY, W, ends, opW=back, ws=ws)[0],
           emu.grouped_wgrad(X, dY, ends, srcA=src, ws=ws)[0])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    Xp, Wp = emu.grouped_split(X, ends, src=src, ws=ws), emu.grouped_split(W, ws=ws)
    emu.grouped_gemm(Xp, Wp, ends, opW=op, ws=ws)
    assert ws.numel() == size and emu.read_flags(ws) == 0
