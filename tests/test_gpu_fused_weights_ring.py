"""FP32 products grouped by expert on the weights themselves, where boxes of weights end past the
matrix: many calls of the same operands give the same bits, which are within the
method's bound.  (A stage that were handed back before it is read would get zeros over its last
values, now and then.)"""
import pytest

import paper_2609_04663_gb300 as emu
from helpers import device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("op", [emu.OP_N, emu.OP_T])
@pytest.mark.parametrize("rows,G,N,K", [(60, 3, 700, 2068), (200, 7, 260, 1036), (9, 9, 1204, 4100), (130, 1, 516, 68), (900, 4, 132, 3332)])
def test_the_same_products_every_time(op, rows, G, N, K):
    import torch
    dev = device()
    g = torch.Generator(device=dev).manual_seed(rows + N)
    X = torch.randn(rows, K, generator=g, device=dev)
    W = torch.randn((G, K, N) if op == emu.OP_N else (G, N, K), generator=g, device=dev)
    cut = torch.randint(0, rows + 1, (G,), generator=g, device=dev).sort().values.int()
    cut[-1] = rows
    Y, ws = emu.grouped_gemm(X, W, cut, op)
    assert emu.read_flags(ws) == 0
    first, at = Y.clone(), 0
    for i, e in enumerate(cut.tolist()):
        M = W[i].double() if op == emu.OP_N else W[i].double().T
        x = X[at:e].double()
        assert bool(((first[at:e].double() - x @ M).abs() <= 1e-5 * (x.abs() @ M.abs())).all())
        at = e
    off = torch.zeros((), dtype=torch.int64, device=dev)
    for _ in range(300):
        emu.grouped_gemm(X, W, cut, op, Y=Y, ws=ws)
        off += (Y != first).sum()
    assert int(off) == 0
