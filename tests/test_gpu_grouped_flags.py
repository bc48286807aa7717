"""Flags of the products grouped by expert: what a call's own splits find is
still in its flag word after the product, and a clean call's word is zero
whatever the workspace held."""
import pytest

import paper_2609_04663_gb300 as emu
from helpers import device

pytestmark = pytest.mark.gpu
BAD_VALUE = emu.FLAG_NONFINITE | emu.FLAG_SLICE


@pytest.fixture(scope="module")
def dev():
    return device()


def operands(dev, dtype, rows=(40, 30), K=64, N=72):
    import torch
    g = torch.Generator(device=dev).manual_seed(1)
    R, dt = sum(rows), getattr(torch, dtype)
    ends = torch.tensor(rows, device=dev).cumsum(0).to(torch.int32)
    X, W, dY = (torch.randn(s, generator=g, device=dev).to(dt) for s in ((R, K), (len(rows), K, N), (R, N)))
    src = torch.randperm(R, generator=g, device=dev).to(torch.int32)
    return X, W, dY, ends, src


def spoiled(src, n):
    bad = src.clone()
    bad[5], bad[50] = -1, n
    return bad


def stale_ws(dev):
    """A workspace whose flag word holds every flag."""
    import torch
    return torch.full((emu.emu_split_workspace_bytes(32),), 255, dtype=torch.uint8, device=dev)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_bad_source_rows(dev, dtype):
    import torch
    X, W, dY, ends, src = operands(dev, dtype)
    bad = spoiled(src, X.shape[0])
    y, ws = emu.grouped_gemm(X, W, ends, src=bad)
    assert emu.read_flags(ws) == emu.FLAG_INDEX
    ok, ws = emu.grouped_gemm(X, W, ends, src=src)
    assert emu.read_flags(ws) == 0
    ok[5], ok[50] = 0, 0
    assert torch.equal(y, ok)
    for kw in ({"srcA": bad}, {"srcB": bad}, {"srcA": bad, "srcB": src}, {"srcA": src, "srcB": bad}):
        _, ws = emu.grouped_wgrad(X, dY, ends, **kw)
        assert emu.read_flags(ws) == emu.FLAG_INDEX, kw
        _, ws = emu.grouped_wgrad(X, dY, ends, **{k: src for k in kw}, ws=ws)
        assert emu.read_flags(ws) == 0, kw


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("wide", [False, True])
def test_bad_source_rows_of_weights_that_are_split_too(dev, dtype, wide):
    """The weights' split (rows that no bulk copy can read) comes after the rows' one."""
    import torch
    X, W, dY, ends, src = operands(dev, dtype)
    if wide:
        big = torch.zeros(2, 64, 75, dtype=W.dtype, device=dev)
        big[:, :, 1:73] = W
        W = big[:, :, 1:73]
    bad = spoiled(src, X.shape[0])
    for Ws in (W, emu.grouped_split(W)):
        _, ws = emu.grouped_gemm(X, Ws, ends, src=bad)
        assert emu.read_flags(ws) == emu.FLAG_INDEX
        _, ws = emu.grouped_gemm(X, Ws, ends, src=src, ws=ws)
        assert emu.read_flags(ws) == 0


@pytest.mark.parametrize("value,flags", [(float("inf"), BAD_VALUE), (float("nan"), BAD_VALUE), (3.4e38, emu.FLAG_SLICE)])
def test_fp32_values_out_of_range(dev, value, flags):
    import torch
    X, W, dY, ends, src = operands(dev, "float32")
    Xb, Wb, db = X.clone(), W.clone(), dY.clone()
    Xb[3, 4] = Wb[1, 2, 3] = db[69, 71] = value
    Xp, Wp = emu.grouped_split(X, ends), emu.grouped_split(W)
    for x, w in ((Xb, W), (X, Wb), (Xb, Wp), (Xp, Wb)):
        _, ws = emu.grouped_gemm(x, w, ends)
        assert emu.read_flags(ws) == flags
    for a, b in ((Xb, dY), (X, db), (Xb, emu.grouped_split(dY, ends)), (Xp, db)):
        _, ws = emu.grouped_wgrad(a, b, ends)
        assert emu.read_flags(ws) == flags
    _, ws = emu.grouped_wgrad(X, db, ends, srcA=spoiled(src, X.shape[0]))
    assert emu.read_flags(ws) == flags | emu.FLAG_INDEX
    _, ws = emu.grouped_gemm(Xp, W, ends)
    assert emu.read_flags(ws) == 0


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_clean_calls_clear_the_word(dev, dtype):
    X, W, dY, ends, src = operands(dev, dtype)
    Xp, Wp, dp = emu.grouped_split(X, ends), emu.grouped_split(W), emu.grouped_split(dY, ends)
    for x, w, s in ((X, Wp, None), (X, Wp, src), (Xp, W, None), (Xp, Wp, None)):
        _, ws = emu.grouped_gemm(x, w, ends, src=s, ws=stale_ws(dev))
        assert emu.read_flags(ws) == 0
    for a, b, s in ((X, dY, None), (X, dY, src), (Xp, dY, None), (X, dp, src), (Xp, dp, None)):
        _, ws = emu.grouped_wgrad(a, b, ends, srcA=s, ws=stale_ws(dev))
        assert emu.read_flags(ws) == 0
    for x, e in ((X, None), (X, ends), (W, None)):
        ws = stale_ws(dev)
        if x.dim() == 3 or e is not None:
            emu.grouped_split(x, e, ws=ws)
            assert emu.read_flags(ws) == 0


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("bad", [[40, 1000], [-5, 70], [50, 30]])
def test_bad_ends(dev, dtype, bad):
    import torch
    X, W, dY, ends, src = operands(dev, dtype)
    e = torch.tensor(bad, dtype=torch.int32, device=dev)
    for s in (None, src):
        _, ws = emu.grouped_gemm(X, W, e, src=s)
        assert emu.read_flags(ws) == emu.FLAG_INDEX
        _, ws = emu.grouped_wgrad(X, dY, e, srcA=s)
        assert emu.read_flags(ws) == emu.FLAG_INDEX


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_empty_products_keep_the_splits_flags(dev, dtype):
    """No columns in the result: nothing is multiplied, but a bad source row is still reported."""
    import torch
    X, W, dY, ends, src = operands(dev, dtype)
    _, ws = emu.grouped_wgrad(X, dY[:, :0], ends, srcA=spoiled(src, X.shape[0]))
    assert emu.read_flags(ws) == emu.FLAG_INDEX
    _, ws = emu.grouped_wgrad(X, dY[:, :0], ends, srcA=src, ws=ws)
    assert emu.read_flags(ws) == 0
