"""FP32 results of BF16 operands over long contractions, against 64 bits.

Tolerances, fixed before the first run.  Products are exact.  Sums are held in
parts of 256 terms, 16 additions of 16 products each, every one truncated at
most two units below FP32's last place of the part's sum so far (2^-22), and the
parts are added with rounding (2^-24 each): an entry is within 16 x 2^-22 + (n / 256)
2^-24 of its absolute sum.  Truncations lean one way; with part sums at most as
large as the result's norm the 2-norm error is within 16 x 2^-23, 2e-6."""
import pytest

import paper_2609_04663_gb300 as emu
from helpers import device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


def values(g, shape, kind):
    """normal: either sign; positive: sums that only grow."""
    import torch
    t = torch.randn(shape, generator=g, device=g.device) if kind == "normal" else torch.rand(shape, generator=g, device=g.device)
    return t.bfloat16()


def close(got, x, w):
    n = x.shape[1]
    ref, mag = x.double() @ w.double(), x.double().abs() @ w.double().abs()
    err = (got.double() - ref).abs()
    entries = bool((err <= (16 * 2.0 ** -22 + n / 256 * 2.0 ** -24) * mag).all())
    return entries and float(err.norm()) <= 2e-6 * float(ref.norm())


@pytest.mark.parametrize("kind", ["normal", "positive"])
@pytest.mark.parametrize("trans", [False, True])
@pytest.mark.parametrize("sizes,K,N", [([40, 0, 24], 4096, 72), ([300, 256, 1], 8192, 264), ([33], 30000, 40),
                                       ([700], 2049, 600), ([16, 17], 257, 136)])
def test_product(dev, kind, trans, sizes, K, N):
    import torch
    g = torch.Generator(device=dev).manual_seed(1)
    rows, G = sum(sizes) + 2, len(sizes)
    X = values(g, (rows, K), kind)
    W = values(g, (G, N, K) if trans else (G, K, N), kind)
    ends = torch.tensor(sizes, device=dev).cumsum(0).to(torch.int32)
    Y = torch.full((rows, N), 7.0, device=dev)
    _, ws = emu.grouped_gemm(X, W, ends, opW=emu.OP_T if trans else emu.OP_N, Y=Y)
    assert emu.read_flags(ws) == 0 and not Y[rows - 2:].any()
    at = 0
    for n, w in zip(sizes, W):
        if n:
            assert close(Y[at:at + n], X[at:at + n], w.T if trans else w)
        at += n


@pytest.mark.parametrize("kind", ["normal", "positive"])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("sizes,M,N", [([5000, 0, 3, 4097], 72, 136), ([20000], 264, 40), ([257, 256, 1023], 300, 520)])
def test_weight_gradient(dev, kind, gather, sizes, M, N):
    """Ragged ends of rows that are used as they stand, and of gathered copies."""
    import torch
    g = torch.Generator(device=dev).manual_seed(2)
    rows = sum(sizes)
    A, B = values(g, (rows, M), kind), values(g, (rows, N), kind)
    src = torch.randperm(rows, generator=g, device=dev).to(torch.int32) if gather else None
    ends = torch.tensor(sizes, device=dev).cumsum(0).to(torch.int32)
    D = torch.full((len(sizes), M, N), 7.0, device=dev)
    _, ws = emu.grouped_wgrad(A, B, ends, srcA=src, D=D)
    assert emu.read_flags(ws) == 0
    As, at = A[src.long()] if gather else A, 0
    for n, d in zip(sizes, D):
        assert close(d, As[at:at + n].T, B[at:at + n]) if n else not d.any()
        at += n


def test_long_sums_do_not_leak_between_groups(dev):
    """NaN in one group's rows and in rows of no group stays there; twice the same bits."""
    import torch
    g = torch.Generator(device=dev).manual_seed(3)
    sizes = [1000, 777, 2050]
    X, B, W = values(g, (3900, 1000), "normal"), values(g, (3900, 72), "normal"), values(g, (3, 1000, 136), "normal")
    ends = torch.tensor(sizes, device=dev).cumsum(0).to(torch.int32)
    outs = []
    for spoil in (False, False, True):
        x = X.clone()
        if spoil:
            x[1000:1777], x[3827:] = float("nan"), float("inf")
        Y, D = torch.empty((3900, 136), device=dev), torch.empty((3, 1000, 72), device=dev)
        emu.grouped_gemm(x, W, ends, Y=Y)
        emu.grouped_wgrad(x, B, ends, D=D)
        outs.append((Y, D))
    (Y, D), again, (Yn, Dn) = outs
    assert torch.equal(Y, again[0]) and torch.equal(D, again[1])
    assert torch.equal(Yn[:1000], Y[:1000]) and torch.equal(Yn[1777:], Y[1777:]) and bool(Yn[1000:1777].isnan().all())
    assert torch.equal(Dn[[0, 2]], D[[0, 2]]) and bool(Dn[1].isnan().all())
