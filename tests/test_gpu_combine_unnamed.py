"""Gradient rows of the weighted sum that no slot names: zero in a dY made by
the call, whatever memory it was given, untouched in a caller's own.

Tolerance: a named row is one product of two FP32 numbers, rounded to the
result's type (2^-23, BF16 2^-8 more)."""
import pytest

import paper_2609_04663_gb300 as emu
from helpers import device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


@pytest.fixture(params=["zeros", "ones"])
def dirty(request, monkeypatch):
    """Every tensor that a call makes starts as NaN, its integers and workspaces as all zero or all one bits."""
    import torch
    plain = emu._empty

    def filled(shape, dtype, dev, stream):
        t = plain(shape, dtype, dev, stream)
        return t.fill_(float("nan")) if t.is_floating_point() else t.fill_(0 if request.param == "zeros" else
                                                                           (255 if dtype is torch.uint8 else -1))
    monkeypatch.setattr(emu, "_empty", filled)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("T,k,cols,extra", [(1, 1, 1, 0), (4, 2, 24, 0), (37, 3, 33, 0), (300, 4, 512, 0), (50, 2, 72, 1),
                                            (1000, 8, 16, -17), (3, 5, 2056, 0), (20, 2, 40, 300)])
def test_unnamed_rows_are_zero(dev, dirty, dtype, weighted, T, k, cols, extra):
    """As many rows as slots (extra 0), more, or fewer; some slots outside."""
    import torch
    g = torch.Generator(device=dev).manual_seed(1)
    S, dt = T * k + extra, getattr(torch, dtype)
    Y, dO = (torch.randn((r, cols), generator=g, device=dev).to(dt) for r in (S, T))
    slots = torch.randperm(max(S, T * k), generator=g, device=dev)[:T * k].to(torch.int32)      # (those from S on are outside)
    slots[:: 7] = -1
    slots[3 :: 11] = S + 5
    slots = slots.view(T, k)
    w = torch.rand((T, k), generator=g, device=dev) + 0.5 if weighted else None
    dY, dw = emu.rows_combine_backward(dO, Y, slots, w)
    ok = (slots >= 0) & (slots < S)
    at = slots[ok].long()
    named = torch.zeros(S, dtype=torch.bool, device=dev)
    named[at] = True
    assert not dY[~named].any() and not dY[~named].isnan().any()
    want = ((w.double()[..., None] if weighted else 1.0) * dO.double()[:, None]).expand(T, k, cols)[ok]
    tol = 2.0 ** -23 + (2.0 ** -8 if dtype == "bfloat16" else 0.0)
    assert bool(((dY[at].double() - want).abs() <= tol * want.abs()).all())
    assert dw is None or not dw[~ok].any()


def test_all_slots_named_and_none(dev, dirty):
    import torch
    dO, Y = torch.randn(6, 40, device=dev), torch.randn(12, 40, device=dev)
    slots = torch.randperm(12, device=dev).to(torch.int32).view(6, 2)
    dY, _ = emu.rows_combine_backward(dO, Y, slots)
    assert torch.equal(dY[slots.long()], dO[:, None].expand(6, 2, 40))
    dY, dw = emu.rows_combine_backward(dO, Y, torch.full_like(slots, -1), torch.ones(6, 2, device=dev))
    assert not dY.any() and not dw.any()


def test_a_given_result_keeps_its_unnamed_rows(dev, dirty):
    import torch
    slots = torch.tensor([[2, -1], [0, 9]], dtype=torch.int32, device=dev)
    dO = torch.randn(2, 24, device=dev)
    dY = torch.full((4, 24), 7.0, device=dev)
    emu.rows_combine_backward(dO, torch.randn(4, 24, device=dev), slots, dY=dY)
    assert torch.equal(dY[[2, 0]], dO) and bool((dY[[1, 3]] == 7.0).all())


def test_no_tokens(dev, dirty):
    import torch
    dY, _ = emu.rows_combine_backward(torch.empty(0, 8, device=dev), torch.randn(5, 8, device=dev),
                                      torch.empty(0, 2, dtype=torch.int32, device=dev))
    assert dY.shape == (5, 8) and not dY.any()
