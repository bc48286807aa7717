"""Sums of 8-bit products next to the largest that one accumulator has to hold (1024 terms of up to 2^14,
2^24 in all), odd ones among them, and large ones that cancel: an accumulator that lost its lowest bit anywhere
would show.  The right value is an integer below 2^31, which 64-bit floating point sums exactly."""
import pytest
import torch

import paper_2609_04663_gb300 as emu
from helpers import device

pytestmark = pytest.mark.gpu


def operands(kind, rows, N, K, g, dev):
    pick = lambda lo, hi, shape: torch.randint(lo, hi + 1, shape, generator=g, device=dev).to(torch.int8)
    at = torch.arange(K, device=dev) % 1024
    if kind == "positive":                       # 1024 terms: 15.9 to 16.5 million
        return pick(127, 127, (rows, K)), pick(125, 127, (N, K))
    if kind == "negative":                       # -16.6 to -16.1 million
        return pick(-128, -127, (rows, K)), pick(125, 127, (N, K))
    if kind == "largest":                        # up to 2^24 itself
        return pick(-128, -127, (rows, K)), pick(-128, -127, (N, K))
    X, W = pick(126, 127, (rows, K)), pick(125, 127, (N, K))
    if kind == "halves":                         # up to 8 million, and back
        return X, torch.where(at < 512, W, -W)
    if kind == "sixteens":                       # up and down between the instructions' contractions
        return X, torch.where(at // 16 % 2 == 0, W, -W)
    assert kind == "one left"                    # all but one term cancels, exactly
    X, W = pick(127, 127, (rows, K)), pick(127, 127, (N, K))
    W = torch.where((at < 512), W, -W)
    W[:, 5] -= 1
    return X, W


#        rows, N and what takes them: integer dot products, single SMs, single SMs with parts of K, pairs
SIZES = [(1, 70), (7, 70), (40, 130), (600, 130), (24, 140), (4000, 1000)]


@pytest.mark.parametrize("kind", ["positive", "negative", "largest", "halves", "sixteens", "one left"])
@pytest.mark.parametrize("K", [1023, 1024, 1025, 2047, 4112, 20001])
@pytest.mark.parametrize("rows,N", SIZES)
def test_every_bit_of_a_sum(rows, N, K, kind):
    dev = device()
    assert (emu.emu_i8_gemm_workspace_bytes(1, rows, N, K, 1) > 0) == (rows == 4000)
    g = torch.Generator(device=dev).manual_seed(rows + K)
    X, W = operands(kind, rows, N, (K + 15) // 16 * 16, g, dev)      # rows on 16 bytes: copied for none
    X, W = X[:, :K], W[:, :K]
    S = X.double() @ W.double().T
    Y, _ = emu.i8_gemm((X, None), (W, None), dtype=torch.int32)
    assert torch.equal(Y.double(), S)
    if K == 1024 and kind in ("positive", "negative", "largest"):    # what the test is about is there
        assert bool((S.abs() > 0.94 * 2 ** 24).all()) and bool((S % 2 == 1).any())


def test_experts_of_many_rows():
    dev = device()
    g = torch.Generator(device=dev).manual_seed(1)
    X, W = operands("positive", 6000, 3300, 2064, g, dev)
    W = W.view(3, 1100, 2064)
    ends = torch.tensor([2500, 2501, 6000], dtype=torch.int32, device=dev)
    assert emu.emu_i8_gemm_workspace_bytes(3, 6000, 1100, 2064, 1) > 0
    Y, _ = emu.i8_gemm((X, None), (W, None), ends=ends, dtype=torch.int32)
    for i, (a, b) in enumerate(((0, 2500), (2500, 2501), (2501, 6000))):
        assert torch.equal(Y[a:b].double(), X[a:b].double() @ W[i].double().T)
