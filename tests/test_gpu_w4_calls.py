"""Calls of the 4-bit products one after another in one workspace."""
import pytest

import paper_2609_04663_gb300 as emu
from helpers import device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


def weights(dev, G, N, K, group, seed=0):
    import torch
    g = torch.Generator(device=dev).manual_seed(seed)
    q = torch.randint(0, 256, (G, N, K // 2), generator=g, device=dev, dtype=torch.uint8)
    return q, torch.rand((G, N, K // group), generator=g, device=dev) + 0.25


def test_a_call_without_rows_ends_before_the_next_one(dev):
    """No group has a row: the product has nothing to wait for, but its rows' slices
    are still being written, where the next call's are to lie."""
    import torch
    rows, K, N = 3000, 4096, 64
    q, s = weights(dev, 2, N, K, 128)
    g = torch.Generator(device=dev).manual_seed(1)
    first, X = (torch.randn((rows, K), generator=g, device=dev) for _ in range(2))
    none = torch.zeros(2, dtype=torch.int32, device=dev)
    ends = torch.tensor([1000, rows], dtype=torch.int32, device=dev)
    want = emu.w4_matvec(X, q, s, ends=ends)
    ws = emu.workspace(emu.emu_w4_workspace_bytes(emu.F32, rows, K), dev)
    for _ in range(20):
        empty = emu.w4_matvec(first, q, s, ends=none, ws=ws)
        got = emu.w4_matvec(X, q, s, ends=ends, ws=ws)
        assert not empty.any() and torch.equal(got, want)
