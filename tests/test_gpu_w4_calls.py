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


def stale(dev, dtype, rows, K):
    """A workspace whose words hold every flag."""
    import torch
    return torch.full((emu.emu_w4_workspace_bytes(emu.F32 if dtype is torch.float32 else emu.BF16, rows, K),), 255,
                      dtype=torch.uint8, device=dev)


@pytest.mark.parametrize("rows,K", [(1, 32), (7, 1024), (30, 16384), (3000, 4096)])
def test_fp32_values_out_of_range_are_flagged(dev, rows, K):
    """The largest values that split into finite slices, and the next one, infinity
    and NaN, first and last: only the row that holds one is touched.  All codes are
    zero points but one of value one: sums stay in range.  2^-23: the third slice's rounding."""
    import torch
    q = torch.full((40, K // 2), 0x88, dtype=torch.uint8, device=dev)
    q[:, 0], q[:, -1] = 0x89, 0x98                     # k = 0 and k = K - 1
    s = torch.full((40, K // 32), 0.5, device=dev)
    g = torch.Generator(device=dev).manual_seed(2)
    X = torch.randn((rows, K), generator=g, device=dev)
    X[:, 0] = X[:, K - 1] = 0.0
    ws = stale(dev, X.dtype, rows, K)
    assert not emu.w4_matvec(X, q, s, ws=ws).any() and emu.read_flags(ws) == 0
    bits = lambda u: torch.tensor(u, dtype=torch.int32).view(torch.float32).item()
    both = emu.FLAG_NONFINITE | emu.FLAG_SLICE
    for value, flags in ((bits(0x7F7F7FFF), 0), (-bits(0x7F7F7FFF), 0), (bits(0x7F7F8000), emu.FLAG_SLICE),
                         (-bits(0x7F7FFFFF), emu.FLAG_SLICE), (float("-inf"), both), (float("nan"), both)):
        for r, k in ((0, 0), (rows - 1, K - 1)):
            X[r, k] = value
            Y = emu.w4_matvec(X, q, s, ws=ws)
            assert emu.read_flags(ws) == flags
            if flags:
                assert bool(Y[r].isnan().all())
            else:
                assert bool(((Y[r].double() - 0.5 * value).abs() <= 2.0 ** -23 * abs(value)).all())
            Y[r] = 0
            assert not Y.any()
            X[r, k] = 0.0


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("cuts,owner", [([4, 9, 12], [0] * 4 + [1] * 5 + [2] * 3), ([4, 1000, 12], [0] * 4 + [1] * 8),
                                        ([-5, 9, 12], [1] * 9 + [2] * 3), ([6, 2, 11], [0] * 6 + [2] * 5 + [-1]),
                                        ([-1, -9, -3], [-1] * 12)])
def test_bad_ends_are_flagged_and_clamped(dev, dtype, aligned, cuts, owner):
    """Ends outside 0 .. rows are clamped, decreasing ones raised to those before them."""
    import torch
    rows, K, N, dt = 12, 128, 70, getattr(torch, dtype)
    q, s = weights(dev, 3, N, K, 64, 3)
    wide = torch.randn((rows, K + 8), generator=torch.Generator(device=dev).manual_seed(4), device=dev).to(dt)
    X = wide[:, :K] if aligned else wide[:, 1:K + 1]
    ends = torch.tensor(cuts, dtype=torch.int32, device=dev)
    bad = cuts != [4, 9, 12]
    for ws in (stale(dev, dt, rows, K), None):
        Y = emu.w4_matvec(X, q, s, ends=ends, ws=ws)
        assert ws is None or emu.read_flags(ws) == (emu.FLAG_INDEX if bad else 0)
        for r, e in enumerate(owner):
            want = emu.w4_matvec(X[r:r + 1], q[e], s[e])[0] if e >= 0 else torch.zeros(N, dtype=dt, device=dev)
            # one row alone may cut K differently: the last bit of a BF16 result, K/16 + 16 roundings of FP32 sums
            tol = 2.0 ** -7 * want.abs() + (K / 16 + 16) * 2.0 ** -22 * 16 * X[r].float().abs().sum()
            assert bool(((Y[r].float() - want.float()).abs() <= tol).all()), r


def test_calls_without_work_clear_the_word(dev):
    import torch
    q, s = weights(dev, 1, 16, 32, 32)
    for rows, N, K in ((0, 16, 32), (2, 0, 32), (2, 16, 0)):
        ws = stale(dev, torch.float32, 2, 32)
        X = torch.zeros((rows, K), device=dev)
        Y = emu.w4_matvec(X, q[0, :N, :K // 2], s[0, :N, :K // 32], ws=ws)
        assert emu.read_flags(ws) == 0 and not Y.any()
