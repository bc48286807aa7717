"""Rows that the products in 8-bit integers take from nowhere (an index outside of X, or no
group) are zero whatever the scales of the channels are, in every kernel."""
import pytest
import torch

import paper_2609_04663_gb300 as emu
from helpers import device

pytestmark = pytest.mark.gpu

#        rows, N, K, groups; the kernel that these sizes get
SIZES = [(5, 90, 130, 3), (6, 200, 96, 8), (40, 150, 200, 3), (900, 144, 400, 3), (24, 140, 4096, 1), (6000, 1100, 400, 3), (6000, 1024, 64, 1)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.int32])
@pytest.mark.parametrize("rows,N,K,G", SIZES)
def test_rows_from_nowhere(rows, N, K, G, dtype):
    dev = device()
    many = emu.emu_i8_gemm_workspace_bytes(G, rows, N, K, 1) > 0
    assert many == (rows == 6000)
    g = torch.Generator(device=dev).manual_seed(rows + N + K)
    X = torch.randint(-128, 128, (50, (K + 15) // 16 * 16), generator=g, device=dev, dtype=torch.int8)[:, :K]
    W = torch.randint(-128, 128, (G, N, (K + 15) // 16 * 16), generator=g, device=dev, dtype=torch.int8)[..., :K]
    xs, v = torch.rand(50, generator=g, device=dev) + 0.5, torch.rand(G, N, generator=g, device=dev) - 0.5
    v[:, 3], v[:, 40], v[:, N - 1] = float("nan"), float("inf"), -float("inf")
    xs[7], xs[9], xs[11] = float("nan"), 0.0, float("inf")
    src = torch.randint(0, 50, (rows,), generator=g, device=dev, dtype=torch.int32)
    src[0], src[2], src[rows - 3] = -1, 50, 2 ** 31 - 1
    ends = torch.tensor([(rows - 1) * (i + 1) // G for i in range(G)], dtype=torch.int32, device=dev)
    Y, _ = emu.i8_gemm((X, xs), (W, v), ends=ends, src=src, dtype=dtype)
    gone = (src < 0) | (src >= 50)
    gone[rows - 1] = True                                    # of no group
    assert not Y[gone].any()
    # all others are what sum, channel and token give, in that order
    of = torch.bucketize(torch.arange(rows, device=dev), ends.long(), right=True).clamp(max=G - 1)
    at = src.long().clamp(0, 49)
    S = torch.empty(rows, N, dtype=torch.float64, device=dev)
    for i in range(G):
        S[of == i] = X[at[of == i]].double() @ W[i].double().T
    want = S.to(torch.int32) if dtype is torch.int32 else (S.float() * v[of] * xs[at][:, None]).to(dtype)
    assert torch.equal(torch.nan_to_num(Y[~gone], nan=1.25), torch.nan_to_num(want[~gone], nan=1.25)) if dtype is not torch.int32 else \
        torch.equal(Y[~gone], want[~gone])
