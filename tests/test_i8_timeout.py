"""A wait that gives up inside of an 8-bit product on single SMs is reported, beside bad indexes,
whether the launch clears the flag word itself (up to 4096 rows) or finds it clear."""
import pytest

import paper_2609_04663_gb300 as emu
from paper_2609_04663_gb300 import _build
from helpers import device


def test_self_test_arguments():
    _build.build()
    P, BIG, f = 16, 1 << 40, emu.emu_selftest_i8_timeout
    #                us G rows N  K  X xrows ldx xs src W ldw sw  ws  ends Y  yt ldy ws bytes stream
    for us in (0, 1000001):
        assert f(us, 1, 40, 8, 16, P, 40, 16, P, None, P, 16, 0, P, None, P, 0, 8, P, BIG, None) == 1
    assert f(1000, 1, 40, 8, 16, P, 40, 16, P, None, P, 16, 0, P, None, P, 0, 8, None, 0, None) == 1      # no workspace
    assert f(1000, 1, 0, 8, 16, P, 40, 16, P, None, P, 16, 0, P, None, P, 0, 8, P, BIG, None) == 1
    assert f(1000, 1, 40, 8, 16, P, 40, 15, P, None, P, 16, 0, P, None, P, 0, 8, P, BIG, None) == 1
    assert f(1000, 1, 40, 8, 16, P, 40, 16, P, None, P, 16, 0, P, None, P, 0, 8, P, 511, None) == 3
    assert f(1000, 1, 1, 8, 16, P, 1, 16, P, None, P, 16, 0, P, None, P, 0, 8, P, BIG, None) == 5         # no waits there
    assert f(1000, 1, 4000, 4000, 16, P, 4000, 16, P, None, P, 16, 0, P, None, P, 0, 4000, P, BIG, None) == 5


@pytest.mark.gpu
@pytest.mark.parametrize("rows,N,K,G", [(40, 200, 96, 1), (24, 140, 4096, 1), (300, 60, 64, 5), (5000, 24, 32, 900)])
def test_a_wait_that_runs_out_is_reported(rows, N, K, G):
    import torch
    dev = device()
    g = torch.Generator(device=dev).manual_seed(rows)
    X = torch.randint(-128, 128, (rows, K), generator=g, device=dev, dtype=torch.int8)
    W = torch.randint(-128, 128, (G, N, K), generator=g, device=dev, dtype=torch.int8)
    src = torch.randperm(rows, generator=g, device=dev).int()
    bad = src.clone()
    bad[rows // 2] = rows
    ends = torch.tensor([(rows - 2) * (i + 1) // G for i in range(G)], dtype=torch.int32, device=dev)
    ws = emu.workspace(emu.emu_split_workspace_bytes(32), dev)
    want, _ = emu.i8_gemm((X, None), (W, None), ends=ends, src=src, dtype=torch.int32)
    Y = torch.full((rows, N), 5, dtype=torch.int32, device=dev)
    for took, flags in ((src, 0), (bad, emu.FLAG_INDEX)):
        ws.fill_(0x7F)                                       # flags as an earlier call may have left them
        assert emu.emu_selftest_i8_timeout(2000, G, rows, N, K, X.data_ptr(), rows, K, None, took.data_ptr(), W.data_ptr(), K,
                                           N * K, None, ends.data_ptr(), Y.data_ptr(), emu.I32, N, ws.data_ptr(), ws.numel(),
                                           emu._stream(None)) == 0
        assert emu.read_flags(ws) == emu.FLAG_TIMEOUT | flags
        assert bool((Y[:rows - 2] == 5).all()) and not Y[rows - 2:].any()
    emu.i8_gemm((X, None), (W, None), ends=ends, src=src, Y=Y, ws=ws)
    assert emu.read_flags(ws) == 0 and torch.equal(Y, want)
    emu.i8_gemm((X, None), (W, None), ends=ends, src=bad, Y=Y, ws=ws)
    assert emu.read_flags(ws) == emu.FLAG_INDEX
