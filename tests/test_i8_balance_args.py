"""The 8-bit and balance entry points reject bad arguments on the host, before any CUDA
call: status codes of the C entry points, ValueError of the tensor calls."""
import pytest

import paper_2609_04663_gb300 as emu
from paper_2609_04663_gb300 import _build


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return emu.load()


P, BIG = 16, 1 << 40


def test_quantise_checks(lib):
    q = emu.emu_i8_quantize
    #        dt G rows cols X ldx sx  codes ldq sq scales ws bytes stream
    assert q(2, 1, 4, 8, P, 8, 0, P, 8, 0, P, None, 0, None) == 1             # type
    assert q(0, 0, 4, 8, P, 8, 0, P, 8, 0, P, None, 0, None) == 1             # no matrices
    assert q(0, 1, 4, 8, P, 7, 0, P, 8, 0, P, None, 0, None) == 1             # ldx < cols
    assert q(0, 1, 4, 8, P, 8, 0, P, 7, 0, P, None, 0, None) == 1             # ldq < cols
    assert q(0, 2, 4, 8, P, 8, 32, P, 8, 31, P, None, 0, None) == 1           # results overlap
    assert q(0, 1, 4, 8, P, 8, 0, P, 8, 0, None, None, 0, None) == 1          # no scales
    assert q(0, 1, 4, 8, None, 8, 0, P, 8, 0, P, None, 0, None) == 1
    assert q(0, 1, 4, 8, P + 2, 8, 0, P, 8, 0, P, None, 0, None) == 2         # FP32 on 2 bytes
    assert q(1, 1, 4, 8, P + 1, 8, 0, P, 8, 0, P, None, 0, None) == 2
    assert q(0, 1, 4, 8, P, 8, 0, P, 8, 0, P + 2, None, 0, None) == 2
    assert q(0, 1, 4, 8, P, 8, 0, P, 8, 0, P, P, 511, None) == 3
    assert q(0, 1, 4, 8, P, 8, 0, P, 8, 0, P, P + 8, 512, None) == 2
    assert q(0, 1 << 20, 1 << 20, 8, P, 8, 1 << 23, P, 8, 1 << 23, P, None, 0, None) == 5
    assert q(0, 1, 4, 1 << 31, P, 1 << 31, 0, P, 1 << 31, 0, P, None, 0, None) == 5


def test_product_checks(lib):
    g = emu.emu_i8_gemm
    #        G rows N  K  X xrows ldx xs src W ldw sw  ws  ends Y  yt ldy ws bytes stream
    assert g(1, 4, 8, 16, P, 4, 16, P, None, P, 16, 0, P, None, P, 3, 8, P, BIG, None) == 1       # type
    assert g(1, 4, 8, 16, P, 3, 16, P, None, P, 16, 0, P, None, P, 0, 8, P, BIG, None) == 1       # xrows < rows
    assert g(1, 4, 8, 16, P, 4, 15, P, None, P, 16, 0, P, None, P, 0, 8, P, BIG, None) == 1       # ldx < K
    assert g(1, 4, 8, 16, P, 4, 16, P, None, P, 15, 0, P, None, P, 0, 8, P, BIG, None) == 1       # ldw < K
    assert g(1, 4, 8, 16, P, 4, 16, P, None, P, 16, 0, P, None, P, 0, 7, P, BIG, None) == 1       # ldy < N
    assert g(2, 4, 8, 16, P, 4, 16, P, None, P, 16, 128, P, None, P, 0, 8, P, BIG, None) == 1     # groups without ends
    assert g(2, 4, 8, 16, P, 4, 16, P, None, P, 16, -1, P, P, P, 0, 8, P, BIG, None) == 1
    assert g(0, 4, 8, 16, P, 4, 16, P, None, P, 16, 0, P, P, P, 0, 8, P, BIG, None) == 1
    assert g(1, 4, 8, 16, P, 4, 16, P, None, P, 16, 0, None, None, P, 2, 8, P, BIG, None) == 1    # sums with scales
    assert g(1, 4, 8, 16, P, 4, 16, P, None, None, 16, 0, P, None, P, 0, 8, P, BIG, None) == 1    # no weights
    assert g(1, 4, 8, 16, P, 4, 16, P, None, P, 16, 0, P, None, None, 0, 8, P, BIG, None) == 1    # no result
    assert g(1, 4, 8, 16, P, 4, 16, P + 2, None, P, 16, 0, P, None, P, 0, 8, P, BIG, None) == 2
    assert g(1, 4, 8, 16, P, 4, 16, P, P + 1, P, 16, 0, P, None, P, 0, 8, P, BIG, None) == 2
    assert g(1, 4, 8, 16, P, 4, 16, P, None, P, 16, 0, P, None, P + 2, 0, 8, P, BIG, None) == 2
    assert g(1, 40, 8, 16, P, 40, 16, P, None, P + 8, 16, 0, P, None, P, 0, 8, None, 0, None) == 1    # weights are copied
    assert g(1, 40, 8, 16, P, 40, 16, P, None, P + 8, 16, 0, P, None, P, 0, 8, P, 512, None) == 3
    assert g(1, 40, 8, 16, P + 8, 40, 16, P, None, P, 16, 0, P, None, P, 0, 8, None, 0, None) == 1    # rows are copied
    assert g(1, 4000, 4000, 16, P, 4000, 16, P, None, P, 16, 0, P, None, P, 0, 4000, None, 0, None) == 1    # rows as FP16
    assert g(1, 4, 8, 16, P, 4, 16, P, None, P, 16, 0, P, None, P, 0, 8, P, 511, None) == 3       # a few: for the flags
    assert g(1, 4, 8, 16, P, 4, 16, P, None, P, 16, 0, P, None, P, 0, 8, P + 8, BIG, None) == 2
    assert g(1, 4, 8, 131072, P, 4, 131072, P, None, P, 131072, 0, P, None, P, 0, 8, P, BIG, None) == 5    # sums past 32 bits
    assert g(1025, 4, 8, 16, P, 4, 16, P, None, P, 16, 128, P, P, P, 0, 8, P, BIG, None) == 5
    assert g(1, 1 << 31, 8, 16, P, 1 << 31, 16, P, None, P, 16, 0, P, None, P, 0, 8, P, BIG, None) == 5
    assert emu.emu_i8_gemm_workspace_bytes(0, 4, 8, 16, 1) == 0
    assert emu.emu_i8_gemm_workspace_bytes(2, 1, 8, 16, 1) == 0 and emu.emu_i8_gemm_workspace_bytes(2, 100, 8, 16, 0) >= 512
    assert emu.emu_i8_gemm_workspace_bytes(2, 100, 8, 16, 1) == 0 and emu.emu_i8_gemm_workspace_bytes(1, 4000, 4000, 16, 1) >= 512


def test_balance_checks(lib):
    b, d = emu.emu_route_balance, emu.emu_route_balance_backward
    need = emu.emu_route_balance_workspace_bytes(1 << 20, 8)
    assert emu.emu_route_balance_workspace_bytes(4, 0) == 0 and emu.emu_route_balance_workspace_bytes(4, 8) == 0 and need > 512
    #        dt T  E  k  z  ldl ex mask coef loss counts tokens ws bytes stream
    assert b(2, 4, 8, 2, P, 8, P, None, 1.0, P, P, P, P, need, None) == 1
    assert b(0, 4, 8, 9, P, 8, P, None, 1.0, P, P, P, P, need, None) == 1        # k > E
    assert b(0, 4, 8, 0, P, 8, P, None, 1.0, P, P, P, P, need, None) == 1
    assert b(0, 4, 8, 2, P, 7, P, None, 1.0, P, P, P, P, need, None) == 1        # ldl < E
    assert b(0, 4, 8, 2, P, 8, None, None, 1.0, P, P, P, P, need, None) == 1     # no experts
    assert b(0, 4, 8, 2, P, 8, P, None, 1.0, None, P, P, P, need, None) == 1
    assert b(0, 4, 8, 2, P, 8, P, None, 1.0, P, None, P, P, need, None) == 1
    assert b(0, 4, 8, 2, P, 8, P, None, 1.0, P, P, None, P, need, None) == 1
    assert b(0, 4, 8, 2, P + 2, 8, P, None, 1.0, P, P, P, P, need, None) == 2
    assert b(0, 4, 8, 2, P, 8, P, None, 1.0, P, P + 2, P, P, need, None) == 2
    assert b(0, 1 << 20, 8, 2, P, 8, P, None, 1.0, P, P, P, P, need - 1, None) == 3
    assert b(0, 1 << 20, 8, 2, P, 8, P, None, 1.0, P, P, P, None, 0, None) == 1
    assert b(0, 4, 8, 2, P, 8, P, None, 1.0, P, P, P, P, 511, None) == 3
    assert b(0, 4, 8, 2, P, 8, P, None, 1.0, P, P, P, P + 8, need, None) == 2
    assert b(0, 4, 2000, 2, P, 2000, P, None, 1.0, P, P, P, P, BIG, None) == 5
    assert b(0, 4, 64, 33, P, 64, P, None, 1.0, P, P, P, P, BIG, None) == 5
    assert b(0, 1 << 30, 8, 2, P, 8, P, None, 1.0, P, P, P, P, need, None) == 5
    #        dt T  E  k  z  ldl counts tokens mask coef dloss add lda d ldd stream
    assert d(0, 4, 8, 2, P, 8, P, P, None, 1.0, None, None, 0, P, 7, None) == 1
    assert d(0, 4, 8, 2, P, 8, P, P, None, 1.0, None, P + 64, 7, P, 8, None) == 1
    assert d(0, 4, 8, 2, P, 8, P, P, None, 1.0, None, P, 9, P, 8, None) == 1     # in place with another pitch
    assert d(0, 4, 8, 2, P, 8, None, P, None, 1.0, None, None, 0, P, 8, None) == 1
    assert d(0, 4, 8, 2, P, 8, P, P, None, 1.0, None, None, 0, None, 8, None) == 1
    assert d(0, 4, 8, 2, P, 8, P, P, None, 1.0, P + 1, None, 0, P, 8, None) == 2
    assert d(0, 0, 8, 2, None, 8, P, P, None, 1.0, None, None, 0, None, 8, None) == 0


def test_tensor_checks_need_no_gpu(lib):
    import torch
    x, w = torch.zeros(4, 16, dtype=torch.int8), torch.zeros(2, 8, 16, dtype=torch.int8)
    xs, ws, ends = torch.zeros(4), torch.zeros(2, 8), torch.tensor([2, 4], dtype=torch.int32)
    z, e = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32)
    for bad in (lambda: emu.i8_quantize(torch.zeros(4, 8)),                            # not on a GPU
                lambda: emu.i8_quantize(torch.zeros(4, 8).half()),
                lambda: emu.i8_quantize(torch.zeros(8)),
                lambda: emu.i8_gemm((x, xs), (w, ws), ends=ends),
                lambda: emu.i8_gemm((x.float(), xs), (w, ws), ends=ends),
                lambda: emu.i8_gemm((x, xs), (w, ws)),
                lambda: emu.route_balance(z, e),
                lambda: emu.route_balance(z.half(), e),
                lambda: emu.route_balance(z, e[:3])):
        with pytest.raises(ValueError):
            bad()
