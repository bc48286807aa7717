"""The expert-layer entry points reject bad arguments on the host, before any
CUDA call: status codes of the C entry points, ValueError of the tensor calls."""
import os
import re

import pytest

import paper_2609_04663_gb300 as emu
from paper_2609_04663_gb300 import _build


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return emu.load()


def test_every_declared_symbol_is_exported_and_bound(lib):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "emu_experts.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(emu_[a-z0-9_]+)\s*\(", text))
    assert len(names) >= 14
    for name in names:
        assert hasattr(lib, name) and name in emu._SIGS, name


def test_argument_checks_need_no_gpu(lib):
    P, big = 16, 1 << 40
    # products grouped by expert
    assert emu.emu_grouped_plane_rows(100, 3) % 16 == 0 and emu.emu_grouped_plane_rows(100, 3) >= 100 + 3 * 15
    g = emu.emu_grouped_prodsum
    #        S  op G  rows N  K  X  ldx pad W  ldw stride ends Y yt ldy ws bytes stream
    assert g(2, 0, 2, 8, 8, 8, P, 8, 0, P, 8, 64, P, P, 0, 8, P, 512, None) == 1      # slices
    assert g(1, 2, 2, 8, 8, 8, P, 8, 0, P, 8, 64, P, P, 0, 8, P, 512, None) == 1      # op
    assert g(1, 0, 0, 8, 8, 8, P, 8, 0, P, 8, 64, P, P, 0, 8, P, 512, None) == 1      # no groups
    assert g(1, 0, 2, 8, 8, 8, P, 8, 0, P, 8, 64, P, P, 0, 7, P, 512, None) == 1      # ldy < N
    assert g(1, 0, 2, 8, 8, 8, P, 8, 0, P, 8, 64, None, P, 0, 8, P, 512, None) == 1   # no ends
    assert g(3, 0, 2, 8, 8, 8, P, 8, 0, P, 8, 72, P, P, 0, 8, P, 512, None) == 1      # slices of weights not dense
    assert g(1, 0, 2, 8, 8, 8, P, 9, 0, P, 8, 64, P, P, 0, 8, P, 512, None) == 2      # row pitch of X
    assert g(1, 0, 2, 8, 8, 8, P, 8, 0, P + 2, 8, 64, P, P, 0, 8, P, 512, None) == 2  # base of W
    assert g(1, 0, 2, 8, 8, 8, P, 8, 0, P, 8, 64, P, P, 0, 8, P, 511, None) == 3      # workspace
    assert g(1, 0, 1025, 8, 8, 8, P, 8, 0, P, 8, 64, P, P, 0, 8, P, 512, None) == 5   # groups
    assert emu.emu_grouped_gemm_f32(0, 2, 8, 8, 8, P, 4, 8, None, P, 8, 64, P, P, 8, P, big, None) == 1   # xrows < rows
    assert emu.emu_grouped_gemm_f32(0, 2, 8, 8, 8, P, 8, 8, None, P, 8, 64, P, P, 8, P, 512, None) == 3
    assert emu.emu_grouped_prodsum_wgrad(1, 2, 8, 8, 8, P, 8, 0, P, 8, 0, P, P, 0, 8, 63, P, 512, None) == 1    # matrices overlap
    assert emu.emu_grouped_prodsum_wgrad(1, 2, 8, 8, 8, P, 12, 0, P, 8, 0, P, P, 0, 8, 64, P, 512, None) == 2
    assert emu.emu_grouped_prodsum_wgrad(3, 2, 8, 8, 8, P, 8, 1, P, 8, 0, P, P, 0, 8, 64, P, 512, None) == 1    # slices at padded rows only
    assert emu.emu_grouped_split(2, 2, 8, 8, P, 8, 64, P, 8, P, 512, None) == 1                          # type
    assert emu.emu_grouped_split(0, 2, 8, 9, P, 9, 72, P, 12, P, 512, None) == 2                         # plane pitch
    assert emu.emu_grouped_split_rows(0, 8, 8, P, 7, 8, None, P, 2, P, 8, P, 512, None) == 1
    # 4-bit weights
    w = emu.emu_w4_matvec
    assert w(0, 1, 1, 8, 64, 48, P, 64, P, P, 0, None, None, P, 8, P, 1 << 20, None) == 1         # group does not divide K
    assert w(0, 1, 1, 8, 64, 16, P, 64, P, P, 0, None, None, P, 8, P, 1 << 20, None) == 1         # group not a multiple of 32
    assert w(0, 2, 1, 8, 64, 32, P, 64, P, P, 0, None, None, P, 8, P, 1 << 20, None) == 1         # groups without ends
    assert w(0, 1, 1, 8, 64, 32, P, 64, P + 4, P, 0, None, None, P, 8, P, 1 << 20, None) == 2
    assert w(0, 1, 1, 8, 64, 32, P, 63, P, P, 0, None, None, P, 8, P, 1 << 20, None) == 1
    assert w(0, 1, 2, 8, 64, 32, P, 64, P, P, 0, None, None, P, 8, P, 767, None) == 3          # room for two rows' slices
    assert w(0, 1, 2, 8, 64, 32, P, 64, P, P, 0, None, None, P, 8, None, 0, None) == 1
    assert w(0, 1, 2, 8, 64, 32, P, 64, P, P, 0, None, P + 2, P, 8, P, 1 << 20, None) == 2      # address of ends
    assert w(1, 1, 131071, 8, 64, 32, P, 64, P, P, 1, None, None, P, 8, None, 0, None) == 5    # rows
    # routing
    assert emu.emu_route(0, 4, 8, 9, 1, P, 8, P, P, P, P, P, P, big, None) == 1       # k > E
    assert emu.emu_route(0, 4, 2000, 2, 1, P, 2000, P, P, P, P, P, P, big, None) == 5
    assert emu.emu_route(0, 4, 8, 2, 1, P, 8, P, P, P, P, P, P, 512, None) == 3
    assert emu.emu_route(0, 1 << 30, 8, 2, 1, P, 8, P, P, P, P, P, P, big, None) == 5
    assert emu.emu_route_backward(0, 4, 8, 2, 1, P, 8, P, P, P, 7, None) == 1
    assert emu.emu_rows_combine(0, 4, 2, 8, P, 8, 7, P, P, P, 8, None) == 1
    assert emu.emu_rows_combine_backward(3, 4, 2, 8, P, 8, P, 8, 8, P, P, P, 8, P, None) == 1


def test_tensor_checks_need_no_gpu():
    import torch
    X, W = torch.zeros(4, 8), torch.zeros(2, 8, 16)
    ends = torch.tensor([2, 4], dtype=torch.int32)
    for bad in (lambda: emu.grouped_gemm(X, W, ends),                                  # not on a GPU
                lambda: emu.grouped_gemm(X, W[:1], ends),
                lambda: emu.grouped_gemm(torch.zeros(4, 9), W, ends),
                lambda: emu.grouped_gemm(X.bfloat16(), W, ends),
                lambda: emu.grouped_gemm(X.half(), W.half(), ends),
                lambda: emu.grouped_split(X),
                lambda: emu.grouped_split(X.double(), ends),
                lambda: emu.w4_matvec(X, torch.zeros(16, 4, dtype=torch.uint8), torch.zeros(16, 1)),
                lambda: emu.route(X.half(), 2),
                lambda: emu.rows_combine(X.half(), ends.view(1, 2))):
        with pytest.raises(ValueError):
            bad()
