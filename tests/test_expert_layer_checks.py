"""Arguments that the expert-layer calls have to reject on the host, before any CUDA call."""
import pytest

import paper_2609_04663_gb300 as emu
from paper_2609_04663_gb300 import _build


@pytest.fixture(scope="module", autouse=True)
def lib():
    _build.build()
    return emu.load()


def test_gradients_of_all_answer_rows():
    P, f = 16, emu.emu_rows_combine_backward_full
    assert emu.emu_rows_combine_workspace_bytes(100) >= 400
    #        type T k cols dO ldo Y yrows ldy slots w dY lddy dw ws bytes stream
    assert f(3, 4, 2, 8, P, 8, P, 8, 8, P, P, P, 8, P, P, 32, None) == 1
    assert f(0, 4, 2, 8, P, 7, P, 8, 8, P, P, P, 8, P, P, 32, None) == 1
    assert f(0, 4, 2, 8, P, 8, P, 8, 8, P, P, P, 8, P, None, 32, None) == 1
    assert f(0, 4, 2, 8, P, 8, P, 8, 8, P, P, P, 8, P, P, 31, None) == 3
    assert f(0, 4, 2, 8, P, 8, P, 8, 8, P, P, P, 8, P, P + 4, 32, None) == 2
    assert f(0, 0, 2, 8, None, 8, P, 8, 8, None, None, None, 8, None, P, 32, None) == 1     # rows to clear
    assert f(0, 0, 2, 8, None, 8, P, 8, 8, None, None, P + 1, 8, None, P, 32, None) == 2
    assert f(0, 0, 2, 8, None, 8, P, 0, 8, None, None, None, 8, None, None, 0, None) == 0


def test_keep_flags_changes_no_check():
    P, K = 16, emu.KEEP_FLAGS
    g = emu.emu_grouped_prodsum
    for S in (2, 0, 4):
        assert g(S | K, 0, 2, 8, 8, 8, P, 8, 0, P, 8, 64, P, P, 0, 8, P, 512, None) == 1
    assert g(1 | K | 0x200, 0, 2, 8, 8, 8, P, 8, 0, P, 8, 64, P, P, 0, 8, P, 512, None) == 1
    assert g(-1, 0, 2, 8, 8, 8, P, 8, 0, P, 8, 64, P, P, 0, 8, P, 512, None) == 1
    assert g(1 | K, 0, 2, 8, 8, 8, P, 8, 0, P, 8, 64, P, P, 0, 8, P, 511, None) == 3
    assert emu.emu_grouped_prodsum_wgrad(3 | K, 2, 8, 8, 8, P, 8, 1, P, 8, 0, P, P, 0, 8, 64, P, 512, None) == 1
    assert emu.emu_grouped_split(2 | K, 2, 8, 8, P, 8, 64, P, 8, P, 512, None) == 1
    assert emu.emu_grouped_split_rows(0 | K, 8, 8, P, 7, 8, None, P, 2, P, 8, P, 512, None) == 1


def test_routing_self_test_arguments():
    P, f = 16, emu.emu_selftest_route_timeout
    for us, T in ((0, 64), (1000001, 64), (1000, 32), (1000, -1)):
        assert f(us, T, 8, 2, P, 8, P, P, P, P, P, P, 1 << 30, None) == 1
    assert f(1000, 64, 8, 2, P, 8, P, P, P, P, P, P, 512, None) == 3
    assert f(1000, 64, 8, 2, P, 8, P, P, P, P + 2, P, P, 1 << 30, None) == 2


def _planes(S, rows, cols, G, plane_rows=None):
    import torch
    n = emu.emu_grouped_plane_rows(rows, G) if plane_rows is None else plane_rows
    return emu.GroupedPlanes(torch.zeros((S, n, emu.gemm_ldk(cols)), dtype=torch.int16), (rows, cols), True)


@pytest.mark.parametrize("made,used", [(4, 512), (512, 4), (1, 2)])
def test_planes_of_token_rows_belong_to_a_number_of_groups(made, used):
    """Rows padded for other groups lie elsewhere, and a plane set made for fewer
    of them ends before the rows that the kernels would read."""
    import torch
    ends = torch.zeros(used, dtype=torch.int32)
    for S, dt in ((3, torch.float32), (1, torch.bfloat16)):
        X, W, B = _planes(S, 40, 24, made), torch.zeros((used, 24, 16), dtype=dt), _planes(S, 40, 16, used)
        for call in (lambda: emu.grouped_gemm(X, W, ends), lambda: emu.grouped_wgrad(X, B, ends),
                     lambda: emu.grouped_wgrad(B, X, ends)):
            with pytest.raises(ValueError, match=f"{used} groups"):
                call()


def test_planes_of_weights_are_whole():
    import torch
    ends = torch.zeros(3, dtype=torch.int32)
    W = emu.GroupedPlanes(torch.zeros((3, 2 * 24, 16), dtype=torch.int16), (3, 24, 16), False)
    with pytest.raises(ValueError, match="3 groups"):
        emu.grouped_gemm(_planes(3, 40, 24, 3), W, ends)


@pytest.mark.parametrize("near", [1, 60, 65535])
def test_sizes_next_to_2_31_are_refused(near):
    """Kernels step over tokens, rows and contractions with 32-bit numbers, by whole
    tiles and shares of a block: a size closer to 2^31 than those would wrap."""
    P, n = 16, 2 ** 31 - near
    assert emu.emu_route(1, n, 1, 1, 1, P, 1, P, P, P, P, P, P, 1 << 40, None) == 5
    assert emu.emu_route(0, n // 2 + 1, 2, 2, 1, P, 2, P, P, P, P, P, P, 1 << 40, None) == 5
    assert emu.emu_selftest_route_timeout(1000, n, 1, 1, P, 1, P, P, P, P, P, P, 1 << 40, None) == 5
    n8 = n // 32 * 32                       # a contraction of whole scale groups
    assert emu.emu_w4_matvec(1, 1, 1, 1, n8, 32, P, n8, P, P, 1, None, None, P, 1, None, 0, None) == 5
    for N, K in ((n, 8), (8, n)):
        assert emu.emu_grouped_prodsum(1, 1, 1, 8, N, K, P, 1 << 32, 0, P, 1 << 32, 0, P, P, 1, N, P, 512, None) == 5
        assert emu.emu_grouped_prodsum_wgrad(1, 1, 8, N, K, P, 1 << 32, 0, P, 1 << 32, 0, P, P, 1, K, 0, P, 512, None) == 5
        assert emu.emu_grouped_gemm_f32(1, 1, 8, N, K, P, 8, K, None, P, K, 0, P, P, N, P, 1 << 62, None) == 5


def test_a_training_steps_workspace_is_enough_for_every_call():
    import torch
    ends = torch.zeros(3, dtype=torch.int32)
    for dt, code in ((torch.float32, emu.F32), (torch.bfloat16, emu.BF16)):
        for K, N in ((24, 200), (200, 24)):
            need = max(emu.emu_grouped_gemm_workspace_bytes(code, 3, 60, *s) for s in ((N, K), (K, N)))
            for W, op in ((torch.zeros(3, K, N, dtype=dt), emu.OP_N), (torch.zeros(3, N, K, dtype=dt), emu.OP_T)):
                X = torch.zeros(60, K, dtype=dt)
                assert emu.grouped_workspace(X, W, ends, op, train=True).numel() >= need
                assert emu.grouped_workspace(X, W, ends, op).numel() >= emu.emu_grouped_gemm_workspace_bytes(code, 3, 60, N, K)


def test_4_bit_workspaces():
    P, w = 16, emu.emu_w4_matvec
    need = emu.emu_w4_workspace_bytes(emu.F32, 2, 64)
    assert need >= emu.emu_split_workspace_bytes(32) + 2 * 64 * 6
    assert w(0, 1, 2, 8, 64, 32, P, 64, P, P, 0, None, None, P, 8, P, need - 1, None) == 3
    assert w(0, 1, 2, 8, 64, 32, P, 64, P, P, 0, None, None, P, 8, P + 8, need, None) == 2
    assert w(1, 1, 2, 8, 64, 32, P, 64, P, P, 1, None, None, P, 8, P, 511, None) == 3            # no room for the flags
    assert w(1, 1, 2, 8, 64, 32, P + 2, 64, P, P, 1, None, None, P, 8, P, 512, None) == 3        # rows that need slices
