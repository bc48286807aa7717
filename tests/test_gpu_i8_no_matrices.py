"""Quantising no matrices at all reports its flags like any other call."""
import pytest
import torch

import paper_2609_04663_gb300 as emu
from helpers import device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(0, 5, 40), (0, 0, 40), (3, 0, 40), (0, 40), (0, 5, 0)])
def test_flags_of_an_empty_call(shape):
    dev = device()
    ws = emu.workspace(emu.emu_split_workspace_bytes(32), dev)
    bad = torch.full((2, 8), float("nan"), device=dev)
    emu.i8_quantize(bad, ws=ws)
    assert emu.read_flags(ws) == emu.FLAG_NONFINITE
    q = emu.i8_quantize(torch.empty(shape, device=dev), ws=ws)
    assert q.codes.shape == shape and q.scales.shape == shape[:-1]
    assert emu.read_flags(ws) == 0
