"""Routing whose blocks wait for one that never comes: the wait ends, the call
reports it, nothing is placed, and the next call is right."""
import pytest

import paper_2609_04663_gb300 as emu
from helpers import device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,E,k", [(33, 8, 2), (5000, 64, 4), (300, 1024, 8)])
def test_a_barrier_that_runs_out_places_nothing(T, E, k):
    import torch
    dev = device()
    g = torch.Generator(device=dev).manual_seed(1)
    x = torch.randn((T, E), generator=g, device=dev)
    want, _ = emu.route(x, k)
    # counts as an earlier call may have left them: far out of range
    ws = torch.full((emu.emu_route_workspace_bytes(T, E, k),), 0x7F, dtype=torch.uint8, device=dev)
    weights = torch.empty((T, k), device=dev)
    experts, slots, rows = (torch.full((T * k,), -7, dtype=torch.int32, device=dev) for _ in range(3))
    ends = torch.full((E,), -7, dtype=torch.int32, device=dev)
    call = (T, E, k, x.data_ptr(), E, weights.data_ptr(), experts.data_ptr(), slots.data_ptr(), rows.data_ptr(),
            ends.data_ptr(), ws.data_ptr(), ws.numel(), emu._stream(None))
    assert emu.emu_selftest_route_timeout(2000, *call) == 0
    assert emu.read_flags(ws) == emu.FLAG_TIMEOUT
    for t in (slots, rows, ends):
        assert bool((t == -7).all())
    assert torch.equal(experts.view(T, k), want.experts) and torch.equal(weights, want.weights)
    r, ws = emu.route(x, k, ws=ws)
    assert emu.read_flags(ws) == 0
    assert all(torch.equal(a, b) for a, b in zip(r, want))
