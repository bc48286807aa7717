"""The routing's balance loss, its counts and its gradient against the formulas in 64
bits and against differences.

Bounds.  A probability: the difference to the largest logit is rounded (2^-24 of at most
the logits' range R, an error of R 2^-24 relative in the exponential), expf is off by 2 units
(2^-22), the sum of E positive terms by at most 32 + 5 additions in a row, then a reciprocal and a
product: (R + 4 + 37 + 2) 2^-24 < (R + 43) 2^-24 relative.  Their sum over T tokens, all positive:
at most T / 32 + 32 + 152 additions in a row (one warp has every 32nd token at most,
32 warps, 152 blocks).  The loss: three factors and a sum over E in at most 32 + 5 + 32 additions.
So its relative error is below (R + T / 32 + 300) 2^-24.  The gradient: p (f - S), S = sum p f
with relative errors of f and p as above and E / 8 + 5 additions: an error of at most
(2 R + 200) 2^-24 of scale p (f + S), and the rounding of the sum with `add` to the result's type."""
import pytest
import torch

import paper_2609_04663_gb300 as emu
from helpers import device

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def dev():
    return device()


def case(dev, T, E, k, dtype, masked, seed=0, scale=1.5):
    g = torch.Generator(device=dev).manual_seed(seed + T + 31 * E + k)
    z = (torch.randn(T, E, generator=g, device=dev) * scale + torch.randn(1, E, generator=g, device=dev)).to(dtype)
    experts = torch.rand(T, E, generator=g, device=dev).topk(k, dim=1).indices.int().contiguous()
    mask = (torch.rand(T, generator=g, device=dev) < 0.6) if masked else None
    add = torch.randn(T, E, generator=g, device=dev).mul_(1e-3 / max(T, 1)).to(dtype)
    return z, experts, mask, add


def formula(z, experts, mask, coef):
    """(loss, counts, n, p, f) in 64 bits."""
    T, E = z.shape
    on = mask if mask is not None else torch.ones(T, dtype=torch.bool, device=z.device)
    n, k = int(on.sum()), experts.shape[1]
    good = experts[on]
    counts = torch.bincount(good[(good >= 0) & (good < E)].reshape(-1).long(), minlength=E)
    x = z.double()
    p = torch.softmax(torch.where(x.isnan(), -float("inf"), x), 1).nan_to_num(0.0)
    p = p * on[:, None]
    f = counts.double() * (coef * E / (max(n, 1) * k))
    return (f * p.sum(0)).sum() / max(n, 1), counts, n, p, f


def space(T, E, dev):
    return emu.workspace(max(emu.emu_route_balance_workspace_bytes(T, E), emu.emu_split_workspace_bytes(32)), dev)


def check(z, experts, mask, add, coef=0.01, dloss=None, flags=0):
    loss, counts, n, p, f = formula(z, experts, mask, coef)
    finite = z[z.isfinite()].double()
    R = float(finite.max() - finite.min()) if finite.numel() else 0.0
    ws = space(*z.shape, z.device)
    b, _ = emu.route_balance(z, experts, coef=coef, mask=mask, ws=ws)
    assert emu.read_flags(ws) == flags
    assert torch.equal(b.loss, emu.route_balance(z, experts, coef=coef, mask=mask)[0].loss)
    assert torch.equal(b.counts.long(), counts) and int(b.tokens) == n
    assert abs(float(b.loss) - float(loss)) <= (R + z.shape[0] / 32 + 300) * U * float(loss)
    scale = (1.0 if dloss is None else float(dloss)) / max(n, 1)
    S = (p * f).sum(1, keepdim=True)
    grad = scale * p * (f - S)
    room = abs(scale) * p * (f + S) * (2 * R + 200) * U
    half = torch.finfo(z.dtype).eps / 2
    for extra in (None, add):
        d = emu.route_balance_backward(z, b, dloss=dloss, coef=coef, mask=mask, add=extra)
        want = grad if extra is None else grad + extra.double()
        assert d.dtype is z.dtype
        # (a result below the smallest normal number is rounded to a multiple of 2^-149, BF16's of 2^-133)
        least = 2.0 ** -149 if z.dtype is torch.float32 else 2.0 ** -133
        bound = room * (1 + half) + want.abs() * (half + U) + (extra.double().abs() * U if extra is not None else 0) + least
        assert bool(((d.double() - want).abs() <= bound).all())
    same = add.clone()
    assert torch.equal(emu.route_balance_backward(z, b, dloss=dloss, coef=coef, mask=mask, add=same, dlogits=same), d)
    return b


SIZES = [(1, 1, 1), (1, 8, 2), (2, 4, 4), (5, 7, 3), (64, 64, 4), (100, 33, 5), (129, 60, 6), (1000, 128, 8), (700, 130, 2),
         (333, 256, 8), (300, 500, 16), (200, 1024, 32), (65, 1023, 9), (4096, 128, 8), (4097, 128, 8), (2049, 200, 3), (600, 700, 4), (5003, 60, 6), (20000, 16, 2), (3000, 512, 1)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("T,E,k", SIZES)
def test_loss_counts_and_gradient(dev, T, E, k, masked, dtype):
    check(*case(dev, T, E, k, dtype, masked), dloss=torch.tensor(-1.75, device=dev))


def test_an_even_routing_has_loss_coef(dev):
    T, E = 512, 64
    z = torch.zeros(T, E, device=dev)
    experts = (torch.arange(T * 4, device=dev).view(T, 4) % E).int()
    b, _ = emu.route_balance(z, experts, coef=0.5)
    assert float(b.loss) == 0.5 and bool((b.counts == T * 4 // E).all())
    d = emu.route_balance_backward(z, b, coef=0.5)
    assert not d.any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_tokens_and_none_that_count(dev, dtype):
    z, experts, _, add = case(dev, 40, 12, 3, dtype, False)
    off = torch.zeros(40, dtype=torch.bool, device=dev)
    b = check(z, experts, off, add)
    assert float(b.loss) == 0.0 and int(b.tokens) == 0 and not b.counts.any()
    assert torch.equal(emu.route_balance_backward(z, b, mask=off, add=add), add)
    assert not emu.route_balance_backward(z, b, mask=off).any()
    b, _ = emu.route_balance(z[:0], experts[:0])
    assert float(b.loss) == 0.0 and not b.counts.any()
    assert emu.route_balance_backward(z[:0], b).shape == (0, 12)


def test_logits_that_are_not_finite(dev):
    inf, nan = float("inf"), float("nan")
    z, experts, _, add = case(dev, 50, 20, 2, torch.float32, False)
    z[3, :19] = -inf                                          # one expert left
    z[4] = -inf                                               # none
    z[5, 2:9] = -inf
    check(z, experts, None, add)
    z[6, 4] = nan                                             # as minus infinity, and flagged
    check(z, experts, None, add, flags=emu.FLAG_NONFINITE)
    # in tokens that do not count, anything goes
    mask = torch.ones(50, dtype=torch.uint8, device=dev)
    mask[6:8] = 0
    z[7], z[6, 5] = nan, inf
    zc = z.clone()
    zc[6:8] = 0
    ws = space(*z.shape, dev)
    a, _ = emu.route_balance(z, experts, mask=mask, ws=ws)
    assert emu.read_flags(ws) == 0
    c, _ = emu.route_balance(zc, experts, mask=mask)
    assert torch.equal(a.loss, c.loss)
    assert torch.equal(emu.route_balance_backward(z, a, mask=mask, add=add), emu.route_balance_backward(zc, c, mask=mask, add=add))
    # plus infinity in one that does: flagged, its own row alone is lost in the gradient
    z[7], z[6], z[9, 1] = 0, 0, inf
    a, _ = emu.route_balance(z, experts, ws=ws)
    assert emu.read_flags(ws) == emu.FLAG_NONFINITE
    d = emu.route_balance_backward(z, a)
    assert bool(d[9].isnan().any()) and bool(d[[i for i in range(50) if i != 9]].isfinite().all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_logits_of_the_largest_magnitudes(dev, dtype):
    # masks of the type's lowest value: as minus infinity beside others, and an even row where there are no others
    lowest, largest = torch.finfo(dtype).min, torch.finfo(dtype).max
    z, experts, _, add = case(dev, 5000, 20, 2, dtype, False)
    same = z.clone()
    z[3, :19], same[3, :19] = lowest, -float("inf")
    z[4], same[4] = lowest, 0
    z[5, 2:9], same[5, 2:9] = lowest, -float("inf")
    z[6, 4], same[6], same[6, 4] = largest, -float("inf"), 0
    z[7], same[7] = largest, 0
    z[8], same[8], same[8, :3] = lowest, -float("inf"), 0
    z[8, :3] = largest
    for T in (50, 5000):
        a, _ = emu.route_balance(z[:T], experts[:T])
        b, _ = emu.route_balance(same[:T], experts[:T])
        assert bool(b.loss.isfinite()) and torch.equal(a.loss, b.loss) and torch.equal(a.counts, b.counts)
        assert torch.equal(emu.route_balance_backward(z[:T], a, add=add[:T]), emu.route_balance_backward(same[:T], b, add=add[:T]))


@pytest.mark.parametrize("T", [30, 6000])
def test_entries_outside_are_not_counted(dev, T):
    z, experts, mask, add = case(dev, T, 24, 4, torch.float32, True)
    experts[2, 1], experts[T - 1, 3], experts[T // 2, 0] = -1, 24, -2 ** 31
    mask[[2, T - 1, T // 2]] = True
    check(z, experts, mask, add, flags=emu.FLAG_INDEX)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_pitches_and_alignments(dev, dtype):
    z, experts, mask, add = case(dev, 300, 64, 4, dtype, True)
    b, _ = emu.route_balance(z, experts, mask=mask)
    d = emu.route_balance_backward(z, b, mask=mask, add=add)
    for left, pitch in ((4, 72), (1, 67), (2, 70), (0, 65)):
        wide = torch.full((300, pitch), 9.0, device=dev, dtype=dtype)
        zz, aa, out = wide.clone(), wide.clone(), wide.clone()
        for t, v in ((zz, z), (aa, add)):
            t[:, left:left + 64] = v
        zz, aa, o = (t[:, left:left + 64] for t in (zz, aa, out))
        b2, _ = emu.route_balance(zz, experts, mask=mask)
        assert torch.equal(b2.counts, b.counts)
        # another order of sums where rows are read value by value: both are within the bound of the formula
        assert abs(float(b2.loss) - float(b.loss)) <= 2 * 400 * U * float(b.loss)
        emu.route_balance_backward(zz, b, mask=mask, add=aa, dlogits=o)
        tol = 2 * torch.finfo(dtype).eps * d.abs().double() + 2 * 300 * U * 0.1 / 100
        assert bool(((o.double() - d.double()).abs() <= tol).all())
        o.fill_(9.0)
        assert bool((out == 9.0).all())


def test_past_two_to_the_31(dev):
    T, E, k = 2_200_000, 1024, 2
    z = torch.empty(T, E, dtype=torch.bfloat16, device=dev).normal_(generator=torch.Generator(device=dev).manual_seed(1))
    experts = torch.stack((torch.arange(T, device=dev) % E, (torch.arange(T, device=dev) * 7 + 1) % E), 1).int()
    b, ws = emu.route_balance(z, experts)
    assert emu.read_flags(ws) == 0 and int(b.tokens) == T
    assert torch.equal(b.counts.long(), torch.bincount(experts.reshape(-1).long(), minlength=E))
    d = emu.route_balance_backward(z, b)
    f = b.counts.double() * (E / (T * k))
    at = torch.tensor([0, 1, 2 ** 21 - 1, 2 ** 21, 2 ** 21 + 1, T - 1], device=dev)
    p = torch.softmax(z[at].double(), 1)
    S = (p * f).sum(1, keepdim=True)
    want, room = p * (f - S) / T, p * (f + S) / T * (2 * 12 + 200) * U
    assert bool(((d[at].double() - want).abs() <= room * (1 + 2 ** -8) + want.abs() * 2 ** -8).all())


def test_gradient_against_differences(dev):
    z, experts, mask, _ = case(dev, 60, 24, 3, torch.float32, True)
    coef = 0.7
    b, _ = emu.route_balance(z, experts, coef=coef, mask=mask)
    d = emu.route_balance_backward(z, b, coef=coef, mask=mask).double()
    g = torch.Generator(device=dev).manual_seed(1)
    for _ in range(5):
        v = torch.randn(z.shape, generator=g, device=dev).double()
        h = 1e-4
        up, down = (formula(z.double() + s * h * v, experts, mask, coef)[0] for s in (1, -1))
        # the third derivative's part is below h^2 |v|^3, the kernel's error below 300 U of the terms
        slope = float(up - down) / (2 * h)
        assert abs(slope - float((d * v).sum())) <= 1e-6 * float((d * v).abs().sum()) + 1e-7


def test_same_bits_streams_and_graphs(dev):
    z, experts, mask, add = case(dev, 9000, 96, 4, torch.bfloat16, True)
    b, ws = emu.route_balance(z, experts, mask=mask)
    d = emu.route_balance_backward(z, b, mask=mask, add=add)
    torch.cuda.synchronize()
    s = torch.cuda.Stream(dev)
    for stream in (None, s, None, s):
        c, _ = emu.route_balance(z, experts, mask=mask, stream=stream)
        e = emu.route_balance_backward(z, c, mask=mask, add=add, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(c.loss, b.loss) and torch.equal(c.counts, b.counts) and torch.equal(d, e)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c, _ = emu.route_balance(z, experts, mask=mask, ws=ws)
        e = emu.route_balance_backward(z, c, mask=mask, add=add)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c.loss, b.loss) and torch.equal(c.counts, b.counts) and torch.equal(d, e)


def test_with_route(dev):
    # as a training step uses it: after route, its gradient added to that of route's weights
    z, _, mask, _ = case(dev, 500, 32, 4, torch.float32, True)
    r, _ = emu.route(z, 4, renorm=False)
    b, _ = emu.route_balance(z, r.experts, coef=0.02, mask=mask)
    assert torch.equal(formula(z, r.experts, mask, 0.02)[1], b.counts.long())
    dw = torch.randn(500, 4, generator=torch.Generator(device=dev).manual_seed(3), device=dev)
    d = emu.route_backward(z, r.experts, dw, renorm=False)
    both = emu.route_balance_backward(z, b, coef=0.02, mask=mask, add=d)
    alone = emu.route_balance_backward(z, b, coef=0.02, mask=mask)
    assert bool(((both.double() - d.double() - alone.double()).abs() <= 2 * U * (both.double().abs() + alone.double().abs())).all())
