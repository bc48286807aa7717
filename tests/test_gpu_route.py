"""Routing and the weighted sum of answers against their definitions in 64
bits.  Whole numbers have to be equal.  Weights and gradients of FP32: the
exponentials, the sum and the quotient are each good to a few units of 2^-24,
the sum of E terms to E of them at most: (E + 16) 2^-23 relative (a gradient:
of the largest product).  Sums over k answers: k 2^-23 of the absolute sum;
dot products over n columns: n 2^-23; BF16 results 2^-8 of themselves more."""
import pytest

import paper_2609_04663_gb300 as emu
from helpers import device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


def reference(x, k, renorm):
    """experts, weights, slots, rows, ends of logits x by the definitions (x on the CPU)."""
    import torch
    x = torch.where(x.isnan(), float("-inf"), x.double())
    T, E = x.shape
    order = torch.sort(x, dim=1, descending=True, stable=True)
    ex = order.indices[:, :k]
    top = order.values[:, :k]
    m = top[:, :1]
    ok = m > float("-inf")
    p = torch.where(ok, (top - m).exp(), 0.0)
    tot = p.sum(1, keepdim=True) if renorm else torch.where(ok, (x - m).exp(), 0.0).sum(1, keepdim=True)
    w = torch.where(ok, p / tot, 0.0)
    by = torch.sort(ex.reshape(-1), stable=True).indices
    slots = torch.empty(T * k, dtype=torch.int64)
    slots[by] = torch.arange(T * k)
    ends = torch.bincount(ex.reshape(-1), minlength=E).cumsum(0)
    return ex, w, slots.view(T, k), by // k, ends


def logits(dev, T, E, dtype, kind, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, E), generator=g) * 2
    if kind == "ties":
        x = (x * 2).round() / 2 * torch.where(torch.rand((T, E), generator=g) < 0.5, 1.0, -1.0)      # negative zeros too
    if kind == "masked":
        x[torch.rand((T, E), generator=g) < 0.6] = float("-inf")
        x[torch.rand((T, E), generator=g) < 0.05] = torch.finfo(dtype).min
        x[::7] = float("-inf")
        x[::5, ::3] = float("nan")
    if kind == "one expert":
        x[:, E // 2] += 50
    return x.to(dtype)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("T,E,k,kind", [
    (1, 1, 1, "plain"), (1, 64, 8, "plain"), (5, 7, 7, "ties"), (33, 32, 2, "masked"), (64, 33, 4, "ties"),
    (1000, 128, 8, "plain"), (777, 257, 16, "masked"), (200, 600, 32, "ties"), (5000, 8, 2, "one expert"),
    (9000, 64, 6, "ties"), (40, 1024, 3, "plain"),
])
def test_route(dev, dtype, renorm, T, E, k, kind):
    import torch
    x = logits(dev, T, E, getattr(torch, dtype), kind, 1)
    ex, w, slots, rows, ends = reference(x, k, renorm)
    r, ws = emu.route(x.to(dev), k, renorm=renorm)
    assert emu.read_flags(ws) == (emu.FLAG_NONFINITE if bool(x.isnan().any()) else 0)
    assert torch.equal(r.experts.cpu().long(), ex)
    assert torch.equal(r.slots.cpu().long(), slots) and torch.equal(r.rows.cpu().long(), rows)
    assert torch.equal(r.ends.cpu().long(), ends)
    assert bool(((r.weights.cpu().double() - w).abs() <= (E + 16) * 2.0 ** -23 * w + 1e-37).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("T,E,k,kind", [(1, 1, 1, "plain"), (37, 16, 3, "plain"), (300, 70, 8, "masked"), (65, 520, 4, "ties")])
def test_route_backward(dev, dtype, renorm, T, E, k, kind):
    """Against the formula by automatic differentiation of the definition in 64 bits."""
    import torch
    x = logits(dev, T, E, getattr(torch, dtype), kind, 2)
    if kind == "masked":
        x[::7, 0] = 0.5                                    # (rows without any expert are looked at below)
    ex, _, _, _, _ = reference(x, k, renorm)
    g = torch.randn((T, k), generator=torch.Generator().manual_seed(3))
    v = torch.where(x.isnan(), float("-inf"), x.double())
    finite = v > float("-inf")
    u = torch.where(finite, v, 0.0).requires_grad_()
    z = torch.where(finite, u, float("-inf"))
    m = z.detach().max(1, keepdim=True).values
    p = torch.where(finite, (z - m).exp(), 0.0)
    sel = p.gather(1, ex)
    w = sel / (sel.sum(1, keepdim=True) if renorm else p.sum(1, keepdim=True))
    (w * g.double()).sum().backward()
    r, _ = emu.route(x.to(dev), k, renorm=renorm)
    d = emu.route_backward(x.to(dev), r.experts, g.to(dev), renorm=renorm).cpu()
    bound = (E + 16) * 2.0 ** -23 * (w.detach() * g.double().abs()).sum(1, keepdim=True).expand(T, E) + 1e-37
    if dtype == "bfloat16":
        bound = bound + 2.0 ** -8 * u.grad.abs()
    assert d.dtype == x.dtype and bool(((d.double() - u.grad).abs() <= bound).all())


def test_route_backward_equals_differences(dev):
    """Central differences of sum(g * weights) in a random direction; the step
    h = 2^-6 leaves a third-order error of at most h^2 times the sum of |g|,
    rounding 2^-22 of it over h."""
    import torch
    g0 = torch.Generator(device=dev).manual_seed(4)
    x = torch.randn(50, 12, device=dev, generator=g0)
    g = torch.randn(50, 3, device=dev, generator=g0)
    v = torch.randn(50, 12, device=dev, generator=g0).clamp(-1, 1)
    h = 2.0 ** -6
    for renorm in (False, True):
        r, _ = emu.route(x, 3, renorm=renorm)
        d = emu.route_backward(x, r.experts, g, renorm=renorm).double()

        def f(y):
            p = (y.double() - y.double().max(1, keepdim=True).values).exp()
            sel = p.gather(1, r.experts.long())
            return (sel / (sel if renorm else p).sum(1, keepdim=True) * g.double()).sum()
        diff = (f(x + h * v) - f(x - h * v)) / (2 * h)
        assert abs(float(diff - (d * v.double()).sum())) <= float(g.abs().sum()) * (h * h + 2.0 ** -22 / h)


def test_rows_without_experts(dev):
    import torch
    x = torch.full((3, 5), float("-inf"), device=dev)
    x[1, 3] = 1.0
    for renorm in (False, True):
        r, _ = emu.route(x, 2, renorm=renorm)
        assert r.experts.tolist() == [[0, 1], [3, 0], [0, 1]]
        assert r.weights.tolist() == [[0, 0], [1, 0], [0, 0]]
        d = emu.route_backward(x, r.experts, torch.ones(3, 2, device=dev), renorm=renorm)
        assert not d.any()


def test_route_strided_logits_and_no_tokens(dev):
    import torch
    big = torch.randn(40, 50, device=dev)
    r, _ = emu.route(big[:, 3:36], 4)
    q, _ = emu.route(big[:, 3:36].contiguous(), 4)
    assert all(torch.equal(a, b) for a, b in zip(r, q))
    r, _ = emu.route(torch.empty(0, 8, device=dev), 2)
    assert r.ends.tolist() == [0] * 8 and r.rows.numel() == 0


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,k,cols,pad", [(1, 1, 1, 0), (3, 2, 8, 0), (40, 4, 2048, 0), (17, 3, 333, 0), (50, 8, 100, 5),
                                          (700, 2, 64, 0)])
def test_combine_and_gradients(dev, dtype, T, k, cols, pad):
    import torch
    dt = getattr(torch, dtype)
    g = torch.Generator(device=dev).manual_seed(5)
    S = T * k + 3                                          # three answers that no token takes
    Y = torch.randn((S, cols + pad), generator=g, device=dev).to(dt)[:, :cols]
    slots = torch.randperm(S, generator=g, device=dev)[:T * k].view(T, k).to(torch.int32)
    w = torch.rand((T, k), generator=g, device=dev)
    dO = torch.randn((T, cols), generator=g, device=dev).to(dt)
    sl = slots.clone()
    if T > 2:
        sl[1, 0], sl[2, k - 1] = -1, S                     # dropped assignments
    ok = ((sl >= 0) & (sl < S)).double()
    Ys = Y.double()[sl.long().clamp(0, S - 1)] * ok[..., None]
    eps = 2.0 ** -8 if dtype == "bfloat16" else 0.0
    for wt in (w, None):
        we = w.double() if wt is not None else torch.ones_like(w).double()
        ref, mag = (Ys * we[..., None]).sum(1), (Ys.abs() * we[..., None]).sum(1)
        O = emu.rows_combine(Y, sl, wt)
        assert O.dtype == dt and bool(((O.double() - ref).abs() <= k * 2.0 ** -23 * mag + eps * ref.abs()).all())
        dY, dw = emu.rows_combine_backward(dO, Y, sl, wt)
        refY = torch.zeros(S, cols, dtype=torch.float64, device=dev)
        take = ok.bool()
        refY[sl[take].long()] = (we[..., None] * dO.double()[:, None]).expand(T, k, cols)[take]
        assert bool(((dY.double() - refY).abs() <= (2.0 ** -23 + eps) * refY.abs()).all())
        if wt is None:
            assert dw is None
        else:
            refw = (Ys * dO.double()[:, None]).sum(-1)
            magw = (Ys.abs() * dO.double().abs()[:, None]).sum(-1)
            assert bool(((dw.double() - refw).abs() <= cols * 2.0 ** -23 * magw).all())


def test_combine_guards(dev):
    import torch
    Y = torch.randn(8, 24, device=dev)
    slots = torch.randperm(8, device=dev).view(4, 2).to(torch.int32)
    O = torch.full((6, 29), 7.0, device=dev)
    emu.rows_combine(Y, slots, O=O[1:5, 2:26])
    assert torch.allclose(O[1:5, 2:26], Y[slots.long()].sum(1))
    O[1:5, 2:26] = 7.0
    assert bool((O == 7.0).all())
    dY = torch.full((10, 27), 7.0, device=dev)
    emu.rows_combine_backward(torch.randn(4, 24, device=dev), Y, slots, dY=dY[1:9, 1:25])
    dY[1:9, 1:25] = 7.0
    assert bool((dY == 7.0).all())


def test_route_feeds_the_products(dev):
    """route -> grouped products -> combine equals the layer written per token."""
    import torch
    g = torch.Generator(device=dev).manual_seed(6)
    T, E, k, K, N = 90, 6, 2, 64, 48
    x, X = torch.randn(T, E, device=dev, generator=g), torch.randn(T, K, device=dev, generator=g)
    W = torch.randn(E, K, N, device=dev, generator=g)
    r, _ = emu.route(x, k)
    Y, _ = emu.grouped_gemm(X, W, r.ends, src=r.rows)
    O = emu.rows_combine(Y, r.slots, r.weights).double()
    per = torch.einsum("tk,tjkn->tjn", X.double(), W.double()[r.experts.long()])
    mag = torch.einsum("tk,tjkn->tjn", X.double().abs(), W.double().abs()[r.experts.long()])
    ref = (per * r.weights.double()[..., None]).sum(1)
    bound = 1e-5 * (mag * r.weights.double()[..., None]).sum(1)
    assert bool(((O - ref).abs() <= bound).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,E,k,kind", [(20001, 36, 5, "masked"), (6000, 70, 32, "ties"), (40000, 3, 1, "one expert"), (33, 1021, 32, "plain")])
def test_route_many_tokens_of_padded_rows(dev, dtype, T, E, k, kind):
    """Several tokens for each warp of every block, logits as a part of wider rows; twice the same."""
    import torch
    x = logits(dev, T, E, getattr(torch, dtype), kind, 5)
    ex, w, slots, rows, ends = reference(x, k, True)
    wide = torch.full((T, E + 3), float("nan"), dtype=x.dtype, device=dev)
    wide[:, :E] = x.to(dev)
    r, ws = emu.route(wide[:, :E], k)
    again, _ = emu.route(wide[:, :E], k)
    assert emu.read_flags(ws) == (emu.FLAG_NONFINITE if bool(x.isnan().any()) else 0)
    assert torch.equal(r.experts.cpu().long(), ex) and torch.equal(r.slots.cpu().long(), slots)
    assert torch.equal(r.rows.cpu().long(), rows) and torch.equal(r.ends.cpu().long(), ends)
    assert bool(((r.weights.cpu().double() - w).abs() <= (E + 16) * 2.0 ** -23 * w + 1e-37).all())
    assert all(torch.equal(a, b) for a, b in zip(r, again))


def test_combine_past_2_31_elements(dev):
    """Answers and their gradients of more than 2^31 elements, the last rows named first."""
    import torch
    T, k, cols = 270000, 2, 4096
    assert T * k * cols > 2 ** 31
    Y = torch.zeros((T * k, cols), dtype=torch.bfloat16, device=dev)
    g = torch.Generator(device=dev).manual_seed(8)
    Y[-8:].normal_(generator=g)
    Y[:8].normal_(generator=g)
    slots = torch.arange(T * k - 1, -1, -1, dtype=torch.int32, device=dev).view(T, k)
    w = torch.rand((T, k), generator=g, device=dev)
    O = emu.rows_combine(Y, slots, w)
    ends = [t for at in (0, T - 4) for t in range(at, at + 4)]
    per = w.double()[ends, :, None] * Y[slots[ends].long()].double()
    bound = k * 2.0 ** -23 * per.abs().sum(1) + 2.0 ** -8 * per.sum(1).abs()
    assert bool(((O[ends].double() - per.sum(1)).abs() <= bound).all())
    dO = torch.zeros_like(O)
    dO[ends] = torch.randn((8, cols), generator=g, device=dev).bfloat16()
    dY, dw = emu.rows_combine_backward(dO, Y, slots, w)
    dot = Y[slots[ends].long()].double() * dO[ends].double()[:, None]
    assert bool(((dw[ends].double() - dot.sum(2)).abs() <= cols * 2.0 ** -23 * dot.abs().sum(2)).all())
    want = w.double()[ends, :, None] * dO[ends].double()[:, None]
    assert bool(((dY[slots[ends].long()].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -23) * want.abs()).all())
    assert not dw[4:T - 4].any() and not dY[8:-8].any()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("cols", [1, 4, 8, 31, 32, 33, 56, 64, 65, 120, 128, 129, 255, 257, 1023])
def test_combine_gradients_of_short_and_odd_rows(dev, dtype, cols):
    """Every share of a warp and both kinds of pieces, slots outside and a last part of a warp among them."""
    import torch
    T, k = 37, 3
    g = torch.Generator(device=dev).manual_seed(9)
    Y, dO = (torch.randn((r, cols), generator=g, device=dev).to(getattr(torch, dtype)) for r in (T * k, T))
    slots = torch.randperm(T * k, generator=g, device=dev).to(torch.int32).view(T, k)
    w = torch.rand((T, k), generator=g, device=dev)
    slots[5, 1], slots[36, 2] = -1, T * k
    dY, dw = emu.rows_combine_backward(dO, Y, slots, w, dY=torch.full_like(Y, 7.0))
    ok = (slots >= 0) & (slots < T * k)
    at = slots.clamp(0, T * k - 1).long()
    dot = Y[at].double() * dO.double()[:, None]
    assert bool(((dw.double() - dot.sum(2)).abs() <= cols * 2.0 ** -23 * dot.abs().sum(2))[ok].all())
    assert not dw[~ok].any()
    want = w.double()[..., None] * dO.double()[:, None]
    tol = 2.0 ** -23 + (2.0 ** -8 if dtype == "bfloat16" else 0.0)
    assert bool(((dY[at].double() - want).abs() <= tol * want.abs())[ok].all())
    named = torch.zeros(T * k, dtype=torch.bool, device=dev)
    named[at[ok]] = True
    assert bool((dY[~named] == 7.0).all())
