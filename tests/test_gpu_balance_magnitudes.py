"""Balance loss and gradient where logits are finite and large: whole rows, single entries
and neighbouring values from 2^19 to the type's largest, against the formulas in 64 bits.

Bounds, with U = 2^-24 and R the largest distance from a row's largest logit among logits that
are no more than 104 below it (others' exponentials are below the smallest normal
number).  An exponent is (x - top) log2 e: the constant is off by 0.22 U of it, one rounding by U
(where top is subtracted first, the difference of values within 104 is exact); an error e of the exponent is
one of 0.694 e in the power, 1.22 R U in all; a common factor of a row (from the rounding of
top log2 e) is in its sum too.  A power of two is off by 2^-22, a sum of up to 32 values in 32
lanes by 36 U, reciprocal and product by one each:
  p: 2 (1.22 R + 4) + 38 < 2.5 R + 48 of U relative, and 2^-125 for what is flushed.
The loss: at most T / 32 + 32 + 152 additions in a row, f 4, three products and 69 additions:
2.5 R + 48 + T / 32 + 264.  The gradient, scale p (f - S) with S = sum p f: p f errs by p's and 4, S by p's, 4
and 37, and times p once more by p's; scale, products and difference by 4: below p (f + S) (5 R + 96 + 49) U;
then one rounding with `add` to the type."""
import pytest
import torch

import paper_2609_04663_gb300 as emu
from helpers import device

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
MAGNITUDES = [2.0 ** 19, 2.0 ** 20, 1.1 * 2 ** 20, 2.0 ** 24, 1e9, 3e9, 5e9, 1e10, 1e12, 1e20, 1e30, 1e37, 9e37, 1.1e38, 3.3e38]


@pytest.fixture(scope="module")
def dev():
    return device()


def rows(dev, E, dtype, g):
    """Rows of every kind for every magnitude and sign, then ordinary ones."""
    plain = lambda: torch.randn(E, generator=g, device=dev)
    some = torch.arange(E, device=dev) % 3 == 1
    out = []
    for m in MAGNITUDES:
        for v in (m, -m):
            near = torch.full((E,), v, device=dev).to(dtype).float()
            step = abs(float(near[0])) * torch.finfo(dtype).eps
            out += [near,                                                       # equal ones
                    torch.where(some, near, plain()),                           # some among ordinary ones
                    torch.where(torch.arange(E, device=dev) == E // 2, near, plain()),
                    torch.where(some, near, -near),                             # of both signs
                    near - step * (torch.arange(E, device=dev) % 5),            # neighbours
                    near + 3 * plain().clamp(-4, 4)]                            # within what the type can tell apart
    z = torch.stack(out).clamp(-3.38e38, 3.38e38).to(dtype)
    assert bool(z.isfinite().all())
    return z


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("E", [3, 20, 64, 128, 200, 500, 700, 1023])
@pytest.mark.parametrize("T", [180, 6000])
def test_large_logits(dev, T, E, dtype):
    g = torch.Generator(device=dev).manual_seed(7 * E + T)
    big = rows(dev, E, dtype, g)
    assert big.shape[0] == 180
    z = torch.cat((big, torch.randn(T - 180, E, generator=g, device=dev).to(dtype)))[torch.randperm(T, generator=g, device=dev)].contiguous()
    k, coef = min(E, 3), 0.7
    experts = torch.rand(T, E, generator=g, device=dev).topk(k, dim=1).indices.int().contiguous()
    add = (torch.randn(T, E, generator=g, device=dev) * 1e-3 / T).to(dtype)
    x = z.double()
    below = x.amax(1, keepdim=True) - x
    R = torch.where(below <= 104, below, torch.zeros_like(below)).amax(1, keepdim=True)
    p = torch.softmax(x, 1)
    counts = torch.bincount(experts.reshape(-1).long(), minlength=E)
    f = counts.double() * (coef * E / (T * k))
    loss = float((f * p.sum(0)).sum()) / T
    ws = emu.workspace(max(emu.emu_route_balance_workspace_bytes(T, E), emu.emu_split_workspace_bytes(32)), dev)
    b, _ = emu.route_balance(z, experts, coef=coef, ws=ws)
    assert emu.read_flags(ws) == 0 and torch.equal(b.counts.long(), counts) and int(b.tokens) == T
    assert abs(float(b.loss) - loss) <= (2.5 * float(R.max()) + 312 + T / 32) * U * loss + 2.0 ** -100
    S = (p * f).sum(1, keepdim=True)
    half = torch.finfo(dtype).eps / 2
    for extra in (None, add):
        d = emu.route_balance_backward(z, b, coef=coef, add=extra).double()
        want = p * (f - S) / T
        room = p * (f + S) / T * (5 * R + 145) * U + 2.0 ** -120
        if extra is not None:
            want, room = want + extra.double(), room + extra.double().abs() * U
        bound = room * (1 + half) + want.abs() * (half + U) + (2.0 ** -149 if dtype is torch.float32 else 2.0 ** -133)
        assert bool(((d - want).abs() <= bound).all())


@pytest.mark.parametrize("fill", [-1e9, -1e10, -1e30])
def test_padded_tokens_without_a_mask(dev, fill):
    # logits of padding filled with a large negative number: an even row each, as in 64 bits
    z = torch.randn(300, 48, generator=torch.Generator(device=dev).manual_seed(1), device=dev)
    z[250:] = fill
    experts = torch.arange(600, device=dev).view(300, 2).remainder(48).int()
    b, _ = emu.route_balance(z, experts)
    even = z.clone()
    even[250:] = 0.0
    c, _ = emu.route_balance(even, experts)
    assert torch.equal(b.loss, c.loss) and bool(b.loss.isfinite())
    assert torch.equal(emu.route_balance_backward(z, b), emu.route_balance_backward(even, c))
