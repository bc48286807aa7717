"""Matrix-vector products with 4-bit weights against the same sums in 64 bits.

Tolerance, fixed before the first run: products are exact; sums of 16 products
are added with truncation inside a scale group and rounded outside of it, at
most K/16 + 16 additions, each within 2^-23 of the sum of absolute products; a
BF16 result is rounded once more (2^-8 of itself)."""
import pytest

import paper_2609_04663_gb300 as emu
from helpers import device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


def make(dev, rows, N, K, group, dtype, zeros, G=0, stype=None, seed=0):
    import torch
    g = torch.Generator(device=dev).manual_seed(seed)
    lead = (G,) if G else ()
    X = torch.randn((rows, K), generator=g, device=dev).to(dtype)
    q = torch.randint(0, 256, lead + (N, K // 2), generator=g, device=dev, dtype=torch.uint8)
    s = (torch.rand(lead + (N, K // group), generator=g, device=dev) + 0.25).to(stype or dtype)
    z = torch.randint(0, 16, lead + (N, K // group), generator=g, device=dev, dtype=torch.uint8) if zeros else None
    return X, q, s, z


def weights(q, s, z, group):
    """The weights' values in 64 bits (exact)."""
    import torch
    w = torch.stack(((q & 15), (q >> 4)), -1).flatten(-2).double().unflatten(-1, (-1, group))
    w = w - (z.double()[..., None] if z is not None else 8.0)
    return (w * s.double()[..., None]).flatten(-2)


def check(Y, X, W):
    import torch
    ref, mag = X.double() @ W.T, X.double().abs() @ W.abs().T
    bound = (X.shape[1] / 16 + 16) * 2.0 ** -23 * mag
    if Y.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * ref.abs()
    return bool(((Y.double() - ref).abs() <= bound).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("rows,N,K,group", [
    (1, 1, 32, 32), (1, 128, 256, 128), (2, 129, 96, 32), (3, 200, 480, 96), (7, 127, 1024, 64), (8, 256, 2048, 128),
    (9, 65, 544, 32), (17, 300, 768, 64), (25, 70, 4096, 4096), (1, 2048, 4096, 128), (2, 96, 2592, 32), (60, 33, 288, 32),
])
def test_one_matrix(dev, dtype, zeros, rows, N, K, group):
    import torch
    X, q, s, z = make(dev, rows, N, K, group, getattr(torch, dtype), zeros)
    assert check(emu.w4_matvec(X, q, s, zeros=z), X, weights(q, s, z, group))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("sizes,tail", [([0, 1, 0, 2], 0), ([3, 0, 30, 1, 0], 5), ([1] * 70, 2), ([0, 0], 3), ([9], 0)])
def test_experts(dev, dtype, sizes, tail):
    import torch
    rows, N, K, group = sum(sizes) + tail, 150, 288, 32
    X, q, s, z = make(dev, rows, N, K, group, getattr(torch, dtype), True, G=len(sizes), seed=1)
    ends = torch.tensor(sizes, device=dev).cumsum(0).to(torch.int32)
    Y = emu.w4_matvec(X, q, s, zeros=z, ends=ends)
    at = 0
    for g, n in enumerate(sizes):
        assert check(Y[at:at + n], X[at:at + n], weights(q[g], s[g], z[g], group))
        at += n
    assert not Y[at:].any()


def test_every_code_and_position(dev):
    """One-hot rows read single weights back: all codes, zero points and places of a word."""
    import torch
    K, N = 64, 256
    q = torch.arange(256, device=dev, dtype=torch.uint8)[:, None].expand(N, K // 2).contiguous()
    z = (torch.arange(N, device=dev) % 16).to(torch.uint8)[:, None].expand(N, 2).contiguous()
    s = torch.ones(N, 2, device=dev)
    W = weights(q, s, z, 32)
    Y = emu.w4_matvec(torch.eye(K, device=dev), q, s, zeros=z)
    assert torch.equal(Y.double(), W.T)


def test_fp32_rows_keep_their_precision(dev):
    """FP32 rows are not rounded to BF16: with one code of one and the rest
    zero points, a row's entry comes back to within its third slice's rounding."""
    import torch
    K = 32
    q = torch.full((1, K // 2), 0x88, dtype=torch.uint8, device=dev)
    q[0, 3] = 0x98                                       # k = 7 has the value 1
    X = torch.randn(5, K, device=dev, generator=torch.Generator(device=dev).manual_seed(3))
    Y = emu.w4_matvec(X, q, torch.ones(1, 1, device=dev))
    assert bool(((Y[:, 0] - X[:, 7]).abs() <= 2.0 ** -23 * X[:, 7].abs()).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_strides_guards_and_scale_types(dev, dtype):
    import torch
    dt = getattr(torch, dtype)
    for stype in (torch.float32, torch.bfloat16):
        X, q, s, z = make(dev, 5, 70, 160, 32, dt, True, stype=stype, seed=4)
        wide = torch.full((5, 171), float("nan"), dtype=dt, device=dev)
        wide[:, 3:163] = X
        out = torch.full((7, 75), 3.0, dtype=dt, device=dev)
        emu.w4_matvec(wide[:, 3:163], q, s, zeros=z, Y=out[1:6, 2:72])
        assert check(out[1:6, 2:72], X, weights(q, s, z, 32))
        out[1:6, 2:72] = 3.0
        assert bool((out == 3.0).all())


def test_rows_do_not_mix(dev):
    import torch
    X, q, s, z = make(dev, 8, 64, 256, 64, torch.bfloat16, True, seed=5)
    want = emu.w4_matvec(X, q, s, zeros=z)
    X[3] = float("nan")
    X[6] = float("inf")
    got = emu.w4_matvec(X, q, s, zeros=z)
    keep = [0, 1, 2, 4, 5, 7]
    assert torch.equal(got[keep], want[keep]) and bool(got[3].isnan().all())


def test_a_row_alone_and_among_others_is_the_same(dev):
    import torch
    X, q, s, z = make(dev, 3, 130, 1024, 128, torch.float32, False, seed=6)
    got = emu.w4_matvec(X, q, s)
    assert torch.equal(got[1:2], emu.w4_matvec(X[1:2], q, s))


def test_empty(dev):
    import torch
    X, q, s, z = make(dev, 0, 16, 32, 32, torch.float32, False)
    assert emu.w4_matvec(X, q, s).shape == (0, 16)


def test_weights_past_4_gib(dev):
    import torch
    G, N, K = 80, 8192, 16384
    q = torch.zeros(G, N, K // 2, dtype=torch.uint8, device=dev)
    q[-1].random_(0, 256, generator=torch.Generator(device=dev).manual_seed(7))
    s = torch.ones(G, N, K // 128, device=dev)
    X = torch.randn(2, K, device=dev, generator=torch.Generator(device=dev).manual_seed(8))
    ends = torch.zeros(G, dtype=torch.int32, device=dev)
    ends[-1] = 2
    # the file's bound: the number of experts changes how K is cut, so last bits may differ from one matrix's
    assert check(emu.w4_matvec(X, q, s, ends=ends), X, weights(q[-1], s[-1], None, 128))


@pytest.mark.parametrize("seed", range(8))
def test_random_shapes(dev, seed):
    import torch
    rng = __import__("random").Random(seed)
    group = rng.choice((32, 64, 96, 128, 160, 256, 512))
    K, N, G = group * rng.randint(1, max(1, 5000 // group)), rng.randint(1, 700), rng.choice((0, 0, 7))
    rows = rng.randint(1, 30)
    dt = rng.choice((torch.float32, torch.bfloat16))
    X, q, s, z = make(dev, rows, N, K, group, dt, rng.random() < 0.5, G=G, seed=seed)
    if not G:
        assert check(emu.w4_matvec(X, q, s, zeros=z), X, weights(q, s, z, group))
        return
    cuts = sorted(rng.randint(0, rows) for _ in range(G - 1)) + [rows]
    Y = emu.w4_matvec(X, q, s, zeros=z, ends=torch.tensor(cuts, dtype=torch.int32, device=dev))
    for g, (a, b) in enumerate(zip([0] + cuts, cuts)):
        if b > a:
            assert check(Y[a:b], X[a:b], weights(q[g], s[g], z[g] if z is not None else None, group))


def test_another_stream(dev):
    import torch
    X, q, s, z = make(dev, 3, 200, 512, 64, torch.float32, True, seed=9)
    want = emu.w4_matvec(X, q, s, zeros=z)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = emu.w4_matvec(X, q, s, zeros=z, stream=st)
    st.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_most_experts_and_many_rows(dev, dtype):
    import torch
    G, N, K, group = 1024, 33, 64, 32
    sizes = [(i * 7) % 4 if i % 3 else 0 for i in range(G)]
    sizes[5] = 150                                         # far more than its share
    rows = sum(sizes) + 2
    X, q, s, z = make(dev, rows, N, K, group, getattr(torch, dtype), True, G=G, seed=10)
    W = weights(q, s, z, group)
    of = torch.repeat_interleave(torch.arange(G, device=dev), torch.tensor(sizes, device=dev))
    Y = emu.w4_matvec(X, q, s, zeros=z, ends=torch.tensor(sizes, device=dev).cumsum(0).to(torch.int32))
    assert not Y[rows - 2:].any()
    for g in (1, 2, 5, 1021, 1022):
        assert check(Y[:rows - 2][of == g], X[:rows - 2][of == g], W[g])
    assert all(check(Y[i:i + 1], X[i:i + 1], W[of[i]]) for i in range(0, rows - 2, 97))
    X, q, s, z = make(dev, 3001, N, K, group, getattr(torch, dtype), True, seed=11)
    assert check(emu.w4_matvec(X, q, s, zeros=z), X, weights(q, s, z, group))
