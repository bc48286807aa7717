"""Products grouped by expert against the same sums in 64 bits.

Tolerances, fixed before the first run.  FP32 mode: |Y - ref| <= 1e-5
(|X||W|), the FP32 mode's bar.  BF16 operands: products are exact and summed
in FP32; with at most n terms the FP32 sum is within n 2^-23 of sum |x||w|
(truncating adds), and a BF16 result is rounded once more (2^-8 of itself).
Gradients are the same sums over other dimensions."""
import numpy as np
import pytest

import paper_2609_04663_gb300 as emu
from helpers import device

pytestmark = pytest.mark.gpu

# group sizes: empty groups first, in the middle and last, single rows, sizes
# around the column tiles of 64 and 256 and the 16-row steps
SIZES = {
    "one row": [0, 1, 0],
    "few rows": [1, 0, 3, 16, 2, 17, 0, 5],
    "ragged": [0, 63, 64, 65, 129, 0, 1, 33, 15],
    "large": [255, 256, 257, 0, 511, 300, 1],
    "one group": [333],
    "all empty": [0, 0, 0],
}


@pytest.fixture(scope="module")
def dev():
    return device()


def make(dev, sizes, K, N, dtype, seed, tail=0, trans=False, gather=False):
    import torch
    g = torch.Generator(device=dev).manual_seed(seed)
    G, rows = len(sizes), sum(sizes) + tail
    ends = torch.tensor(np.cumsum(sizes), dtype=torch.int32, device=dev)
    src = None
    if gather:
        T = max(1, rows // 3)
        src = torch.randint(0, T, (rows,), generator=g, device=dev, dtype=torch.int32)
    X = torch.randn((T if gather else rows, K), generator=g, device=dev).to(dtype)
    W = torch.randn((G, N, K) if trans else (G, K, N), generator=g, device=dev).to(dtype)
    dY = torch.randn((rows, N), generator=g, device=dev).to(dtype)
    return X, W, dY, ends, src


def spans(sizes):
    e = np.concatenate([[0], np.cumsum(sizes)])
    return [(int(a), int(b)) for a, b in zip(e, e[1:])]


def reference(X, W, dY, sizes, trans):
    """Y, dX, dW in FP64, and the same with absolute values."""
    import torch
    out = []
    for f in (lambda t: t.double(), lambda t: t.double().abs()):
        x, w, d = f(X), f(W), f(dY)
        w = w.transpose(1, 2) if trans else w
        Y = torch.zeros(x.shape[0], w.shape[2], dtype=torch.float64, device=X.device)
        dX, dW = torch.zeros_like(x), torch.zeros_like(w)
        for g, (a, b) in enumerate(spans(sizes)):
            Y[a:b], dX[a:b], dW[g] = x[a:b] @ w[g], d[a:b] @ w[g].T, x[a:b].T @ d[a:b]
        out.append((Y, dX, dW.transpose(1, 2) if trans else dW))
    return out


def within(got, ref, mag, terms, f32_mode):
    import torch
    if f32_mode:
        bound = 1e-5 * mag
    else:
        bound = terms * 2.0 ** -23 * mag
        if got.dtype == torch.bfloat16:
            bound = bound + 2.0 ** -8 * ref.abs()
    return bool(((got.double() - ref).abs() <= bound).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("trans", [False, True])
@pytest.mark.parametrize("name,K,N", [
    ("one row", 64, 128), ("few rows", 8, 16), ("few rows", 136, 264), ("ragged", 200, 384), ("large", 96, 520),
    ("one group", 1000, 136), ("all empty", 64, 64), ("ragged", 33, 77), ("few rows", 1, 1), ("large", 129, 255),
])
def test_products_and_gradients(dev, dtype, trans, name, K, N):
    import torch
    dt, sizes = getattr(torch, dtype), SIZES[name]
    X, W, dY, ends, _ = make(dev, sizes, K, N, dt, 1, tail=3, trans=trans)
    (Y, dX, dW), (aY, aX, aW) = reference(X, W, dY, sizes, trans)
    op, back = (emu.OP_T, emu.OP_N) if trans else (emu.OP_N, emu.OP_T)
    f32 = dtype == "float32"
    y, ws = emu.grouped_gemm(X, W, ends, opW=op)
    assert emu.read_flags(ws) == 0 and y.dtype == dt
    assert within(y, Y, aY, K, f32)
    dx, ws = emu.grouped_gemm(dY, W, ends, opW=back)
    assert emu.read_flags(ws) == 0 and within(dx, dX, aX, N, f32)
    dw, ws = emu.grouped_wgrad(dY, X, ends) if trans else emu.grouped_wgrad(X, dY, ends)
    assert emu.read_flags(ws) == 0 and within(dw, dW, aW, max(sizes), f32)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("name,K,N", [("few rows", 72, 40), ("ragged", 61, 130), ("large", 128, 256)])
def test_gathered_rows(dev, dtype, name, K, N):
    import torch
    sizes = SIZES[name]
    X, W, dY, ends, src = make(dev, sizes, K, N, getattr(torch, dtype), 2, gather=True)
    (Y, _, dW), (aY, _, aW) = reference(X[src.long()], W, dY, sizes, False)
    y, ws = emu.grouped_gemm(X, W, ends, src=src)
    assert emu.read_flags(ws) == 0 and within(y, Y, aY, K, dtype == "float32")
    dw, ws = emu.grouped_wgrad(X, dY, ends, srcA=src)
    assert emu.read_flags(ws) == 0 and within(dw, dW, aW, max(sizes), dtype == "float32")


def test_planes_stand_for_their_operands(dev):
    import torch
    X, W, dY, ends, src = make(dev, SIZES["ragged"], 96, 200, torch.float32, 3, gather=True)
    xp, wp, dp = emu.grouped_split(X, ends, src=src), emu.grouped_split(W), emu.grouped_split(dY, ends)
    assert torch.equal(emu.grouped_gemm(xp, wp, ends)[0], emu.grouped_gemm(X, W, ends, src=src)[0])
    assert torch.equal(emu.grouped_gemm(dp, wp, ends, opW=emu.OP_T)[0], emu.grouped_gemm(dY, W, ends, opW=emu.OP_T)[0])
    assert torch.equal(emu.grouped_gemm(dp, W, ends, opW=emu.OP_T)[0], emu.grouped_gemm(dY, W, ends, opW=emu.OP_T)[0])
    assert torch.equal(emu.grouped_wgrad(xp, dp, ends)[0], emu.grouped_wgrad(X, dY, ends, srcA=src)[0])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_other_groups_do_not_leak(dev, dtype):
    """NaN and infinity in one group's rows and in rows of no group stay there;
    a group's gradient sees its own rows only."""
    import torch
    dt, sizes = getattr(torch, dtype), [7, 20, 0, 70, 3]
    X, W, dY, ends, _ = make(dev, sizes, 64, 136, dt, 4, tail=9)
    clean = [emu.grouped_gemm(X, W, ends)[0], emu.grouped_wgrad(X, dY, ends)[0]]
    X2, d2 = X.clone(), dY.clone()
    X2[7:27], d2[7:27] = float("nan"), float("inf")
    X2[100:], d2[100:] = float("nan"), float("nan")
    y, dw = emu.grouped_gemm(X2, W, ends)[0], emu.grouped_wgrad(X2, d2, ends)[0]
    keep = [0, 2, 3, 4]
    assert torch.equal(dw[keep], clean[1][keep]) and bool(dw[1].isnan().all())
    assert torch.equal(y[:7], clean[0][:7]) and torch.equal(y[27:], clean[0][27:])
    assert bool(y[7:27].isnan().all()) and not y[100:].any()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_strides_and_guards(dev, dtype):
    """Row pitches wider than the rows, results inside canaries."""
    import torch
    dt, sizes = getattr(torch, dtype), SIZES["ragged"]
    X, W, dY, ends, _ = make(dev, sizes, 72, 90, dt, 5)
    Xw = torch.full((X.shape[0], 96), float("nan"), dtype=dt, device=dev)
    Xw[:, 8:80] = X
    Ww = torch.full((len(sizes), 80, 104), float("nan"), dtype=dt, device=dev)
    Ww[:, :72, 3:93] = W                       # a base that no bulk copy can start from
    Yw = torch.full((X.shape[0] + 4, 101), 7.0, dtype=dt, device=dev)
    want = emu.grouped_gemm(X, W, ends)[0]
    emu.grouped_gemm(Xw[:, 8:80], Ww[:, :72, 3:93], ends, Y=Yw[2:-2, 5:95])
    assert torch.equal(Yw[2:-2, 5:95], want)
    Yw[2:-2, 5:95] = 7.0
    assert bool((Yw == 7.0).all())
    Dw = torch.full((len(sizes), 75, 97), 7.0, dtype=dt, device=dev)
    want = emu.grouped_wgrad(X, dY, ends)[0]
    emu.grouped_wgrad(Xw[:, 8:80], dY, ends, D=Dw[:, 1:73, 2:92])
    assert torch.equal(Dw[:, 1:73, 2:92], want)
    Dw[:, 1:73, 2:92] = 7.0
    assert bool((Dw == 7.0).all())


def test_bf16_operands_with_fp32_results(dev):
    import torch
    sizes = SIZES["large"]
    X, W, dY, ends, _ = make(dev, sizes, 128, 264, torch.bfloat16, 6)
    (Y, _, dW), (aY, _, aW) = reference(X, W, dY, sizes, False)
    y = torch.empty(Y.shape, device=dev)
    d = torch.empty(dW.shape, device=dev)
    emu.grouped_gemm(X, W, ends, Y=y)
    emu.grouped_wgrad(X, dY, ends, D=d)
    assert within(y, Y, aY, 128, False) and within(d, dW, aW, 511, False)


def test_bad_indices_are_flagged_and_stay_inside(dev):
    import torch
    sizes = [40, 30]
    X, W, dY, ends, src = make(dev, sizes, 64, 64, torch.float32, 7, gather=True)
    bad = src.clone()
    bad[5], bad[50] = -1, X.shape[0]
    y, ws = emu.grouped_gemm(X, W, ends, src=bad)
    assert emu.read_flags(ws) == emu.FLAG_INDEX
    ok = emu.grouped_gemm(X, W, ends, src=src)[0]
    ok[5], ok[50] = 0, 0
    assert torch.equal(y, ok)
    for e in ([40, 1000], [-5, 70], [50, 30]):
        _, ws = emu.grouped_gemm(X[src.long()], W, torch.tensor(e, dtype=torch.int32, device=dev))
        assert emu.read_flags(ws) & emu.FLAG_INDEX


def test_wgrad_equals_differences(dev):
    """dW against central differences of f(W) = sum(dY * Y(W)) in a random
    direction: f is linear in W, so the difference quotient is exact up to the
    FP32 mode's own error (1e-5 of the absolute sums on each of two values)."""
    import torch
    sizes = SIZES["ragged"]
    X, W, dY, ends, _ = make(dev, sizes, 40, 48, torch.float32, 8)
    dW = emu.grouped_wgrad(X, dY, ends)[0].double()
    V = torch.randn(W.shape, device=dev)
    f = lambda w: (emu.grouped_gemm(X, w, ends)[0].double() * dY.double()).sum()
    mag = (reference(X, W.abs() + V.abs(), dY, sizes, False)[1][0] * dY.double().abs()).sum()
    assert abs(float((f(W + V) - f(W - V)) / 2 - (dW * V.double()).sum())) <= 2e-5 * float(mag)


def test_zero_sizes(dev):
    import torch
    e = torch.tensor([0, 0], dtype=torch.int32, device=dev)
    z = lambda *s: torch.zeros(s, device=dev)
    assert emu.grouped_gemm(z(0, 8), z(2, 8, 16), e)[0].shape == (0, 16)
    assert not emu.grouped_gemm(z(3, 0), z(2, 0, 16), torch.tensor([1, 3], dtype=torch.int32, device=dev))[0].any()
    d = torch.full((2, 8, 16), 5.0, device=dev)
    emu.grouped_wgrad(z(0, 8), z(0, 16), e, D=d)
    assert not d.any()


def test_another_stream(dev):
    import torch
    X, W, dY, ends, src = make(dev, SIZES["large"], 128, 256, torch.float32, 9, gather=True)
    want = emu.grouped_gemm(X, W, ends, src=src)[0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = emu.grouped_gemm(X, W, ends, src=src, stream=s)[0]
    s.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows_each", [3, 40, 200])
def test_shared_weights_of_all_groups(dev, dtype, rows_each):
    """One matrix expanded over the groups (distance 0) is the plain product."""
    import torch
    dt = getattr(torch, dtype)
    sizes = [rows_each, 0, rows_each + 1]
    X, W, dY, ends, _ = make(dev, sizes, 64, 80, dt, 10)
    Ws = W[:1].expand(3, 64, 80)
    (Y, dX, _), (aY, aX, _) = reference(X, Ws, dY, sizes, False)
    y, _ = emu.grouped_gemm(X, Ws, ends)
    dx, _ = emu.grouped_gemm(dY, Ws, ends, opW=emu.OP_T)
    assert within(y, Y, aY, 64, dtype == "float32") and within(dx, dX, aX, 80, dtype == "float32")


@pytest.mark.parametrize("rows", [8, 5120])
def test_weights_past_4_gib(dev, rows):
    """The last group's matrix lies past 2^32 bytes."""
    import torch
    G, K, N = 40, 8192, 8192
    W = torch.zeros(G, K, N, dtype=torch.bfloat16, device=dev)
    W[-1].normal_(generator=torch.Generator(device=dev).manual_seed(11))
    X = torch.randn(rows, K, device=dev, generator=torch.Generator(device=dev).manual_seed(12)).bfloat16()
    ends = torch.zeros(G, dtype=torch.int32, device=dev)
    ends[-1] = rows
    y, ws = emu.grouped_gemm(X, W, ends)
    one, _ = emu.grouped_gemm(X, W[-1:], ends[-1:])
    assert emu.read_flags(ws) == 0
    assert float((y.float() - one.float()).abs().max()) <= 2.0 ** -8 * float(one.float().abs().max())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("seed", range(6))
def test_random_shapes(dev, dtype, seed):
    """Sizes, orders and paths at random: few and many rows, odd widths, gathers."""
    import torch
    rng = np.random.default_rng(100 + seed)
    G = int(rng.integers(1, 12))
    sizes = [int(v) for v in rng.integers(0, [4, 70, 600][seed % 3], G)]
    K, N = (int(v) for v in rng.integers(1, 700, 2))
    if seed % 2:
        K, N = K // 8 * 8 + 8, N // 64 * 64 + 64
    trans = bool(rng.integers(0, 2))
    dt = getattr(torch, dtype)
    X, W, dY, ends, src = make(dev, sizes, K, N, dt, seed, tail=int(rng.integers(0, 3)), trans=trans, gather=seed % 2 == 0)
    Xg = X[src.long()] if src is not None else X
    (Y, dX, dW), (aY, aX, aW) = reference(Xg, W, dY, sizes, trans)
    op, back = (emu.OP_T, emu.OP_N) if trans else (emu.OP_N, emu.OP_T)
    f32 = dtype == "float32"
    if dY.shape[0] == 0:
        return
    assert within(emu.grouped_gemm(X, W, ends, opW=op, src=src)[0], Y, aY, K, f32)
    assert within(emu.grouped_gemm(dY, W, ends, opW=back)[0], dX, aX, N, f32)
    dw = emu.grouped_wgrad(dY, X, ends, srcB=src)[0] if trans else emu.grouped_wgrad(X, dY, ends, srcA=src)[0]
    assert within(dw, dW, aW, max(sizes + [1]), f32)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_most_groups(dev, dtype):
    """1024 groups, most of them empty or of one row: product, both gradients."""
    import torch
    rng = np.random.default_rng(13)
    sizes = [int(v) for v in rng.choice((0, 0, 1, 1, 2, 19), 1024)]
    X, W, dY, ends, src = make(dev, sizes, 40, 72, getattr(torch, dtype), 14, tail=3, gather=True)
    (Y, dX, dW), (aY, aX, aW) = reference(X[src.long()], W, dY, sizes, False)
    f32 = dtype == "float32"
    assert within(emu.grouped_gemm(X, W, ends, src=src)[0], Y, aY, 40, f32)
    assert within(emu.grouped_gemm(dY, W, ends, opW=emu.OP_T)[0], dX, aX, 72, f32)
    assert within(emu.grouped_wgrad(X, dY, ends, srcA=src)[0], dW, aW, 19, f32)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows_past_2_31_elements(dev, dtype):
    """Token rows and results of more than 2^31 elements: the first and last rows
    of the product and of the rows' gradient, parts of the weights' gradient."""
    import torch
    dt, f32 = getattr(torch, dtype), dtype == "float32"
    G, rows, K, N = 3, 66000, 16, 32776
    g = torch.Generator(device=dev).manual_seed(15)
    X, W = torch.randn(rows, K, generator=g, device=dev).to(dt), torch.randn(G, K, N, generator=g, device=dev).to(dt)
    dY = torch.randn(rows, N, generator=g, device=dev).to(dt)
    ends = torch.tensor([100, 100, rows], dtype=torch.int32, device=dev)
    assert rows * N > 2 ** 31
    y, _ = emu.grouped_gemm(X, W, ends)
    dx, _ = emu.grouped_gemm(dY, W, ends, opW=emu.OP_T)
    for at, w in ((slice(0, 100), W[0].double()), (slice(rows - 70, rows), W[2].double())):
        x, d = X[at].double(), dY[at].double()
        assert within(y[at], x @ w, x.abs() @ w.abs(), K, f32)
        assert within(dx[at], d @ w.T, d.abs() @ w.abs().T, N, f32)
    del y, dx
    dw, _ = emu.grouped_wgrad(X, dY, ends)
    x = X[100:].double()
    for at in (slice(0, 65), slice(N - 65, N)):
        d = dY[100:, at].double()
        assert within(dw[2][:, at], x.T @ d, x.abs().T @ d.abs(), rows, f32)
    assert not dw[1].any()
