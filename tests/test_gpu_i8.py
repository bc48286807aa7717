"""Quantisation of rows to 8-bit integers and products of 8-bit integers against
their definitions in 64 bits.

Codes, scales and integer sums have one right value each: they have to be equal.  A
product with scales rounds its sum to FP32 and multiplies twice: three roundings of
2^-24 relative to the value, (1 + 2^-24)^3 - 1 < 3.01 * 2^-24; BF16 results take one more of 2^-8."""
import numpy as np
import pytest
import torch

import paper_2609_04663_gb300 as emu
from helpers import device

pytestmark = pytest.mark.gpu

F32_TOL = 3.01 * 2.0 ** -24
BF16_TOL = 2.0 ** -8 + F32_TOL * (1 + 2.0 ** -8)


@pytest.fixture(scope="module")
def dev():
    return device()


def gen(dev, seed):
    return torch.Generator(device=dev).manual_seed(seed)


# ------------------------------------------------------------------ quantise
def quantized(X):
    """(codes, scales) by the definition, in 64 bits: a quotient of two FP32 numbers is at least
    2^-26 of its size away from a border that it is not on, and 64 bits hold 2^-53."""
    x = X.double()
    amax = x.abs().amax(-1) if x.shape[-1] else torch.zeros(x.shape[:-1], dtype=torch.float64, device=x.device)
    s = (amax / 127).float()
    d = torch.where(s > 0, s, torch.ones_like(s)).double()
    q = torch.round(x / d[..., None]).clamp(-127, 127) * (s > 0)[..., None]
    return q.to(torch.int8), s


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (3, 8), (2, 33), (5, 128), (9, 500), (1, 512), (7, 513), (4, 1024),
                                       (3, 1027), (2, 4096), (3, 4097), (2, 16384), (1, 16391), (2, 40000), (1500, 96)])
def test_codes_and_scales_are_the_definition(dev, rows, cols, dtype):
    g = gen(dev, rows * 131 + cols)
    X = (torch.randn(rows, cols, generator=g, device=dev) * torch.exp(2 * torch.randn(rows, 1, generator=g, device=dev))).to(dtype)
    q = emu.i8_quantize(X)
    codes, scales = quantized(X)
    assert torch.equal(q.scales, scales)
    assert torch.equal(q.codes, codes)


def test_quotients_on_and_next_to_borders(dev):
    # scale 1 (largest magnitude 127), then halves exactly on the border and one FP32 step to
    # either side; a row of the same times 3 / 1024 has another scale and no ties
    n = np.arange(-126, 127, dtype=np.float32) + np.float32(0.5)
    row = np.concatenate([n, np.nextafter(n, np.float32(1e9)), np.nextafter(n, np.float32(-1e9)), [np.float32(127)]])
    X = torch.from_numpy(np.stack([row, row * np.float32(3 / 1024), -row])).to(dev)
    q = emu.i8_quantize(X)
    codes, scales = quantized(X)
    assert float(scales[0]) == 1.0 and torch.equal(q.scales, scales) and torch.equal(q.codes, codes)
    assert q.codes[0, :4].tolist() == [-126, -124, -124, -122]                        # -125.5, -124.5, .. to even


def test_extreme_rows(dev):
    big, tiny, sub = 3.4e38, 1.2e-38, 1.4e-45
    rows = [[0.0] * 9, [-0.0] * 9, [big, -big, big / 2, big / 254, 1.0, 0, 0, 0, 0], [tiny, -tiny / 2, tiny / 254, 0, 0, 0, 0, 0, 0],
            [sub * 200, sub * 100, sub, -sub * 180, 0, 0, 0, 0, 0], [sub * 180, -sub * 90, 0, 0, 0, 0, 0, 0, 0],
            [sub, sub, 0, 0, 0, 0, 0, 0, 0], [1e-25, 3e-27, -1e-26, 5e-26, 0, 0, 0, 0, 0]]
    X = torch.tensor(rows, dtype=torch.float32, device=dev)
    q = emu.i8_quantize(X)
    codes, scales = quantized(X)
    assert torch.equal(q.scales, scales) and torch.equal(q.codes, codes)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("cols,at", [(40, 39), (3000, 2999), (70000, 69000)])
def test_rows_that_are_not_finite(dev, cols, at, bad, dtype):
    X = torch.randn(5, cols, generator=gen(dev, 3), device=dev).to(dtype)
    want, scales = quantized(X)
    X[2, at] = bad
    ws = emu.workspace(emu.emu_split_workspace_bytes(32), dev)
    q = emu.i8_quantize(X, ws=ws)
    assert emu.read_flags(ws) == emu.FLAG_NONFINITE
    keep = [0, 1, 3, 4]
    assert torch.equal(q.codes[keep], want[keep]) and torch.equal(q.scales[keep], scales[keep])
    assert bool(q.scales[2].isnan()) and not q.codes[2].any()
    X[2, at] = 0.0
    emu.i8_quantize(X, ws=ws)
    assert emu.read_flags(ws) == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_matrices_pitches_and_given_results(dev, dtype):
    g = gen(dev, 5)
    big = torch.randn(3, 10, 101, generator=g, device=dev).to(dtype)
    X = big[:, 1:8, 3:72]                                       # any alignment, distance and pitch of their own
    out = torch.full((3, 9, 90), 99, dtype=torch.int8, device=dev)
    codes = out[:, 1:8, 5:74]
    sc = torch.empty(3, 7, device=dev)
    q = emu.i8_quantize(X, codes=codes, scales=sc)
    want, scales = quantized(X)
    assert torch.equal(codes, want) and torch.equal(sc, scales) and q.codes.data_ptr() == codes.data_ptr()
    codes.fill_(99)
    assert bool((out == 99).all())                              # nothing else was written
    empty = emu.i8_quantize(torch.empty(0, 5, dtype=dtype, device=dev))
    assert empty.codes.shape == (0, 5) and empty.scales.shape == (0,)
    none = emu.i8_quantize(torch.empty(4, 0, dtype=dtype, device=dev))
    assert none.codes.shape == (4, 0) and none.scales.tolist() == [0.0] * 4


# ------------------------------------------------------------------- products
def make(dev, rows, N, K, G=0, seed=0, pad=0):
    g = gen(dev, seed + rows + 7 * N + 31 * K)
    lead = (G,) if G else ()
    X = torch.randint(-128, 128, (rows, K + pad), generator=g, device=dev, dtype=torch.int8)[:, :K]
    W = torch.randint(-128, 128, lead + (N, K + pad), generator=g, device=dev, dtype=torch.int8)[..., :K]
    xs = torch.rand(rows, generator=g, device=dev) * 0.1 + 0.01
    ws = torch.rand(lead + (N,), generator=g, device=dev) * 0.1 + 0.01
    return (X, xs), (W, ws)


def spans(ends, rows):
    out, at = [], 0
    for e in ends:
        e = min(max(e, at), rows)
        out.append((at, e))
        at = e
    return out


def sums(X, W, ends=None, src=None):
    """The sums in 64 bits, as integers (64-bit floating point holds them exactly)."""
    x = X[src.long().clamp(0, X.shape[0] - 1)].double() if src is not None else X.double()
    if src is not None:
        x[(src < 0) | (src >= X.shape[0])] = 0
    if ends is None:
        return x @ W.double().T
    Y = torch.zeros(x.shape[0], W.shape[1], dtype=torch.float64, device=x.device)
    for e, (a, b) in enumerate(spans(ends, x.shape[0])):
        Y[a:b] = x[a:b] @ W[e].double().T
    return Y


def scaled(S, xs, ws, ends=None, src=None):
    r = S.shape[0]
    t = torch.arange(r, device=S.device) if src is None else src.long().clamp(0, xs.shape[0] - 1)
    Y = S * xs[t].double()[:, None]
    if ends is None:
        return Y * ws.double()
    for e, (a, b) in enumerate(spans(ends, r)):
        Y[a:b] *= ws[e].double()
    return Y


def space(X, W, ends=None, src=None):
    """A workspace that is enough for the call however W lies, or for its flags."""
    rows, G = src.numel() if src is not None else X[0].shape[0], 1 if ends is None else len(ends)
    need = emu.emu_i8_gemm_workspace_bytes(G, rows, W[0].shape[-2], W[0].shape[-1], 0)
    return emu.workspace(max(need, emu.emu_split_workspace_bytes(32)), X[0].device)


def check(X, W, ends=None, src=None, flags=0):
    e = None if ends is None else torch.tensor(ends, dtype=torch.int32, device=X[0].device)
    S = sums(X[0], W[0], ends, src)
    ws = space(X, W, ends, src)
    Y, _ = emu.i8_gemm(X, W, ends=e, src=src, dtype=torch.int32, ws=ws)
    assert emu.read_flags(ws) == flags
    assert torch.equal(Y.double(), S), float((Y.double() - S).abs().max())
    want = scaled(S, X[1], W[1], ends, src)
    for dtype, tol in ((torch.float32, F32_TOL), (torch.bfloat16, BF16_TOL)):
        Y, _ = emu.i8_gemm(X, W, ends=e, src=src, dtype=dtype, ws=ws)
        assert emu.read_flags(ws) == flags and Y.dtype is dtype
        assert torch.equal(Y, emu.i8_gemm(X, W, ends=e, src=src, dtype=dtype)[0])      # in a workspace of its own, or none
        assert bool(((Y.double() - want).abs() <= tol * want.abs()).all())


SIZES = [(1, 1, 1), (1, 5, 16), (1, 517, 333), (1, 4096, 4096), (2, 64, 64), (3, 130, 129), (4, 96, 512), (5, 257, 1024),
         (8, 128, 1025), (9, 300, 2049), (16, 640, 1008), (17, 129, 4097), (33, 1000, 2048), (64, 384, 512), (65, 511, 700),
         (128, 256, 1024), (130, 1000, 1100), (256, 512, 1040), (257, 264, 3000), (700, 130, 64), (1030, 700, 2064),
         (2500, 2500, 100), (515, 4100, 1300)]


@pytest.mark.parametrize("rows,N,K", SIZES)
def test_one_matrix(dev, rows, N, K):
    check(*make(dev, rows, N, K))


@pytest.mark.parametrize("K", [1, 2, 15, 17, 63, 127, 129])
@pytest.mark.parametrize("rows,N", [(1, 1), (9, 1), (40, 127), (300, 2), (700, 257)])
def test_short_contractions_and_narrow_results(dev, rows, N, K):
    check(*make(dev, rows, N, K))


@pytest.mark.parametrize("rows,N,K", [(1, 40, 333), (6, 40, 333), (20, 200, 333), (300, 300, 1029)])
def test_rows_on_16_bytes_within_a_wider_pitch(dev, rows, N, K):
    check(*make(dev, rows, N, K, pad=-K % 16))
    check(*make(dev, rows, N, K, pad=1))


GROUPS = [([3, 3, 7, 8], 8), ([0, 0, 0], 4), ([5], 9), ([1, 2, 3, 4, 5, 6], 6), ([16, 16, 40, 41, 41, 100], 100),
          ([64, 65, 300, 300, 301], 310), ([0, 700, 700], 700), ([255, 511, 513, 1000], 1003)]


@pytest.mark.parametrize("ends,rows", GROUPS)
@pytest.mark.parametrize("N,K", [(37, 70), (272, 1088), (600, 2050)])
def test_groups(dev, ends, rows, N, K):
    check(*make(dev, rows, N, K, G=len(ends)), ends=ends)


@pytest.mark.parametrize("ends,rows", GROUPS)
def test_gathered_rows(dev, ends, rows):
    X, W = make(dev, 50, 144, 400, G=len(ends))
    src = torch.randint(0, 50, (rows,), generator=gen(dev, rows), device=dev, dtype=torch.int32)
    check(X, W, ends=ends, src=src)


@pytest.mark.parametrize("rows", [6, 120, 900])
def test_bad_rows_and_ends_are_flagged(dev, rows):
    X, W = make(dev, 50, 144, 400, G=3)
    src = torch.randint(0, 50, (rows,), generator=gen(dev, rows), device=dev, dtype=torch.int32)
    bad = src.clone()
    bad[1], bad[rows - 1], bad[rows // 2] = -1, 50, 2 ** 31 - 1
    check(X, W, ends=[2, rows // 2, rows], src=bad, flags=emu.FLAG_INDEX)
    check(X, W, ends=[rows // 2, 2, rows], src=src, flags=emu.FLAG_INDEX)
    check(X, W, ends=[-5, 4, rows + 9], src=src, flags=emu.FLAG_INDEX)


@pytest.mark.parametrize("rows", [3, 200])
def test_no_rows_to_take_and_nothing_to_multiply(dev, rows):
    X, W = make(dev, 5, 40, 64)
    none = (X[0][:0], X[1][:0])
    src = torch.arange(rows, dtype=torch.int32, device=dev)
    ws = space(none, W, src=src)
    Y, _ = emu.i8_gemm(none, W, src=src, dtype=torch.float32, ws=ws)
    assert emu.read_flags(ws) == emu.FLAG_INDEX and Y.shape == (rows, 40) and not Y.any()
    Y, _ = emu.i8_gemm(none, W, ws=ws)
    assert Y.shape == (0, 40) and emu.read_flags(ws) == 0
    Y, _ = emu.i8_gemm((X[0][:, :0], X[1]), (W[0][:, :0], W[1]))
    assert Y.shape == (5, 40) and not Y.any()
    Y, _ = emu.i8_gemm(X, (W[0][:0], W[1][:0]))
    assert Y.shape == (5, 0)


@pytest.mark.parametrize("rows", [2, 60, 600])
def test_scales_left_out(dev, rows):
    (x, xs), (w, v) = make(dev, rows, 80, 192)
    S = sums(x, w)
    for X, W, want in (((x, None), (w, v), S * v.double()), ((x, xs), (w, None), S * xs.double()[:, None]), ((x, None), (w, None), S)):
        Y, _ = emu.i8_gemm(X, W, dtype=torch.float32)
        assert bool(((Y.double() - want).abs() <= F32_TOL * want.abs()).all())


def test_past_two_to_the_31(dev):
    # weights of 4.9 GB: the last group's lie past 2^32 bytes
    G, N, K = 5, 8192, 119984
    W = torch.empty(G, N, K, dtype=torch.int8, device=dev).random_(-128, 128, generator=gen(dev, 1))
    v = torch.rand(G, N, device=dev)
    some = torch.randint(0, N, (50,), device=dev)
    for rows in (2, 20):
        X = torch.empty(rows, K, dtype=torch.int8, device=dev).random_(-128, 128, generator=gen(dev, rows))
        xs = torch.rand(rows, device=dev)
        ends = torch.tensor([0, 0, 0, 0, rows], dtype=torch.int32, device=dev)
        ws = space((X, xs), (W, v), ends)
        Y, _ = emu.i8_gemm((X, xs), (W, v), ends=ends, dtype=torch.int32, ws=ws)
        assert torch.equal(Y[:, some].double(), X.double() @ W[4][some].double().T) and emu.read_flags(ws) == 0
    del W
    # and an answer of 4.6 GB
    X, W = make(dev, 70001, 32768, 64)
    Y, ws = emu.i8_gemm(X, W)
    at = torch.tensor([0, 1, 65535, 65536, 70000], device=dev)
    want = scaled(sums(X[0][at], W[0]), X[1][at], W[1])
    assert bool(((Y[at].double() - want).abs() <= BF16_TOL * want.abs()).all()) and emu.read_flags(ws) == 0


def test_quantise_past_two_to_the_31(dev):
    X = torch.empty(40000, 65536, dtype=torch.bfloat16, device=dev).normal_(generator=gen(dev, 2))
    q = emu.i8_quantize(X)
    at = torch.tensor([0, 17, 32767, 32768, 39999], device=dev)
    codes, scales = quantized(X[at])
    assert torch.equal(q.codes[at], codes) and torch.equal(q.scales[at], scales)


@pytest.mark.parametrize("rows,N,K", [(1030, 700, 2064), (4000, 1000, 1040), (20, 4096, 5136), (6, 900, 2064)])
def test_the_same_sums_every_time(dev, rows, N, K):
    # a stage's last bytes must not be given up before they are read: K that ends inside of one, many times
    X, W = make(dev, rows, N, K)
    S = sums(X[0], W[0]).int()
    off = torch.zeros((), dtype=torch.int64, device=dev)
    for _ in range(500):
        off += (emu.i8_gemm(X, W, dtype=torch.int32)[0] != S).sum()
    assert int(off) == 0


@pytest.mark.parametrize("N,K", [(1300, 333), (1301, 1100), (1024, 17), (1500, 129), (1100, 2064)])
@pytest.mark.parametrize("ends", [None, [4000, 4000, 4001, 5300, 5990], [1, 300, 2300, 4444, 6000]])
def test_many_rows(dev, ends, N, K):
    # sizes that pairs of SMs get, of any alignment, gathered
    G = len(ends) if ends else 0
    assert emu.emu_i8_gemm_workspace_bytes(max(G, 1), 6000, N, K, 1) > 0
    X, W = make(dev, 6000 if not ends else 777, N, K, G=G)
    if not ends:
        return check(X, W)
    src = torch.randint(0, 777, (6000,), generator=gen(dev, N), device=dev, dtype=torch.int32)
    check(X, W, ends=ends, src=src)


@pytest.mark.parametrize("K", [2064, 2050, 4112])
@pytest.mark.parametrize("per", [65, 49, 17])
def test_parts_of_the_contraction_and_several_tiles_each(dev, per, K):
    # more tiles than clusters that share a contraction: sums are handed over again and again
    G, N = 7, 600
    ends = [per * (g + 1) for g in range(6)] + [448]
    X, W = make(dev, 448, N, K, G=G)
    check(X, W, ends=ends)
    src = torch.randint(0, 448, (448,), generator=gen(dev, K), device=dev, dtype=torch.int32)
    check(X, W, ends=ends, src=src)


def test_many_groups(dev):
    rng = np.random.default_rng(0)
    for per in (1, 40):
        ends = np.cumsum(rng.integers(0, 2 * per, size=1024)).tolist()
        check(*make(dev, ends[-1] + 3, 20, 48, G=1024), ends=ends)


@pytest.mark.parametrize("rows", [1, 7, 20, 150, 600])
def test_largest_sums(dev, rows):
    # the longest contraction, all codes at the end of their range: the sums reach 2^31 - 16384
    K = 131071
    X = torch.full((rows, K), -128, dtype=torch.int8, device=dev)
    W = torch.full((130, K), -128, dtype=torch.int8, device=dev)
    W[1::2] = 127
    ws = space((X, None), (W, None))
    Y, _ = emu.i8_gemm((X, None), (W, None), dtype=torch.int32, ws=ws)
    assert emu.read_flags(ws) == 0
    assert bool((Y[:, 0::2] == 128 * 128 * K).all()) and bool((Y[:, 1::2] == -128 * 127 * K).all())


@pytest.mark.parametrize("rows,N,K", [(1, 100, 96), (3, 37, 33), (40, 150, 96), (300, 131, 200), (600, 500, 1200)])
@pytest.mark.parametrize("dtype", [torch.int32, torch.float32, torch.bfloat16])
def test_results_in_a_pitch_of_their_own(dev, rows, N, K, dtype):
    X, W = make(dev, rows, N, K)
    for left, right in ((0, 8), (1, 2), (3, 0)):
        out = torch.full((rows + 2, N + left + right), 77, dtype=dtype, device=dev)
        Y = out[1:-1, left:left + N]
        emu.i8_gemm(X, W, Y=Y)
        want, _ = emu.i8_gemm(X, W, dtype=dtype)
        assert torch.equal(Y, want)
        Y.fill_(77)
        assert bool((out == 77).all())


def test_shared_and_overlapping_weights(dev):
    # one matrix for all groups (distance 0), and matrices that share rows
    (x, xs), (w, _) = make(dev, 200, 64, 96)
    ends = [50, 120, 200]
    v = torch.rand(3, 64, device=dev)
    check((x, xs), (w[None].expand(3, 64, 96), v), ends=ends)
    check((x[:9].contiguous(), xs[:9].contiguous()), (w[None].expand(3, 64, 96), v), ends=[2, 3, 9])
    _, (tall, _) = make(dev, 1, 96, 96)
    check((x, xs), (tall.as_strided((3, 64, 96), (16 * 96, 96, 1)), v), ends=ends)


def test_scales_that_are_not_finite_reach_only_their_own(dev):
    (x, xs), (w, v) = make(dev, 300, 200, 320)
    xs[7], v[11] = float("nan"), float("inf")
    Y, _ = emu.i8_gemm((x, xs), (w, v), dtype=torch.float32)
    assert bool(Y[7].isnan().all()) and bool((~Y[:7, 11].isfinite()).all())
    Y[7], Y[:, 11] = 0, 0
    assert bool(Y.isfinite().all())


@pytest.mark.parametrize("rows,N,K,G", [(1, 512, 512, 0), (48, 1000, 2048, 0), (900, 300, 500, 3)])
def test_other_streams_graphs_and_two_calls_at_once(dev, rows, N, K, G):
    ends = None if not G else torch.tensor([rows // 5, rows // 2, rows], dtype=torch.int32, device=dev)
    a, b = make(dev, rows, N, K, G, seed=1), make(dev, rows, N, K, G, seed=2)
    want = [emu.i8_gemm(*p, ends=ends)[0] for p in (a, b)]
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(dev), torch.cuda.Stream(dev)
    got = []
    for _ in range(5):
        for s, p in ((s1, a), (s2, b)):
            got.append(emu.i8_gemm(*p, ends=ends, stream=s)[0])
    torch.cuda.synchronize()
    for i, y in enumerate(got):
        assert torch.equal(y, want[i % 2])
    # captured and replayed, two graphs with one workspace, other inputs in the same place
    (x, xs), W = a
    ws = space((x, xs), W, ends)
    Y1, _ = emu.i8_gemm((x, xs), W, ends=ends, ws=ws)
    Y2 = torch.empty_like(Y1)
    graphs = []
    torch.cuda.synchronize()
    for Y in (Y1, Y2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            emu.i8_gemm((x, xs), W, ends=ends, Y=Y, ws=ws)
        graphs.append(gr)
    for inputs, y in ((a[0], want[0]), (b[0], emu.i8_gemm(b[0], W, ends=ends)[0])):
        x.copy_(inputs[0])
        xs.copy_(inputs[1])
        Y1.zero_()
        Y2.zero_()
        for gr in graphs * 2:
            gr.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y1, y) and torch.equal(Y2, y) and emu.read_flags(ws) == 0


def test_quantise_multiply_twice(dev):
    # the run of an 8-bit expert's two matrices: its error is the quantisation's alone
    g = gen(dev, 9)
    x = torch.randn(40, 256, generator=g, device=dev).bfloat16()
    W1, W2 = (torch.randn(4, n, k, generator=g, device=dev) for n, k in ((512, 256), (256, 512)))
    ends = torch.tensor([10, 10, 33, 40], dtype=torch.int32, device=dev)
    src = torch.randperm(40, generator=g, device=dev).int()
    q1, q2 = emu.i8_quantize(W1), emu.i8_quantize(W2)
    ws = emu.workspace(max(emu.emu_i8_gemm_workspace_bytes(4, 40, 512, 256, 0), emu.emu_i8_gemm_workspace_bytes(4, 40, 256, 512, 0)), dev)
    h, _ = emu.i8_gemm(emu.i8_quantize(x), q1, ends=ends, src=src, ws=ws)
    y, _ = emu.i8_gemm(emu.i8_quantize(h), q2, ends=ends, ws=ws)
    # (the sums as integers first: those of scaled codes would leave 2^-53 of their terms where the sum is 0)
    cx, cw1, cw2 = quantized(x), quantized(W1), quantized(W2)
    hw = scaled(sums(cx[0], cw1[0], ends.tolist(), src), cx[1], cw1[1], ends.tolist(), src)
    assert bool(((h.double() - hw).abs() <= BF16_TOL * hw.abs()).all())
    ch = quantized(h)
    yw = scaled(sums(ch[0], cw2[0], ends.tolist()), ch[1], cw2[1], ends.tolist())
    assert bool(((y.double() - yw).abs() <= BF16_TOL * yw.abs()).all())
