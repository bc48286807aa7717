"""Cases, inputs and plain forms of the expert layers' 8-bit and balance
operators: quantisation of rows to 8-bit integers with a scale for each row,
matrix products in 8-bit integers with scales for each token and channel (dense
or grouped by expert), and the routing's balance loss with its counts and gradient.

``own`` selects what ``run`` computes with: False, elementary torch operations;
True, this package's kernels, called as a user's program calls them.  ``exact``
gives the same results from the definitions in 64 bits."""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


# ------------------------------------------------------------------- cases
def listed():
    return [
        # one token's activations before an 8-bit product of a decoding step: latency
        dict(name="quantize one token", op="quantize", rows=1, cols=4096, dtype="bf16"),
        # FP32 rows of odd width, so of every alignment
        dict(name="quantize odd f32", op="quantize", rows=1537, cols=1027, dtype="f32"),
        # a prompt's activations, or a layer's weights, channel by channel
        dict(name="quantize 16384 rows", op="quantize", rows=16384, cols=4096, dtype="bf16"),
        # one token through one projection: the weights are read once
        dict(name="i8 one token", op="i8", rows=1, experts=0, active=0, K=4096, N=4096, dtype="bf16", gather=False,
             tail=0),
        # a few tokens through their experts, gathered by routing's order
        dict(name="i8 experts", op="i8", rows=16, experts=64, active=12, K=4096, N=2048, dtype="bf16", gather=True,
             tail=0),
        # a serving batch through a wide projection, FP32 answers
        dict(name="i8 batch of 48", op="i8", rows=48, experts=0, active=0, K=5120, N=8192, dtype="f32", gather=False,
             tail=0),
        # odd sizes throughout, gathered rows, rows that belong to no expert, an empty expert
        dict(name="i8 odd experts", op="i8", rows=1537, experts=7, active=6, K=333, N=517, dtype="f32", gather=True,
             tail=13),
        # prompts of several requests through the experts
        dict(name="i8 experts prompt", op="i8", rows=8192, experts=32, active=32, K=2048, N=4096, dtype="bf16",
             gather=True, tail=0),
        # long prompts through one projection (the largest case)
        dict(name="i8 prompt", op="i8", rows=16384, experts=0, active=0, K=8192, N=4096, dtype="bf16", gather=False,
             tail=0),
        # a small step's loss and gradient: latency
        dict(name="balance 64 tokens", op="balance", tokens=64, experts=64, k=4, dtype="f32", masked=False, add=False),
        # packed sequences of odd length, a third of the tokens is padding
        dict(name="balance odd masked", op="balance", tokens=5003, experts=60, k=6, dtype="f32", masked=True, add=True),
        # a training step's loss, counts and gradient, added to the gradient of the routing's weights
        dict(name="balance 32768 tokens", op="balance", tokens=32768, experts=128, k=8, dtype="bf16", masked=False,
             add=True),
    ]


def _log(rng, lo, hi):
    return min(max(int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))), lo), hi)


def _width(rng, lo, hi):
    """A matrix dimension: mostly a multiple of 16 or 64, at times any number."""
    step = rng.choice((1, 16, 64, 64))
    return max(lo, _log(rng, lo, hi) // step * step)


def draw(rng):
    most = {}
    for c in listed():
        w, m = work(c), most.setdefault(c["op"], [0.0, 0.0])
        m[0], m[1] = max(m[0], w["bytes"]), max(m[1], w["flops"])
    op = rng.choice(("quantize", "i8", "i8", "i8", "balance"))
    while True:
        dtype = rng.choice(("f32", "bf16"))
        if op == "quantize":
            c = dict(op=op, rows=_log(rng, 1, 32768), cols=_width(rng, 32, 16384), dtype=dtype)
        elif op == "i8":
            E, rows = rng.choice((0, 0, _log(rng, 2, 64))), _log(rng, 1, 16384)
            c = dict(op=op, rows=rows, experts=E, active=max(1, min(E, rows, int(E * rng.uniform(0.3, 1.2)))) if E else 0,
                     K=_width(rng, 32, 16384), N=_width(rng, 32, 16384), dtype=dtype, gather=rng.random() < 0.5,
                     tail=rng.choice((0, 0, 5)) if E else 0)
        else:
            E = _log(rng, 4, 512)
            c = dict(op=op, tokens=_log(rng, 1, 65536), experts=E, k=rng.randint(1, min(16, E)), dtype=dtype,
                     masked=rng.random() < 0.5, add=rng.random() < 0.5)
        w = work(c)
        held = max(1, c.get("experts", 0)) * c.get("K", 0) * c.get("N", 0)     # elements of all weights
        if w["bytes"] <= most[op][0] and w["flops"] <= most[op][1] and held <= 64 * 2048 * 4096:
            return c


# -------------------------------------------------------------------- work
def work(c):
    s = SIZE[c["dtype"]]
    if c["op"] == "quantize":
        R, K = c["rows"], c["cols"]
        return {"bytes": R * K * (s + 1) + 4 * R, "flops": 3.0 * R * K}
    if c["op"] == "i8":
        R, K, N = c["rows"], c["K"], c["N"]
        T = max(1, R // 4) if c["gather"] else R
        return {"bytes": T * K + max(1, c["active"]) * (K + 4) * N + R * N * s + 4 * T, "flops": 2.0 * R * K * N}
    T, E, k = c["tokens"], c["experts"], c["k"]
    b = T * E * s * (3 if c["add"] else 2) + 4 * T * k + 4 * E     # logits, experts, gradients to add; gradients out
    return {"bytes": b + (T if c["masked"] else 0), "flops": 12.0 * T * E}


# ------------------------------------------------------------------ inputs
def _ends(c, seed):
    """Group ends of `rows` rows spread unevenly over `active` of the experts."""
    rng = random.Random(seed)
    E, rows, active = c["experts"], c["rows"], c["active"]
    picked = sorted(rng.sample(range(E), active))
    share = [math.exp(0.5 * rng.gauss(0, 1)) for _ in picked]
    total, left, size = sum(share), rows - active, [1] * active
    for i, q in enumerate(share):
        size[i] += int(left * q / total)
    size[rng.randrange(active)] += rows - sum(size)
    count = [0] * E
    for p, n in zip(picked, size):
        count[p] = n
    ends, at = [], 0
    for n in count:
        at += n
        ends.append(at)
    return ends, max(count)


def _normal(g, shape, dtype, scale=1.0):
    t = torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)
    return t.mul_(scale) if scale != 1.0 else t


def _codes(g, shape):
    """8-bit codes of normally distributed values whose largest lies near four deviations."""
    t = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, 32.0, generator=g)
    return t.round_().clamp_(-127, 127).to(torch.int8)


def _scales(g, shape):
    return torch.rand(shape, generator=g, device="cuda") * 0.02 + 0.005


def prepare(case, seed):
    c, dt = dict(case), DTYPES[case["dtype"]]
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["op"] == "quantize":
        # rows of different size, as activations have them
        s["X"] = _normal(g, (c["rows"], c["cols"]), dt) * torch.exp(_normal(g, (c["rows"], 1), torch.float32)).to(dt)
    elif c["op"] == "i8":
        R, E, K, N = c["rows"] + c["tail"], c["experts"], c["K"], c["N"]
        lead = (E,) if E else ()
        T = max(1, R // 4) if c["gather"] else R
        s["X"] = (_codes(g, (T, K)), _scales(g, (T,)))
        s["W"] = (_codes(g, lead + (N, K)), _scales(g, lead + (N,)) / math.sqrt(K))
        s["src"] = torch.randint(0, T, (R,), generator=g, device="cuda", dtype=torch.int32) if c["gather"] else None
        s["ends"], s["most"] = None, R
        if E:
            ends, s["most"] = _ends(c, seed)
            s["ends"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
    else:
        T, E, k = c["tokens"], c["experts"], c["k"]
        # some experts are liked better than others; the gradient to add is of the loss's own size, so
        # that neither hides the other's errors
        s["logits"] = _normal(g, (T, E), dt, 1.5) + _normal(g, (1, E), dt, 0.5)
        s["experts"] = torch.topk(s["logits"].float(), k, dim=1).indices.to(torch.int32).contiguous()
        s["mask"] = torch.rand(T, generator=g, device="cuda") < 0.67 if c["masked"] else None
        s["add"] = _normal(g, (T, E), dt, 1e-4 / max(1, T)) if c["add"] else None
        s["dloss"] = torch.rand((), generator=g, device="cuda") + 0.5
        s["coef"] = 0.01
    return s


# ------------------------------------------------------------- plain forms
def _plain_quantize(s):
    """A row's scale is its largest magnitude over 127, rounded to FP32; a code is
    the value over the scale, rounded to the nearest integer (ties to even).  The
    quotients are taken in 64 bits: in 32 they can round onto a border of two results.
    Codes are whole numbers that this definition fixes, and returned as such."""
    X = s["X"].float()
    scales = (X.abs().amax(1).double() / 127).float()
    q = torch.round(X.double() / torch.where(scales > 0, scales, 1.0).double()[:, None])
    return {"codes": q.clamp(-127, 127).to(torch.int8), "scales": scales}


def _plain_i8(s):
    c, (X, xs), (W, ws), dt = s["case"], s["X"], s["W"], DTYPES[s["case"]["dtype"]]
    R = c["rows"] + c["tail"]
    if s["src"] is not None:
        X, xs = X[s["src"].long()], xs[s["src"].long()]
    Xf = X.float()
    if s["ends"] is None:
        return {"Y": ((Xf @ W.float().T) * ws * xs[:, None]).to(dt)}
    ends, E = s["ends"].long(), c["experts"]
    slot = torch.arange(R, device=X.device)
    of = torch.searchsorted(ends, slot, right=True)             # expert of each row; E: none
    there = (of < E)[:, None]
    of = of.clamp(max=E - 1)
    if R <= E:                                                  # few rows: each with its own expert's matrix
        Y = torch.bmm(W[of].float(), Xf[:, :, None])[:, :, 0]
    else:
        starts = torch.cat([ends.new_zeros(1), ends[:-1]])
        at = starts[:, None] + torch.arange(s["most"], device=X.device)
        Xp = torch.where((at < ends[:, None])[..., None], Xf[at.clamp(max=R - 1)], 0.0)
        Y = torch.bmm(Xp, W.float().transpose(1, 2))[of, (slot - starts[of]).clamp(max=s["most"] - 1)]
    return {"Y": torch.where(there, Y * ws[of] * xs[:, None], 0.0).to(dt)}


def _plain_balance(s):
    """loss = coef E / (n k) sum_e counts_e P_e over the n tokens that count, P_e their
    mean softmax probability of expert e; counts are constants in the gradient."""
    c, x, mask = s["case"], s["logits"].float(), s["mask"]
    T, E, k = c["tokens"], c["experts"], c["k"]
    on = mask.float() if mask is not None else torch.ones(T, device=x.device)
    p = torch.exp(x - x.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True) * on[:, None]
    n = on.sum()
    counts = torch.zeros(E, dtype=torch.int64, device=x.device)
    counts.scatter_add_(0, s["experts"].reshape(-1).long(), on.long().repeat_interleave(k))
    many = n.clamp(min=1.0)
    f = s["coef"] * E / (many * k) * counts.float()
    loss = (f * (p.sum(0) / many)).sum()
    d = s["dloss"] / many * p * (f - (p * f).sum(1, keepdim=True))
    if s["add"] is not None:
        d = d + s["add"].float()
    return {"loss": loss, "counts": counts.to(torch.int32), "dlogits": d.to(s["logits"].dtype)}


PLAIN = {"quantize": _plain_quantize, "i8": _plain_i8, "balance": _plain_balance}


# -------------------------------------------------------------- the kernels
def _own_quantize(s, emu):
    q = emu.i8_quantize(s["X"])
    return {"codes": q.codes, "scales": q.scales}


def _own_i8(s, emu):
    Y, _ = emu.i8_gemm(s["X"], s["W"], ends=s["ends"], src=s["src"], dtype=DTYPES[s["case"]["dtype"]])
    return {"Y": Y}


def _own_balance(s, emu):
    b, _ = emu.route_balance(s["logits"], s["experts"], coef=s["coef"], mask=s["mask"])
    d = emu.route_balance_backward(s["logits"], b, dloss=s["dloss"], coef=s["coef"], mask=s["mask"], add=s["add"])
    return {"loss": b.loss, "counts": b.counts, "dlogits": d}


OWN = {"quantize": _own_quantize, "i8": _own_i8, "balance": _own_balance}


def run(state):
    op = state["case"]["op"]
    if own:
        import paper_2609_04663_gb300 as emu
        return OWN[op](state, emu)
    return PLAIN[op](state)


# ------------------------------------------------------------------- exact
def exact(case, seed):
    """The same results in 64 bits, expert by expert and block of rows by block of rows."""
    s = prepare(case, seed)
    c = s["case"]
    if c["op"] == "quantize":
        codes, scales = [], []
        for x in s["X"].split(2048):
            x = x.double()
            # the definition rounds a scale to FP32 before it divides by it
            a = (x.abs().max(1).values / 127).float()
            whole = torch.floor(x / a.double()[:, None])
            rest = x - whole * a.double()[:, None]              # exact: 8 and 24 bits
            up = 2 * rest - a.double()[:, None]
            codes.append((whole + ((up > 0) | ((up == 0) & (whole % 2 != 0)))).clamp(-127, 127).to(torch.int8))
            scales.append(a.double())
        return {"codes": torch.cat(codes), "scales": torch.cat(scales)}
    if c["op"] == "i8":
        R, N = c["rows"] + c["tail"], c["N"]
        at = s["src"].long() if s["src"] is not None else torch.arange(R, device=s["X"][0].device)
        ends = [0] + (s["ends"].tolist() if s["ends"] is not None else [R])
        Y = torch.zeros(R, N, dtype=torch.float64, device=at.device)
        for e, (a, b) in enumerate(zip(ends, ends[1:])):
            w, v = (t[e] if s["ends"] is not None else t for t in s["W"])
            w, v = w.double() if b > a else w, v.double()
            for i in range(a, b, 4096):
                j = at[i:min(b, i + 4096)]
                Y[i:min(b, i + 4096)] = (s["X"][0][j].double() @ w.T) * (s["X"][1][j].double()[:, None] * v)
        return {"Y": Y}
    x, E, k = s["logits"].double(), c["experts"], c["k"]
    on = s["mask"] if s["mask"] is not None else torch.ones(len(x), dtype=torch.bool, device=x.device)
    counts = torch.bincount(s["experts"][on].reshape(-1).long(), minlength=E)
    n, p = int(on.sum()), torch.softmax(x, 1)
    f = counts.double() * (s["coef"] * E / (max(n, 1) * k))
    loss = p[on].sum(0) @ f / max(n, 1)
    d = torch.zeros_like(x)
    d[on] = (p * (f - (p @ f)[:, None]))[on] * (s["dloss"].double() / max(n, 1))
    if s["add"] is not None:
        d += s["add"].double()
    return {"loss": loss, "counts": counts.int(), "dlogits": d}
