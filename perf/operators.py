"""Cases, inputs and plain forms of the expert-layer operators: routing of
tokens to experts, matrix products grouped by expert, matrix-vector products
with 4-bit weights, and the weighted sum of the experts' answers.

``own`` selects what ``run`` computes with: False, elementary torch operations
in 32 bits; True, this package's kernels, called as a user's program calls
them (the workspaces and results that such a program keeps are in the state).
``exact`` gives the same results from the definitions in 64 bits."""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


# ------------------------------------------------------------------- cases
def listed():
    return [
        # one decoding step of a few sequences: latency of the routing itself
        dict(name="route 8 tokens", op="route", tokens=8, experts=64, k=4, dtype="f32", renorm=True, train=False),
        # a training step's routing, probabilities over all experts, with the logits' gradient
        dict(name="route 32768 train", op="route", tokens=32768, experts=128, k=8, dtype="bf16", renorm=False,
             train=True),
        # one token decoded: each of its experts' matrices is read for one row
        dict(name="experts one token", op="grouped", rows=4, experts=32, active=4, K=2048, N=4096, dtype="bf16",
             trans=True, train=False, gather=False, tail=0),
        # a small serving batch in FP32: sixteen rows or so for each expert
        dict(name="experts batch f32", op="grouped", rows=256, experts=16, active=16, K=1024, N=2048, dtype="f32",
             trans=False, train=False, gather=False, tail=0),
        # odd sizes throughout, gathered rows, rows that belong to no expert, an empty expert; a training step
        dict(name="experts odd f32", op="grouped", rows=1537, experts=7, active=6, K=333, N=517, dtype="f32",
             trans=False, train=True, gather=True, tail=13),
        # training in FP32: product and both gradients
        dict(name="experts train f32", op="grouped", rows=16384, experts=16, active=16, K=2048, N=2048, dtype="f32",
             trans=False, train=True, gather=False, tail=0),
        # training in BF16 with the rows gathered from the tokens: product and both gradients (the largest case)
        dict(name="experts train bf16", op="grouped", rows=32768, experts=64, active=64, K=2048, N=4096, dtype="bf16",
             trans=False, train=True, gather=True, tail=0),
        # one token through one projection with 4-bit weights
        dict(name="w4 one token", op="w4", rows=1, experts=0, active=0, N=4096, K=4096, group=128, dtype="bf16",
             zeros=False),
        # a few tokens through their experts' 4-bit weights
        dict(name="w4 experts", op="w4", rows=16, experts=64, active=12, N=2048, K=4096, group=32, dtype="bf16",
             zeros=True),
        # several FP32 rows through one large matrix (an output head)
        dict(name="w4 seven rows f32", op="w4", rows=7, experts=0, active=0, N=16384, K=8192, group=64, dtype="f32",
             zeros=True),
        # the experts' answers of a decoding step added up
        dict(name="combine 4 tokens", op="combine", tokens=4, k=4, cols=2048, dtype="bf16", train=False),
        # the same in a training step, with the gradients of the answers and of the weights
        dict(name="combine 16384 train", op="combine", tokens=16384, k=4, cols=2048, dtype="bf16", train=True),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return min(max(v + (v == 3 << 10), lo), hi)


def _width(rng, lo, hi):
    """A matrix dimension: mostly a multiple of 8 or 64, at times any number."""
    v = _log(rng, lo, hi)
    step = rng.choice((1, 8, 64, 64))
    v = max(lo, v // step * step)
    return v + step if v == 3 << 10 else v


def draw(rng):
    most = {}
    for c in listed():
        w, m = work(c), most.setdefault(c["op"], [0.0, 0.0])
        m[0], m[1] = max(m[0], w["bytes"]), max(m[1], w["flops"])
    op = rng.choice(("route", "grouped", "grouped", "w4", "combine"))
    while True:
        dtype = rng.choice(("f32", "bf16"))
        if op == "route":
            E = _log(rng, 4, 512)
            c = dict(op=op, tokens=_log(rng, 1, 65536), experts=E, k=rng.randint(1, min(16, E)), dtype=dtype,
                     renorm=rng.random() < 0.5, train=rng.random() < 0.5)
        elif op == "grouped":
            E, rows = _log(rng, 1, 128), _log(rng, 1, 65536)
            c = dict(op=op, rows=rows, experts=E, active=max(1, min(E, rows, int(E * rng.uniform(0.5, 1.2)))),
                     K=_width(rng, 32, 8192), N=_width(rng, 32, 8192), dtype=dtype, trans=rng.random() < 0.5,
                     train=rng.random() < 0.5, gather=rng.random() < 0.5, tail=rng.choice((0, 0, 5)))
        elif op == "w4":
            E, rows = rng.choice((0, 0, _log(rng, 2, 64))), _log(rng, 1, 16)
            group = rng.choice((32, 64, 128))
            K = max(1, _log(rng, 128, 16384) // group) * group
            c = dict(op=op, rows=rows, experts=E, active=max(1, min(E, rows, int(E * rng.uniform(0.2, 1)))) if E else 0,
                     N=_width(rng, 64, 16384), K=K + group if K == 3 << 10 else K, group=group, dtype=dtype,
                     zeros=rng.random() < 0.5)
        else:
            c = dict(op=op, tokens=_log(rng, 1, 32768), k=rng.randint(1, 8), cols=_width(rng, 64, 8192), dtype=dtype,
                     train=rng.random() < 0.5)
        w = work(c)
        held = max(1, c.get("experts", 0)) * c.get("K", 0) * c.get("N", 0)     # elements of all weights
        if w["bytes"] <= most[op][0] and w["flops"] <= most[op][1] and held <= 64 * 2048 * 4096:
            return c


# -------------------------------------------------------------------- work
def work(c):
    s = SIZE[c["dtype"]]
    if c["op"] == "route":
        T, E, k = c["tokens"], c["experts"], c["k"]
        b, f = T * E * s + T * k * 16 + 4 * E, 3.0 * T * E
        if c["train"]:       # logits and the weights' gradients read, the logits' gradients written
            b, f = b + T * E * 2 * s + T * k * 8, f + 6.0 * T * E
        return {"bytes": b, "flops": f}
    if c["op"] == "grouped":
        R, K, N = c["rows"], c["K"], c["N"]
        T = max(1, R // 4) if c["gather"] else R
        f, b = 2.0 * R * K * N, (T * K + R * N + c["active"] * K * N) * s
        if c["train"]:       # dX = dY.W^T and dW = X^T.dY besides
            f, b = 3 * f, b + (R * (2 * N + K) + T * K + (c["active"] + c["experts"]) * K * N) * s
        return {"bytes": b, "flops": f}
    if c["op"] == "w4":
        R, K, N, g = c["rows"], c["K"], c["N"], c["group"]
        each = N * K // 2 + N * (K // g) * (s + (1 if c["zeros"] else 0))
        return {"bytes": max(1, c["active"]) * each + R * (K + N) * s, "flops": 2.0 * R * K * N}
    T, k, D = c["tokens"], c["k"], c["cols"]
    b, f = T * k * (D * s + 8) + T * D * s, 2.0 * T * k * D
    if c["train"]:           # dO and Y read, dY and dw written
        b, f = b + T * D * s + 2 * T * k * D * s + 12 * T * k, f + 3.0 * T * k * D
    return {"bytes": b, "flops": f}


# ------------------------------------------------------------------ inputs
def _ends(c, seed):
    """Group ends of `rows` rows spread unevenly over `active` of the experts."""
    rng = random.Random(seed)
    E, rows, active = c["experts"], c["rows"], c["active"]
    picked = sorted(rng.sample(range(E), active))
    share = [math.exp(0.5 * rng.gauss(0, 1)) for _ in picked]
    total, left, size = sum(share), rows - active, [1] * active
    for i, q in enumerate(share):
        n = int(left * q / total)
        size[i] += n
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


def prepare(case, seed):
    c, dt = dict(case), DTYPES[case["dtype"]]
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["op"] == "route":
        T, E, k = c["tokens"], c["experts"], c["k"]
        s["logits"] = _normal(g, (T, E), dt, 1.5)
        s["dweights"] = _normal(g, (T, k), torch.float32)
    elif c["op"] == "grouped":
        ends, s["most"] = _ends(c, seed)
        R, E, K, N = c["rows"] + c["tail"], c["experts"], c["K"], c["N"]
        s["ends"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
        T = max(1, R // 4) if c["gather"] else R
        s["X"] = _normal(g, (T, K), dt)
        s["src"] = torch.randint(0, T, (R,), generator=g, device="cuda", dtype=torch.int32) if c["gather"] else None
        s["W"] = _normal(g, (E, N, K) if c["trans"] else (E, K, N), dt, 1.0 / math.sqrt(K))
        s["dY"] = _normal(g, (R, N), dt) if c["train"] else None
    elif c["op"] == "w4":
        R, N, K, q = c["rows"], c["N"], c["K"], c["group"]
        lead = (c["experts"],) if c["experts"] else ()
        s["X"] = _normal(g, (R, K), dt)
        s["Wq"] = torch.randint(0, 256, lead + (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
        s["scales"] = (torch.rand(lead + (N, K // q), generator=g, device="cuda") * 0.02 + 0.005).to(dt)
        s["zeros"] = (torch.randint(0, 16, lead + (N, K // q), generator=g, device="cuda", dtype=torch.uint8)
                      if c["zeros"] else None)
        s["ends"] = torch.tensor(_ends(c, seed)[0], dtype=torch.int32, device="cuda") if lead else None
    else:
        T, k, D = c["tokens"], c["k"], c["cols"]
        s["Y"] = _normal(g, (T * k, D), dt)
        s["slots"] = torch.randperm(T * k, generator=g, device="cuda").to(torch.int32).view(T, k)
        s["weights"] = torch.rand((T, k), generator=g, device="cuda")
        s["dO"] = _normal(g, (T, D), dt) if c["train"] else None
    if own:
        import paper_2609_04663_gb300 as emu
        emu.load()
        if c["op"] == "route":
            s["ws"] = emu.workspace(emu.emu_route_workspace_bytes(c["tokens"], c["experts"], c["k"]))
        elif c["op"] == "grouped":
            s["ws"] = emu.grouped_workspace(s["X"], s["W"], s["ends"], emu.OP_T if c["trans"] else emu.OP_N, s["src"],
                                            train=c["train"])
    return s


# ------------------------------------------------------------- plain forms
def _plain_route(s):
    c = s["case"]
    T, E, k = c["tokens"], c["experts"], c["k"]
    x = s["logits"].float()
    order = torch.sort(x, dim=1, descending=True, stable=True)
    top, experts = order.values[:, :k], order.indices[:, :k]
    p = torch.exp(top - top[:, :1])
    if c["renorm"]:
        weights = p / p.sum(1, keepdim=True)
    else:
        full = torch.exp(x - top[:, :1])
        total = full.sum(1, keepdim=True)
        weights = p / total
    by = torch.sort(experts.reshape(-1), stable=True).indices
    slots = torch.empty(T * k, dtype=torch.int32, device=x.device)
    slots[by] = torch.arange(T * k, dtype=torch.int32, device=x.device)
    ends = torch.cumsum((experts.reshape(-1, 1) == torch.arange(E, device=x.device)).sum(0), 0).to(torch.int32)
    out = {"weights": weights, "experts": experts.to(torch.int32), "slots": slots.view(T, k),
           "rows": (by // k).to(torch.int32), "ends": ends}
    if c["train"]:
        gw = weights * s["dweights"]
        inner = gw.sum(1, keepdim=True)
        if c["renorm"]:
            d = torch.zeros_like(x).scatter_(1, experts, gw - weights * inner)
        else:
            d = -(full / total) * inner
            d.scatter_add_(1, experts, gw)
        out["dlogits"] = d.to(s["logits"].dtype)
    return out


def _plain_grouped(s):
    c, X, W, ends, dt = s["case"], s["X"], s["W"], s["ends"].long(), s["X"].dtype
    E, R = c["experts"], c["rows"] + c["tail"]
    slot = torch.arange(R, device=X.device)
    of = torch.searchsorted(ends, slot, right=True)             # expert of each row; E: none
    there = (of < E)[:, None]
    of = of.clamp(max=E - 1)
    Xs = (X[s["src"].long()] if s["src"] is not None else X).float()
    if not c["train"] and R <= E:                               # few rows: each with its own expert's matrix
        Wr = W[of].float()
        Y = torch.bmm(Xs[:, None], Wr.transpose(1, 2) if c["trans"] else Wr)[:, 0]
        return {"Y": torch.where(there, Y, 0.0).to(dt)}
    starts = torch.cat([ends.new_zeros(1), ends[:-1]])
    at = starts[:, None] + torch.arange(s["most"], device=X.device)
    mine = (at < ends[:, None])[..., None]
    at = at.clamp(max=R - 1)
    back = slot - starts[of]                                    # place of each row within its expert
    Wf = W.float()
    Wkn = Wf.transpose(1, 2) if c["trans"] else Wf
    Xp = torch.where(mine, Xs[at], 0.0)
    Y = torch.bmm(Xp, Wkn)[of, back.clamp(max=s["most"] - 1)]
    out = {"Y": torch.where(there, Y, 0.0).to(dt)}
    if c["train"]:
        dYp = torch.where(mine, s["dY"].float()[at], 0.0)
        dX = torch.bmm(dYp, Wkn.transpose(1, 2))[of, back.clamp(max=s["most"] - 1)]
        out["dX"] = torch.where(there, dX, 0.0).to(dt)
        dW = torch.bmm(dYp.transpose(1, 2), Xp) if c["trans"] else torch.bmm(Xp.transpose(1, 2), dYp)
        out["dW"] = dW.to(dt)
    return out


def _plain_w4(s):
    c, Wq, scales, zeros = s["case"], s["Wq"], s["scales"], s["zeros"]
    if s["ends"] is not None:                                   # each row with its own expert's matrix
        of = torch.searchsorted(s["ends"].long(), torch.arange(c["rows"], device=Wq.device), right=True)
        Wq, scales, zeros = Wq[of], scales[of], zeros[of] if zeros is not None else None
    q = torch.stack((Wq & 15, Wq >> 4), -1).flatten(-2).float()
    q = q.unflatten(-1, (-1, c["group"])) - (zeros.float()[..., None] if zeros is not None else 8.0)
    W = (q * scales.float()[..., None]).flatten(-2)
    X = s["X"].float()
    Y = torch.bmm(W, X[:, :, None])[:, :, 0] if s["ends"] is not None else X @ W.T
    return {"Y": Y.to(s["X"].dtype)}


def _plain_combine(s):
    at = s["slots"].reshape(-1).long()
    T, k = s["slots"].shape
    Ys = s["Y"][at].float().view(T, k, -1)
    out = {"O": (Ys * s["weights"][..., None]).sum(1).to(s["Y"].dtype)}
    if s["case"]["train"]:
        dO = s["dO"].float()
        dY = torch.empty_like(s["Y"])
        dY[at] = (s["weights"][..., None] * dO[:, None]).to(dY.dtype).flatten(0, 1)
        out["dY"], out["dweights"] = dY, (Ys * dO[:, None]).sum(-1)
    return out


PLAIN = {"route": _plain_route, "grouped": _plain_grouped, "w4": _plain_w4, "combine": _plain_combine}


# -------------------------------------------------------------- the kernels
def _own_route(s, emu):
    c = s["case"]
    r, _ = emu.route(s["logits"], c["k"], renorm=c["renorm"], ws=s["ws"])
    out = {"weights": r.weights, "experts": r.experts, "slots": r.slots, "rows": r.rows, "ends": r.ends}
    if c["train"]:
        out["dlogits"] = emu.route_backward(s["logits"], r.experts, s["dweights"], renorm=c["renorm"])
    return out


def _own_grouped(s, emu):
    c, X, W, dY, ends, src, ws = s["case"], s["X"], s["W"], s["dY"], s["ends"], s["src"], s["ws"]
    op, back = (emu.OP_T, emu.OP_N) if c["trans"] else (emu.OP_N, emu.OP_T)
    if not c["train"]:
        return {"Y": emu.grouped_gemm(X, W, ends, opW=op, src=src, ws=ws)[0]}
    if c["dtype"] == "f32":      # each operand of a training step is in two products: split it once
        X, dY = emu.grouped_split(X, ends, src=src, ws=ws), emu.grouped_split(dY, ends, ws=ws)
        W, src = emu.grouped_split(W, ws=ws), None
    out = {"Y": emu.grouped_gemm(X, W, ends, opW=op, src=src, ws=ws)[0],
           "dX": emu.grouped_gemm(dY, W, ends, opW=back, ws=ws)[0]}
    if c["trans"]:
        out["dW"] = emu.grouped_wgrad(dY, X, ends, srcB=src, ws=ws)[0]
    else:
        out["dW"] = emu.grouped_wgrad(X, dY, ends, srcA=src, ws=ws)[0]
    return out


def _own_w4(s, emu):
    return {"Y": emu.w4_matvec(s["X"], s["Wq"], s["scales"], zeros=s["zeros"], ends=s["ends"])}


def _own_combine(s, emu):
    out = {"O": emu.rows_combine(s["Y"], s["slots"], s["weights"])}
    if s["case"]["train"]:
        out["dY"], out["dweights"] = emu.rows_combine_backward(s["dO"], s["Y"], s["slots"], s["weights"])
    return out


OWN = {"route": _own_route, "grouped": _own_grouped, "w4": _own_w4, "combine": _own_combine}


def run(state):
    op = state["case"]["op"]
    if own:
        import paper_2609_04663_gb300 as emu
        return OWN[op](state, emu)
    return PLAIN[op](state)


# ------------------------------------------------------------------- exact
def _spans(ends):
    e = [0] + [int(v) for v in ends.tolist()]
    return [(a, b) for a, b in zip(e, e[1:])]


def exact(case, seed):
    """The same results in 64 bits, expert by expert and token by token from the definitions."""
    s = prepare(case, seed)
    c = s["case"]
    if c["op"] == "route":
        k, x = c["k"], s["logits"].double()
        T, E = x.shape
        # rank of an expert: how many have a larger logit, or the same and a lower index
        rank = torch.empty(T, E, dtype=torch.int64, device=x.device)
        lower = torch.ones(E, E, dtype=torch.bool, device=x.device).tril(-1)
        for a in range(0, T, 256):
            u = x[a:a + 256]
            ahead = (u[:, None, :] > u[:, :, None]) | ((u[:, None, :] == u[:, :, None]) & lower)
            rank[a:a + 256] = ahead.sum(2)
        experts = torch.argsort(rank, 1)[:, :k]
        chosen = torch.gather(x, 1, experts)
        p = torch.softmax(x, 1)
        w = torch.softmax(chosen, 1) if c["renorm"] else torch.gather(p, 1, experts)
        key = experts.reshape(-1) * (T * k) + torch.arange(T * k, device=x.device)
        by = torch.argsort(key)
        out = {"weights": w, "experts": experts.int(), "slots": torch.argsort(by).view(T, k).int(),
               "rows": (by // k).int(), "ends": torch.bincount(experts.reshape(-1), minlength=E).cumsum(0).int()}
        if c["train"]:
            sel, g = rank < k, torch.zeros_like(x).scatter_(1, experts, s["dweights"].double())
            q = torch.where(sel, p, 0.0)
            if c["renorm"]:
                q = q / q.sum(1, keepdim=True)
                out["dlogits"] = q * (g - (q * g).sum(1, keepdim=True))
            else:
                out["dlogits"] = q * g - p * (q * g).sum(1, keepdim=True)
        return out
    if c["op"] == "grouped":
        X = s["X"][s["src"].long()] if s["src"] is not None else s["X"]
        Y = torch.zeros(X.shape[0], c["N"], dtype=torch.float64, device=X.device)
        dX = torch.zeros(X.shape, dtype=torch.float64, device=X.device) if c["train"] else None
        dW = torch.zeros(s["W"].shape, dtype=torch.float64, device=X.device) if c["train"] else None
        for e, (a, b) in enumerate(_spans(s["ends"])):
            if a == b:
                continue
            x, w = X[a:b].double(), s["W"][e].double()
            w = w.T if c["trans"] else w
            Y[a:b] = x @ w
            if c["train"]:
                d = s["dY"][a:b].double()
                dX[a:b] = d @ w.T
                dW[e] = d.T @ x if c["trans"] else x.T @ d
        return {"Y": Y, "dX": dX, "dW": dW} if c["train"] else {"Y": Y}
    if c["op"] == "w4":
        X, spans = s["X"].double(), _spans(s["ends"]) if s["ends"] is not None else [(0, c["rows"])]
        Y = torch.zeros(c["rows"], c["N"], dtype=torch.float64, device=X.device)
        for e, (a, b) in enumerate(spans):
            if a == b:
                continue
            pick = (lambda t: t[e]) if c["experts"] else (lambda t: t)
            b8 = pick(s["Wq"])
            w = torch.empty(c["N"], c["K"], dtype=torch.float64, device=X.device)
            w[:, 0::2], w[:, 1::2] = (b8 % 16).double(), torch.div(b8, 16, rounding_mode="floor").double()
            z = pick(s["zeros"]).double() if s["zeros"] is not None else torch.full_like(pick(s["scales"]).double(), 8)
            w = (w - z.repeat_interleave(c["group"], 1)) * pick(s["scales"]).double().repeat_interleave(c["group"], 1)
            Y[a:b] = X[a:b] @ w.T
        return {"Y": Y}
    Y, w, at = s["Y"].double(), s["weights"].double(), s["slots"].long()
    O = sum(w[:, j, None] * Y[at[:, j]] for j in range(c["k"]))
    if not c["train"]:
        return {"O": O}
    dO, dY = s["dO"].double(), torch.zeros_like(Y)
    dw = torch.empty_like(w)
    for j in range(c["k"]):
        dY[at[:, j]] = w[:, j, None] * dO
        dw[:, j] = (Y[at[:, j]] * dO).sum(1)
    return {"O": O, "dY": dY, "dweights": dw}
