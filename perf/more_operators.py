"""Cases and plain forms of the operators beside a trained partition head: softmax cross entropy over many classes without
keeping the logits, and its backward pass; the matrix product in 8-bit integers with scales for each row and column; and a
whole layer of experts (router, both products of the chosen parts, their sum) for a few rows.

``run`` computes an operator either through the package (``own`` true) or in its plain form: elementary torch
operations in 32 bits, rounded once at the end.  ``exact`` states the same definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16, "int8": torch.int8}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2, "int8": 1}


# ------------------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # validation of one small batch while training on the 10,000-vertex graph, in 32 bits
        {"name": "entropy, 128 rows of 32 bits", "op": "entropy", "rows": 128, "in": 64, "classes": 32, "dtype": "fp32",
         "bias": True, "dead": 0.0},
        # every vertex of the 169,343-vertex graph against the 4096 clusters that its numbering is made of
        {"name": "entropy, 169343 rows, 4096 classes", "op": "entropy", "rows": 169343, "in": 128, "classes": 4096,
         "dtype": "bf16", "bias": False, "dead": 0.05},
        # 32-bit training with widths that no 16-byte access divides, each row with a weight of its own
        {"name": "entropy backward, ragged 32 bits", "op": "entropy_backward", "rows": 2999, "in": 65, "classes": 257,
         "dtype": "fp32", "bias": True, "dead": 0.1, "weighted": True},
        # the same training step as the second case
        {"name": "entropy backward, 169343 rows", "op": "entropy_backward", "rows": 169343, "in": 128, "classes": 4096,
         "dtype": "bf16", "bias": False, "dead": 0.05, "weighted": False},
        # link prediction: which of the 169,343 vertices is a row's neighbour (a class for every vertex)
        {"name": "entropy backward, 169343 classes", "op": "entropy_backward", "rows": 4096, "in": 256, "classes": 169343,
         "dtype": "fp16", "bias": True, "dead": 0.0, "weighted": False},
        # one new vertex through a hidden layer
        {"name": "integers, one row", "op": "integers", "rows": 1, "in": 1024, "out": 1024, "result": "bf16", "act": "gelu",
         "bias": True, "residual": True},
        # a small batch with odd widths, to 32-bit logits
        {"name": "integers, ragged", "op": "integers", "rows": 301, "in": 515, "out": 257, "result": "fp32", "act": "none",
         "bias": True, "residual": False},
        # the head's widening layer for every vertex of the 169,343-vertex graph (bound by memory)
        {"name": "integers, 169343 rows", "op": "integers", "rows": 169343, "in": 128, "out": 512, "result": "bf16",
         "act": "relu", "bias": True, "residual": False},
        # a large layer (bound by the tensor cores)
        {"name": "integers, 8192 x 4096 x 4096", "op": "integers", "rows": 8192, "in": 4096, "out": 4096, "result": "bf16",
         "act": "none", "bias": False, "residual": False},
        # one new vertex, two of 64 experts
        {"name": "experts, one row", "op": "experts", "rows": 1, "in": 1024, "hidden": 4096, "out": 1024, "experts": 64, "k": 2,
         "dtype": "bf16", "weights": "bf16", "act": "gelu", "biases": True, "residual": True, "renormalize": True, "closed": 0.0},
        # a few queries at once, most experts are wanted by some row; weights in 8 bits
        {"name": "experts, 16 rows, weights of 8 bits", "op": "experts", "rows": 16, "in": 1024, "hidden": 4096, "out": 1024,
         "experts": 32, "k": 2, "dtype": "bf16", "weights": "int8", "act": "silu", "biases": False, "residual": True,
         "renormalize": False, "closed": 0.0},
        # odd widths in 32 bits, some parts closed
        {"name": "experts, ragged 32 bits", "op": "experts", "rows": 7, "in": 333, "hidden": 1029, "out": 77, "experts": 5, "k": 3,
         "dtype": "fp32", "weights": "fp32", "act": "relu", "biases": True, "residual": False, "renormalize": True, "closed": 0.2},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["entropy", "entropy_backward", "entropy_backward", "integers", "integers", "experts", "experts"])
    if op.startswith("entropy"):
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        n_in = _log(rng, 8, 1024)
        if rng.random() < 0.5:      # half of the widths are multiples of 16
            n_in = 16 * max(1, n_in // 16)
        classes = _log(rng, 2, 200_000)
        most = min(4e8, 8e10 / n_in) / (6.0 if dtype == "fp32" else 1.0)
        rows = _log(rng, 1, max(1, min(200_000, int(most / classes))))
        case = {"op": op, "rows": rows, "in": n_in, "classes": classes, "dtype": dtype, "bias": rng.random() < 0.5,
                "dead": rng.choice([0.0, 0.0, 0.1, 0.5])}
        if op == "entropy_backward":
            case["weighted"] = rng.random() < 0.3
        return case
    if op == "integers":
        n_in, n_out = _log(rng, 8, 4096), _log(rng, 8, 4096)
        if rng.random() < 0.5:      # half of the layers have widths that are multiples of 64
            n_in, n_out = 64 * max(1, n_in // 64), 64 * max(1, n_out // 64)
        rows = _log(rng, 1, max(1, min(200_000, int(1.2e11 / (n_in * n_out)), (1 << 26) // max(n_in, n_out))))
        return {"op": op, "rows": rows, "in": n_in, "out": n_out, "result": rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                "act": rng.choice(["none", "relu", "gelu", "silu"]), "bias": rng.random() < 0.7, "residual": rng.random() < 0.5}
    n_in, hidden, out = _log(rng, 16, 2048), _log(rng, 16, 4096), _log(rng, 16, 2048)
    if rng.random() < 0.5:
        n_in, hidden, out = (16 * max(1, v // 16) for v in (n_in, hidden, out))
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    weights = rng.choice([dtype, "int8"])
    experts = _log(rng, 2, max(2, min(128, (1 << 28) // (hidden * (n_in + out)))))
    k = min(experts, rng.choice([1, 2, 2, 4]))
    rows = _log(rng, 1, max(1, min(64, (1 << 28) // (k * hidden * max(n_in, out)))))
    return {"op": op, "rows": rows, "in": n_in, "hidden": hidden, "out": out, "experts": experts, "k": k, "dtype": dtype,
            "weights": weights, "act": rng.choice(["relu", "gelu", "silu"]), "biases": rng.random() < 0.5,
            "residual": rng.random() < 0.5, "renormalize": rng.random() < 0.5, "closed": rng.choice([0.0, 0.0, 0.2])}


# ------------------------------------------------------------------------------------------------ inputs

def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _to_integers(x):
    """Rows (the last axis) in 8-bit integers, and the scale of each."""
    scale = x.abs().amax(-1) / 127.0
    return torch.round(x / scale[..., None]).to(torch.int8), scale


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    op, rows = case["op"], case["rows"]
    if op.startswith("entropy"):
        n_in, classes, dt = case["in"], case["classes"], DTYPES[case["dtype"]]
        w = _randn(g, classes, n_in).mul_(1.0 / math.sqrt(n_in))
        t = torch.randint(0, classes, (rows,), generator=g, device="cuda")
        x = _randn(g, rows, n_in).add_(w[t], alpha=4.0)           # what training has reached: the right class stands out
        dead = torch.rand(rows, generator=g, device="cuda") < case["dead"]
        s["x"], s["w"] = x.to(dt), w.to(dt)
        s["t"] = t.masked_fill(dead, -1).int()                    # padding rows have no class
        s["b"] = _randn(g, classes).mul_(0.5) if case["bias"] else None
        if op == "entropy_backward":
            s["lse"], s["counted"] = _lse(s), (s["t"] >= 0).sum().reshape(1)   # what the forward left
            s["dloss"] = torch.full((1,), 1.0, device="cuda")
            s["drow"] = torch.rand(rows, generator=g, device="cuda").mul_(1.0 / rows) if case["weighted"] else None
        return s
    if op == "integers":
        n_in, n_out = case["in"], case["out"]
        s["x"], s["x_scale"] = _to_integers(_randn(g, rows, n_in))
        s["w"], s["w_scale"] = _to_integers(_randn(g, n_out, n_in).mul_(1.0 / math.sqrt(n_in)))
        s["b"] = _randn(g, n_out).mul_(0.1) if case["bias"] else None
        s["r"] = _randn(g, rows, n_out).to(DTYPES[case["result"]]) if case["residual"] else None
        return s
    n_in, hidden, out, experts, dt = case["in"], case["hidden"], case["out"], case["experts"], DTYPES[case["dtype"]]
    s["x"] = _randn(g, rows, n_in).to(dt)
    s["router"] = _randn(g, experts, n_in).mul_(1.5 / math.sqrt(n_in)).to(dt)
    s["router_bias"] = _randn(g, experts).mul_(0.1)
    s["router_bias"][:int(case["closed"] * experts)] = -math.inf
    w1, w2 = _randn(g, experts, hidden, n_in).mul_(1.0 / math.sqrt(n_in)), _randn(g, experts, out, hidden).mul_(1.0 / math.sqrt(hidden))
    s["w1_scale"] = s["w2_scale"] = None
    if case["weights"] == "int8":
        (s["w1"], s["w1_scale"]), (s["w2"], s["w2_scale"]) = _to_integers(w1), _to_integers(w2)
    else:
        s["w1"], s["w2"] = w1.to(dt), w2.to(dt)
    s["b1"] = _randn(g, experts, hidden).mul_(0.1) if case["biases"] else None
    s["b2"] = _randn(g, experts, out).mul_(0.1) if case["biases"] else None
    s["r"] = _randn(g, rows, out).to(dt) if case["residual"] else None
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _logits(s):
    l = s["x"].float() @ s["w"].float().T
    return l if s["b"] is None else l + s["b"]


def _lse(s):
    l = _logits(s)
    top = l.amax(1, keepdim=True)
    return (torch.log(torch.exp(l - top).sum(1, keepdim=True)) + top)[:, 0]


def _entropy(s):
    l = _logits(s)
    top = l.amax(1, keepdim=True)
    lse = (torch.log(torch.exp(l - top).sum(1, keepdim=True)) + top)[:, 0]
    live = s["t"] >= 0
    at = l.gather(1, s["t"].clamp(min=0).long()[:, None])[:, 0]
    row_loss = torch.where(live, lse - at, torch.zeros_like(lse))
    counted = live.sum().reshape(1)
    return {"loss": row_loss.sum().reshape(1) / counted.clamp(min=1), "row_loss": row_loss, "lse": lse * live, "counted": counted}


def _entropy_backward(s):
    dt, live = DTYPES[s["dtype"]], s["t"] >= 0
    g = s["dloss"] / s["counted"].clamp(min=1).float()
    g = live * (g if s["drow"] is None else g + s["drow"])
    p = torch.exp(_logits(s) - s["lse"][:, None])
    at = s["t"].clamp(min=0).long()[:, None]
    p.scatter_add_(1, at, -torch.ones_like(s["lse"])[:, None])
    p.mul_(g[:, None])
    return {"dx": (p @ s["w"].float()).to(dt), "dweight": (p.T @ s["x"].float()).to(dt), "dbias": p.sum(0)}


def _act(z, act):
    if act == "relu":
        return torch.maximum(z, torch.zeros_like(z))
    if act == "gelu":
        return z * 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _integers(s):
    z = (s["x"].float() @ s["w"].float().T) * s["x_scale"][:, None] * s["w_scale"]
    if s["b"] is not None:
        z = z + s["b"]
    y = _act(z, s["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    return y.to(DTYPES[s["result"]])


def _weights_of(w, scale, ids):
    chosen = w[ids].float()
    return chosen if scale is None else chosen * scale[ids][..., None]


def _experts(s):
    x, k = s["x"].float(), s["k"]
    l = x @ s["router"].float().T + s["router_bias"]
    top = l.amax(1, keepdim=True)
    e = torch.exp(l - top)
    p = e / e.sum(1, keepdim=True)
    best, ids = torch.sort(l, dim=1, descending=True, stable=True)
    best, ids = best[:, :k], ids[:, :k]
    got = best > -math.inf
    w = torch.where(got, p.gather(1, ids), torch.zeros_like(best))
    if s["renormalize"]:
        w = w / w.sum(1, keepdim=True)
    y = torch.zeros(x.shape[0], s["w2"].shape[1], device=x.device)
    for i in range(k):
        at = ids[:, i]
        z = (_weights_of(s["w1"], s["w1_scale"], at) @ x[:, :, None])[:, :, 0]
        h = _act(z if s["b1"] is None else z + s["b1"][at], s["act"])
        o = (_weights_of(s["w2"], s["w2_scale"], at) @ h[:, :, None])[:, :, 0]
        y = y + w[:, i:i + 1] * (o if s["b2"] is None else o + s["b2"][at])
    if s["r"] is not None:
        y = y + s["r"].float()
    return {"out": y.to(DTYPES[s["dtype"]]), "ids": torch.where(got, ids, torch.full_like(ids, -1)).int(), "weights": w}


# ------------------------------------------------------------------------------------------------ one pass

def _run_own(s):
    import paper_2604_01000_b200 as ep
    op = s["op"]
    if op == "entropy":
        r = ep.ep_cross_entropy(s["x"], s["w"], s["t"], s["b"])
        return {"loss": r.loss, "row_loss": r.row_loss, "lse": r.lse, "counted": r.counted}
    if op == "entropy_backward":
        r = ep.CrossEntropyResult(None, None, s["lse"], s["counted"])
        got = ep.ep_cross_entropy_backward(s["x"], s["w"], s["t"], r, s["b"], s["dloss"], s["drow"])
        return {"dx": got.dx, "dweight": got.dweight, "dbias": got.dbias}
    if op == "integers":
        return ep.ep_linear(s["x"], s["w"], s["b"], s["act"], s["r"], s["x_scale"], s["w_scale"], DTYPES[s["result"]]).out
    r = ep.ep_experts(s["x"], s["router"], s["w1"], s["w2"], s["k"], s["router_bias"], s["b1"], s["b2"], s["act"], s["renormalize"],
                      s["r"], s["w1_scale"], s["w2_scale"])
    return {"out": r.out, "ids": r.ids, "weights": r.weights}


def run(state):
    if own:
        return _run_own(state)
    return {"entropy": _entropy, "entropy_backward": _entropy_backward, "integers": _integers, "experts": _experts}[state["op"]](state)


def work(case):
    op, rows = case["op"], case["rows"]
    if op.startswith("entropy"):
        size, n_in, classes = SIZE[case["dtype"]], case["in"], case["classes"]
        operands = size * n_in * (rows + classes) + 4 * rows + (4 * classes if case["bias"] else 0)
        products = 2 * rows * n_in * classes
        if op == "entropy":
            return {"bytes": operands + 8 * rows, "flops": products}
        return {"bytes": operands + size * n_in * (rows + classes) + 4 * rows + 4 * classes + (4 * rows if case["weighted"] else 0),
                "flops": 3 * products}                          # the logits, which nobody kept, and two products
    if op == "integers":
        n_in, n_out, result = case["in"], case["out"], SIZE[case["result"]]
        return {"bytes": n_in * (rows + n_out) + result * rows * n_out * (1 + int(case["residual"])) + 4 * (rows + n_out)
                + (4 * n_out if case["bias"] else 0), "flops": 2 * rows * n_in * n_out}
    n_in, hidden, out, experts, k = case["in"], case["hidden"], case["out"], case["experts"], case["k"]
    size, per = SIZE[case["dtype"]], SIZE[case["weights"]]
    wanted = experts * (1.0 - (1.0 - k / experts) ** rows)      # experts that some row chooses
    expert = per * hidden * (n_in + out) + (4 * (hidden + out) if case["weights"] == "int8" else 0)
    expert += 4 * (hidden + out) if case["biases"] else 0
    rest = size * (rows * (n_in + out * (1 + int(case["residual"]))) + experts * n_in) + 4 * experts + 8 * rows * k
    return {"bytes": int(wanted * expert) + rest, "flops": 2 * rows * (experts * n_in + k * hidden * (n_in + out))}


# ------------------------------------------------------------------------------------------------ in 64 bits

def _exact_act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op.startswith("entropy"):
        x, w = s["x"].double(), s["w"].double()
        b = torch.zeros((), dtype=torch.float64, device=x.device) if s["b"] is None else s["b"].double()
        live = s["t"] >= 0
        counted = max(1, int(live.sum()))
        rows = max(1, (1 << 28) // case["classes"])              # this many at a time
        if op == "entropy":
            lse, row_loss = torch.zeros_like(x[:, 0]), torch.zeros_like(x[:, 0])
            for i in range(0, case["rows"], rows):
                l, t = torch.einsum("rk,ck->rc", x[i:i + rows], w) + b, s["t"][i:i + rows].long()
                z = torch.logsumexp(l, 1)
                row_loss[i:i + rows] = z - l[torch.arange(len(t), device=t.device), t.clamp(min=0)]
                lse[i:i + rows] = z
            row_loss, lse = row_loss.masked_fill(~live, 0.0), lse.masked_fill(~live, 0.0)
            return {"loss": row_loss.sum().reshape(1) / counted, "row_loss": row_loss, "lse": lse, "counted": None}
        weight = torch.full_like(x[:, 0], float(s["dloss"]) / counted)
        if s["drow"] is not None:
            weight = weight + s["drow"].double()
        weight = weight.masked_fill(~live, 0.0)
        dx, dw = torch.zeros_like(x), torch.zeros_like(w)
        db = torch.zeros(case["classes"], dtype=torch.float64, device=x.device)
        for i in range(0, case["rows"], rows):
            l, t = torch.einsum("rk,ck->rc", x[i:i + rows], w) + b, s["t"][i:i + rows].long()
            p = torch.exp(l - s["lse"][i:i + rows].double()[:, None])          # (lse is an input, as it was rounded)
            p[torch.arange(len(t), device=t.device), t.clamp(min=0)] -= 1.0
            p *= weight[i:i + rows, None]
            dx[i:i + rows] = torch.einsum("rc,ck->rk", p, w)
            dw += torch.einsum("rc,rk->ck", p, x[i:i + rows])
            db += torch.einsum("rc->c", p)
        return {"dx": dx, "dweight": dw, "dbias": db}
    if op == "integers":
        z = torch.einsum("mk,nk->mn", s["x"].double(), s["w"].double())
        z = s["x_scale"].double()[:, None] * z * s["w_scale"].double()[None, :] + (0.0 if s["b"] is None else s["b"].double())
        return _exact_act(z, case["act"]) + (0.0 if s["r"] is None else s["r"].double())
    x, k = s["x"].double(), case["k"]
    l = torch.einsum("rn,en->re", x, s["router"].double()) + s["router_bias"].double()
    p = torch.softmax(l, 1)
    column, left = torch.arange(case["experts"], device=x.device), l.clone()
    y = torch.zeros(case["rows"], case["out"], dtype=torch.float64, device=x.device)
    slots, weights = [], []
    for _ in range(k):                                            # the best expert that is left, the first of equals
        best = left.max(1, keepdim=True).values
        first = torch.where(left == best, column, case["experts"]).min(1).values
        none = torch.isneginf(best[:, 0])
        slots.append(first)
        weights.append(p.gather(1, first[:, None])[:, 0].masked_fill(none, 0.0))
        left = left.scatter(1, first[:, None], -math.inf)
    w = torch.stack(weights, 1)
    if case["renormalize"]:
        w = w / w.sum(1, keepdim=True)
    for i, at in enumerate(slots):
        for r in range(case["rows"]):
            e = int(at[r])
            w1, w2 = s["w1"][e].double(), s["w2"][e].double()
            if s["w1_scale"] is not None:
                w1, w2 = w1 * s["w1_scale"][e].double()[:, None], w2 * s["w2_scale"][e].double()[:, None]
            z = torch.mv(w1, x[r]) + (0.0 if s["b1"] is None else s["b1"][e].double())
            o = torch.mv(w2, _exact_act(z, case["act"])) + (0.0 if s["b2"] is None else s["b2"][e].double())
            y[r] += w[r, i] * o
    return {"out": y + (0.0 if s["r"] is None else s["r"].double()), "ids": None, "weights": w}
