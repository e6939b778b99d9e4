"""Cases and plain forms of the operators of a trained partition head: the root-mean-square norm with the residual's
addition (and an 8-bit output with scales), the matrix product with bias, activation and residual, and the routing of
rows to parts with its counts and balance loss.  Each with its backward pass.

``run`` computes an operator either through the package (``own`` true) or in its plain form: elementary torch
operations in 32 bits, rounded once at the end.  ``exact`` states the same definitions in 64 bits.
"""
import math

import torch

own = False

EPS = 1e-6
E4M3_MAX = 448.0
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2, "e4m3": 1}


# ------------------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # one new vertex: its row is normalised and handed to an 8-bit product
        {"name": "norm, one row to 8 bits", "op": "norm", "rows": 1, "width": 1024, "dtype": "bf16", "out": "e4m3",
         "residual": True},
        # the embeddings of the 169,343-vertex graph, from 32 bits to the 16 bits the products take
        {"name": "norm, 169343 rows", "op": "norm", "rows": 169343, "width": 128, "dtype": "fp32", "out": "bf16",
         "residual": True},
        # training on all 2,449,029 vertices at once
        {"name": "norm backward, 2449029 rows", "op": "norm_backward", "rows": 2449029, "width": 128, "dtype": "bf16",
         "grad": "bf16", "residual": True},
        # one new vertex through a hidden layer
        {"name": "linear, one row", "op": "linear", "rows": 1, "in": 1024, "out": 1024, "dtype": "bf16", "result": "bf16",
         "act": "gelu", "bias": True, "residual": True, "preact": False},
        # a batch of queries through 8-bit weights
        {"name": "linear, 2000 rows of 8 bits", "op": "linear", "rows": 2000, "in": 4096, "out": 4096, "dtype": "e4m3",
         "result": "bf16", "act": "silu", "bias": True, "residual": True, "preact": False},
        # the widening layer of a training step on the 169,343-vertex graph (bound by memory)
        {"name": "linear, 169343 rows", "op": "linear", "rows": 169343, "in": 128, "out": 512, "dtype": "bf16",
         "result": "bf16", "act": "relu", "bias": True, "residual": False, "preact": True},
        # a large layer (bound by the tensor cores)
        {"name": "linear, 8192 x 4096 x 4096", "op": "linear", "rows": 8192, "in": 4096, "out": 4096, "dtype": "fp16",
         "result": "fp16", "act": "none", "bias": True, "residual": True, "preact": False},
        # 32-bit training on the 10,000-vertex graph, with widths that no 16-byte access divides
        {"name": "linear backward, ragged 32 bits", "op": "linear_backward", "rows": 10000, "in": 65, "out": 257,
         "dtype": "fp32", "grad": "fp32", "act": "gelu"},
        # a training step on the 232,965-vertex graph: the sum over rows is the long one
        {"name": "linear backward, 232965 rows", "op": "linear_backward", "rows": 232965, "in": 256, "out": 256,
         "dtype": "bf16", "grad": "bf16", "act": "gelu"},
        # one new vertex to two of 64 parts
        {"name": "route, one row", "op": "route", "rows": 1, "parts": 64, "k": 2, "dtype": "fp32", "renormalize": True,
         "valid": False, "closed": 0.0},
        # every vertex of the 2,449,029-vertex graph to one of 32 parts
        {"name": "route, 2449029 rows", "op": "route", "rows": 2449029, "parts": 32, "k": 1, "dtype": "fp32",
         "renormalize": False, "valid": False, "closed": 0.0},
        # training with padding rows, parts closed to some rows and an odd number of parts
        {"name": "route backward, 169343 rows", "op": "route_backward", "rows": 169343, "parts": 257, "k": 8,
         "dtype": "bf16", "renormalize": True, "valid": True, "closed": 0.1},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm_backward", "linear", "linear", "linear_backward", "route", "route_backward"])
    if op.startswith("norm"):
        width = _log(rng, 8, 8192)
        rows = _log(rng, 1, max(1, min(1 << 20, (1 << 27) // width)))
        dtype = rng.choice(["fp32", "bf16", "fp16"])
        case = {"op": op, "rows": rows, "width": width, "dtype": dtype, "residual": rng.random() < 0.6}
        if op == "norm":
            case["out"] = rng.choice([dtype, "e4m3"] + (["bf16", "fp16"] if dtype == "fp32" else []))
        else:
            case["grad"] = rng.choice([dtype] + (["bf16", "fp16"] if dtype == "fp32" else []))
        return case
    if op.startswith("linear"):
        n_in, n_out = _log(rng, 8, 4096), _log(rng, 8, 4096)
        if rng.random() < 0.5:      # half of the layers have widths that are multiples of 64
            n_in, n_out = 64 * max(1, n_in // 64), 64 * max(1, n_out // 64)
        times = 2 if op == "linear_backward" else 1
        rows = _log(rng, 1, max(1, min(200_000, int(1.2e11 / (2 * times * n_in * n_out)), (1 << 26) // max(n_in, n_out))))
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"] + (["e4m3"] if op == "linear" else []))
        case = {"op": op, "rows": rows, "in": n_in, "out": n_out, "dtype": dtype,
                "act": rng.choice(["none", "relu", "gelu", "silu"])}
        if op == "linear":
            case["result"] = rng.choice({"e4m3": ["bf16", "fp16", "fp32"], "fp32": ["fp32"]}.get(dtype, [dtype, dtype, "fp32"]))
            case.update(bias=rng.random() < 0.7, residual=rng.random() < 0.5, preact=rng.random() < 0.3)
        else:
            case["grad"] = rng.choice([dtype, dtype, "fp32"])
        return case
    parts = _log(rng, 2, 4096)
    rows = _log(rng, 1, max(1, min(1 << 20, (1 << 25) // parts)))
    return {"op": op, "rows": rows, "parts": parts, "k": min(parts, rng.choice([1, 1, 2, 4, 8])),
            "dtype": rng.choice(["fp32", "bf16", "fp16"]), "renormalize": rng.random() < 0.5,
            "valid": rng.random() < 0.5, "closed": rng.choice([0.0, 0.0, 0.1])}


# ------------------------------------------------------------------------------------------------ inputs

def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _embeddings(g, rows, width):
    """Rows of a 40-component Gaussian mixture."""
    centres = _randn(g, 40, width)
    which = torch.randint(0, 40, (rows,), generator=g, device="cuda")
    return _randn(g, rows, width).mul_(0.7).add_(centres[which])


def _unit_rows(g, rows, width):
    """What a norm leaves: rows of root mean square one."""
    x = _embeddings(g, rows, width)
    return x.mul_(torch.rsqrt(x.square().mean(1, keepdim=True) + EPS))


def _to_8_bits(x):
    scale = x.abs().amax(1) / E4M3_MAX
    return (x / scale[:, None]).to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    op, rows, dt = case["op"], case["rows"], DTYPES[case["dtype"]]
    if op in ("norm", "norm_backward"):
        width = case["width"]
        s["weight"] = _randn(g, width).mul_(0.2).add_(1.0)
        s["x"] = _embeddings(g, rows, width).to(dt)          # the backward's hidden rows, x + residual
        if op == "norm":
            s["r"] = _embeddings(g, rows, width).mul_(0.5).to(dt) if case["residual"] else None
        else:
            s["dout"] = _randn(g, rows, width).mul_(0.1).to(DTYPES[case["grad"]])
            s["dhidden"] = _randn(g, rows, width).mul_(0.1).to(dt) if case["residual"] else None
        return s
    if op in ("linear", "linear_backward"):
        n_in, n_out = case["in"], case["out"]
        x, w = _unit_rows(g, rows, n_in), _randn(g, n_out, n_in).mul_(1.0 / math.sqrt(n_in))
        bias = _randn(g, n_out).mul_(0.1)
        s["x_scale"] = s["w_scale"] = None
        if dt == torch.float8_e4m3fn:
            (s["x"], s["x_scale"]), (s["w"], s["w_scale"]) = _to_8_bits(x), _to_8_bits(w)
        else:
            s["x"], s["w"] = x.to(dt), w.to(dt)
        if op == "linear":
            s["b"] = bias if case["bias"] else None
            s["r"] = _randn(g, rows, n_out).to(DTYPES[case["result"]]) if case["residual"] else None
        else:
            z = s["x"].float() @ s["w"].float().T + bias
            s["z"] = z.to(dt) if case["act"] != "none" else None    # the forward's stored value before the activation
            s["dout"] = _randn(g, rows, n_out).mul_(0.01).to(DTYPES[case["grad"]])
        return s
    parts, k = case["parts"], case["k"]
    centres = _randn(g, 40, parts).mul_(1.5)                 # rows of one component favour the same parts
    which = torch.randint(0, 40, (rows,), generator=g, device="cuda")
    logits = _randn(g, rows, parts).add_(centres[which])
    if case["closed"]:
        logits.masked_fill_(torch.rand(rows, parts, generator=g, device="cuda") < case["closed"], -math.inf)
    s["logits"] = logits.to(dt)
    s["live"] = (torch.rand(rows, generator=g, device="cuda") >= 0.05).to(torch.uint8) if case["valid"] else None
    if op == "route_backward":                               # what the forward left, and the gradients that came back
        s["ids"], s["weights"], s["counts"], s["prob"], s["loss"], s["routed"] = _route(
            s["logits"], k, s["live"], case["renormalize"])
        s["dweights"] = _randn(g, rows, k).mul_(0.1)
        s["dloss"] = torch.full((1,), 0.01, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _norm(s):
    h = s["x"].float() if s["r"] is None else s["x"].float() + s["r"].float()
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["weight"]
    hidden = None if s["r"] is None else h.to(DTYPES[s["dtype"]])
    if s["out"] != "e4m3":
        return {"out": y.to(DTYPES[s["out"]]), "hidden": hidden}
    scale = y.abs().amax(1) / E4M3_MAX
    inverse = torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))
    return {"out": (y * inverse[:, None]).to(torch.float8_e4m3fn), "scale": scale, "hidden": hidden}


def _norm_backward(s):
    h, dy = s["x"].float(), s["dout"].float()
    rho = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    a = dy * s["weight"]
    dx = rho * (a - h * (rho * rho) * (a * h).mean(1, keepdim=True))
    if s["dhidden"] is not None:
        dx = dx + s["dhidden"].float()
    return {"dx": dx.to(DTYPES[s["dtype"]]), "dweight": (dy * (h * rho)).sum(0)}


def _act(z, act):
    if act == "relu":
        return torch.maximum(z, torch.zeros_like(z))
    if act == "gelu":
        return z * 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    sig = 1.0 / (1.0 + torch.exp(-z))
    return sig * (1.0 + z * (1.0 - sig))


def _linear(s):
    z = s["x"].float() @ s["w"].float().T
    if s["x_scale"] is not None:
        z = z * s["x_scale"][:, None] * s["w_scale"]
    if s["b"] is not None:
        z = z + s["b"]
    y = _act(z, s["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    out = DTYPES[s["result"]]
    return {"out": y.to(out), "preact": z.to(out) if s["preact"] else None}


def _linear_backward(s):
    dt = DTYPES[s["dtype"]]
    dz = s["dout"].float()
    if s["act"] != "none":
        dz = dz * _act_slope(s["z"].float(), s["act"])
    return {"dx": (dz @ s["w"].float()).to(dt), "dweight": (dz.T @ s["x"].float()).to(dt), "dbias": dz.sum(0)}


def _softmax(logits, live):
    """Probabilities in 32 bits, zero in rows that take no part; and which rows do."""
    l = logits.float()
    top = l.amax(1, keepdim=True)
    part = (top > -math.inf) & (live[:, None] != 0) if live is not None else top > -math.inf
    e = torch.where(part, torch.exp(l - top), torch.zeros_like(l))
    return l, e / torch.where(part, e.sum(1, keepdim=True), torch.ones_like(top)), part


def _route(logits, k, live, renormalize):
    parts = logits.shape[1]
    l, p, part = _softmax(logits, live)
    top, ids = torch.sort(l, dim=1, descending=True, stable=True)
    top, ids = top[:, :k], ids[:, :k]
    got = part & (top > -math.inf)
    w = torch.where(got, p.gather(1, ids), torch.zeros_like(top))
    if renormalize:
        w = w / torch.where(part, w.sum(1, keepdim=True), torch.ones_like(w[:, :1]))
    counts = torch.zeros(parts, dtype=torch.int64, device=l.device).scatter_add_(0, ids.reshape(-1), got.reshape(-1).long())
    routed = part.sum().reshape(1)
    rows = routed.clamp(min=1).float()
    prob = p.sum(0) / rows
    loss = (parts / (k * rows)) * (counts.float() * prob).sum()
    return torch.where(got, ids, torch.full_like(ids, -1)).int(), w, counts, prob, loss, routed


def _route_backward(s):
    k, parts = s["k"], s["parts"]
    _, p, part = _softmax(s["logits"], s["live"])
    rows = s["routed"].clamp(min=1).float()
    slope = s["dloss"] * (parts / k) * s["counts"].float() / (rows * rows)
    got = s["ids"] >= 0
    at = s["ids"].clamp(min=0).long()
    dw = torch.where(got, s["dweights"], torch.zeros_like(s["dweights"]))
    if s["renormalize"]:
        total = torch.where(got, p.gather(1, at), torch.zeros_like(dw)).sum(1, keepdim=True)
        dw = (dw - (dw * s["weights"]).sum(1, keepdim=True)) / torch.where(part, total, torch.ones_like(total))
        dw = torch.where(got, dw, torch.zeros_like(dw))
    grad = (part * slope).scatter_add(1, at, dw)
    return {"dlogits": (p * (grad - (p * grad).sum(1, keepdim=True))).to(DTYPES[s["dtype"]])}


# ------------------------------------------------------------------------------------------------ one pass

def _run_own(s):
    import paper_2604_01000_b200 as ep
    op = s["op"]
    if op == "norm":
        r = ep.ep_rms_norm(s["x"], s["weight"], s["r"], EPS, DTYPES[s["out"]])
        got = {"out": r.out, "hidden": None if s["r"] is None else r.hidden}
        if s["out"] == "e4m3":
            got["scale"] = r.scale
        return got
    if op == "norm_backward":
        r = ep.ep_rms_norm_backward(s["dout"], s["x"], s["weight"], EPS, s["dhidden"])
        return {"dx": r.dx, "dweight": r.dweight}
    if op == "linear":
        r = ep.ep_linear(s["x"], s["w"], s["b"], s["act"], s["r"], s["x_scale"], s["w_scale"], DTYPES[s["result"]], s["preact"])
        return {"out": r.out, "preact": r.preact}
    if op == "linear_backward":
        r = ep.ep_linear_backward(s["dout"], s["x"], s["w"], s["z"], s["act"])
        return {"dx": r.dx, "dweight": r.dweight, "dbias": r.dbias}
    if op == "route":
        r = ep.ep_route(s["logits"], s["k"], s["live"], s["renormalize"])
        return dict(zip(("ids", "weights", "counts", "prob", "loss", "routed"), r))
    r = ep.RouteResult(s["ids"], s["weights"], s["counts"], s["prob"], s["loss"], s["routed"])
    return {"dlogits": ep.ep_route_backward(s["logits"], r, s["dweights"], s["dloss"], s["live"], s["renormalize"])}


def run(state):
    if own:
        return _run_own(state)
    op = state["op"]
    if op == "route":
        return dict(zip(("ids", "weights", "counts", "prob", "loss", "routed"),
                        _route(state["logits"], state["k"], state["live"], state["renormalize"])))
    return {"norm": _norm, "norm_backward": _norm_backward, "linear": _linear, "linear_backward": _linear_backward,
            "route_backward": _route_backward}[op](state)


def work(case):
    op, rows = case["op"], case["rows"]
    size = SIZE[case["dtype"]]
    if op == "norm":
        n = rows * case["width"]
        moved = n * (size + SIZE[case["out"]] + (2 * size if case["residual"] else 0)) + 4 * case["width"]
        return {"bytes": moved + (4 * rows if case["out"] == "e4m3" else 0), "flops": 6 * n}
    if op == "norm_backward":
        n = rows * case["width"]
        return {"bytes": n * (2 * size + SIZE[case["grad"]] + (size if case["residual"] else 0)) + 8 * case["width"],
                "flops": 12 * n}
    if op.startswith("linear"):
        n_in, n_out = case["in"], case["out"]
        if op == "linear":
            result = SIZE[case["result"]]
            outs = 1 + int(case["residual"]) + int(case["preact"])
            extra = 4 * (rows + n_out) if case["dtype"] == "e4m3" else 0
            return {"bytes": size * (rows * n_in + n_out * n_in) + result * rows * n_out * outs + extra
                    + (4 * n_out if case["bias"] else 0), "flops": 2 * rows * n_in * n_out}
        reads = rows * n_out * (SIZE[case["grad"]] + (size if case["act"] != "none" else 0))
        return {"bytes": reads + 2 * size * (rows * n_in + n_out * n_in) + 4 * n_out, "flops": 4 * rows * n_in * n_out}
    n, k = rows * case["parts"], case["k"]
    mask = rows if case["valid"] else 0
    if op == "route":
        return {"bytes": n * size + rows * k * 8 + mask + 12 * case["parts"], "flops": 5 * n}
    return {"bytes": 2 * n * size + rows * k * 12 + mask + 8 * case["parts"], "flops": 8 * n}


# ------------------------------------------------------------------------------------------------ in 64 bits

def _exact_act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _exact_slope(z, act):
    if act == "relu":
        return torch.heaviside(z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)


def _exact_probabilities(s):
    l = s["logits"].double()
    dead = torch.isneginf(l).all(1)
    if s["live"] is not None:
        dead = dead | (s["live"] == 0)
    p = torch.exp(l - torch.logsumexp(l, 1, keepdim=True))
    return l, p.masked_fill(dead[:, None], 0.0), dead


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        h = s["x"].double()
        if s["r"] is not None:
            h = h + s["r"].double()
        y = s["weight"].double() * h / torch.sqrt(torch.mean(h ** 2, 1, keepdim=True) + EPS)
        got = {"out": y, "hidden": None if s["r"] is None else h}
        if case["out"] == "e4m3":
            got["scale"] = torch.max(torch.abs(y), 1).values / E4M3_MAX
            got["out"] = y / got["scale"][:, None]
        return got
    if op == "norm_backward":
        h, dy, w = s["x"].double(), s["dout"].double(), s["weight"].double()
        ms = torch.mean(h ** 2, 1, keepdim=True) + EPS
        unit = h / torch.sqrt(ms)
        dunit = dy * w
        dx = (dunit - unit * torch.mean(dunit * unit, 1, keepdim=True)) / torch.sqrt(ms)
        if s["dhidden"] is not None:
            dx = dx + s["dhidden"].double()
        return {"dx": dx, "dweight": torch.einsum("rw,rw->w", dy, unit)}
    if op == "linear":
        x, w = s["x"].double(), s["w"].double()
        if s["x_scale"] is not None:
            x, w = x * s["x_scale"].double()[:, None], w * s["w_scale"].double()[:, None]
        z = torch.einsum("mk,nk->mn", x, w) + (0.0 if s["b"] is None else s["b"].double())
        y = _exact_act(z, case["act"]) + (0.0 if s["r"] is None else s["r"].double())
        return {"out": y, "preact": z if case["preact"] else None}
    if op == "linear_backward":
        dz = s["dout"].double()
        if case["act"] != "none":
            dz = dz * _exact_slope(s["z"].double(), case["act"])
        return {"dx": torch.einsum("mn,nk->mk", dz, s["w"].double()),
                "dweight": torch.einsum("mn,mk->nk", dz, s["x"].double()), "dbias": torch.einsum("mn->n", dz)}
    l, p, dead = _exact_probabilities(s)
    rows, parts, k = case["rows"], case["parts"], case["k"]
    routed = max(1, int((~dead).sum()))
    if op == "route":
        column = torch.arange(parts, device=l.device)
        left, chosen = l.masked_fill(dead[:, None], -math.inf), []
        counts, weights = torch.zeros(parts, device=l.device, dtype=torch.float64), []
        for _ in range(k):                                    # the best column that is left, the first of equals
            best = left.max(1, keepdim=True).values
            first = torch.where(left == best, column, parts).min(1).values
            none = torch.isneginf(best[:, 0])
            weights.append(p.gather(1, first[:, None])[:, 0].masked_fill(none, 0.0))
            counts += torch.bincount(first[~none], minlength=parts).double()
            left = left.scatter(1, first[:, None], -math.inf)
        w = torch.stack(weights, 1)
        if case["renormalize"]:
            w = w / w.sum(1, keepdim=True).masked_fill(dead[:, None], 1.0)
        prob = p.sum(0) / routed
        loss = parts * torch.dot(counts / (k * routed), prob)
        return {"ids": None, "weights": w, "counts": None, "prob": prob, "loss": loss.reshape(1), "routed": None}
    # d loss / d logit_j = sum_i (d loss / d p_i) p_i (delta_ij - p_j)
    got = s["ids"] >= 0
    at = s["ids"].long().clamp(min=0)
    chosen = p.gather(1, at) * got
    dchosen = s["dweights"].double() * got
    if case["renormalize"]:
        total = chosen.sum(1, keepdim=True).masked_fill(dead[:, None], 1.0)
        dchosen = (dchosen / total - (dchosen * chosen).sum(1, keepdim=True) / total ** 2) * got
    dp = torch.zeros_like(p) + s["dloss"].double() * parts * s["counts"].double() / (k * routed) / routed
    dp = dp.scatter_add(1, at, dchosen).masked_fill(dead[:, None], 0.0)
    return {"dlogits": p * dp - p * (p * dp).sum(1, keepdim=True)}
