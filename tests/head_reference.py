"""Plain 64-bit statements of the partition head's operators, and the rounding units the tests' bounds are made of."""
import math

import torch

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float8_e4m3fn: 2.0 ** -4}
# half the spacing of the smallest numbers of each type: what rounding to zero can cost
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float8_e4m3fn: 2.0 ** -10}
FP32 = 2.0 ** -24


def norm(x, weight, residual, eps):
    h = x.double() if residual is None else x.double() + residual.double()
    rho = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    g = torch.ones(x.shape[1], dtype=torch.float64, device=x.device) if weight is None else weight.double()
    return h, rho, h * rho * g


def norm_backward(dout, h, weight, eps, dhidden):
    h, dy = h.double(), dout.double()
    g = torch.ones(h.shape[1], dtype=torch.float64, device=h.device) if weight is None else weight.double()
    rho = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    a = dy * g
    dx = rho * (a - h * rho ** 2 * (a * h).mean(1, keepdim=True))
    size = rho * (a.abs() + h.abs() * rho ** 2 * (a * h).abs().mean(1, keepdim=True))
    if dhidden is not None:
        dx, size = dx + dhidden.double(), size + dhidden.double().abs()
    return dx, size, (dy * h * rho).sum(0), (dy * h * rho).abs().sum(0)


def act(z, name):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def route(logits, k, valid, renormalize):
    """(ids, weights, counts, prob, loss, routed, p) row by row, as the definition reads."""
    rows, parts = logits.shape
    l = logits.double().cpu()
    ids = torch.full((rows, k), -1, dtype=torch.int32)
    w = torch.zeros(rows, k, dtype=torch.float64)
    p = torch.zeros(rows, parts, dtype=torch.float64)
    counts = torch.zeros(parts, dtype=torch.int64)
    routed = 0
    for r in range(rows):
        if valid is not None and not bool(valid[r]):
            continue
        row = l[r]
        if not bool((row > -math.inf).any()):
            continue
        routed += 1
        top = max(v for v in row.tolist() if v == v)
        e = torch.exp(row - top)
        p[r] = e / e.sum()
        order = sorted((c for c in range(parts) if row[c] > -math.inf), key=lambda c: (-float(row[c]), c))[:k]
        for i, c in enumerate(order):
            ids[r, i] = c
            w[r, i] = p[r, c]
            counts[c] += 1
        if renormalize:
            w[r] /= w[r].sum()
    n = max(routed, 1)
    prob = p.sum(0) / n
    loss = parts * float((counts.double() / (k * n) * prob).sum())
    return ids, w, counts, prob, loss, routed, p


def route_backward(p, ids, counts, routed, k, renormalize, dweights, dloss):
    """(dlogits, the size of the terms it is summed from)."""
    rows, parts = p.shape
    n = max(routed, 1)
    dlogits, size = torch.zeros_like(p), torch.zeros_like(p)
    for r in range(rows):
        if not bool((p[r] != 0).any()):
            continue
        dp = dloss * parts * counts.double() / (k * n) / n
        big = dp.abs().clone()
        chosen = [(i, int(c)) for i, c in enumerate(ids[r]) if c >= 0]
        total = sum(float(p[r, c]) for _, c in chosen)
        if dweights is not None:
            pulled = sum(float(dweights[r, i]) * float(p[r, c]) for i, c in chosen) / total if renormalize else 0.0
            for i, c in chosen:
                dw = float(dweights[r, i])
                dp[c] += (dw - pulled) / total if renormalize else dw
                big[c] += (abs(dw) + abs(pulled)) / total if renormalize else abs(dw)
        dlogits[r] = p[r] * (dp - (p[r] * dp).sum())
        size[r] = p[r] * (big + (p[r] * big).sum())
    return dlogits, size


def within(got, want, bound, what):
    """Every element of got within `bound` of want, both finite."""
    got, want, bound = got.double().cpu(), want.double().cpu(), bound.double().cpu()
    assert got.shape == want.shape, what
    off = (got - want).abs()
    bad = ~(off <= bound)
    if bool(bad.any()):
        i = torch.nonzero(bad)[0].tolist()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {got[tuple(i)]} for "
                             f"{want[tuple(i)]}, bound {bound[tuple(i)]}")


def misaligned(t):
    """A contiguous copy of t that starts one element past a 16-byte boundary."""
    room = torch.empty(t.numel() + 16, dtype=t.dtype, device=t.device)
    view = room[1:1 + t.numel()].view(t.shape)
    view.copy_(t)
    return view


def entropy(x, weight, targets, bias):
    """(lse, row_loss, loss, counted, logits): rows whose target is -1 (or whose classes are all closed) take no part."""
    l = x.double() @ weight.double().T
    if bias is not None:
        l = l + bias.double()
    t = targets.long()
    live = (t >= 0) & (t < weight.shape[0])
    lse = torch.logsumexp(l, 1)
    live = live & ~torch.isneginf(lse)
    at = l.gather(1, t.clamp(0, weight.shape[0] - 1)[:, None])[:, 0]
    row_loss = torch.where(live, lse - at, torch.zeros_like(lse))
    return lse, row_loss, row_loss.sum() / max(1, int(live.sum())), int(live.sum()), l


def entropy_slopes(l, lse, targets, dloss, drow, counted):
    """(G, p |g|): the logits' gradient from a given lse, and the size of its terms."""
    t = targets.long()
    live = (t >= 0) & (t < l.shape[1]) & ~torch.isneginf(lse)
    g = torch.zeros_like(lse.double()) if dloss is None else torch.full_like(lse.double(), float(dloss) / max(1, counted))
    if drow is not None:
        g = g + drow.double()
    g = torch.where(live, g, torch.zeros_like(g))
    p = torch.where(live[:, None], torch.exp(l - lse.double()[:, None]), torch.zeros_like(l))
    G = p.clone()
    rows = torch.nonzero(live)[:, 0]
    G[rows, t[rows]] -= 1.0
    return G * g[:, None], p * g.abs()[:, None]
