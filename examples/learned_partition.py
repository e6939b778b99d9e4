"""A partition that is learned instead of clustered, and that then answers for new vertices one at a time.

    python examples/learned_partition.py [--vertices 10000] [--parts 8] [--steps 200]

A head on the embeddings sends every vertex to its best part(s) and is trained to rebuild the embedding from the centroid
of that part, under a balance loss that keeps the parts equally large.  It starts from K-Means (ep_kmeans), whose
parts are as unequal as the embeddings make them.  Printed are edge cut and vertex balance (ep_partition_quality) of
K-Means and of the head, and, for a few vertices served one by one through 8-bit weights, whether they get the part
that the whole pass gave them.

    u      = norm(x)                       ep_rms_norm, fp32 to bf16
    a      = gelu(u W1^T + b1)             ep_linear
    n      = norm(a W2^T + b2 + u)         ep_linear; the sum inside ep_rms_norm
    logits = n Wr^T + br                   ep_linear, fp32 result
    ids, weights, balance loss             ep_route
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2604_01000_b200 as ep  # noqa: E402
import synth  # noqa: E402

BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn


class PartitionHead:
    """The head's parameters (fp32; the products take bf16 copies), its passes, and Adam on its gradients."""

    def __init__(self, width: int, parts: int, centroids: torch.Tensor, hidden: int = 256, seed: int = 0, sharpness: float = 4.0):
        g = torch.Generator(device=centroids.device).manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device=centroids.device) / s[-1] ** 0.5   # noqa: E731
        zeros = lambda *s: torch.zeros(*s, device=centroids.device)                              # noqa: E731
        # the router starts as "nearest centroid": |n - c|^2 = |n|^2 - 2 n.c + |c|^2
        self.p = {"g1": torch.ones_like(centroids[0]), "w1": rand(hidden, width), "b1": zeros(hidden),
                  "w2": 0.02 * rand(width, hidden), "b2": zeros(width), "g2": torch.ones_like(centroids[0]),
                  "wr": sharpness * centroids / width, "br": -0.5 * sharpness * centroids.square().sum(1) / width}
        self.m = {n: torch.zeros_like(t) for n, t in self.p.items()}
        self.v = {n: torch.zeros_like(t) for n, t in self.p.items()}
        self.t = 0

    def forward(self, x: torch.Tensor, k: int):
        p = self.p
        w = {n: p[n].to(BF16) for n in ("w1", "w2", "wr")}
        u = ep.ep_rms_norm(x, p["g1"], out_dtype=BF16).out
        a = ep.ep_linear(u, w["w1"], p["b1"], "gelu", preact=True)
        y = ep.ep_linear(a.out, w["w2"], p["b2"]).out
        n = ep.ep_rms_norm(y, p["g2"], u)
        logits = ep.ep_linear(n.out, w["wr"], p["br"], out_dtype=torch.float32).out
        return logits, ep.ep_route(logits, k), (x, u, a, n, w)

    def backward(self, kept, logits, routed, dweights, dloss) -> dict:
        x, u, a, n, w = kept
        p = self.p
        dlogits = ep.ep_route_backward(logits, routed, dweights, dloss)
        r = ep.ep_linear_backward(dlogits, n.out, w["wr"])
        s = ep.ep_rms_norm_backward(r.dx, n.hidden, p["g2"])          # s.dx: of y and, alike, of the residual u
        l2 = ep.ep_linear_backward(s.dx, a.out, w["w2"])
        l1 = ep.ep_linear_backward(l2.dx, u, w["w1"], a.preact, "gelu")
        first = ep.ep_rms_norm_backward(l1.dx + s.dx, x, p["g1"])
        return {"g1": first.dweight, "w1": l1.dweight.float(), "b1": l1.dbias, "w2": l2.dweight.float(), "b2": l2.dbias,
                "g2": s.dweight, "wr": r.dweight.float(), "br": r.dbias}

    def step(self, grads: dict, lr: float):
        self.t += 1
        for n, g in grads.items():
            self.m[n].mul_(0.9).add_(g, alpha=0.1)
            self.v[n].mul_(0.99).addcmul_(g, g, value=0.01)
            up = (self.m[n] / (1 - 0.9 ** self.t)) / ((self.v[n] / (1 - 0.99 ** self.t)).sqrt() + 1e-8)
            self.p[n].sub_(lr * up)

    def serving(self):
        """A function from one or more embeddings to part ids, through weights in 8 bits that are laid out once."""
        p = self.p
        q = {n: ep.ep_quantize_rows(p[n]) for n in ("w1", "w2", "wr")}

        def answer(x: torch.Tensor) -> torch.Tensor:
            u = ep.ep_rms_norm(x, p["g1"], out_dtype=BF16).out
            u8 = ep.ep_quantize_rows(u)
            a = ep.ep_linear(u8.q, q["w1"].q, p["b1"], "gelu", None, u8.scale, q["w1"].scale).out
            a8 = ep.ep_quantize_rows(a)
            y = ep.ep_linear(a8.q, q["w2"].q, p["b2"], "none", None, a8.scale, q["w2"].scale).out
            n = ep.ep_rms_norm(y, p["g2"], u, out_dtype=E4M3)
            logits = ep.ep_linear(n.out, q["wr"].q, p["br"], "none", None, n.scale, q["wr"].scale, torch.float32).out
            return ep.ep_route(logits, 1).ids
        return answer


def train(x: torch.Tensor, parts: int, steps: int, balance: float = 1.0, lr: float = 1e-3, k: int = 1):
    """(head, K-Means result on the normalised rows, history of (rebuilding loss, balance loss))."""
    unit = ep.ep_rms_norm(x).out
    km = ep.ep_kmeans(unit, parts, 20, unit[:parts].contiguous())
    head, history = PartitionHead(x.shape[1], parts, km.centroids), []
    dloss = torch.full((1,), balance, device=x.device)
    for _ in range(steps):
        logits, r, kept = head.forward(x, k)
        chosen = km.centroids[r.ids.long()]                               # rows x k x width
        off = (r.weights[:, :, None] * chosen).sum(1) - unit
        dweights = (2.0 / unit.numel()) * torch.einsum("rw,rkw->rk", off, chosen).contiguous()
        history.append((off.square().mean(), r.loss))
        head.step(head.backward(kept, logits, r, dweights, dloss), lr)
    return head, km, [(float(a), float(b)) for a, b in history]


def quality(rowptr, colidx, assign, parts: int):
    """(edge-cut ratio, vertex balance) of a partition."""
    q = ep.ep_partition_quality(rowptr, colidx, assign, parts)
    return float(q.edge_cut) / max(1, colidx.numel()), float(q.part_vertices.max()) * parts / assign.numel()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--vertices", type=int, default=10_000)
    ap.add_argument("--parts", type=int, default=8)
    ap.add_argument("--steps", type=int, default=200)
    a = ap.parse_args(argv)
    work = synth.scaled(synth.WORKLOADS["cfg1"], a.vertices)
    x = synth.embeddings(work, device="cuda:0")
    rowptr, colidx = synth.graph(work, device="cuda:0")
    head, km, history = train(x, a.parts, a.steps)
    ids = head.forward(x, 1)[1].ids.view(-1)
    print("rebuilding loss %.4f -> %.4f, balance loss %.4f -> %.4f" % (history[0][0], history[-1][0], history[0][1], history[-1][1]))
    for name, part in (("K-Means", km.assign), ("learned", ids)):
        print("%s: edge-cut ratio %.4f, vertex balance %.3f" % ((name,) + quality(rowptr, colidx, part, a.parts)))
    answer = head.serving()
    some = range(0, a.vertices, max(1, a.vertices // 64))
    same = sum(int(answer(x[i:i + 1])) == int(ids[i]) for i in some)
    print("one by one in 8 bits: %d of %d vertices as in the whole pass" % (same, len(some)))
    ep.default_context().check()


if __name__ == "__main__":
    main()
