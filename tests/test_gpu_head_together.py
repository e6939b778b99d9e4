"""The head's operators in a row, as they are used: K-Means' clusters are learned by cross entropy on a hidden layer, the trained
layer answers in 8-bit integers, and a layer of experts, one set of weights for each cluster, answers for single rows."""
import pytest
import torch

import head_reference as ref

pytestmark = pytest.mark.gpu

F32, BF16, I8 = torch.float32, torch.bfloat16, torch.int8


def ep():
    import paper_2604_01000_b200 as m
    return m


def clustered(rows, width, clusters, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    centres = torch.randn(clusters, width, generator=g, device="cuda")
    which = torch.randint(0, clusters, (rows,), generator=g, device="cuda")
    return torch.randn(rows, width, generator=g, device="cuda") * 0.3 + centres[which], g


def network(width, hidden, classes, g):
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda") / s[-1] ** 0.5   # noqa: E731
    return {"g": torch.ones(width, device="cuda"), "w1": rand(hidden, width), "b1": torch.zeros(hidden, device="cuda"),
            "w2": rand(classes, hidden), "b2": torch.zeros(classes, device="cuda")}


def gradients(p, x, targets):
    """The loss and its gradients by the library, the products in bf16."""
    m = ep()
    w1, w2 = p["w1"].to(BF16), p["w2"].to(BF16)
    u = m.ep_rms_norm(x, p["g"], out_dtype=BF16).out
    a = m.ep_linear(u, w1, p["b1"], "gelu", preact=True)
    r = m.ep_cross_entropy(a.out, w2, targets, p["b2"])
    last = m.ep_cross_entropy_backward(a.out, w2, targets, r, p["b2"], torch.ones(1, device="cuda"))
    first = m.ep_linear_backward(last.dx, u, w1, a.preact, "gelu")
    norm = m.ep_rms_norm_backward(first.dx.float(), x, p["g"])
    return r.loss, {"g": norm.dweight, "w1": first.dweight.float(), "b1": first.dbias, "w2": last.dweight.float(), "b2": last.dbias}


def loss_in_64_bits(p, x, targets):
    h, _, u = ref.norm(x, p["g"], None, 1e-6)
    a = ref.act(u @ p["w1"].double().T + p["b1"].double(), "gelu")
    return ref.entropy(a, p["w2"], targets, p["b2"])[2]


def test_a_head_learns_the_clusters_and_answers_in_integers():
    m = ep()
    x, g = clustered(4001, 64, 24, 1)
    km = m.ep_kmeans(x, 24, 10, x[:24].contiguous())
    targets = km.assign.clone()
    targets[::17] = -1                                         # vertices that are kept from training
    p = network(64, 96, 24, g)
    # the gradients along a direction against differences of the 64-bit loss: bf16 operands and gradients, 2^-8 each, through three
    # products, leave 2^-5 of the sizes that are summed
    loss, grads = gradients(p, x, targets)
    assert abs(float(loss) - float(loss_in_64_bits(p, x, targets))) <= 2.0 ** -5 * float(loss)
    for name, grad in grads.items():
        d = grad / grad.norm()
        h = 1e-3
        up, down = ({**p, name: p[name].double() + s * h * d.double()} for s in (1, -1))
        diff = float(loss_in_64_bits(up, x, targets) - loss_in_64_bits(down, x, targets)) / (2 * h)
        assert abs(diff - float(grad.norm())) <= 2.0 ** -4 * float(grad.norm()), name
    for _ in range(60):
        _, grads = gradients(p, x, targets)
        for name, grad in grads.items():
            p[name] -= 2.0 * grad
    # what it has learned, whole and row by row in 8-bit integers
    u = m.ep_rms_norm(x, p["g"], out_dtype=BF16).out
    a = m.ep_linear(u, p["w1"].to(BF16), p["b1"], "gelu").out
    whole = m.ep_linear(a, p["w2"].to(BF16), p["b2"], out_dtype=F32).out
    q1, q2 = m.ep_quantize_rows(p["w1"], I8), m.ep_quantize_rows(p["w2"], I8)

    def answer(rows):
        n = m.ep_rms_norm(rows, p["g"], out_dtype=I8)
        h = m.ep_quantize_rows(m.ep_linear(n.out, q1.q, p["b1"], "gelu", None, n.scale, q1.scale).out, I8)
        return m.ep_linear(h.q, q2.q, p["b2"], "none", None, h.scale, q2.scale, F32).out
    # rows and weights are within half of 1/127 of their largest: far less than what separates the best class where it is clear
    clear = whole.topk(2).values
    clear = (clear[:, 0] - clear[:, 1]) > 0.5 * whole.abs().amax(1)
    assert int(clear.sum()) > 100
    got = answer(x)
    assert torch.equal(got.argmax(1)[clear], whole.argmax(1)[clear])
    for i in torch.nonzero(clear)[:20, 0].tolist():
        assert int(answer(x[i:i + 1]).argmax()) == int(whole[i].argmax())
    m.default_context().check()


def test_experts_are_the_products_of_their_parts():
    # the layer for few rows against the same layer made of ep_route and, part by part, ep_linear; bf16 rows, weights of both kinds
    m = ep()
    x, g = clustered(48, 128, 12, 2)
    x = x.to(BF16)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda") / s[-1] ** 0.5   # noqa: E731
    router, w1, w2 = rand(12, 128).to(BF16), rand(12, 256, 128), rand(12, 64, 256)
    b1, b2 = rand(12, 256), rand(12, 64)
    q1, q2 = m.ep_quantize_rows(w1.view(-1, 128), I8), m.ep_quantize_rows(w2.view(-1, 256), I8)
    routed = m.ep_route(m.ep_linear(x, router, out_dtype=F32).out, 2, None, True)
    for whole in (True, False):
        if whole:
            got = m.ep_experts(x, router, w1.to(BF16), w2.to(BF16), 2, None, b1, b2, "gelu", True)
            first, second = w1.to(BF16), w2.to(BF16)
        else:
            got = m.ep_experts(x, router, q1.q.view(w1.shape), q2.q.view(w2.shape), 2, None, b1, b2, "gelu", True, None,
                               q1.scale.view(12, 256), q2.scale.view(12, 64))
            first = (q1.q.float() * q1.scale[:, None]).view(w1.shape)
            second = (q2.q.float() * q2.scale[:, None]).view(w2.shape)
        assert torch.equal(got.ids, routed.ids)
        want = torch.zeros(48, 64, device="cuda", dtype=torch.float64)
        for part in range(12):
            for slot in range(2):
                rows = torch.nonzero(routed.ids[:, slot] == part)[:, 0]
                if len(rows) == 0:
                    continue
                h = m.ep_linear(x[rows].float(), first[part].float(), b1[part], "gelu").out
                y = m.ep_linear(h, second[part].float(), b2[part]).out
                want[rows] += routed.weights[rows, slot, None].double() * y.double()
        ref.within(got.out, want, 2.0 ** -8 * want.abs() + 2.0 ** -12, "out")   # rounded once, fp32 products on both sides
    m.default_context().check()
