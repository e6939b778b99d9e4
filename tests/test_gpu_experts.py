"""ep_experts against 64-bit formulas.

Bounds.  A dot product of n numbers, summed in fp32 by 32 lanes that take at least every 64th pair, is within (n / 32 + 16) 2^-24 of
the sum of its terms' sizes; 8-bit weights add one rounding for their scale.  Router logits are off by that (e), weights by 2 e + 2^-19 of
themselves (renormalised: twice that), hidden values by their product's error, by 2^-20 of what the activation adds and by its slope (at
most 1.13), outputs by what the errors of hidden values and weights make in them; one rounding ends it.
Rows of 16 bits may hold their hidden values as two bf16 numbers, 2^-17 of themselves off.
"""
import math

import pytest
import torch

import head_reference as ref

pytestmark = pytest.mark.gpu

F32, BF16, F16, I8 = torch.float32, torch.bfloat16, torch.float16, torch.int8


def ep():
    import paper_2604_01000_b200 as m
    return m


def rand(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def layer(rows, n_in, hidden, n_out, parts, dtype, weights, seed):
    """(x, router, w1, w2, w1_scale, w2_scale)"""
    x, router = rand((rows, n_in), dtype, seed), rand((parts, n_in), dtype, seed + 1, 1.5 * n_in ** -0.5)
    w1, w2 = rand((parts, hidden, n_in), F32, seed + 2, n_in ** -0.5), rand((parts, n_out, hidden), F32, seed + 3, hidden ** -0.5)
    if weights != I8:
        return x, router, w1.to(dtype), w2.to(dtype), None, None
    q1 = ep().ep_quantize_rows(w1.view(-1, n_in), I8)
    q2 = ep().ep_quantize_rows(w2.view(-1, hidden), I8)
    return x, router, q1.q.view(w1.shape), q2.q.view(w2.shape), q1.scale.view(parts, hidden), q2.scale.view(parts, n_out)


def dot_error(n):
    return (n / 32 + 16) * 2.0 ** -24


def check(x, router, w1, w2, s1, s2, k=1, router_bias=None, b1=None, b2=None, act="gelu", renormalize=False, residual=None, valid=None):
    r = ep().ep_experts(x, router, w1, w2, k, router_bias, b1, b2, act, renormalize, residual, s1, s2, valid)
    rows, parts, n_out, dt = x.shape[0], router.shape[0], w2.shape[1], x.dtype
    assert r.out.dtype == dt and r.out.shape == (rows, n_out) and r.ids.dtype == torch.int32 and r.weights.dtype == F32
    l = x.double() @ router.double().T
    e = (x.double().abs() @ router.double().abs().T) * dot_error(x.shape[1]) + 2.0 ** -23 * l.abs()
    if router_bias is not None:
        l = l + router_bias.double()
    ids, w = ref.route(l, k, valid, renormalize)[:2]
    ids, w = ids.cuda(), w.cuda()
    assert torch.equal(r.ids, ids)
    off = w * (4 * e.amax(1, keepdim=True) + 2.0 ** -18)
    ref.within(r.weights, w, off + 2.0 ** -126, "weights")
    total, error = torch.zeros(rows, n_out, dtype=torch.float64, device="cuda"), torch.zeros(rows, n_out, dtype=torch.float64, device="cuda")
    for row in range(rows):
        for i in range(k):
            p = int(ids[row, i])
            if p < 0:
                continue
            a, b = w1[p].double(), w2[p].double()
            if s1 is not None:
                a, b = a * s1[p].double()[:, None], b * s2[p].double()[:, None]
            z, S = a @ x[row].double(), a.abs() @ x[row].double().abs()
            z = z if b1 is None else z + b1[p].double()
            dz = S * (dot_error(x.shape[1]) + 2.0 ** -24) + 2.0 ** -23 * z.abs()
            h = ref.act(z, act)
            dh = 1.13 * dz + 2.0 ** -20 * (h.abs() + z.abs() * 2.0 ** -4)
            if dt != F32:
                dh = dh + 2.0 ** -17 * h.abs()
            y, dy = b @ h, b.abs() @ dh + (b.abs() @ h.abs()) * (dot_error(w1.shape[1]) + 2.0 ** -24)
            y = y if b2 is None else y + b2[p].double()
            total[row] += w[row, i] * y
            error[row] += w[row, i] * (dy + 2.0 ** -22 * y.abs()) + off[row, i] * y.abs()
    if residual is not None:
        total = total + residual.double()
        error = error + 2.0 ** -23 * residual.double().abs()
    ref.within(r.out, total, error + ref.UNIT[dt] * (total.abs() + error) + ref.TINY[dt], "out")
    return r


SHAPES = [(1, 64, 128, 64, 8, 2), (1, 1024, 4096, 1024, 64, 2), (1, 1, 1, 1, 1, 1), (2, 33, 65, 17, 3, 3), (3, 500, 77, 130, 5, 1), (7, 333, 1029, 77, 5, 3),
          (16, 128, 256, 512, 32, 2), (9, 72, 40, 24, 2, 1), (33, 48, 96, 1000, 7, 4), (64, 64, 64, 64, 300, 8), (64, 16, 32, 8, 4096, 32), (40, 96, 2000, 33, 40, 32),
          (40, 64, 1528, 72, 40, 4), (64, 48, 4096, 24, 12, 2), (9, 32, 2064, 40, 40, 6), (20, 112, 1936, 130, 60, 3)]


@pytest.mark.parametrize("rows,n_in,hidden,n_out,parts,k", SHAPES)
@pytest.mark.parametrize("dtype,weights", [(BF16, BF16), (F16, F16), (F32, F32), (BF16, I8), (F16, I8), (F32, I8)])
def test_shapes(rows, n_in, hidden, n_out, parts, k, dtype, weights):
    args = layer(rows, n_in, hidden, n_out, parts, dtype, weights, 1)
    check(*args, k=k)
    check(*args, k, rand((parts,), F32, 6, 0.1), rand((parts, hidden), F32, 7, 0.1), rand((parts, n_out), F32, 8, 0.1), "silu", True,
          rand((rows, n_out), dtype, 9))


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("bias", [BF16, F16])
def test_activations_and_bias_types(act, bias):
    args = layer(5, 64, 96, 48, 6, BF16, BF16, 10)
    check(*args, 2, rand((6,), bias, 11), rand((6, 96), bias, 12), None, act)
    check(*args, 2, None, None, rand((6, 48), bias, 13), act)


def test_closed_parts_and_rows_that_take_no_part():
    args = layer(12, 40, 56, 24, 6, F32, F32, 14)
    b = rand((6,), F32, 15)
    b[[0, 2, 5]] = -math.inf
    valid = torch.tensor([1, 0, 1, 1, 0, 1, 1, 1, 1, 1, 0, 1], device="cuda", dtype=torch.uint8)
    res = rand((12, 24), F32, 16)
    for residual in (None, res):
        r = check(*args, 5, b, None, None, "gelu", True, residual, valid)      # more slots than open parts
        assert bool((r.ids[valid == 0] == -1).all()) and bool((r.ids[valid == 1][:, 3:] == -1).all())
        assert torch.equal(r.out[valid == 0], torch.zeros_like(res[valid == 0]) if residual is None else res[valid == 0])
        r = check(*args, 2, torch.full((6,), -math.inf, device="cuda"), None, None, "gelu", False, residual)
        assert bool((r.ids == -1).all()) and torch.equal(r.out, torch.zeros_like(res) if residual is None else res)
    check(*args, 2, valid=valid.bool())
    # what a row that takes no part holds does not matter
    x = args[0].clone()
    x[valid == 0] = math.nan
    want, got = (ep().ep_experts(y, *args[1:4], 2, valid=valid) for y in (args[0], x))
    assert all(torch.equal(p, q) for p, q in zip(want, got))


def test_parts_that_nobody_chose_do_not_matter():
    x, router, w1, w2, _, _ = layer(3, 32, 64, 32, 16, BF16, BF16, 17)
    want = ep().ep_experts(x, router, w1, w2, 2)
    others = torch.tensor(sorted(set(range(16)) - set(want.ids.flatten().tolist())), device="cuda")
    w1, w2 = w1.clone(), w2.clone()
    w1[others], w2[others] = math.nan, math.inf
    got = ep().ep_experts(x, router, w1, w2, 2)
    assert all(torch.equal(p, q) for p, q in zip(want, got))


def test_equal_logits_and_spoiled_rows():
    x, router, w1, w2, _, _ = layer(6, 32, 48, 16, 9, F32, F32, 18)
    r = check(x, torch.zeros_like(router), w1, w2, None, None, 4, None, None, None, "relu", True)
    assert torch.equal(r.ids, torch.arange(4, device="cuda", dtype=torch.int32).expand(6, 4))
    bad = x.clone()
    bad[2, 3] = math.nan
    want, got = ep().ep_experts(x, router, w1, w2, 2), ep().ep_experts(bad, router, w1, w2, 2)
    fine = torch.arange(6, device="cuda") != 2
    assert torch.equal(got.out[fine], want.out[fine]) and bool((got.ids[2] == -1).all())
    # one NaN among the logits: never chosen, but nothing is known of the row's weights
    b = torch.zeros(9, device="cuda")
    b[4] = math.nan
    got = ep().ep_experts(x, router, w1, w2, 2, b)
    assert bool((got.ids != 4).all()) and bool(torch.isnan(got.weights).all()) and bool(torch.isnan(got.out).all())


def test_the_router_is_ep_route():
    m = ep()
    x, router, w1, w2, _, _ = layer(50, 96, 32, 32, 70, BF16, BF16, 19)
    b = rand((70,), F32, 20)
    logits = m.ep_linear(x, router, b, out_dtype=F32).out
    for renormalize in (False, True):
        want, got = m.ep_route(logits, 6, None, renormalize), m.ep_experts(x, router, w1, w2, 6, b, renormalize=renormalize)
        assert torch.equal(want.ids, got.ids)
        ref.within(got.weights, want.weights, 2.0 ** -16 * want.weights, "weights")


def test_a_row_does_not_depend_on_how_many_others_come_with_it():
    args = layer(64, 128, 256, 128, 8, BF16, I8, 21)
    whole = ep().ep_experts(*args[:4], 2, w1_scale=args[4], w2_scale=args[5])
    for n in (1, 2, 7, 33):
        got = ep().ep_experts(args[0][:n], *args[1:4], 2, w1_scale=args[4], w2_scale=args[5])
        assert torch.equal(got.ids, whole.ids[:n])
        ref.within(got.out, whole.out[:n].double(), 2 * ref.UNIT[BF16] * whole.out[:n].double().abs() + 2.0 ** -12, "out")


def test_strided_rows_and_misaligned_buffers():
    for dtype, weights in ((BF16, BF16), (F32, F32), (BF16, I8)):
        _, router, w1, w2, s1, s2 = layer(6, 64, 96, 48, 6, dtype, weights, 22)
        big, res = rand((12, 200), dtype, 23), rand((6, 96), dtype, 24)
        for x in (big[:6, 8:72], big[::2, 3:67], ref.misaligned(big[:6, :64].contiguous())):
            check(x, router, w1, w2, s1, s2, 2, residual=res[:, 5:53])
        check(big[:6, :64], *(ref.misaligned(t) for t in (router, w1, w2)), s1, s2, 2)


def test_no_rows():
    args = layer(0, 64, 96, 48, 6, BF16, BF16, 25)
    r = ep().ep_experts(*args[:4], 2)
    assert r.out.shape == (0, 48) and r.ids.shape == (0, 2)


def test_captured_beside_another_stream():
    m = ep()
    sets = [layer(4, 256, 512, 256, 16, BF16, BF16, 26), layer(30, 128, 256, 64, 8, BF16, I8, 30)]
    run = lambda a: list(m.ep_experts(*a[:4], 2, w1_scale=a[4], w2_scale=a[5]))   # noqa: E731
    want = [run(a) for a in sets]
    torch.cuda.synchronize()
    graphs, outs, streams = [], [], []
    for a in sets:
        s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(run(a))
        graphs.append(g)
        streams.append(s)
    for _ in range(5):
        for o in outs:
            for t in o:
                t.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for o, w in zip(outs, want) for p, q in zip(o, w))


def test_refusals():
    m = ep()
    x, router, w1, w2, _, _ = layer(5, 16, 24, 8, 6, BF16, BF16, 34)
    q1, q2 = w1.to(I8), w2.to(I8)
    s1, s2 = torch.ones(6, 24, device="cuda"), torch.ones(6, 8, device="cuda")
    for bad in (lambda: m.ep_experts(x.float(), router, w1, w2), lambda: m.ep_experts(x, router[:, :8], w1, w2),
                lambda: m.ep_experts(x, router[:5], w1, w2), lambda: m.ep_experts(x, router, w1[:, :, :8], w2),
                lambda: m.ep_experts(x, router, w1, w2[:, :, :8]), lambda: m.ep_experts(x, router, w1, q2),
                lambda: m.ep_experts(x, router, q1, q2), lambda: m.ep_experts(x, router, q1, q2, w1_scale=s1),
                lambda: m.ep_experts(x, router, q1, q2, w1_scale=s1, w2_scale=s2[:, :7]), lambda: m.ep_experts(x, router, w1, w2, w1_scale=s1, w2_scale=s2),
                lambda: m.ep_experts(x, router, w1, w2, 0), lambda: m.ep_experts(x, router, w1, w2, 7),
                lambda: m.ep_experts(x, router, w1, w2, activation="tanh"), lambda: m.ep_experts(x, router, w1, w2, b1=s2),
                lambda: m.ep_experts(x, router, w1, w2, b1=s1, b2=s2.half()), lambda: m.ep_experts(x, router, w1, w2, residual=s2[:5]),
                lambda: m.ep_experts(x, router, w1, w2, valid=torch.ones(4, device="cuda", dtype=torch.uint8)),
                lambda: m.ep_experts(x.cpu(), router, w1, w2), lambda: m.ep_experts(x, router, w1[0], w2),
                lambda: m.ep_experts(x.repeat(13, 1), router, w1, w2)):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("rows", [1, 64])
def test_parts_whose_offsets_pass_32_bits(rows):
    """520 parts of 2048 x 4096 and 4096 x 2048 integers; the first and the last two are open, and come out as of a layer of these three."""
    parts, n, hidden, chosen = 520, 4096, 2048, [0, 518, 519]
    g = torch.Generator(device="cuda").manual_seed(5)
    w1 = torch.zeros(parts, hidden, n, device="cuda", dtype=torch.int8)
    w2 = torch.zeros(parts, n, hidden, device="cuda", dtype=torch.int8)
    for e in chosen:
        w1[e] = torch.randint(-127, 128, (hidden, n), generator=g, device="cuda")
        w2[e] = torch.randint(-127, 128, (n, hidden), generator=g, device="cuda")
    s1, s2 = (torch.rand(parts, m, generator=g, device="cuda") * 1e-4 + 1e-4 for m in (hidden, n))
    x = torch.randn(rows, n, generator=g, device="cuda").to(BF16)
    router = torch.randn(parts, n, generator=g, device="cuda").mul_(n ** -0.5).to(BF16)
    closed = torch.full((parts,), -math.inf, device="cuda")
    closed[chosen] = 0.0
    got = ep().ep_experts(x, router, w1, w2, 2, router_bias=closed, w1_scale=s1, w2_scale=s2)
    want = ep().ep_experts(x, router[chosen].contiguous(), w1[chosen].contiguous(), w2[chosen].contiguous(), 2, w1_scale=s1[chosen].contiguous(),
                           w2_scale=s2[chosen].contiguous())
    assert torch.equal(got.ids, torch.tensor(chosen, device="cuda", dtype=torch.int32)[want.ids.long()])
    assert float((got.out.double() - want.out.double()).norm()) <= 2.0 ** -6 * float(want.out.double().norm())
