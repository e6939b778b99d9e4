"""ep_cross_entropy and ep_cross_entropy_backward against 64-bit formulas.

Bounds.  A logit with S = sum |x| |w| is off by at most e = summing(n_in) S + 2^-23 |l| (the tensor core's sums as for ep_linear,
then the bias).  Exponentials are within 2^-20 of themselves beside 2^-22 |l - m| (two roundings of the argument, and
|l - m| exp(l - m) < 1); their sum over C classes within (C / 32 + 64) 2^-24 of itself.  So lse is off by at most
max e + 2^-19 + 2^-22 max|l| + (C / 32 + 64) 2^-24, and a row's loss by that and its target's e.  The backward is given lse: an
element of G is off by |g| p (e + 2^-19 + 2^-22 (|l| + |lse|)) and by one rounding to the operands' type; exponentials
below 2^-126 are zero, which costs |g| 2^-126.
"""
import math

import pytest
import torch

import head_reference as ref

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def ep():
    import paper_2604_01000_b200 as m
    return m


def rand(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def some_targets(rows, classes, seed, dead=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randint(0, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
    return t.masked_fill(torch.rand(rows, generator=g, device="cuda") < dead, -1)


def summing(k, runs):
    return (32 if runs else k / 16 + 4) * 2.0 ** -22


def logit_error(x, w, l):
    S = x.double().abs() @ w.double().abs().T
    return S * summing(x.shape[1], x.dtype == F32) + 2.0 ** -23 * torch.where(torch.isfinite(l), l.abs(), torch.zeros_like(l))


def finite_max(l):
    return torch.where(torch.isfinite(l), l.abs(), torch.zeros_like(l)).amax(1)


def forward(x, w, t, b=None):
    r = ep().ep_cross_entropy(x, w, t, b)
    lse, row_loss, loss, counted, l = ref.entropy(x, w, t, b)
    C = w.shape[0]
    assert int(r.counted) == counted and r.loss.shape == (1,) and r.lse.dtype == F32
    e = logit_error(x, w, l)
    off = e.amax(1) + 2.0 ** -19 + 2.0 ** -22 * finite_max(l) + (C / 32 + 64) * 2.0 ** -24
    live = (t >= 0) & (t < C) & ~torch.isneginf(lse)
    assert bool((r.row_loss[~live] == 0).all())
    ref.within(r.lse[live], lse[live], off[live] + ref.FP32 * lse[live].abs(), "lse")
    fine = live & torch.isfinite(row_loss)
    off = 2 * off + 2.0 ** -23 * (lse.abs() + row_loss.abs())
    ref.within(r.row_loss[fine], row_loss[fine], off[fine], "row_loss")
    assert bool(torch.isposinf(r.row_loss[live & ~fine]).all())
    if bool(fine.all() or (~live | fine).all()):
        ref.within(r.loss[0], loss, off[live].mean() + ref.FP32 * loss.abs() if counted else torch.tensor(0.0), "loss")
    return r


def backward(x, w, t, r, b=None, dloss=None, drow=None, **need):
    got = ep().ep_cross_entropy_backward(x, w, t, r, b, dloss, drow, **need)
    rows, n_in, C, dt = x.shape[0], x.shape[1], w.shape[0], x.dtype
    l = x.double() @ w.double().T
    l = l if b is None else l + b.double()
    e = logit_error(x, w, l)
    G, size = ref.entropy_slopes(l, r.lse, t, dloss, drow, int(r.counted))
    live = (t >= 0) & (t < C) & ~torch.isneginf(r.lse)
    x = torch.where(live[:, None], x, torch.zeros_like(x))      # rows that take no part count for nothing, whatever they hold
    e, l = torch.where(live[:, None], e, torch.zeros_like(e)), torch.where(live[:, None] & torch.isfinite(l), l, torch.zeros_like(l))
    lse = torch.where(live, r.lse.double(), torch.zeros_like(r.lse.double()))
    off = size * (e + 2.0 ** -19 + 2.0 ** -22 * (l.abs() + lse.abs()[:, None])) + 2.0 ** -23 * G.abs()
    off = off + 2.0 ** -126 * (size.sum(1, keepdim=True) + 1)      # (the sizes of a row add up to |g|)
    rounded = off + (ref.UNIT[dt] if dt != F32 else 2.0 ** -22) * G.abs()
    if dt == F16 and G.numel():
        rounded = rounded + 2.0 ** -38 * float(size.sum(1).max())
    xd, wd = x.double(), w.double()
    if got.dx is not None:
        want, S = G @ wd, G.abs() @ wd.abs()
        d = rounded @ wd.abs() + S * (summing(C, dt == F32) + 64 * ref.FP32)
        ref.within(got.dx, want, d + ref.UNIT[dt] * (want.abs() + d) + ref.TINY[dt], "dx")
        assert bool((got.dx[~live] == 0).all())
    if got.dweight is not None:
        want, S = G.T @ xd, G.abs().T @ xd.abs()
        d = rounded.T @ xd.abs() + S * (summing(rows, dt == F32) + 64 * ref.FP32)
        ref.within(got.dweight, want, d + ref.UNIT[dt] * (want.abs() + d) + ref.TINY[dt], "dweight")
    if got.dbias is not None:
        d = rounded.sum(0) + G.abs().sum(0) * (64 + rows / 16) * 2.0 ** -23
        ref.within(got.dbias, G.sum(0), d, "dbias")
    return got


def trained(rows, n_in, classes, dtype, seed, dead=0.0):
    w = rand((classes, n_in), dtype, seed, n_in ** -0.5)
    t = some_targets(rows, classes, seed + 1, dead)
    x = (rand((rows, n_in), F32, seed + 2) + 4 * w.float()[t.clamp(min=0).long()]).to(dtype)
    return x, w, t


SHAPES = [(1, 8, 2), (1, 64, 4096), (2, 65, 3), (7, 128, 1), (8, 1, 77), (33, 257, 129), (64, 128, 256), (128, 64, 32), (129, 100, 1000),
          (300, 72, 5003), (1000, 128, 4096), (2999, 65, 257), (70, 48, 40000), (4097, 16, 33), (500, 256, 700), (129, 272, 300),
          (1000, 129, 5000), (257, 1024, 1000)]


@pytest.mark.parametrize("rows,n_in,classes", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_shapes(rows, n_in, classes, dtype):
    x, w, t = trained(rows, n_in, classes, dtype, 1)
    b = rand((classes,), F32, 4, 0.5)
    backward(x, w, t, forward(x, w, t), None, torch.ones(1, device="cuda"))
    t = some_targets(rows, classes, 5, 0.3)
    r = forward(x, w, t, b)
    backward(x, w, t, r, b, torch.full((1,), -0.7, device="cuda"), rand((rows,), F32, 6, 1.0 / rows))
    backward(x, w, t, r, b, None, rand((rows,), F32, 7))


@pytest.mark.parametrize("rows,n_in,classes", [(20000, 40, 2500), (2500, 40, 20000), (17000, 24, 17000), (20000, 264, 2500), (2500, 264, 20000),
                                                  (40000, 200, 300), (300, 200, 40000)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_several_pieces(rows, n_in, classes, dtype):
    x, w, t = trained(rows, n_in, classes, dtype, 8, 0.1)
    b = rand((classes,), dtype, 9, 0.5)
    r = forward(x, w, t, b)
    got = backward(x, w, t, r, b, torch.ones(1, device="cuda"))
    again = ep().ep_cross_entropy_backward(x, w, t, r, b, torch.ones(1, device="cuda"))
    assert all(torch.equal(p, q) for p, q in zip(got, again))        # the same from run to run


@pytest.mark.parametrize("rows,n_in", [(300, 64), (6000, 64), (3000, 264)])
def test_what_is_not_wanted_is_not_made(rows, n_in):
    x, w, t = trained(rows, n_in, 100, BF16, 10)
    r = forward(x, w, t)
    one = torch.ones(1, device="cuda")
    whole = backward(x, w, t, r, None, one)
    for i, name in enumerate(("need_dx", "need_dweight", "need_dbias")):
        got = backward(x, w, t, r, None, one, **{name: False})
        assert got[i] is None and all(torch.equal(a, b) for j, (a, b) in enumerate(zip(got, whole)) if j != i)
    assert all(g is None for g in ep().ep_cross_entropy_backward(x, w, t, r, None, one, None, False, False, False))


# (up to 2^25 products go by other kernels than more, rows of up to 256 elements by others than wider ones)
@pytest.mark.parametrize("rows,n_in", [(500, 96), (3000, 96), (1800, 256), (700, 296)])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_rows_without_a_class_count_for_nothing_whatever_they_hold(dtype, rows, n_in):
    x, w, t = trained(rows, n_in, 300, dtype, 11, 0.2)
    b, one = rand((300,), F32, 12), torch.ones(1, device="cuda")
    r = forward(x, w, t, b)
    clean = backward(x, w, t, r, b, one, rand((rows,), F32, 13))
    spoiled = x.clone()
    spoiled[t < 0] = torch.tensor([math.nan, math.inf, -math.inf, 1.0] * (n_in // 4), device="cuda").to(dtype)
    drow = rand((rows,), F32, 13)
    drow[t < 0] = math.nan
    q = ep().ep_cross_entropy(spoiled, w, t, b)
    assert all(torch.equal(p, s) for p, s in zip(r, q))
    got = ep().ep_cross_entropy_backward(spoiled, w, t, q, b, one, drow)
    assert all(torch.equal(p, s) for p, s in zip(got, clean))
    got = ep().ep_cross_entropy_backward(ref.misaligned(spoiled), w, t, q, b, one, drow)
    assert all(torch.equal(p, s) for p, s in zip(got, clean))


@pytest.mark.parametrize("rows,n_in", [(200, 64), (9000, 64), (2000, 272)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_closed_classes(dtype, rows, n_in):
    x, w, t = trained(rows, n_in, 70, dtype, 14)
    b = rand((70,), F32, 15)
    b[::3] = -math.inf
    r = forward(x, w, t, b)
    assert bool(torch.isinf(r.row_loss[(t % 3 == 0)]).all()) and bool(torch.isinf(r.loss).all())
    got = backward(x, w, t, r, b, torch.ones(1, device="cuda"))
    t = (t // 3 * 3 + 1).clamp(max=67)
    r = forward(x, w, t, b)
    assert bool(torch.isfinite(r.loss).all())
    got = backward(x, w, t, r, b, torch.ones(1, device="cuda"))
    assert bool((got.dbias[::3] == 0).all()) and bool((got.dweight[::3] == 0).all())
    # nothing left: no row takes part
    r = ep().ep_cross_entropy(x, w, t, torch.full((70,), -math.inf, device="cuda"))
    assert int(r.counted) == 0 and float(r.loss) == 0 and bool((r.row_loss == 0).all()) and bool(torch.isneginf(r.lse).all())
    got = ep().ep_cross_entropy_backward(x, w, t, r, torch.full((70,), -math.inf, device="cuda"), torch.ones(1, device="cuda"))
    assert all(bool((g == 0).all()) for g in got)


@pytest.mark.parametrize("rows", [150, 14000])
def test_far_logits_and_spoiled_rows(rows):
    # logits of hundreds: one class has all of it; masks of the type's lowest value beside it
    for dtype in (BF16, F32):
        x, w = rand((rows, 32), dtype, 16, 30.0), rand((90, 32), dtype, 17, 5.0)
        t = some_targets(rows, 90, 18)
        b = torch.zeros(90, device="cuda")
        b[:40] = torch.finfo(F32).min
        r = forward(x, w, t.clamp(min=40), b)
        backward(x, w, t.clamp(min=40), r, b, torch.ones(1, device="cuda"))
        bad = x.clone()
        bad[7, 3] = math.nan
        r = ep().ep_cross_entropy(bad, w, t)
        assert bool(torch.isnan(r.row_loss[7])) and bool(torch.isnan(r.loss).all()) and int(torch.isnan(r.lse).sum()) == 1


@pytest.mark.parametrize("rows,n_in", [(40, 16), (40000, 96), (14000, 264)])
def test_targets_outside_the_classes_are_told_and_skipped(rows, n_in):
    m = ep()
    x, w, t = trained(rows, n_in, 10, BF16, 19)
    m.default_context().check()
    bad = t.clone()
    bad[3], bad[4], bad[5] = 10, -2, 2 ** 31 - 1
    left = t.clone()
    left[3:6] = -1
    want = m.ep_cross_entropy(x, w, left)
    m.default_context().check()
    got = m.ep_cross_entropy(x, w, bad)
    assert m.default_context().poll_status() == 4
    assert all(torch.equal(p, q) for p, q in zip(got, want)) and int(got.counted) == rows - 3
    one = torch.ones(1, device="cuda")
    got = m.ep_cross_entropy_backward(x, w, bad, want, None, one)
    assert m.default_context().poll_status() == 4
    assert all(torch.equal(p, q) for p, q in zip(got, m.ep_cross_entropy_backward(x, w, left, want, None, one)))


def test_no_rows_and_none_that_count():
    m = ep()
    w, one = rand((30, 20), BF16, 20), torch.ones(1, device="cuda")
    x, t = torch.empty(0, 20, device="cuda", dtype=BF16), torch.empty(0, device="cuda", dtype=torch.int32)
    r = m.ep_cross_entropy(x, w, t)
    assert float(r.loss) == 0 and int(r.counted) == 0 and r.lse.shape == (0,)
    got = m.ep_cross_entropy_backward(x, w, t, r, None, one)
    assert got.dx.shape == (0, 20) and not bool(got.dweight.any()) and not bool(got.dbias.any())
    x, t = rand((50, 20), BF16, 21), torch.full((50,), -1, device="cuda", dtype=torch.int32)
    r = m.ep_cross_entropy(x, w, t)
    assert float(r.loss) == 0 and int(r.counted) == 0
    got = m.ep_cross_entropy_backward(x, w, t, r, None, one, torch.ones(50, device="cuda"))
    assert not any(bool(g.any()) for g in got)


@pytest.mark.parametrize("rows", [130, 7000])
def test_strided_rows_and_misaligned_buffers(rows):
    for dtype in (BF16, F32, F16):
        big, wide = rand((rows, 200), dtype, 22), rand((70, 160), dtype, 23, 0.1)
        t, one = some_targets(rows, 70, 24), torch.ones(1, device="cuda")
        for x, w in ((big[:, 8:136], wide[:, 16:144]), (big[:, 3:80], wide[:, 5:82]), (big[:, :160], wide), (big[:, 1:161], wide)):
            backward(x, w, t, forward(x, w, t), None, one)
        half = some_targets(rows // 2, 70, 25)
        x = big[::2, :160]
        backward(x, wide, half, forward(x, wide, half, ref.misaligned(rand((70,), dtype, 26))), ref.misaligned(rand((70,), dtype, 26)), one)


def test_gradients_against_differences():
    # along a direction d: (loss(x + h d) - loss(x - h d)) / 2 h is off by h^2 / 6 of the third derivative (of a softmax's lse along
    # logits that move by at most D: at most 2 D^3) and by the loss' own error over h
    x, w, t = trained(60, 24, 40, F32, 27, 0.2)
    b = rand((40,), F32, 28)
    one = torch.ones(1, device="cuda")
    got = ep().ep_cross_entropy_backward(x, w, t, ep().ep_cross_entropy(x, w, t, b), b, one)
    h = 2.0 ** -10
    for name, grad in zip("xwb", got):
        d = torch.sign(rand(grad.shape, F32, 29))
        args = {"x": x, "w": w, "b": b}
        up, down = dict(args), dict(args)
        up[name], down[name] = args[name] + h * d, args[name] - h * d
        diff = (ep().ep_cross_entropy(up["x"], up["w"], t, up["b"]).loss.double() -
                ep().ep_cross_entropy(down["x"], down["w"], t, down["b"]).loss.double()) / (2 * h)
        moved = 1.0 if name == "b" else (w if name == "x" else x).abs().sum(1).max()
        bound = h * h / 6 * 2 * float(moved) ** 3 + 2.0 ** -16 / h
        assert abs(float(diff) - float((grad.double() * d.double()).sum())) <= bound, name


def test_small_gradients_of_fp16_are_kept():
    # a mean over many rows puts whole gradients below fp16's range
    for rows, n_in in ((5000, 32), (20000, 32), (3000, 264)):   # 64 classes each
        x, w, t = trained(rows, n_in, 64, F16, 30)
        r = forward(x, w, t)
        backward(x, w, t, r, None, torch.full((1,), 1e-4, device="cuda"))
        backward(x, w, t, r, None, torch.full((1,), 3e4, device="cuda"))


def test_captured_beside_another_stream():
    m = ep()
    x, w, t = trained(700, 64, 900, BF16, 31, 0.1)
    y, v, u = trained(900, 32, 300, BF16, 32, 0.1)
    one = torch.ones(1, device="cuda")
    def both(a, b, c):   # noqa: E306
        r = m.ep_cross_entropy(a, b, c)
        return [*r, *m.ep_cross_entropy_backward(a, b, c, r, None, one)]
    want, other = both(x, w, t), both(y, v, u)
    torch.cuda.synchronize()
    graphs, outs, streams = [], [], []
    for args in ((x, w, t), (y, v, u)):
        s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(both(*args))
        graphs.append(g)
        streams.append(s)
    for _ in range(5):
        for o in outs:
            for p in o:
                p.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[0], want)) and all(torch.equal(a, b) for a, b in zip(outs[1], other))


def test_refusals():
    m = ep()
    x, w, t = trained(10, 16, 5, BF16, 33)
    one = torch.ones(1, device="cuda")
    r = m.ep_cross_entropy(x, w, t)
    for bad in (lambda: m.ep_cross_entropy(x.float(), w, t), lambda: m.ep_cross_entropy(x, w[:, :8], t), lambda: m.ep_cross_entropy(x, w, t.long()),
                lambda: m.ep_cross_entropy(x, w, t[:9]), lambda: m.ep_cross_entropy(x, w, t.cpu()), lambda: m.ep_cross_entropy(x.t(), w, t),
                lambda: m.ep_cross_entropy(x, w, t, one), lambda: m.ep_cross_entropy(x.to(torch.int8), w.to(torch.int8), t),
                lambda: m.ep_cross_entropy_backward(x, w, t, r, None, torch.ones(2, device="cuda")),
                lambda: m.ep_cross_entropy_backward(x, w, t, r, None, one.double()),
                lambda: m.ep_cross_entropy_backward(x, w, t, r, None, one, torch.ones(9, device="cuda")),
                lambda: m.ep_cross_entropy_backward(x, w, t, r._replace(lse=r.lse[:5]), None, one)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(m.EmbedPartError):
        m.ep_cross_entropy(torch.empty(4, 70000, device="cuda", dtype=BF16), torch.empty(3, 70000, device="cuda", dtype=BF16), t[:4])
    with pytest.raises(m.EmbedPartError):
        m.ep_cross_entropy(torch.empty(4, 0, device="cuda", dtype=BF16), torch.empty(3, 0, device="cuda", dtype=BF16), t[:4])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n_in", [17, 128, 256, 727, 1024, 4096])
@pytest.mark.parametrize("stands_out", [0.0, 4.0])
def test_sums_of_logits_lose_nothing_on_average(dtype, n_in, stands_out):
    """The tensor cores cut sums off toward zero, a share of the sum that is given back.  With one class lse is the logit itself.  Of many
    rows' logits the common share that is missing: a quarter of what was cut off, (2.5 + 1.5 steps) 1e-8 for bf16 and (5 + 1.9 steps) 1e-8 for
    fp16 with a step of 16 products, and the roundings of the factors 1 / log 2 and log 2, 2^-24 each of themselves: 1.2e-7."""
    rows, g = 65536, torch.Generator(device="cuda").manual_seed(n_in)
    w = torch.randn(1, n_in, device="cuda", generator=g) / n_in ** 0.5
    x = torch.randn(rows, n_in, device="cuda", generator=g) + stands_out * w
    x, w = x.to(dtype), w.to(dtype)
    lse = ep().ep_cross_entropy(x, w, torch.zeros(rows, device="cuda", dtype=torch.int32)).lse.double()
    want = (x.double() * w.double()).sum(1)
    steps = (n_in + 15) // 16
    lost = (2.5 + 1.5 * steps if dtype is torch.bfloat16 else 5 + 1.9 * steps) * 1e-8
    share = ((lse - want) * want).sum() / (want * want).sum()
    assert abs(share.item()) <= 0.25 * lost + 1.2e-7


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,n_in,classes", [(23406, 727, 23), (20000, 250, 5), (20000, 1000, 40)])
def test_bias_gradient_of_many_rows_and_few_classes(dtype, rows, n_in, classes):
    """What a logit is off in common is off in a sum over rows, too, where the slopes themselves nearly cancel: dbias is some 1e-3 and its
    slopes up to 1.  With a quarter of what the sums lose (above) left, a row's logit l is off by less than 0.25 lost |l|, its slopes by less
    than that and 2^-23 |l| more for the exponents' roundings, and dbias by no more than their mean."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    w = torch.randn(classes, n_in, device="cuda", generator=g) / n_in ** 0.5
    t = torch.randint(0, classes, (rows,), device="cuda", generator=g)
    x = torch.randn(rows, n_in, device="cuda", generator=g) + 4 * w[t]
    x, w = x.to(dtype), w.to(dtype)
    l = x.double() @ w.double().T
    result = ep().ep_cross_entropy(x, w, t.int())._replace(lse=torch.logsumexp(l, 1).float())
    got = ep().ep_cross_entropy_backward(x, w, t.int(), result, None, torch.ones(1, device="cuda"))
    p = torch.exp(l - result.lse.double()[:, None])
    p[torch.arange(rows, device="cuda"), t] -= 1.0
    steps = (n_in + 15) // 16
    lost = (2.5 + 1.5 * steps if dtype is torch.bfloat16 else 5 + 1.9 * steps) * 1e-8
    most = (0.25 * lost + 2.0 ** -23) * l.abs().amax(1).mean()
    assert (got[2].double() - p.mean(0)).abs().max() <= most


@pytest.mark.parametrize("dtype,rows", [(torch.bfloat16, 17 * 2048 + 300), (torch.float32, 34 * 1024 + 7)])
def test_bias_gradient_over_more_pieces_of_rows_than_are_kept(dtype, rows):
    """16384 classes by 2048 rows (16 bits) or 1024 (32) make a piece; more than 16 pieces' sums are joined on the way.  Slopes by the bounds
    above, their sums rounded a few times: 2^-21 of the sum of magnitudes."""
    n_in, classes = 264, 16384
    x, w = rand((rows, n_in), dtype, 1), rand((classes, n_in), dtype, 2, 0.05)
    t = some_targets(rows, classes, 3, dead=0.1)
    result = ep().ep_cross_entropy(x, w, t)
    got = ep().ep_cross_entropy_backward(x, w, t, result, None, torch.ones(1, device="cuda"), need_dx=False, need_dweight=False)[2]
    want, off = torch.zeros(classes, device="cuda", dtype=torch.float64), torch.zeros(classes, device="cuda", dtype=torch.float64)
    live = t >= 0
    R = int(live.sum())
    for i in range(0, rows, 4096):
        l = x[i:i + 4096].double() @ w.double().T
        lse = result.lse[i:i + 4096].double()[:, None]
        p = torch.exp(l - lse)
        e = logit_error(x[i:i + 4096], w, l) + 2.0 ** -19 + 2.0 ** -22 * (l.abs() + lse.abs())
        hot = torch.nn.functional.one_hot(t[i:i + 4096].clamp(min=0).long(), classes)
        want += ((p - hot) * live[i:i + 4096, None]).sum(0) / R
        off += ((p * e + 2.0 ** -21 * (p + hot)) * live[i:i + 4096, None]).sum(0) / R
    ref.within(got, want, off, "dbias")


def near(got, want, what):
    """Addresses are what is tested: values of another row would be off by as much as they are large."""
    got, want = got.double(), want.double()
    assert float((got - want).norm()) <= 2.0 ** -6 * float(want.norm()), what


@pytest.mark.parametrize("n_in", [257, 256])
def test_weights_whose_offsets_pass_32_bits(n_in):
    classes, rows = (1 << 24) - 5, 24
    chosen = torch.cat([torch.arange(700), torch.arange(classes // 2, classes // 2 + 700), torch.arange(classes - 700, classes)]).cuda()
    some = rand((len(chosen), n_in), BF16, 1, n_in ** -0.5)
    w = torch.zeros(classes, n_in, device="cuda", dtype=BF16)
    w[chosen] = some
    bias = torch.full((classes,), -math.inf, device="cuda")
    bias[chosen] = 0.5
    t = some_targets(rows, len(chosen), 2)
    t[0], t[1] = len(chosen) - 1, 0
    x = (rand((rows, n_in), F32, 3) + 4 * some.float()[t.long()]).to(BF16)
    far = chosen[t.long()].int()
    r, few = ep().ep_cross_entropy(x, w, far, bias), ep().ep_cross_entropy(x, some, t)
    near(r.lse, few.lse + 0.5, "lse")
    near(r.row_loss, few.row_loss, "row_loss")
    one = torch.ones(1, device="cuda")
    got, want = ep().ep_cross_entropy_backward(x, w, far, r, bias, one), ep().ep_cross_entropy_backward(x, some, t, few, None, one)
    near(got.dx, want.dx, "dx")
    near(got.dweight[chosen], want.dweight, "dweight")
    near(got.dbias[chosen], want.dbias, "dbias")
    got.dweight[chosen] = 0
    got.dbias[chosen] = 0
    assert int(torch.count_nonzero(got.dbias)) == 0
    assert all(int(torch.count_nonzero(part)) == 0 for part in got.dweight.split(1 << 20))


@pytest.mark.parametrize("rows,n_in", [(1 << 25, 136), ((1 << 24) - 77, 264)])
def test_rows_whose_offsets_pass_32_bits(rows, n_in):
    classes = 5
    chosen = torch.cat([torch.arange(400), torch.arange(rows // 2, rows // 2 + 400), torch.arange(rows - 400, rows)]).cuda()
    w = rand((classes, n_in), BF16, 1, n_in ** -0.5)
    t = some_targets(len(chosen), classes, 2)
    some = (rand((len(chosen), n_in), F32, 3) + 4 * w.float()[t.long()]).to(BF16)
    x = torch.zeros(rows, n_in, device="cuda", dtype=BF16)
    x[chosen] = some
    x[rows // 4] = math.nan
    far = torch.full((rows,), -1, device="cuda", dtype=torch.int32)
    far[chosen] = t
    r, few = ep().ep_cross_entropy(x, w, far), ep().ep_cross_entropy(some, w, t)
    assert int(r.counted) == len(chosen)
    near(r.lse[chosen], few.lse, "lse")
    near(r.loss, few.loss, "loss")
    one = torch.ones(1, device="cuda")
    got, want = ep().ep_cross_entropy_backward(x, w, far, r, None, one), ep().ep_cross_entropy_backward(some, w, t, few, None, one)
    near(got.dx[chosen], want.dx, "dx")
    near(got.dweight, want.dweight, "dweight")
    near(got.dbias, want.dbias, "dbias")
    got.dx[chosen] = 0
    assert all(int(torch.count_nonzero(part)) == 0 for part in got.dx.split(1 << 21))
