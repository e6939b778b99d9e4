"""Cross entropy where its logits are far from zero or exact, and each of its kernels by sizes that reach it, against 64-bit formulas.

The backward of 16-bit rows has three kernels: rows * classes * n_in up to 2^26 (rows and classes rounded up to 64s) with n_in <= 128 go by
one, other rows of up to 256 elements by another, wider ones by a third.  NARROW and WIDE are sizes of the second and third.
Bounds are those of test_gpu_entropy.py unless a test gives its own.
"""
import math

import pytest
import torch

import head_reference as ref
from test_gpu_entropy import BF16, F16, F32, backward, ep, forward, rand, some_targets, trained

pytestmark = pytest.mark.gpu


def one():
    return torch.ones(1, device="cuda")


def goes_by_tiles(rows, n_in, classes):
    return n_in > 128 or -(-rows // 64) * 64 * (-(-classes // 64) * 64) * n_in > 2 ** 26


# ---------------------------------------------------------------------------------------------- logits that are far from zero together
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("classes", [2, 10, 70])
@pytest.mark.parametrize("rows,n_in", [(17000, 64), (300, 200), (300, 264)])
@pytest.mark.parametrize("by", ["bias", "weights"])
def test_a_common_shift_of_the_logits(dtype, classes, rows, n_in, by):
    # a softmax is the same; classes that only fill a tile up have logits of zero, far above all others
    assert goes_by_tiles(rows, n_in, classes)
    for shift in (-2.0, -20.0, -120.0, 60.0):
        x, w = rand((rows, n_in), dtype, 1), rand((classes, n_in), dtype, 2, n_in ** -0.5)
        t, b = some_targets(rows, classes, 3, 0.1), None
        if by == "bias":
            b = rand((classes,), F32, 4, 0.5) + shift
        else:   # (powers of two and their sums: exact)
            x[:, 0], w[:, 0] = 4.0, shift / 4
        r = forward(x, w, t, b)
        got = backward(x, w, t, r, b, one(), rand((rows,), F32, 5, 1.0 / rows))
        assert all(bool(torch.isfinite(g).all()) for g in got)


# ---------------------------------------------------------------------------------------------- sums of logits
def one_class(x, w):
    """The logits themselves, as lse of a single class."""
    return ep().ep_cross_entropy(x, w, torch.zeros(x.shape[0], device="cuda", dtype=torch.int32)).lse.double()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n_in", [60, 256, 264, 1024, 4096, 65536])
def test_logits_of_one_element_are_exact(dtype, n_in):
    """One product of 8 by 8 or 11 by 11 bits fits fp32: what is off is 1 / log 2 and log 2 and the products with them, 2^-24 of the logit
    each.  Up to 256 elements a sum is given back what dense ones lose of it on average: (5 + 1.9 * 16) 1e-8 of itself at most."""
    rows = 200
    w, at = rand((1, n_in), dtype, 1), torch.arange(rows, device="cuda") * 37 % n_in
    x = torch.zeros(rows, n_in, device="cuda", dtype=dtype)
    x[torch.arange(rows, device="cuda"), at] = rand((rows,), dtype, 2, 16.0)
    want = (x.double() * w.double()).sum(1)
    most = 2.0 ** -22 + (3.54e-7 if n_in <= 256 else 0.0)
    ref.within(one_class(x, w), want, most * want.abs(), "lse")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n_in", [300, 1024, 4096, 65536])
def test_logits_of_one_sign(dtype, n_in):
    """Sums of one sign lose the most, with every step of 16 products 1e-7 of the result, which is below 2^-23.  After 16 steps at most they are
    added up to nearest, which costs 2^-24 of the sum each time (twice as many of them are allowed for)."""
    x, w = rand((64, n_in), dtype, 1).abs(), rand((1, n_in), dtype, 2).abs()
    want = (x.double() * w.double()).sum(1)
    ref.within(one_class(x, w), want, (16 * 2.0 ** -23 + -(-n_in // 128) * 2.0 ** -24 + 2.0 ** -22) * want, "lse")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n_in", [264, 1024, 4096, 65536])
def test_slopes_of_exact_logits(dtype, n_in):
    """dbias of a single row is that row of G, not rounded to the operands' type: p is off by 2^-20 of itself beside what the exponent's two
    roundings cost, 2^-22 (|l| + |lse|)."""
    classes = 40
    x, w = torch.zeros(1, n_in, device="cuda", dtype=dtype), rand((classes, n_in), dtype, 1)
    x[0, n_in // 2] = 1.0
    w[:, n_in // 2] = torch.linspace(56, 64, classes, device="cuda").to(dtype)
    t = torch.zeros(1, device="cuda", dtype=torch.int32)
    l = w[:, n_in // 2].double()
    lse = torch.logsumexp(l, 0)
    r = ep().ep_cross_entropy(x, w, t)._replace(lse=lse.float()[None])
    got = ep().ep_cross_entropy_backward(x, w, t, r, None, one()).dbias
    p = torch.exp(l - r.lse.double())
    want = p.clone()
    want[0] -= 1.0
    ref.within(got, want, p * (2.0 ** -20 + 2.0 ** -22 * (l.abs() + lse.abs())) + 2.0 ** -24 * want.abs(), "dbias")


# ---------------------------------------------------------------------------------------------- a class closed by the type's lowest value
@pytest.mark.parametrize("dtype,bias_dtype", [(BF16, F32), (BF16, BF16), (F16, F32), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("rows,n_in", [(50, 24), (400, 264)])
def test_loss_against_a_class_of_the_lowest_bias(dtype, bias_dtype, rows, n_in):
    x, w, t = trained(rows, n_in, 90, dtype, 1)
    b = rand((90,), bias_dtype, 2)
    b[30:60] = torch.finfo(bias_dtype).min
    r = forward(x, w, t, b)
    assert bool(((t >= 30) & (t < 60)).any())
    got = backward(x, w, t, r, b, one())
    assert bool((got.dbias[30:60] <= 0).all())


# ---------------------------------------------------------------------------------------------- each kernel of the backward
NARROW = [(30000, 64, 100), (17000, 96, 100), (1800, 200, 100)]
WIDE = [(1200, 264, 300)]


@pytest.mark.parametrize("rows,n_in,classes", NARROW + WIDE)
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_only_what_is_wanted(dtype, rows, n_in, classes):
    assert goes_by_tiles(rows, n_in, classes)
    x, w, t = trained(rows, n_in, classes, dtype, 10, 0.1)
    b = rand((classes,), F32, 11)
    r = forward(x, w, t, b)
    whole = backward(x, w, t, r, b, one())
    for wanted in ((0,), (1,), (2,), (0, 1), (0, 2), (1, 2)):
        got = backward(x, w, t, r, b, one(), **{n: i in wanted for i, n in enumerate(("need_dx", "need_dweight", "need_dbias"))})
        assert all(torch.equal(got[i], whole[i]) if i in wanted else got[i] is None for i in range(3)), wanted


@pytest.mark.parametrize("rows,n_in", [(40000, 32), (2000, 160), (1000, 272)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_far_logits_of_each_kernel(dtype, rows, n_in):
    # logits of hundreds: one class has all of it; masks of the type's lowest value beside it
    assert goes_by_tiles(rows, n_in, 90)
    x, w = rand((rows, n_in), dtype, 16, 30.0), rand((90, n_in), dtype, 17, 5.0)
    t = some_targets(rows, 90, 18).clamp(min=40)
    b = torch.zeros(90, device="cuda")
    b[:40] = torch.finfo(F32).min
    r = forward(x, w, t, b)
    backward(x, w, t, r, b, one())
    bad = x.clone()
    bad[7, 3] = math.nan
    r = ep().ep_cross_entropy(bad, w, t, b)
    got = ep().ep_cross_entropy_backward(bad, w, t, r, b, one())
    spoiled = torch.isnan(got.dx).any(1)
    assert bool(spoiled[7]) and int(spoiled.sum()) == 1


@pytest.mark.parametrize("rows,n_in", [(40000, 32), (2000, 160), (1000, 272)])
def test_fp16_gradients_of_any_size(rows, n_in):
    # a mean over many rows puts whole gradients below fp16's range
    assert goes_by_tiles(rows, n_in, 64)
    x, w, t = trained(rows, n_in, 64, F16, 30)
    r = forward(x, w, t)
    for g in (1e-4, 3e4, -1e-30, 1e-40):
        backward(x, w, t, r, None, torch.full((1,), g, device="cuda"))
    drow = rand((rows,), F32, 31) * torch.logspace(-6, 2, rows, device="cuda")
    drow[::5] = 0
    backward(x, w, t, r, None, None, drow)


@pytest.mark.parametrize("sizes", [((2500, 64, 900), (900, 200, 300)), ((3000, 128, 200), (900, 264, 300))])
def test_graphs_of_each_kernel_on_two_streams(sizes):
    m = ep()
    cases = [trained(rows, n_in, classes, dtype, 31 + i, 0.1) for i, ((rows, n_in, classes), dtype) in enumerate(zip(sizes, (BF16, F16)))]
    assert all(goes_by_tiles(*s) for s in sizes)
    ones = one()

    def both(a, b, c):
        r = m.ep_cross_entropy(a, b, c)
        return [*r, *m.ep_cross_entropy_backward(a, b, c, r, None, ones)]
    want = [both(*c) for c in cases]
    torch.cuda.synchronize()
    graphs, outs, streams = [], [], []
    for c in cases:
        s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(both(*c))
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
        assert all(torch.equal(a, b) for o, w in zip(outs, want) for a, b in zip(o, w))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n_in", [64, 130, 256, 264])
def test_rows_without_a_class_and_spoiled_ones_of_each_kernel(dtype, n_in):
    rows, classes = (20000, 70) if n_in <= 128 else (1500, 70)
    assert goes_by_tiles(rows, n_in, classes)
    x, w, t = trained(rows, n_in, classes, dtype, 40, 0.3)
    b, drow = rand((classes,), F32, 41) - 30, rand((rows,), F32, 42)
    r = forward(x, w, t, b)
    clean = backward(x, w, t, r, b, one(), drow)
    bad = x.clone()
    bad[t < 0] = torch.tensor([math.nan, math.inf], device="cuda").repeat(n_in // 2).to(dtype)
    q = ep().ep_cross_entropy(bad, w, t, b)
    assert all(torch.equal(p, s) for p, s in zip(r, q))
    got = ep().ep_cross_entropy_backward(bad, w, t, q, b, one(), drow.masked_fill(t < 0, math.nan))
    assert all(torch.equal(p, s) for p, s in zip(got, clean))


# ---------------------------------------------------------------------------------------------- what all elements of a gradient have in common
def common_share(got, want):
    """How much of `want` is missing in all of got: roundings by chance add up to nothing."""
    got, want = got.double(), want.double()
    return float(((got - want) * want).sum() / (want * want).sum())


@pytest.mark.parametrize("dtype,rows,n_in,classes", [(BF16, 255 * 64, 64, 3000), (BF16, 255 * 8, 200, 3000), (BF16, 255 * 8, 272, 3000),
                                                     (BF16, 255 * 8, 272, 40000), (F16, 2047 * 8, 64, 3000), (F16, 2047, 200, 3000), (F16, 2047, 272, 3000)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_a_mean_loss_scales_no_gradient(dtype, rows, n_in, classes, sign):
    """1 / rows lies half-way between two numbers of 8 (11) bits: as such in every row's target, a gradient would be off by 2^-8 (2^-11) throughout.
    Roundings by chance of n elements leave about UNIT / sqrt(n); sums in the tensor cores lose 1e-7 a step, some of it of one sign.  What may stay
    in common: 1 - p is rounded to 1 where the target's p is below half the spacing there (2^-9, 2^-12), so that it is off by p; the mean of p bounds
    that.  The result's own rounding is left out by rounding what is wanted, too (a single row's x times 1 / rows is rounded alike throughout)."""
    x, w = rand((rows, n_in), dtype, 1, 0.3), rand((classes, n_in), dtype, 2, n_in ** -0.5)
    t = some_targets(rows, classes, 3)
    r = forward(x, w, t)
    got = backward(x, w, t, r, None, sign * one())
    l = x.double() @ w.double().T
    G = ref.entropy_slopes(l, r.lse, t, sign * one(), None, rows)[0]
    p = torch.exp(l.gather(1, t.long()[:, None])[:, 0] - r.lse.double())
    for g, want in ((got.dx, G @ w.double()), (got.dweight, G.T @ x.double())):
        most = ref.UNIT[dtype] * 8 / math.sqrt(want.numel()) + 1e-7 * max(rows, classes) / 16 * 0.1 + 1e-6 + float(p.mean())
        if dtype == F16:      # below fp16's smallest normal number roundings are larger
            most = most + 2.0 ** -25 / float(want.abs().mean()) * 8 / math.sqrt(want.numel())
        assert abs(common_share(g, want.to(dtype))) <= most


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n_in", [64, 200])
def test_long_sums_over_classes_and_over_rows(dtype, n_in):
    """A column of W (of x) that is 1 throughout: its gradient dx is g (sum of p - 1) = 0, and that of W is dbias.  The tensor cores cut off 1e-7 of a sum of
    one sign with every 16 products; after 512 steps (fp16; bf16 4096) a sum is put away: 2^-23 512 of it, instead of all 10584.  G's roundings: the
    target's 1 - p by half the spacing below 1, UNIT / 2; by chance UNIT p a class, less than UNIT / 64 in all; exponentials and lse 2^-19."""
    steps = 512 if dtype == F16 else 4096
    rows, classes = 128 * 148 + 50, 169343
    x, w = rand((rows, n_in), dtype, 1), rand((classes, n_in), dtype, 2, n_in ** -0.5)
    w[:, 0], x[:, 1] = 1.0, 1.0
    t = some_targets(rows, classes, 3)
    r = ep().ep_cross_entropy(x, w, t)
    got = ep().ep_cross_entropy_backward(x, w, t, r, None, one() * rows, need_dweight=False, need_dbias=False)
    off = steps * 2.0 ** -23 + ref.UNIT[dtype] / 2 + ref.UNIT[dtype] / 64 + 2.0 ** -19
    ref.within(got.dx[:, 0], torch.zeros(rows), torch.full((rows,), off), "dx")
    # on average what rounding leaves is the mean of p where 1 - p is rounded to 1
    p = torch.exp(-r.row_loss.double())
    assert abs(float(got.dx[:, 0].double().mean())) <= steps * 2.0 ** -23 + float(p.clamp(max=ref.UNIT[dtype] / 2).mean()) + 2.0 ** -19
    # and over rows: the parts of dbias of one sign are the probabilities' sum and the targets'
    rows, classes = 169343, 128 * 148 + 50
    x, w, t = rand((rows, n_in), dtype, 4), w[:classes], some_targets(rows, classes, 5)
    x[:, 1] = 1.0
    r = ep().ep_cross_entropy(x, w, t)
    got = ep().ep_cross_entropy_backward(x, w, t, r, None, one() * rows, need_dx=False)
    sizes = 2 * torch.bincount(t.long(), minlength=classes).double() + got.dbias.double()
    off = (steps * 2.0 ** -23 + ref.UNIT[dtype] / 64) * sizes + ref.UNIT[dtype] * got.dbias.double().abs() + ref.UNIT[dtype] * sizes.sqrt()
    ref.within(got.dweight[:, 1], got.dbias, off, "dweight")


@pytest.mark.parametrize("n_in", [64, 200])
def test_sums_that_are_put_away_on_the_way(n_in):
    # a block's stretch is more than the 64 tiles of 128 rows after which fp16 sums are put away, and neither begins nor ends with a row tile
    rows, classes = 128 * 148 + 50, 9000
    x, w, t = trained(rows, n_in, classes, F16, 50, 0.1)
    b = rand((classes,), F32, 51)
    r = forward(x, w, t, b)
    whole = backward(x, w, t, r, b, one() * 1000)
    again = ep().ep_cross_entropy_backward(x, w, t, r, b, one() * 1000, need_dx=False)
    assert torch.equal(again.dweight, whole.dweight) and torch.equal(again.dbias, whole.dbias)
