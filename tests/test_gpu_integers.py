"""8-bit integers: ep_quantize_rows and ep_rms_norm to int8, and ep_linear of int8, against 64-bit formulas.

Bounds.  The products' sums are exact integers; turning one into fp32 costs 2^-24 of it, the scales' product and its product with
the sum 2^-24 each, so z is within 3 2^-24 |z - bias| + 2^-24 |z| of itself; activations and the residual as for ep_linear
(2^-20 of their terms), and one rounding ends it.  An integer of ep_quantize_rows lies within 1/2 + 127 (3 2^-24) of x / scale.
"""
import math

import pytest
import torch

import head_reference as ref

pytestmark = pytest.mark.gpu

F32, BF16, F16, I8 = torch.float32, torch.bfloat16, torch.float16, torch.int8
NEAR = 0.5 + 127 * 3 * 2.0 ** -24


def ep():
    import paper_2604_01000_b200 as m
    return m


def rand(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def integers(shape, seed, low=-128):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(low, 128, shape, generator=g, device="cuda", dtype=torch.int8)


def scales(n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.rand(n, generator=g, device="cuda") * 0.01 + 1e-4


def exact_products(x, w):
    return (x.double() @ w.double().T)      # integers below 2^53


def check(x, w, xs, ws, bias=None, act="none", residual=None, out=BF16, preact=False):
    r = ep().ep_linear(x, w, bias, act, residual, xs, ws, out, preact)
    assert r.out.dtype == out and (r.preact is None) == (not preact)
    s = exact_products(x, w) * xs.double()[:, None] * ws.double()
    z = s + (0.0 if bias is None else bias.double())
    work = 2.0 ** -24 * (3 * s.abs() + z.abs()) + 2.0 ** -149
    if preact:
        ref.within(r.preact, z, work + ref.UNIT[out] * (z.abs() + work) + ref.TINY[out], "preact")
    y, res = ref.act(z, act), 0.0 if residual is None else residual.double()
    work = 1.2 * work + 2.0 ** -24 * (y + res).abs() if act in ("none", "relu") else 1.2 * work + 2.0 ** -20 * (y.abs() + z.abs() * 2.0 ** -4)
    total = y + res
    ref.within(r.out, total, work + ref.UNIT[out] * (total.abs() + work) + ref.TINY[out], "out")
    return r


SHAPES = [(1, 1024, 1024), (1, 5, 3), (2, 33, 77), (3, 16, 130), (7, 500, 64), (8, 4096, 65), (9, 64, 64), (17, 8, 8), (64, 128, 256), (127, 80, 130),
          (128, 64, 128), (129, 65, 257), (300, 515, 257), (200, 4096, 64), (513, 1, 1), (1000, 256, 1000), (2000, 640, 384), (40, 16384, 33)]


@pytest.mark.parametrize("rows,n_in,n_out", SHAPES)
@pytest.mark.parametrize("out", [BF16, F16, F32])
def test_shapes(rows, n_in, n_out, out):
    x, w = integers((rows, n_in), 1), integers((n_out, n_in), 2)
    xs, ws = scales(rows, 3) / n_in ** 0.5, scales(n_out, 4)
    check(x, w, xs, ws, None, "none", None, out)
    check(x, w, xs, ws, rand((n_out,), F32, 5), "gelu", rand((rows, n_out), out, 6), out, True)
    check(x, w, xs, ws, rand((n_out,), BF16, 5), "silu", None, out)


@pytest.mark.parametrize("rows", [1, 5, 8, 9, 150, 700])
def test_sums_are_exact_however_long(rows):
    # the largest sums there are, and sums past 2^24, whose last bits fp32 would not keep; scale 1: the integer itself, rounded once
    for n_in in (3000, 65536):
        x, w = integers((rows, n_in), 7, 100), integers((40, n_in), 8, 100)
        x[0], w[0], w[1] = -128, -128, 127
        one_r, one_c = torch.ones(rows, device="cuda"), torch.ones(40, device="cuda")
        want = exact_products(x, w)
        assert float(want.abs().max()) >= 128.0 * 127 * n_in
        got = ep().ep_linear(x, w, None, "none", None, one_r, one_c, F32).out
        assert torch.equal(got, want.float())


def test_a_row_does_not_depend_on_how_many_others_come_with_it():
    x, w = integers((600, 2500), 9), integers((300, 2500), 10)
    xs, ws, b = scales(600, 11), scales(300, 12), rand((300,), F32, 13)
    whole = ep().ep_linear(x, w, b, "gelu", None, xs, ws, F32).out
    for n in (1, 3, 8, 9, 130, 599):
        assert torch.equal(ep().ep_linear(x[:n], w, b, "gelu", None, xs[:n], ws, F32).out, whole[:n])


def test_strided_rows_and_misaligned_buffers():
    big, wide = integers((300, 400), 14), integers((70, 300), 15)
    for rows in (4, 150):
        res = rand((rows, 96), BF16, 16)
        xs, ws = scales(rows, 17), scales(70, 18)
        for x, w in ((big[:rows, 16:144], wide[:, 32:160]), (big[:rows, 3:80], wide[:, 5:82]), (big[:2 * rows:2, :300], wide)):
            check(x, w, xs, ws, None, "relu", res[:, 1:71])
            check(x, w, xs, ws, None, "relu", None, F32)
        check(ref.misaligned(big[:rows, :300].contiguous()), ref.misaligned(wide), xs, ws, rand((70,), F16, 19), "none", ref.misaligned(res[:, :70].contiguous()))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,width", [(1, 1), (3, 7), (5, 128), (17, 1000), (200, 4096), (9, 16384), (1000, 33)])
def test_quantized_rows(dtype, rows, width):
    m = ep()
    for x in (rand((rows, width), dtype, 20, 3.0), ref.misaligned(rand((rows, width), dtype, 21, 1e-3))):
        r = m.ep_quantize_rows(x, torch.int8)
        assert r.q.dtype == I8 and r.scale.dtype == F32
        want = x.double().abs().amax(1) / 127
        ref.within(r.scale, want, ref.FP32 * want, "scale")
        assert bool((r.q.abs().amax(1) == 127).all())
        ref.within(r.q, x.double() / r.scale.double()[:, None], torch.full((rows, width), NEAR), "q")


def test_rows_that_have_no_scale():
    m = ep()
    x = rand((6, 64), F32, 22)
    x[1] = 0
    x[2, 5] = math.nan
    x[3, 6] = -math.inf
    x[4] *= 1e-41                       # scales below the smallest normal number keep few bits
    x[5] *= 1e37
    r = m.ep_quantize_rows(x, torch.int8)
    assert float(r.scale[1]) == 0 and not bool(r.q[1:4].any())
    assert math.isnan(float(r.scale[2])) and math.isinf(float(r.scale[3]))
    off = (r.q[4].double() * r.scale[4].double() - x[4].double()).abs()
    assert float(off.max()) <= 0.5 * float(r.scale[4]) + 127 * 2.0 ** -150
    assert int(r.q[5].abs().max()) == 127
    tiny = torch.arange(0, 200, device="cuda", dtype=F32)[:, None] * 2.0 ** -149 * torch.ones(1, 16, device="cuda")
    q = m.ep_quantize_rows(tiny, torch.int8)
    assert int(q.q.min()) >= 0          # never past 127
    # what stands for NaN makes NaN, beside rows that are fine
    w, ws = integers((20, 64), 23), scales(20, 24)
    for n in (6, 60):
        y = m.ep_linear(r.q.repeat(n // 6, 1), w, None, "none", None, r.scale.repeat(n // 6), ws, F32).out.view(-1, 6, 20)
        assert bool(torch.isnan(y[:, 2:4]).all()) and bool(torch.isfinite(y[:, [0, 1, 4, 5]]).all())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,width", [(1, 1024), (300, 96), (77, 515)])
def test_norm_to_integers_feeds_the_product(dtype, rows, width):
    m = ep()
    x, g, res = rand((rows, width), dtype, 25), rand((width,), F32, 26) * 0.1 + 1, rand((rows, width), dtype, 27)
    n = m.ep_rms_norm(x, g, res, 1e-6, torch.int8)
    h, _, y = ref.norm(x, g, res, 1e-6)
    assert n.out.dtype == I8 and n.hidden.dtype == dtype
    top = y.abs().amax(1)
    ref.within(n.scale, top / 127, 2.0 ** -20 * top / 127, "scale")
    # y is within 2^-20 of itself before it is rounded to an integer
    ref.within(n.out, y / n.scale.double()[:, None], torch.full((rows, width), NEAR + 127 * 2.0 ** -20), "out")
    wq = m.ep_quantize_rows(rand((88, width), BF16, 28), torch.int8)
    check(n.out, wq.q, n.scale, wq.scale, None, "none", None, BF16)


def test_e4m3_stays_the_choice_when_none_is_made():
    r = ep().ep_quantize_rows(rand((4, 32), F32, 29))
    assert r.q.dtype == torch.float8_e4m3fn


def test_no_rows():
    m = ep()
    q = m.ep_quantize_rows(torch.empty(0, 32, device="cuda"), I8)
    r = m.ep_linear(q.q, integers((5, 32), 30), None, "none", None, q.scale, scales(5, 31), F32)
    assert r.out.shape == (0, 5)


def test_captured_beside_another_stream():
    m = ep()
    args = [(integers((700, 640), 32), integers((500, 640), 33), scales(700, 34), scales(500, 35)),
            (integers((40, 8192), 36), integers((64, 8192), 37), scales(40, 38), scales(64, 39)),
            (integers((2, 512), 40), integers((300, 512), 41), scales(2, 42), scales(300, 43))]
    run = lambda x, w, xs, ws: m.ep_linear(x, w, None, "gelu", None, xs, ws, BF16).out   # noqa: E731
    want = [run(*a) for a in args]
    torch.cuda.synchronize()
    graphs, outs, streams = [], [], []
    for a in args:
        s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(run(*a))
        graphs.append(g)
        streams.append(s)
    for _ in range(5):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_refusals():
    m = ep()
    x, w, xs, ws = integers((10, 16), 44), integers((5, 16), 45), scales(10, 46), scales(5, 47)
    for bad in (lambda: m.ep_linear(x, w), lambda: m.ep_linear(x, w, None, "none", None, xs), lambda: m.ep_linear(x, w.to(torch.float8_e4m3fn), None, "none", None, xs, ws),
                lambda: m.ep_linear(x, w, None, "none", None, xs, ws, I8), lambda: m.ep_linear(x, w, None, "none", None, xs[:9], ws),
                lambda: m.ep_linear(x, w, None, "none", None, xs.double(), ws), lambda: m.ep_linear(x.to(torch.uint8), w, None, "none", None, xs, ws),
                lambda: m.ep_quantize_rows(x, I8), lambda: m.ep_quantize_rows(rand((4, 4), F32, 48), torch.uint8),
                lambda: m.ep_quantize_rows(rand((4, 4), F32, 48), BF16), lambda: m.ep_rms_norm(rand((4, 4), F32, 48), out_dtype=torch.uint8),
                lambda: m.ep_linear_backward(rand((10, 5), F32, 49), x, w), lambda: m.ep_route(x, 1)):
        with pytest.raises(ValueError):
            bad()
