"""The partition head's operators at the ends of their range, against 64-bit formulas.

Bounds, with u the rounding unit of the output's type.  GELU's lower side is z m, m = tail(|z|) exp(-z^2 / 2): the
exponential's argument is rounded twice (2^-23 z^2 / 2 each), the special function unit and the polynomial add a few 2^-22, and
z itself may be 2^-22 of itself off, which its lower side shows (z^2 + 1) times: 2^-20 (z^2 + 4) of the value covers all of it.
SiLU alike with |z| for z^2.  Exponentials and reciprocals below 2^-126 are zero.
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


def through(z, act, rows, out):
    """act(z) by a product of one input column of ones; z's type is the operands'."""
    return ep().ep_linear(torch.ones(rows, 1, device="cuda", dtype=z.dtype), z[:, None].contiguous(), None, act, out_dtype=out).out


@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16)])
@pytest.mark.parametrize("rows", [5, 200])
def test_gelu_keeps_its_lower_tail(dtype, out, rows):
    z = torch.linspace(-12, 3, 301, device="cuda").to(dtype)
    got, zd = through(z, "gelu", rows, out), z.double()
    want = ref.act(zd, "gelu")
    bound = want.abs() * (2.0 ** -20 * (zd * zd + 4) + 1.01 * ref.UNIT[out]) + ref.TINY[out] + 12 * 2.0 ** -126
    ref.within(got, want.expand(rows, -1), bound.expand(rows, -1), "gelu")


def test_gelu_slope_keeps_its_lower_tail():
    # W = I: dx is dz, rounded once; the terms Phi(z) and z phi(z) of the slope cancel near -0.75
    z = torch.linspace(-12, 3, 304, device="cuda").to(BF16).repeat(40, 1)
    eye = torch.eye(304, device="cuda", dtype=BF16)
    dx = ep().ep_linear_backward(torch.ones_like(z), torch.ones_like(z), eye, z, "gelu", need_dweight=False).dx
    zd = z.double()
    want = ref.slope(zd, "gelu")
    terms = 0.5 * torch.special.erfc(-zd / math.sqrt(2)) + zd.abs() * torch.exp(-zd * zd / 2) / math.sqrt(2 * math.pi)
    ref.within(dx, want, terms * 2.0 ** -20 * (zd * zd + 4) + 1.01 * ref.UNIT[BF16] * want.abs() + 12 * 2.0 ** -126, "slope")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [5, 200])
def test_silu_far_below_zero(dtype, rows):
    z = torch.tensor([-1e38, -3e30, -1e9, -1e4, -200.0, -100.0, -90.0, -87.0, -80.0, -60.0, -10.0, -1.0, 0.0, 5.0, 90.0, 1e38],
                     device="cuda").to(dtype)
    got, zd = through(z, "silu", rows, dtype), z.double()
    want = ref.act(zd, "silu")
    bound = want.abs() * (2.0 ** -20 * (zd.abs().clamp(max=200) + 4) + 1.01 * ref.UNIT[dtype]) + 200 * 2.0 ** -126
    ref.within(got, want.expand(rows, -1), bound.expand(rows, -1), "silu")
    low = through(torch.full((8,), -math.inf, device="cuda", dtype=dtype), "silu", rows, dtype)
    assert bool((torch.isnan(low) | (low == 0)).all())   # (the formula's own: -infinity / infinity; its limit is 0)
    r = ep().ep_linear_backward(torch.ones(20, 16, device="cuda"), torch.ones(20, 8, device="cuda"), torch.ones(16, 8, device="cuda"),
                                z.float().repeat(20, 1), "silu")
    slope = ref.slope(zd, "silu")
    slope[:6] = torch.exp(zd[:6]) * (1 + zd[:6])         # (the reference's product is 0 times infinity there)
    slope[0], slope[15] = 0.0, 1.0
    ref.within(r.dbias, 20 * slope, 20 * (slope.abs() * 2.0 ** -18 * (zd.abs().clamp(max=200) + 4) + 200 * 2.0 ** -126), "slope")


@pytest.mark.parametrize("rows", [1, 3, 8, 40])
@pytest.mark.parametrize("n_in,n_out", [(96, 64), (33, 7), (2048, 5)])
def test_an_infinity_in_fp32_is_nan_whatever_the_number_of_rows(rows, n_in, n_out):
    g = torch.Generator(device="cuda").manual_seed(50)
    x, w = torch.randn(rows, n_in, generator=g, device="cuda"), torch.randn(n_out, n_in, generator=g, device="cuda") * 0.1
    clean = ep().ep_linear(x, w).out
    for bad in (math.inf, -math.inf, math.nan):
        a, b = x.clone(), w.clone()
        a[rows - 1, n_in - 1] = bad
        out = ep().ep_linear(a, w).out
        assert bool(torch.isnan(out[rows - 1]).all()) and torch.equal(out[:rows - 1], clean[:rows - 1])
        b[2, 1] = bad
        out = ep().ep_linear(x, b).out
        keep = [c for c in range(n_out) if c != 2]
        assert bool(torch.isnan(out[:, 2]).all()) and torch.equal(out[:, keep], clean[:, keep])


def test_a_sum_that_overflows_is_an_infinity():
    x, w = torch.full((2, 40), 1e20, device="cuda"), torch.full((9, 40), 1e20, device="cuda")
    assert bool(torch.isposinf(ep().ep_linear(x, w).out).all()) and bool(torch.isneginf(ep().ep_linear(-x, w).out).all())


def fp16_gradients(dout, x, w, z, act):
    """dx, dweight and dbias of fp16 operands against fp64.  dz keeps 11 bits wherever |dz| is above 2^-26 of the largest
    |dout| and loses 2^-38 of that largest otherwise; the sums truncate 2^-22 a step of 16; one rounding ends it."""
    r = ep().ep_linear_backward(dout, x, w, z, act)
    slope = torch.ones_like(dout, dtype=torch.float64) if act == "none" else ref.slope(z.double(), act)
    dz, lost = dout.double() * slope, 2.0 ** -38 * float(dout.double().abs().max())
    unit = ref.UNIT[F16]
    for got, a, b, steps in ((r.dx, dz, w.double(), w.shape[0] / 16), (r.dweight, dz.T, x.double(), x.shape[0] / 16)):
        want, size = a @ b, a.abs() @ b.abs()
        e = size * (2.0 ** -18 + unit + (steps + 4) * 2.0 ** -22) + lost * b.abs().sum(0)
        ref.within(got, want, e + unit * (want.abs() + e) + ref.TINY[F16], "gradient")
        assert float(want.abs().min()) > 2.0 ** -14          # (a result that fp16 holds)
    want = dz.sum(0)
    ref.within(r.dbias, want, dz.abs().sum(0) * (2.0 ** -18 + (64 + x.shape[0] / 64) * 2.0 ** -23), "dbias")


@pytest.mark.parametrize("rows,n_in,n_out", [(20000, 64, 128), (20001, 33, 17)])
@pytest.mark.parametrize("grad", [F32, F16])
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
def test_fp16_gradients_below_what_fp16_holds(rows, n_in, n_out, grad, act):
    # a mean over very many rows without a loss scale: every element of dz is near or below fp16's smallest numbers, the
    # sums over rows are not
    g = torch.Generator(device="cuda").manual_seed(51)
    uniform = lambda *s: torch.rand(*s, generator=g, device="cuda") + 0.5   # noqa: E731
    x, w = uniform(rows, n_in).to(F16), (uniform(n_out, n_in) * 30000).to(F16)
    z = (uniform(rows, n_out) * 0.1).to(F16)
    fp16_gradients((uniform(rows, n_out) * (2.0 ** -27 if grad == F32 else 2.0 ** -23)).to(grad), x, w, z, act)


@pytest.mark.parametrize("act", ["none", "gelu"])
def test_fp16_gradients_above_what_fp16_holds(act):
    g = torch.Generator(device="cuda").manual_seed(52)
    uniform = lambda *s: torch.rand(*s, generator=g, device="cuda") + 0.5   # noqa: E731
    x, w, z = (uniform(300, 40) * 1e-5).to(F16), (uniform(24, 40) * 1e-4).to(F16), uniform(300, 24).to(F16)
    fp16_gradients(uniform(300, 24) * 1e6, x, w, z, act)
    big = torch.full((300, 24), 65504.0, device="cuda", dtype=F16)          # times a slope above 1
    fp16_gradients(big, x, w, torch.full_like(z, 1.5), "gelu")


def test_fp16_gradients_that_are_zero_or_not_finite():
    x, w = torch.ones(40, 16, device="cuda", dtype=F16), torch.ones(24, 16, device="cuda", dtype=F16)
    zero = ep().ep_linear_backward(torch.zeros(40, 24, device="cuda"), x, w)
    assert not bool(zero.dx.any()) and not bool(zero.dweight.any()) and not bool(zero.dbias.any())
    dout = torch.full((40, 24), 1e-9, device="cuda")
    clean = ep().ep_linear_backward(dout * 1e4, x, w)
    for bad in (math.nan, math.inf):
        d = dout * 1e4
        d[3, 5] = bad
        r = ep().ep_linear_backward(d, x, w)
        keep = [i for i in range(40) if i != 3]
        assert torch.equal(r.dx[keep], clean.dx[keep]) and not bool(torch.isfinite(r.dx[3]).any())
        cols = [i for i in range(24) if i != 5]
        assert torch.equal(r.dweight[cols], clean.dweight[cols]) and not bool(torch.isfinite(r.dweight[5]).any())


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_long_sums_do_not_drift(dtype):
    # 400000 rows of one sign into a weight gradient wide enough that no idle block takes a share of its sum.  Sums that are
    # truncated at every step lose about 1e-7 of themselves a step (25000 steps here): the mean of the errors must stay
    # within a quarter of the type's rounding unit, whatever the number of rows
    rows, n = 400_000, 2048
    g = torch.Generator(device="cuda").manual_seed(53)
    x = ((torch.rand(rows, n, generator=g, device="cuda", dtype=F16) + 1) * 0.5).to(dtype)
    dout = ((torch.rand(rows, n, generator=g, device="cuda", dtype=F16) + 1) * 2.0 ** -11).to(dtype)
    want = torch.zeros(n, n, device="cuda", dtype=torch.float64)
    for at in range(0, rows, 50_000):
        want += dout[at:at + 50_000].double().T @ x[at:at + 50_000].double()
    got = ep().ep_linear_backward(dout, x, torch.ones(n, n, device="cuda", dtype=dtype), need_dx=False, need_dbias=False).dweight
    off, unit = (got.double() - want) / want, ref.UNIT[dtype]
    assert abs(float(off.mean())) <= unit / 4 and float(off.abs().max()) <= unit * 1.26


@pytest.mark.parametrize("dtype,rows,n_out,n_in", [(F16, 131_150, 2100, 1997), (BF16, 131_150, 2100, 1997), (F16, 20_011, 4999, 5008),
                                                   (F16, 1_200_005, 40, 56), (BF16, 70_003, 4000, 4008), (F16, 9_000, 300, 20_000)])
def test_long_sums_of_either_sign(dtype, rows, n_out, n_in):
    # lengths that end inside a step, widths that leave by whole pieces and by single elements, in shares and in one.  A run
    # has at most 512 (fp16) or 4096 steps, each of which costs 2^-22 of its terms; then one rounding
    g = torch.Generator(device="cuda").manual_seed(54)
    x = torch.randn(rows, n_in, generator=g, device="cuda").to(dtype)
    dout = torch.randn(rows, n_out, generator=g, device="cuda").to(dtype)
    got = ep().ep_linear_backward(dout, x, torch.ones(n_out, n_in, device="cuda", dtype=dtype), need_dx=False, need_dbias=False).dweight
    steps = 520 if dtype == F16 else 4110
    for at in range(0, n_out, 1700):                     # (the reference, some rows of dweight at a time)
        cols = slice(at, min(at + 100, n_out))
        want = torch.zeros(cols.stop - cols.start, n_in, device="cuda", dtype=torch.float64)
        size = torch.zeros_like(want)
        for r in range(0, rows, 20_000):
            a, b = dout[r:r + 20_000, cols].double(), x[r:r + 20_000].double()
            want += a.T @ b
            size += a.abs().T @ b.abs()
        e = size * steps * 2.0 ** -22
        ref.within(got[cols], want, e + ref.UNIT[dtype] * (want.abs() + e), "dweight")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,n_in,n_out", [(2000, 40_000, 5008), (2000, 40_001, 5001), (9000, 9000, 9008), (40, 65536, 24)])
def test_long_rows_through_the_whole_epilogue(dtype, rows, n_in, n_out):
    # of one sign, so that S is z itself; the first three so wide that no idle block takes a share
    g = torch.Generator(device="cuda").manual_seed(57)
    x = ((torch.rand(rows, n_in, generator=g, device="cuda") + 1) * 0.5).to(dtype)
    w = ((torch.rand(n_out, n_in, generator=g, device="cuda") + 1) * 2.0 ** -11).to(dtype)
    bias, res = torch.randn(n_out, generator=g, device="cuda"), torch.randn(rows, n_out, generator=g, device="cuda").to(dtype)
    r = ep().ep_linear(x, w, bias, "relu", res, preact=True)
    z = x.double() @ w.double().T
    unit, e = ref.UNIT[dtype], z * (520 if dtype == F16 else 2510) * 2.0 ** -22
    ref.within(r.preact, z + bias, e + unit * (z + bias.abs()) * 1.01, "preact")
    want = (z + bias).clamp(min=0) + res.double()
    ref.within(r.out, want, 1.01 * e + unit * (z + bias.abs() + res.double().abs()) * 1.01, "out")
    off = (r.preact.double() - (z + bias)) / z
    assert abs(float(off.mean())) <= unit / 4


@pytest.mark.parametrize("parts", [8, 130, 1100])
@pytest.mark.parametrize("renormalize", [True, False])
def test_the_gradient_of_a_slot_that_no_part_took_does_not_matter(parts, renormalize):
    g = torch.Generator(device="cuda").manual_seed(55)
    l = torch.randn(60, parts, generator=g, device="cuda")
    l[::3] = -math.inf
    l[::3, 5] = 1.0                                      # one part is open: slots 1 to 3 stay empty
    l[6] = -math.inf                                     # none is
    r = ep().ep_route(l, 4, None, renormalize)
    assert r.ids[0].tolist() == [5, -1, -1, -1] and r.ids[6].tolist() == [-1] * 4
    dw, dl = torch.randn(60, 4, generator=g, device="cuda"), torch.ones(1, device="cuda")
    want = ep().ep_route_backward(l, r, torch.where(r.ids < 0, 0.0, dw), dl, None, renormalize)
    for bad in (math.nan, math.inf, -math.inf):
        assert torch.equal(ep().ep_route_backward(l, r, torch.where(r.ids < 0, bad, dw), dl, None, renormalize), want)
    assert bool(torch.isfinite(want).all())


@pytest.mark.parametrize("parts", [8, 130, 1100])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_that_take_no_part_have_no_gradient_of_a_loss_that_is_not_finite(parts, dtype):
    g = torch.Generator(device="cuda").manual_seed(56)
    l = torch.randn(60, parts, generator=g, device="cuda").to(dtype)
    valid = torch.ones(60, dtype=torch.uint8, device="cuda")
    valid[::3] = 0
    l[7] = -math.inf
    r = ep().ep_route(l, 2, valid)
    for bad in (math.nan, math.inf):
        d = ep().ep_route_backward(l, r, torch.ones(60, 2, device="cuda"), torch.full((1,), bad, device="cuda"), valid)
        assert not bool(d[::3].any()) and not bool(d[7].any()) and not bool(torch.isfinite(d[1]).all())


def test_other_threads_run_while_a_call_waits():
    # PyGILState_Check in the place of a C function answers 1, an error status, where the caller still holds the interpreter's lock
    import ctypes

    from paper_2604_01000_b200 import binding
    m, x = ep(), torch.ones(4, 64, device="cuda")
    w, h = torch.ones(8, 64, device="cuda"), torch.ones(4, 64, device="cuda")
    calls = {"ep_rms_norm": lambda: m.ep_rms_norm(x), "ep_quantize_rows": lambda: m.ep_quantize_rows(x),
             "ep_rms_norm_backward": lambda: m.ep_rms_norm_backward(h, x), "ep_linear": lambda: m.ep_linear(x, w),
             "ep_linear_backward": lambda: m.ep_linear_backward(torch.ones(4, 8, device="cuda"), x, w),
             "ep_route": lambda: m.ep_route(x), "ep_route_backward": lambda: m.ep_route_backward(x, r)}
    r = m.ep_route(x)
    head = binding._load_head()
    lib = binding.load_library()
    real = {n: ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in binding._HEAD_CALLS}
    held = ctypes.cast(ctypes.pythonapi.PyGILState_Check, ctypes.c_void_p).value
    try:
        for name, call in calls.items():
            head.bind(dict(real, **{name: held}), binding._raise_status)
            call()
    finally:
        head.bind(real, binding._raise_status)
    assert torch.equal(m.ep_route(x).ids, r.ids)


def test_two_threads_on_two_streams_of_one_context():
    import threading

    m, ctx = ep(), ep().default_context()
    g = torch.Generator(device="cuda").manual_seed(58)
    sets = []
    for n in (3000, 4001):
        x, w = torch.randn(n, 192, generator=g, device="cuda").to(BF16), torch.randn(96, 192, generator=g, device="cuda").to(BF16)
        sets.append((x, w))

    def passes(x, w):
        n = m.ep_rms_norm(x)
        y = m.ep_linear(n.out, w, None, "gelu", preact=True)
        r = m.ep_route(y.out, 2)
        d = m.ep_linear_backward(m.ep_route_backward(y.out, r, r.weights, r.loss), n.out, w, y.preact, "gelu")
        return [*y, *r, *d, m.ep_rms_norm_backward(d.dx, n.hidden).dx]
    alone = [passes(*s) for s in sets]
    torch.cuda.synchronize()
    before, got, failed = ctx.launch_count(), [None, None], []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(50):
                    got[i] = passes(*sets[i])
                torch.cuda.current_stream().synchronize()
        except Exception as e:   # noqa: BLE001
            failed.append(e)
    ctx.set_profile(True)
    try:
        threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        times = [ctx.profile_read(name) for name in ("norm", "linear", "route")]
        ctx.set_profile(False)
    assert not failed, failed
    for a, b in zip(alone, got):
        for p, q in zip(a, b):
            assert torch.equal(p, q)
    assert [n for _, n in times] == [200, 200, 200] and all(ms > 0 for ms, _ in times)
    single = ctx.launch_count()
    for s in sets:
        passes(*s)
    assert single - before == 50 * (ctx.launch_count() - single)
    ctx.check()


def test_calls_inside_a_cuda_graph():
    m = ep()
    g = torch.Generator(device="cuda").manual_seed(59)
    x, w = torch.randn(3000, 100, generator=g, device="cuda").to(F16), torch.randn(60, 100, generator=g, device="cuda").to(F16)

    def passes():
        n = m.ep_rms_norm(x)
        y = m.ep_linear(n.out, w, None, "silu", preact=True)
        r = m.ep_route(y.out, 2, None, True)
        d = m.ep_linear_backward(m.ep_route_backward(y.out, r, r.weights, r.loss, None, True).float(), n.out, w, y.preact, "silu")
        return [*y, *r, *d, *m.ep_rms_norm_backward(d.dx, n.hidden)]
    passes()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = passes()
    x.copy_(torch.randn(3000, 100, generator=g, device="cuda"))
    graph.replay()
    for a, b in zip(passes(), got):
        assert torch.equal(a, b)


def test_clustering_works_without_the_heads_extension(monkeypatch):
    from paper_2604_01000_b200 import binding
    monkeypatch.setattr(binding, "_head", None)
    monkeypatch.setattr(binding, "_PKG", "/nonexistent")
    ctx = binding.Context(0)
    try:
        x = torch.randn(500, 16, device="cuda")
        assert ctx.kmeans(x, 4, 2, x[:4].contiguous()).assign.shape == (500,)
        with pytest.raises(FileNotFoundError):
            ctx.route(x)
    finally:
        ctx.close()


@pytest.mark.parametrize("d", [40, 64, 2048])
def test_infinities_in_8_bits(d):
    x = torch.randn(5, d, generator=torch.Generator(device="cuda").manual_seed(60), device="cuda")
    x[1, 3], x[3, d - 1] = math.inf, -math.inf
    n, q = ep().ep_rms_norm(x, out_dtype=torch.float8_e4m3fn), ep().ep_quantize_rows(x)
    for row in (1, 3):
        assert bool(torch.isnan(n.out[row].float()).all()) and bool(torch.isnan(n.scale[row]))
        assert bool(torch.isnan(q.q[row].float() * q.scale[row]).all()) and math.isinf(float(q.scale[row]))
    for row in (0, 2, 4):
        assert bool(torch.isfinite(n.out[row].float()).all()) and bool(torch.isfinite(q.q[row].float()).all())


def test_no_gradient_is_recorded():
    x, w = torch.ones(4, 16, device="cuda", requires_grad=True), torch.ones(8, 16, device="cuda", requires_grad=True)
    assert not ep().ep_linear(x, w).out.requires_grad and not ep().ep_rms_norm(x).out.requires_grad
    assert not ep().ep_route(x).weights.requires_grad
