"""ep_rms_norm, ep_quantize_rows and ep_rms_norm_backward against the 64-bit formulas.

Bounds.  With u the rounding unit of the output's type, an output is off by u of itself (one rounding) plus the fp32
work: a sum of d terms kept by at least 8 threads of at most 64 terms in a row each and a tree of at most 9 steps, a
reciprocal square root and a few products, each within 2^-23 relative: (d / 8 limited to 64, + 32) 2^-23 in all.
"""
import math

import pytest
import torch

import head_reference as ref

pytestmark = pytest.mark.gpu

F32, BF16, F16, E4M3 = torch.float32, torch.bfloat16, torch.float16, torch.float8_e4m3fn


def ep():
    import paper_2604_01000_b200 as m
    return m


def fp32_work(d):
    return (min(d / 8, 64) + 32) * 2.0 ** -23


def make(rows, d, dtype, seed=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(rows, d, generator=g, device="cuda") * scale).to(dtype)


def check(x, weight, residual, eps, out_dtype, want_rows=None):
    r = ep().ep_rms_norm(x, weight, residual, eps, out_dtype)
    h, rho, y = ref.norm(x, weight, residual, eps)
    d = x.shape[1]
    lost = 0 if residual is None else ref.FP32 * (x.double().abs() + residual.double().abs()) * rho
    if weight is not None and residual is not None:
        lost = lost * weight.double().abs()
    work = y.abs() * fp32_work(d) + lost
    if residual is not None:
        ref.within(r.hidden, h, ref.UNIT[x.dtype] * h.abs() * 1.001 + ref.FP32 * (x.double().abs() + residual.double().abs())
                   + ref.TINY[x.dtype], "hidden")
    else:
        assert r.hidden is x
    if out_dtype == E4M3:
        top = y.abs().amax(1)
        ref.within(r.scale, top / 448, top / 448 * fp32_work(d) * 2 + lost_top(lost) / 448 + 2.0 ** -149, "scale")
        s = r.scale.double()[:, None]
        step = torch.maximum((y.abs() + work) * ref.UNIT[E4M3], s * 2.0 ** -10)
        ref.within(r.out.double() * s, y, step * (1 + 2.0 ** -10) + 2 * work, "out")
    else:
        assert r.scale is None and r.out.dtype == out_dtype
        ref.within(r.out, y, (y.abs() + work) * ref.UNIT[out_dtype] + work + ref.TINY[out_dtype], "out")
    return r


def lost_top(lost):
    return 0 if isinstance(lost, int) else lost.amax(1)


@pytest.mark.parametrize("d", [1, 3, 8, 31, 32, 64, 100, 128, 129, 255, 256, 512, 1000, 1024, 2048, 4099, 8192, 16384])
@pytest.mark.parametrize("dtype,out", [(F32, F32), (F32, BF16), (F32, F16), (F32, E4M3), (BF16, BF16), (BF16, E4M3), (F16, F16),
                                       (F16, E4M3)])
def test_forward(d, dtype, out):
    rows = 37 if d <= 1024 else 5
    g = make(1, d, F32, 1)[0] * 0.2 + 1
    check(make(rows, d, dtype, 2), g, make(rows, d, dtype, 3), 1e-6, out)
    check(make(rows, d, dtype, 4), None, None, 1e-6, out)


@pytest.mark.parametrize("rows", [1, 2, 31, 33, 4097, 20011])
@pytest.mark.parametrize("d", [64, 200, 1056])
def test_row_counts(rows, d):
    check(make(rows, d, BF16, 5), make(1, d, BF16, 6)[0], make(rows, d, BF16, 7), 1e-5, BF16)


def test_misaligned_buffers_and_parameter_types():
    for dtype in (F32, BF16, F16):
        x, r = ref.misaligned(make(9, 96, dtype, 8)), ref.misaligned(make(9, 96, dtype, 9))
        for wt in (F32, dtype):
            check(x, make(1, 97, wt, 10)[0][1:], r, 1e-6, dtype)


def test_rows_of_zeros_and_extremes():
    x = torch.zeros(4, 160, device="cuda")
    x[1] = 1e-30
    x[2, 7] = 1e18
    for out in (F32, E4M3):
        r = ep().ep_rms_norm(x, None, None, 1e-6, out)
        assert bool((r.out[0].float() == 0).all())
        value = r.out.float() if out == F32 else r.out.float() * r.scale[:, None]
        assert bool(torch.isfinite(value).all())
        want = ref.norm(x, None, None, 1e-6)[2]
        assert abs(float(value[2, 7]) - float(want[2, 7])) <= 1e-5 * float(want[2, 7])
    assert float(ep().ep_rms_norm(x, None, None, 0.0, E4M3).scale[1]) == pytest.approx(1 / 448, rel=1e-5)
    bad = torch.ones(3, 40, device="cuda")
    bad[1, 3] = math.nan
    r = ep().ep_rms_norm(bad, None, None, 1e-6, E4M3)
    assert bool(torch.isnan(r.scale[1])) and bool(torch.isfinite(r.scale[[0, 2]]).all())
    assert bool(torch.isnan(r.out.float()[1]).all()) and bool(torch.isfinite(r.out.float()[[0, 2]]).all())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("d", [1, 17, 64, 300, 2000])
def test_quantize_rows(dtype, d):
    x = make(23, d, dtype, 11, 3.0)
    x[4] = 0
    q, scale = ep().ep_quantize_rows(x)
    xd = x.double()
    top = xd.abs().amax(1)
    ref.within(scale, top / 448, top * 2.0 ** -22 / 448 + 2.0 ** -149, "scale")
    s = scale.double()[:, None]
    ref.within(q.double() * s, xd, torch.maximum(xd.abs() * ref.UNIT[E4M3], s * 2.0 ** -10) * (1 + 2.0 ** -10) + xd.abs() * 2.0 ** -21, "q")
    assert float(q.float().abs().max()) == 448.0


@pytest.mark.parametrize("d", [1, 8, 33, 64, 128, 200, 256, 500, 1024, 1500, 4096, 8192, 16384])
@pytest.mark.parametrize("dtype,grad", [(F32, F32), (F32, BF16), (F32, F16), (BF16, BF16), (F16, F16)])
def test_backward(d, dtype, grad):
    rows = 301 if d <= 1024 else 7
    g = make(1, d, F32, 12)[0] * 0.2 + 1
    h, dy, dh = make(rows, d, dtype, 13), make(rows, d, grad, 14), make(rows, d, dtype, 15)
    for weight, extra in ((g, dh), (None, None)):
        r = ep().ep_rms_norm_backward(dy, h, weight, 1e-6, extra)
        dx, size, dg, dg_size = ref.norm_backward(dy, h, weight, 1e-6, extra)
        ref.within(r.dx, dx, ref.UNIT[dtype] * dx.abs() * 1.01 + size * 2 * fp32_work(d) + ref.TINY[dtype], "dx")
        # sums over rows: at most 64 rows in a row per thread here, then trees
        ref.within(r.dweight, dg, dg_size * (64 + fp32_work(d) / 2.0 ** -23) * 2.0 ** -23, "dweight")


def test_backward_many_rows_misaligned_and_without_dweight():
    h, dy = ref.misaligned(make(5003, 66, BF16, 16)), ref.misaligned(make(5003, 66, BF16, 17))
    r = ep().ep_rms_norm_backward(dy, h, None, 1e-6, None)
    dx, size, dg, dg_size = ref.norm_backward(dy, h, None, 1e-6, None)
    ref.within(r.dx, dx, ref.UNIT[BF16] * dx.abs() * 1.01 + size * 2 * fp32_work(66), "dx")
    ref.within(r.dweight, dg, dg_size * 200 * 2.0 ** -23, "dweight")
    alone = ep().ep_rms_norm_backward(dy, h, None, 1e-6, None, need_dweight=False)
    assert alone.dweight is None and torch.equal(alone.dx, r.dx)


def test_gradient_against_differences():
    # f = sum(out * G); along v the difference quotient of step 2^-6 is off by its square times the third derivative
    # (order one here) and by fp32 noise of f over the step: 1e-3 of |gradient| |v| covers both
    x, G, v = make(12, 96, F32, 18), make(12, 96, F32, 19), make(12, 96, F32, 20)
    w, vw = make(1, 96, F32, 21)[0] * 0.2 + 1, make(1, 96, F32, 22)[0]
    f = lambda a, b: float((ep().ep_rms_norm(a, b, None, 1e-6).out.double() * G.double()).sum())   # noqa: E731
    r = ep().ep_rms_norm_backward(G, x, w, 1e-6)
    t = 2.0 ** -6
    for got, vec, diff in ((r.dx, v, (f(x + t * v, w) - f(x - t * v, w)) / (2 * t)),
                           (r.dweight, vw, (f(x, w + t * vw) - f(x, w - t * vw)) / (2 * t))):
        slope = float((got.double() * vec.double()).sum())
        assert abs(slope - diff) <= 1e-3 * float(got.norm()) * float(vec.norm())


def test_same_from_run_to_run_and_on_another_stream():
    h, dy, g = make(3001, 128, BF16, 23), make(3001, 128, BF16, 24), make(1, 128, F32, 25)[0]
    a, b = ep().ep_rms_norm(h, g, dy, 1e-6), ep().ep_rms_norm_backward(dy, h, g)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c, e = ep().ep_rms_norm(h, g, dy, 1e-6), ep().ep_rms_norm_backward(dy, h, g)
    s.synchronize()
    assert torch.equal(a.out, c.out) and torch.equal(b.dx, e.dx) and torch.equal(b.dweight, e.dweight)


def test_no_rows():
    x = torch.empty(0, 64, device="cuda", dtype=BF16)
    assert ep().ep_rms_norm(x, None, x, 1e-6, E4M3).out.shape == (0, 64)
    r = ep().ep_rms_norm_backward(x, x)
    assert r.dx.shape == (0, 64) and bool((r.dweight == 0).all())
    assert ep().ep_quantize_rows(x).q.shape == (0, 64)


def test_offsets_past_32_bits():
    rows, d = (1 << 31) // 128 + 1000, 128
    x = torch.zeros(rows, d, device="cuda", dtype=BF16)
    x[-500:] = make(500, d, BF16, 26)
    r = ep().ep_rms_norm(x, None, None, 1e-6)
    ref.within(r.out[-500:], ref.norm(x[-500:], None, None, 1e-6)[2], ref.norm(x[-500:], None, None, 1e-6)[2].abs() * 2.0 ** -8, "out")
    del r
    dx = ep().ep_rms_norm_backward(x, x, None, 1e-6, None).dx
    want, size, _, _ = ref.norm_backward(x[-500:], x[-500:], None, 1e-6, None)
    ref.within(dx[-500:], want, ref.UNIT[BF16] * want.abs() * 1.01 + size * 2 * fp32_work(d), "dx")


def test_refusals():
    m = ep()
    x = make(4, 64, F32, 27)
    for bad in (lambda: m.ep_rms_norm(x.cpu()), lambda: m.ep_rms_norm(x.double()), lambda: m.ep_rms_norm(x[0]),
                lambda: m.ep_rms_norm(x[:, ::2]), lambda: m.ep_rms_norm(x, x[0, :5]), lambda: m.ep_rms_norm(x, x),
                lambda: m.ep_rms_norm(x, None, x[:2]), lambda: m.ep_rms_norm(x, None, x.to(BF16)),
                lambda: m.ep_rms_norm(x.to(BF16), None, None, 1e-6, F16), lambda: m.ep_rms_norm(x.to(BF16), None, None, 1e-6, F32),
                lambda: m.ep_rms_norm_backward(x.to(F16), x.to(BF16)), lambda: m.ep_rms_norm_backward(x[:2], x),
                lambda: m.ep_rms_norm_backward(x, x, None, 1e-6, x.to(BF16)), lambda: m.ep_quantize_rows(x.to(E4M3))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: m.ep_rms_norm(x, None, None, -1.0), lambda: m.ep_rms_norm(x, None, None, math.nan),
                lambda: m.ep_rms_norm(x, None, None, math.inf), lambda: m.ep_rms_norm(torch.zeros(1, 16385, device="cuda")),
                lambda: m.ep_rms_norm(torch.zeros(3, 0, device="cuda")),
                lambda: m.ep_rms_norm_backward(torch.zeros(1, 16385, device="cuda"), torch.zeros(1, 16385, device="cuda"))):
        with pytest.raises(m.EmbedPartError):
            bad()
    ctx = m.default_context()
    assert ctx._lib.ep_rms_norm(None, None, 0, None, None, 0, 1, 8, 1e-6, None, 0, None, None, None) == 1
    assert ctx._lib.ep_rms_norm(ctx._h, None, 0, None, None, 0, 1, 8, 1e-6, None, 0, None, None, None) == 1
    assert ctx._lib.ep_rms_norm_backward_workspace_bytes(ctx._h, 4, 0) == 0
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    assert ctx._lib.ep_rms_norm_backward(ctx._h, x.data_ptr(), 0, x.data_ptr(), 0, None, 0, None, 4, 64, 1e-6, x.data_ptr(),
                                         x.data_ptr(), ws.data_ptr(), 256, None) == 3
    ctx.check()
