"""ep_linear and ep_linear_backward against 64-bit products.

Bounds.  With S = sum |x| |w| of an output, the tensor core adds 16 products (32 of 8-bit inputs) a step and truncates:
at most 2^-22 S a step (2^-23 of the running sum, and the same again for aligning a step's products), so (n_in / 16 + 4)
2^-22 S where sums run through, 32 2^-22 S where they are kept in runs (fp32 outputs).  Three bf16 parts leave out
products below 2^-22 S together.  The epilogue's fp32 work is within 2^-20 of its terms, and one rounding ends it.
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


def rand(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def summing(k, runs):
    return (32 if runs else k / 16 + 4) * 2.0 ** -22


def check(x, w, bias=None, act="none", residual=None, out_dtype=None, preact=False, x_scale=None, w_scale=None):
    r = ep().ep_linear(x, w, bias, act, residual, x_scale, w_scale, out_dtype, preact)
    out_dtype = out_dtype or (BF16 if x.dtype == E4M3 else x.dtype)
    assert r.out.dtype == out_dtype and (r.preact is None) == (not preact)
    xd, wd = x.double(), w.double()
    if x_scale is not None:
        xd, wd = xd * x_scale.double()[:, None], wd * w_scale.double()[:, None]
    z, S = xd @ wd.T, xd.abs() @ wd.abs().T
    b = torch.zeros(w.shape[0], dtype=torch.float64, device="cuda") if bias is None else bias.double()
    z = z + b
    y, res = ref.act(z, act), 0.0 if residual is None else residual.double()
    work = S * summing(x.shape[1], out_dtype == F32) + 2.0 ** -20 * (z.abs() + b.abs())
    if preact:
        ref.within(r.preact, z, work + ref.UNIT[out_dtype] * (z.abs() + work) + ref.TINY[out_dtype], "preact")
    total = y + res
    work = 1.2 * work + 2.0 ** -20 * (y.abs() + (0.0 if residual is None else res.abs()))
    ref.within(r.out, total, work + ref.UNIT[out_dtype] * (total.abs() + work) + ref.TINY[out_dtype], "out")
    return r


SHAPES = [(1, 64, 64), (1, 1000, 77), (2, 33, 5), (3, 128, 40), (7, 16, 300), (8, 2048, 129), (9, 64, 64), (17, 8, 8), (64, 128, 256),
          (127, 72, 130), (128, 64, 128), (129, 65, 257), (300, 520, 48), (200, 4096, 64), (513, 1, 1), (1000, 256, 1000),
          (2000, 640, 384)]


@pytest.mark.parametrize("rows,n_in,n_out", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_shapes(rows, n_in, n_out, dtype):
    x, w = rand((rows, n_in), dtype, 1), rand((n_out, n_in), dtype, 2, n_in ** -0.5)
    check(x, w)
    check(x, w, rand((n_out,), F32, 3), "gelu", rand((rows, n_out), dtype, 4), None, True)
    if dtype != F32:
        check(x, w, rand((n_out,), dtype, 3), "none", None, F32)


@pytest.mark.parametrize("rows,n_in,n_out", [(1, 256, 100), (4, 48, 64), (9, 128, 64), (130, 100, 257), (300, 1024, 512)])
@pytest.mark.parametrize("out", [BF16, F16, F32])
def test_eight_bits(rows, n_in, n_out, out):
    m = ep()
    xq, xs = m.ep_quantize_rows(rand((rows, n_in), F32, 5))
    wq, ws = m.ep_quantize_rows(rand((n_out, n_in), F32, 6, n_in ** -0.5))
    check(xq, wq, rand((n_out,), F32, 7), "silu", rand((rows, n_out), out, 8), out, True, xs, ws)
    check(xq, wq, None, "none", None, out, False, xs, ws)


def test_norm_in_8_bits_feeds_the_product():
    m = ep()
    x, g = rand((200, 192), F32, 9), rand((192,), F32, 10) * 0.1 + 1
    n = m.ep_rms_norm(x, g, None, 1e-6, E4M3)
    wq, ws = m.ep_quantize_rows(rand((96, 192), BF16, 11))
    check(n.out, wq, None, "none", None, BF16, False, n.scale, ws)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("rows", [5, 200])
def test_activations_over_their_range(act, rows):
    # one input column of 1: z is the weight, from -30 to 30 and the special points
    z = torch.cat([torch.linspace(-30, 30, 101), torch.tensor([0.0, -0.0, 1e-6, -1e-6, 88.0, -88.0, 200.0, -200.0])]).cuda()
    x, w = torch.ones(rows, 1, device="cuda"), z[:, None].contiguous()
    check(x, w, None, act, None, F32, True)


def test_strided_rows_and_misaligned_buffers():
    for dtype in (BF16, F32, F16):
        for rows in (4, 150):
            big, wide, res = rand((rows, 200), dtype, 12), rand((70, 160), dtype, 13, 0.1), rand((rows, 96), dtype, 14)
            check(big[:, 8:136], wide[:, 16:144], None, "relu", res[:, 16:86], preact=True)
            check(big[:, 3:80], wide[:, 5:82], None, "relu", res[:, 1:71])
            check(ref.misaligned(big), ref.misaligned(rand((66, 200), dtype, 15, 0.1)), None, "none",
                  ref.misaligned(rand((rows, 66), dtype, 16)))
            check(big[::2], rand((64, 200), dtype, 17, 0.1))


def test_bias_types():
    x, w = rand((40, 64), BF16, 18), rand((48, 64), BF16, 19, 0.1)
    for t in (F32, BF16, F16):
        check(x, w, rand((48,), t, 20))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_long_sums_of_one_sign(dtype):
    # truncation always loses: sums of positive terms show it most
    x, w = rand((130, 16384), dtype, 21).abs(), rand((64, 16384), dtype, 22, 0.01).abs()
    check(x, w, out_dtype=F32)
    check(x, w)


def backward(x, w, dout, z, act, **kw):
    r = ep().ep_linear_backward(dout, x, w, z, act, **kw)
    dz = dout.double() * (1.0 if act == "none" else ref.slope(z.double(), act))
    dt = x.dtype
    xd, wd = x.double(), w.double()
    # dz: two exponentials' worth of fp32 work (2^-18), then one rounding to the operands' type
    u = 2.0 ** -18 + (ref.UNIT[dt] if dt != F32 else 2.0 ** -22)
    size = dout.double().abs() if act == "none" else dout.double().abs() * (1.2 + 0 * dz)
    size = torch.maximum(size * 2.0 ** -8, dz.abs())   # where the slope cancels, its terms still count
    if r.dx is not None:
        want, S = dz @ wd, size @ wd.abs()
        e = S * (u + summing(w.shape[0], dt == F32))
        ref.within(r.dx, want, e + ref.UNIT[dt] * (want.abs() + e) + (w.shape[0] + 1) * ref.TINY[dt] * float(wd.abs().max() + 1), "dx")
    if r.dweight is not None:
        want, S = dz.T @ xd, size.T @ xd.abs()
        e = S * (u + summing(x.shape[0], dt == F32))
        ref.within(r.dweight, want, e + ref.UNIT[dt] * (want.abs() + e) + (x.shape[0] + 1) * ref.TINY[dt] * float(xd.abs().max() + 1),
                   "dweight")
    if r.dbias is not None:
        ref.within(r.dbias, dz.sum(0), size.sum(0) * (2.0 ** -18 + (64 + x.shape[0] / 64) * 2.0 ** -23), "dbias")
    return r


@pytest.mark.parametrize("rows,n_in,n_out", [(1, 64, 64), (5, 33, 17), (130, 64, 128), (257, 100, 72), (300, 65, 257), (1000, 256, 64),
                                             (3001, 40, 300), (700, 512, 520)])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_backward(rows, n_in, n_out, dtype):
    x, w = rand((rows, n_in), dtype, 23), rand((n_out, n_in), dtype, 24, n_in ** -0.5)
    dout, z = rand((rows, n_out), dtype, 25), rand((rows, n_out), dtype, 26)
    backward(x, w, dout, z, "gelu")
    backward(x, w, dout, None, "none")
    if dtype != F32:
        backward(x, w, dout.float(), z, "silu")
        backward(x, w, dout.float(), None, "none")


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_slopes_over_their_range(act):
    z = torch.cat([torch.linspace(-30, 30, 100), torch.tensor([0.0, -0.0, 88.0, -88.0])]).cuda().repeat(20, 1)
    x, w = torch.ones(20, 8, device="cuda"), torch.ones(104, 8, device="cuda")
    r = ep().ep_linear_backward(torch.ones_like(z), x, w, z, act)
    want = ref.slope(z.double(), act).sum(0)
    ref.within(r.dbias, want, want.abs() * 2.0 ** -18 + 20 * 2.0 ** -20, "dbias")


def test_backward_strided_misaligned_and_partial():
    for dtype in (BF16, F32):
        big, wide = rand((333, 150), dtype, 27), rand((50, 150), dtype, 28, 0.1)
        dout, z = ref.misaligned(rand((333, 50), dtype, 29)), ref.misaligned(rand((333, 50), dtype, 30))
        backward(big[:, 8:72], wide[:, 16:80], dout, z, "relu")
        full = backward(big[:, 3:70], wide[:, 1:68], dout, z, "silu")
        x, w = big[:, 3:70], wide[:, 1:68]
        only = ep().ep_linear_backward(dout, x, w, z, "silu", need_dweight=False, need_dbias=False)
        assert only.dweight is None and only.dbias is None and torch.equal(only.dx, full.dx)
        only = ep().ep_linear_backward(dout, x, w, z, "silu", need_dx=False, need_dbias=False)
        assert only.dx is None and torch.equal(only.dweight, full.dweight)
        only = ep().ep_linear_backward(dout, x, w, z, "silu", need_dx=False, need_dweight=False)
        assert torch.equal(only.dbias, full.dbias)


def test_gradient_against_differences():
    # f = sum(out G): its third derivative along v is below 10 |G| |v|^3 here; steps of 2^-6 and fp32 noise stay within
    # 2e-3 of |gradient| |v|
    rows, n_in, n_out = 24, 40, 56
    x, w, b = rand((rows, n_in), F32, 31), rand((n_out, n_in), F32, 32, 0.15), rand((n_out,), F32, 33)
    G, t = rand((rows, n_out), F32, 34), 2.0 ** -6
    for act in ("none", "gelu", "silu"):
        f = lambda a, c, d: float((ep().ep_linear(a, c, d, act).out.double() * G.double()).sum())   # noqa: E731
        z = ep().ep_linear(x, w, b, act, preact=True).preact
        r = ep().ep_linear_backward(G, x, w, z, act)
        vx, vw, vb = rand(x.shape, F32, 35, 0.5), rand(w.shape, F32, 36, 0.1), rand(b.shape, F32, 37)
        for got, v, diff in ((r.dx, vx, f(x + t * vx, w, b) - f(x - t * vx, w, b)),
                             (r.dweight, vw, f(x, w + t * vw, b) - f(x, w - t * vw, b)),
                             (r.dbias, vb, f(x, w, b + t * vb) - f(x, w, b - t * vb))):
            slope = float((got.double() * v.double()).sum())
            assert abs(slope - diff / (2 * t)) <= 2e-3 * float(got.norm()) * float(v.norm())


def test_same_from_run_to_run_and_on_another_stream():
    x, w = rand((4000, 320), BF16, 38), rand((200, 320), BF16, 39, 0.1)
    dout, z = rand((4000, 200), BF16, 40), rand((4000, 200), BF16, 41)
    a, b = ep().ep_linear(x, w, None, "gelu"), ep().ep_linear_backward(dout, x, w, z, "gelu")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c, d = ep().ep_linear(x, w, None, "gelu"), ep().ep_linear_backward(dout, x, w, z, "gelu")
    s.synchronize()
    assert torch.equal(a.out, c.out)
    for p, q in zip(b, d):
        assert torch.equal(p, q)


@pytest.mark.parametrize("rows", [3, 40])
def test_not_finite_values_stay_in_their_rows(rows):
    for dtype in (BF16, F32):
        x, w = rand((rows, 96), dtype, 42), rand((64, 96), dtype, 43, 0.1)
        clean = ep().ep_linear(x, w).out
        x[1, 5], x[2, 7] = math.nan, math.inf
        out = ep().ep_linear(x, w).out
        keep = [r for r in range(rows) if r not in (1, 2)]
        assert torch.equal(out[keep], clean[keep])
        assert bool(torch.isnan(out[1]).all()) and not bool(torch.isfinite(out[2]).any())


def test_no_rows():
    x, w = torch.empty(0, 64, device="cuda", dtype=BF16), rand((32, 64), BF16, 44)
    r = ep().ep_linear(x, w, preact=True)
    assert r.out.shape == (0, 32) and r.preact.shape == (0, 32)
    d = ep().ep_linear_backward(r.out, x, w, r.preact, "gelu")
    assert d.dx.shape == (0, 64) and not bool(d.dweight.any()) and not bool(d.dbias.any())


def test_offsets_past_32_bits():
    rows, n = (1 << 31) // 512 + 100, 512
    x, w = torch.zeros(rows, 16, device="cuda", dtype=BF16), rand((n, 16), BF16, 45)
    x[-50:] = rand((50, 16), BF16, 46)
    out = ep().ep_linear(x, w).out
    assert torch.equal(out[-50:], ep().ep_linear(x[-50:].contiguous(), w).out) and not bool(out[:50].any())
    r = ep().ep_linear_backward(out, x, w)
    tail = out[-50:].double()
    want = tail.T @ x[-50:].double()
    ref.within(r.dweight, want, (tail.abs().T @ x[-50:].double().abs()) * 2.0 ** -18 + want.abs() * 2.0 ** -8, "dweight")
    want = tail @ w.double()
    ref.within(r.dx[-50:], want, (tail.abs() @ w.double().abs()) * 2.0 ** -16 + want.abs() * 2.0 ** -8, "dx")


def test_refusals():
    m = ep()
    x, w = rand((20, 64), BF16, 47), rand((32, 64), BF16, 48)
    q, s = m.ep_quantize_rows(x)
    wq, ws = m.ep_quantize_rows(w)
    out = torch.zeros(20, 32, device="cuda", dtype=BF16)
    for bad in (lambda: m.ep_linear(x.cpu(), w), lambda: m.ep_linear(x.double(), w.double()), lambda: m.ep_linear(x, w.half()),
                lambda: m.ep_linear(x, w[:, :32]), lambda: m.ep_linear(x.T, w), lambda: m.ep_linear(x[:1].expand(20, 64), w),
                lambda: m.ep_linear(x, w, out[0, :5]), lambda: m.ep_linear(x, w, None, "tanh"),
                lambda: m.ep_linear(x, w, None, "none", out.float()), lambda: m.ep_linear(x, w, None, "none", out[:5]),
                lambda: m.ep_linear(x, w, None, "none", None, None, None, F16), lambda: m.ep_linear(q, wq),
                lambda: m.ep_linear(x, w, x_scale=s, weight_scale=ws), lambda: m.ep_linear(q, wq, x_scale=s),
                lambda: m.ep_linear(q, wq, None, "none", None, s, ws, E4M3),
                lambda: m.ep_linear_backward(out, x, w, None, "gelu"), lambda: m.ep_linear_backward(out.half(), x, w),
                lambda: m.ep_linear_backward(out[:, :16], x, w), lambda: m.ep_linear_backward(out, x, w, out[:4], "relu"),
                lambda: m.ep_linear_backward(out, q, wq)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(m.EmbedPartError):
        m.ep_linear(torch.zeros(2, 65537, device="cuda"), torch.zeros(2, 65537, device="cuda"))
    with pytest.raises(m.EmbedPartError):
        m.ep_linear(torch.zeros(2, 0, device="cuda"), torch.zeros(2, 0, device="cuda"))
    ctx = m.default_context()
    lib, p = ctx._lib, x.data_ptr()
    assert lib.ep_linear(None, p, 64, p, 64, 1, None, None, None, 0, 0, None, 0, p, 1, None, 1, 8, 8, p, 256, None) == 1
    assert lib.ep_linear(ctx._h, p, 64, p, 64, 1, None, None, None, 0, 9, None, 0, p, 1, None, 1, 8, 8, p, 256, None) == 1
    assert lib.ep_linear(ctx._h, p, 7, p, 64, 1, None, None, None, 0, 0, None, 0, p, 1, None, 1, 8, 8, p, 256, None) == 1
    assert lib.ep_linear(ctx._h, p + 1, 64, p, 64, 1, None, None, None, 0, 0, None, 0, p, 1, None, 1, 8, 8, p, 256, None) == 1
    assert lib.ep_linear(ctx._h, p, 64, p, 64, 1, None, None, None, 0, 0, None, 0, p, 1, None, 1, 8, 8, None, 0, None) == 3
    assert lib.ep_linear(ctx._h, None, 64, p, 64, 1, None, None, None, 0, 0, None, 0, p, 1, None, 1, 8, 8, p, 256, None) == 1
    assert lib.ep_linear_workspace_bytes(ctx._h, 10, 0, 8, 1, 1, 1) == 0 and lib.ep_linear_workspace_bytes(ctx._h, 10, 8, 8, 1, 2, 1) == 0
    ctx.check()
