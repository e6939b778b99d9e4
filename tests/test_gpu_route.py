"""ep_route and ep_route_backward against the 64-bit definitions; ids, counts and routed are exact.

Bounds.  p = exp(l - top) / sum: the exponential's argument is rounded (2^-24 |l - top|, times one for the product with
log2 e) and the function itself is within 2^-21; the sum adds at most 32 terms in a row per thread and a tree.  So p is
within (|l - top| + 64) 2^-22 of itself, renormalised weights within three times that, and sums over rows, kept in fp32
per thread over at most 64 rows in these tests, within 64 2^-24 more.
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


def make(rows, parts, dtype, seed, scale=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(rows, parts, generator=g, device="cuda") * scale).to(dtype)


def spread(logits):
    l = logits.double()
    l = l[torch.isfinite(l)]
    return float(l.max() - l.min()) if l.numel() else 0.0


def check(logits, k, valid, renormalize, seed=0):
    rows, parts = logits.shape
    r = ep().ep_route(logits, k, valid, renormalize)
    ids, w, counts, prob, loss, routed, p = ref.route(logits, k, valid, renormalize)
    assert torch.equal(r.ids.cpu(), ids)
    assert torch.equal(r.counts.cpu(), counts) and int(r.routed) == routed
    rel = (spread(logits) + 64) * 2.0 ** -22
    ref.within(r.weights, w, w * (3 * rel if renormalize else rel) + 2.0 ** -126, "weights")
    ref.within(r.prob, prob, prob * (rel + 64 * ref.FP32) + 2.0 ** -126, "prob")
    assert abs(float(r.loss) - loss) <= loss * (rel + 64 * ref.FP32)

    g = torch.Generator(device="cuda").manual_seed(seed + 1000)
    dw = torch.randn(rows, k, generator=g, device="cuda")
    dl = torch.full((1,), 0.7, device="cuda")
    for a, b in ((dw, dl), (None, dl), (dw, None)):
        got = ep().ep_route_backward(logits, r, a, b, valid, renormalize)
        want, size = ref.route_backward(p, ids, counts, routed, k, renormalize, None if a is None else a.cpu(),
                                        0.0 if b is None else float(dl))
        ref.within(got, want, ref.UNIT[logits.dtype] * want.abs() * 1.01 + size * 8 * rel + ref.TINY[logits.dtype] + 2.0 ** -126,
                   "dlogits")
        assert got.dtype == logits.dtype
    ep().default_context().check()
    return r


@pytest.mark.parametrize("parts", [1, 2, 3, 4, 7, 8, 16, 31, 32, 33, 64, 100, 128, 257, 512, 777, 1024, 1025, 2048, 4095, 4096])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_shapes_and_types(parts, dtype):
    rows = 67 if parts <= 256 else 9
    for k in sorted({1, min(2, parts), min(8, parts)}):
        check(make(rows, parts, dtype, parts + k), k, None, k > 1, k)
        check(make(rows, parts, dtype, parts + k + 1), k, None, False, k)


@pytest.mark.parametrize("k", [5, 31, 32])
def test_many_slots(k):
    for parts in (32, 40, 1500):
        check(make(11, parts, F32, k + parts), k, None, True)
        check(make(11, parts, BF16, k + parts), k, None, False)


@pytest.mark.parametrize("rows", [1, 2, 63, 2500])
def test_row_counts(rows):
    check(make(rows, 12, F32, rows), 2, None, True)


def test_ties_go_to_the_lower_part():
    l = torch.zeros(5, 300, device="cuda")
    l[1, 100:200] = 1.0
    l[2] = -0.0
    l[2, 7] = 0.0
    l[3] = torch.finfo(F32).min
    for dtype in (F32, BF16, F16):
        lt = l.clone()
        lt[3] = torch.finfo(dtype).min
        r = check(lt.to(dtype), 4, None, True)
        assert r.ids[0].tolist() == [0, 1, 2, 3] and r.ids[1].tolist() == [100, 101, 102, 103]
        assert r.ids[2].tolist() == [0, 1, 2, 3] and r.ids[3].tolist() == [0, 1, 2, 3]
        assert float(r.weights[3].min()) == pytest.approx(0.25, rel=1e-6)


@pytest.mark.parametrize("parts", [6, 64, 130, 1100])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_closed_parts_and_rows_that_take_no_part(parts, dtype):
    l = make(90, parts, dtype, parts)
    g = torch.Generator(device="cuda").manual_seed(3)
    l[torch.rand(90, parts, generator=g, device="cuda") < 0.5] = -math.inf
    l[7] = -math.inf                        # nothing is open
    l[8] = -math.inf
    l[8, parts - 1] = -5.0                  # one part is
    l[9, :] = torch.finfo(dtype).min        # masked with the type's lowest value instead
    l[9, 2] = 1.0
    valid = (torch.rand(90, generator=g, device="cuda") > 0.2)
    valid[7:10] = True
    for v in (None, valid, valid.to(torch.uint8)):
        for renormalize in (True, False):
            r = check(l, 3, v, renormalize)
            assert r.ids[7].tolist() == [-1, -1, -1] and r.ids[8].tolist() == [parts - 1, -1, -1]
            assert float(r.weights[8, 0]) == 1.0


def test_no_row_takes_part():
    l = make(40, 16, F32, 1)
    valid = torch.zeros(40, dtype=torch.uint8, device="cuda")
    for logits, v in ((l, valid), (torch.full_like(l, -math.inf), None)):
        r = check(logits, 2, v, True)
        assert int(r.routed) == 0 and float(r.loss) == 0 and not bool(r.prob.any()) and not bool(r.counts.any())


def test_what_masked_rows_hold_does_not_matter():
    l = make(600, 40, BF16, 2)
    valid = torch.ones(600, dtype=torch.uint8, device="cuda")
    valid[::3] = 0
    dw = torch.randn(600, 2, device="cuda")
    dl = torch.ones(1, device="cuda")
    a = ep().ep_route(l, 2, valid, True)
    ga = ep().ep_route_backward(l, a, dw, dl, valid, True)
    poisoned = l.clone()
    poisoned[::3] = math.nan
    poisoned[3] = math.inf
    b = ep().ep_route(poisoned, 2, valid, True)
    gb = ep().ep_route_backward(poisoned, b, dw, dl, valid, True)
    for x, y in zip(a, b):
        assert torch.equal(x, y)
    assert torch.equal(ga, gb) and not bool(ga[::3].any())


def test_nan_and_infinity_in_a_row_that_takes_part():
    l = make(6, 40, F32, 4)
    l[1, 5] = math.nan
    l[2, 6] = math.inf
    r = ep().ep_route(l, 2)
    clean = ep().ep_route(make(6, 40, F32, 4), 2)
    assert 5 not in r.ids[1].tolist() and int(r.ids[2, 0]) == 6
    for row in (0, 3, 4, 5):
        assert torch.equal(r.ids[row], clean.ids[row]) and torch.equal(r.weights[row], clean.weights[row])
    assert bool(torch.isnan(r.weights[1:3]).all()) and bool(torch.isnan(r.loss)) and int(r.routed) == 6


def test_misaligned_logits():
    check(ref.misaligned(make(30, 64, BF16, 5)), 2, None, True)
    check(ref.misaligned(make(30, 64, F32, 6)), 1, None, False)


def test_large_logits_do_not_overflow():
    check(make(50, 33, F32, 7, 100.0), 2, None, True)
    check(make(50, 33, F32, 8, 1.0) + 1e4, 2, None, False)


def test_gradient_against_differences():
    # parts 0.4 apart in every row, so that a step of 2^-7 leaves the choice alone; the quotient is off by the step's
    # square times the third derivative (below 10 here) and fp32 noise over the step: 2e-3 of |gradient| |v|
    g = torch.Generator(device="cuda").manual_seed(9)
    rows, parts, k = 20, 10, 3
    order = torch.rand(rows, parts, generator=g, device="cuda").argsort(1)
    l = order.float() * 0.4 - 2
    G, v = torch.randn(rows, k, generator=g, device="cuda"), torch.randn(rows, parts, generator=g, device="cuda")
    for renormalize in (False, True):
        def f(x):
            r = ep().ep_route(x, k, None, renormalize)
            return float((r.weights.double() * G.double()).sum()) + 30.0 * float(r.loss.double())
        r = ep().ep_route(l, k, None, renormalize)
        grad = ep().ep_route_backward(l, r, G, torch.full((1,), 30.0, device="cuda"), None, renormalize)
        t = 2.0 ** -7
        diff = (f(l + t * v) - f(l - t * v)) / (2 * t)
        assert abs(float((grad.double() * v.double()).sum()) - diff) <= 2e-3 * float(grad.norm()) * float(v.norm())


@pytest.mark.parametrize("parts", [1, 5, 40, 700, 2000])
def test_a_single_renormalised_weight_is_one_and_has_no_gradient(parts):
    for dtype in (F32, BF16):
        l = make(50, parts, dtype, 15)
        r = ep().ep_route(l, 1, None, True)
        assert bool((r.weights == 1).all())
        dw = torch.randn(50, 1, device="cuda")
        assert not bool(ep().ep_route_backward(l, r, dw, None, None, True).any())


def test_balance_loss_of_even_and_of_one_sided_routing():
    even = torch.full((64, 8), -4.0, device="cuda")
    even[torch.arange(64), torch.arange(64) % 8] = 4.0
    assert float(ep().ep_route(even, 1).loss) == pytest.approx(1.0, rel=1e-5)
    one = torch.full((64, 8), -40.0, device="cuda")
    one[:, 3] = 40.0
    assert float(ep().ep_route(one, 1).loss) == pytest.approx(8.0, rel=1e-5)


def test_same_from_run_to_run_and_on_another_stream():
    l = make(30011, 64, BF16, 10)
    a = ep().ep_route(l, 2, None, True)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b = ep().ep_route(l, 2, None, True)
    s.synchronize()
    for x, y in zip(a, b):
        assert torch.equal(x, y)
    assert int(a.counts.sum()) == 60022


def test_routed_ids_are_an_assignment():
    l = make(5000, 7, F32, 11)
    r = ep().ep_route(l, 1)
    perm = ep().ep_reorder(r.ids.view(-1), 7).perm
    sizes = torch.bincount(r.ids.view(-1).long(), minlength=7)
    assert torch.equal(sizes, r.counts) and bool((r.ids.view(-1)[perm.long()].diff() >= 0).all())


def test_no_rows():
    l = torch.empty(0, 9, device="cuda")
    r = ep().ep_route(l, 2)
    assert r.ids.shape == (0, 2) and int(r.routed) == 0 and not bool(r.counts.any()) and float(r.loss) == 0
    assert ep().ep_route_backward(l, r, torch.empty(0, 2, device="cuda"), torch.ones(1, device="cuda")).shape == (0, 9)


def test_offsets_past_32_bits():
    rows, parts = (1 << 31) // 64 + 300, 64
    l = torch.zeros(rows, parts, device="cuda", dtype=BF16)
    tail = make(200, parts, BF16, 12)
    l[-200:] = tail
    r = ep().ep_route(l, 2)
    want = ep().ep_route(tail, 2)
    assert torch.equal(r.ids[-200:], want.ids) and torch.equal(r.weights[-200:], want.weights) and int(r.routed) == rows
    d = ep().ep_route_backward(l, r, torch.ones(rows, 2, device="cuda"), None)
    w = ep().ep_route_backward(tail, want, torch.ones(200, 2, device="cuda"), None)
    assert torch.equal(d[-200:], w)


def test_an_id_out_of_range_is_reported_and_skipped():
    m = ep()
    ctx = m.default_context()
    ctx.check()
    l = make(4, 8, F32, 13)
    r = m.ep_route(l, 2)
    ids = r.ids.clone()
    ids[2, 0], ids[3, 1] = 8, -2
    m.ep_route_backward(l, r._replace(ids=ids), torch.ones(4, 2, device="cuda"), None)
    with pytest.raises(m.EmbedPartError) as e:
        ctx.check()
    assert e.value.status == 4
    ctx.check()


def test_refusals():
    m = ep()
    l = make(4, 8, F32, 14)
    r = m.ep_route(l, 2)
    dw = torch.ones(4, 2, device="cuda")
    for bad in (lambda: m.ep_route(l.cpu()), lambda: m.ep_route(l.double()), lambda: m.ep_route(l[0]), lambda: m.ep_route(l, 0),
                lambda: m.ep_route(l, 9), lambda: m.ep_route(make(2, 40, F32, 1), 33), lambda: m.ep_route(l[:, :6]),
                lambda: m.ep_route(l, 1, torch.ones(3, dtype=torch.uint8, device="cuda")),
                lambda: m.ep_route(l, 1, torch.ones(4, device="cuda")),
                lambda: m.ep_route_backward(l[:2].contiguous(), r, dw), lambda: m.ep_route_backward(l, r, dw[:, :1]),
                lambda: m.ep_route_backward(l, r, dw.double()), lambda: m.ep_route_backward(l, r, dw, torch.ones(2, device="cuda")),
                lambda: m.ep_route_backward(l, r._replace(counts=r.counts[:5]), dw)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(m.EmbedPartError):
        m.ep_route(torch.zeros(1, 4097, device="cuda"))
    ctx = m.default_context()
    assert ctx._lib.ep_route_workspace_bytes(ctx._h, 4, 0) == 0
    assert ctx._lib.ep_route(None, None, 0, 1, 8, 1, None, 0, None, None, None, None, None, None, None, 0, None) == 1
    out = torch.zeros(64, dtype=torch.int64, device="cuda").data_ptr()
    assert ctx._lib.ep_route(ctx._h, l.data_ptr(), 0, 4, 8, 1, None, 0, out, out, out, out, out, out, out, 0, None) == 3
    ctx.check()
