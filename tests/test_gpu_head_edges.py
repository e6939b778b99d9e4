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
