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
