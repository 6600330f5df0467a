"""Activations of infinite values, whichever way a result is finished: what the definition gives in 64
bits, z Phi(z) and z sigmoid(z) being infinite at +infinity and not a number at -infinity (a product
of infinity and zero), their slopes not a number at either (the sum's second part is one)."""
import math

import pytest
import torch

from paper_2207_10731_gb300 import sequence
from tests.seq_util import normal
from tests.test_gpu_linear import act, slope

pytestmark = pytest.mark.gpu

INF = float("inf")
# tokens, in, out: few tokens, whole tiles of one CTA and of a pair, rows off the grid, a split
# contraction
SHAPES = [(1, 1, 3), (8, 64, 136), (200, 72, 64), (700, 200, 1024), (300, 33, 35), (70, 8192, 40)]


def same(got, want):
    assert torch.equal(got.isnan(), want.isnan())
    odd = want.isinf()
    assert torch.equal(got.isinf(), odd) and torch.equal(got[odd].double(), want[odd])


@pytest.mark.parametrize("name", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("wide", [False, True])
def test_infinite_values(name, shape, wide):
    t, n, m = shape
    x = normal(1, t, n, dtype=torch.bfloat16, scale=n ** -0.5)
    w = normal(2, n, m, dtype=torch.bfloat16)
    bias = normal(3, m)
    bias[0], bias[m - 1] = INF, -INF
    kind = torch.float32 if wide else torch.bfloat16
    y, z = sequence.linear_forward(x, w, bias, name, keep=True, out_dtype=kind)
    want = (x.double() @ w.double() + bias.double())
    assert (z[:, 0] == INF).all() and (z[:, m - 1] == -INF).all()
    same(y, act(want, name))
    assert (y[:, 0] == INF).all()
    # and onto the residual
    r = normal(4, t, m, dtype=kind)
    same(sequence.linear_forward(x, w, bias, name, r, out_dtype=kind), act(want, name) + r.double())


@pytest.mark.parametrize("name", ["relu", "gelu", "silu"])
def test_large_finite_values(name):
    # up to the largest fp32 number, through the bias
    z = torch.tensor([1e5, 1e19, 1.9e19, 1e38, 3.4028235e38], device="cuda")
    z = torch.cat([z, -z])
    one = torch.ones(1, 1, dtype=torch.bfloat16, device="cuda")
    nothing = torch.zeros(1, z.numel(), dtype=torch.bfloat16, device="cuda")
    y = sequence.linear_forward(one, nothing, z, name, out_dtype=torch.float32)
    want = act(z.double(), name)
    assert torch.equal(y[0].double(), want.float().double())


@pytest.mark.parametrize("name", ["relu", "gelu", "silu"])
def test_slopes_of_infinite_values(name):
    z = torch.tensor([[INF, -INF, 3.0, -2.0, 65504.0, -65504.0]], dtype=torch.float16, device="cuda")
    one = torch.ones(1, 1, dtype=torch.float16, device="cuda")
    g = torch.ones(1, 6, device="cuda")
    _, _, db = sequence.linear_backward(g, one, z, z, name, dx=False, dweight=False)
    want = slope(z[0].double(), name)
    assert torch.equal(db.isnan(), want.isnan())
    near = ~want.isnan()
    assert (db[near].double() - want[near]).abs().max() < 1e-5


def test_the_definition_at_infinity():
    z = torch.tensor([INF, -INF], dtype=torch.float64)
    for name, two in (("relu", [INF, 0.0]), ("gelu", [INF, math.nan]), ("silu", [INF, math.nan])):
        same(act(z, name), torch.tensor(two, dtype=torch.float64))
