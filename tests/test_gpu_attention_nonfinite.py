"""Attention over packed sequences where operands are infinite or NaN: what a row
sees reaches it, what it does not see does not, and neither costs much more than
a clean call."""
import math

import pytest
import torch

from tests.test_gpu_attention import inputs, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nq,nk", [([150], [150]), ([3, 40], [7, 200]), ([1, 1], [6000, 3000])])
@pytest.mark.parametrize("status", [False, True])
@pytest.mark.parametrize("where", ["first key", "first keys", "all keys", "query"])
def test_a_nan_score_reaches_its_row_wherever_it_stands(nq, nk, status, where):
    # a softmax with one NaN score is NaN, also where no other score came before it
    q, k, v, _ = inputs(nq, nk, 4, 2, 64, seed=200)
    clean = run(q, k, v, None, nq, nk, True, status=status)
    k2, q2 = k.clone(), q.clone()
    if where == "query":
        q2[:nq[0]] = float("nan")
    else:
        k2[:{"first key": 1, "first keys": 5, "all keys": nk[0]}[where]] = float("nan")
    out, lse = run(q2, k2, v, None, nq, nk, True, status=status)
    assert out[:nq[0]].isnan().all() and lse[:nq[0]].isnan().all()
    assert torch.equal(out[nq[0]:], clean[0][nq[0]:]) and torch.equal(lse[nq[0]:], clean[1][nq[0]:])


def test_a_score_of_minus_infinity_has_no_weight():
    q, k, v, _ = inputs([200], [200], 2, 1, 64, seed=210)
    q, k = q.abs(), k.abs()
    k[0] = -math.inf
    out, lse = run(q, k, v, None, [200], [200], True)
    clean = run(q[1:], k[1:], v[1:], None, [199], [199], True)
    # the row that sees nothing else has no softmax; the others are those without the key
    assert out[0].isnan().all() and (lse[0] == -math.inf).all()
    assert (out[1:].float() - clean[0].float()).abs().max() <= 2 ** -7 * clean[0].abs().max()
    assert (lse[1:] - clean[1]).abs().max() <= 1e-4
