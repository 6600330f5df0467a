"""Layouts and sizes that lead the sequence operators onto paths of their own.
Bounds as in the operators' own tests."""
import pytest
import torch

from paper_2207_10731_gb300 import sequence
from tests.seq_util import TYPES, U32, check, normal
from tests.test_gpu_attention import compare, inputs, offsets, run
from tests.test_gpu_dropout import mask
from tests.test_gpu_layer_norm import backward_reference, reference

pytestmark = pytest.mark.gpu


def cut(x, before, after):
    """The same rows inside a wider buffer of sevens."""
    wide = torch.full((x.shape[0], x.shape[1] + before + after), 7.0, dtype=x.dtype, device="cuda")
    wide[:, before:before + x.shape[1]] = x
    return wide, wide[:, before:before + x.shape[1]]


@pytest.mark.parametrize("cols", [1, 3, 8, 31, 64, 128, 129, 333, 512, 513, 1000, 2049, 4097, 8193, 12001, 16384])
@pytest.mark.parametrize("a,b", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("f16", "f16")])
def test_norm_of_rows_that_lie_differently_in_each_tensor(cols, a, b):
    # x, y, the gradient and dx each off the grid in their own way: one element at a time
    rows = max(3, min(700, 60000 // cols))
    x = (normal(40 + cols, rows, cols) * 1.5 + normal(41, rows, 1)).to(TYPES[a])
    w, c = 1 + normal(42, cols, scale=0.3), normal(43, cols)
    wide, x = cut(x, 3, 2)
    out_wide, out = cut(torch.zeros(rows, cols, dtype=TYPES[b], device="cuda"), 1, 7)
    y, mean, rstd = sequence.layer_norm_forward(x, w, c, eps=1e-5, out=out)
    ref, m, r, bound, m_bound, r_bound = reference(x, w, c, 1e-5)
    check(mean, m, m_bound, "mean")
    check(rstd, r, r_bound, "rstd")
    check(y, ref, bound, "y")
    assert (out_wide[:, :1] == 7).all() and (out_wide[:, 1 + cols:] == 7).all()
    _, g = cut(normal(44, rows, cols, dtype=TYPES[b]), 5, 4)
    dx_wide, dx = cut(torch.zeros_like(x), 2, 1)
    got = sequence.layer_norm_backward(g, x, w, mean, rstd, out=dx)
    want = backward_reference(g, x, w, mean, rstd)
    for name, value, limit, have in zip(("dx", "dweight", "dbias"), want[:3], want[3:], got):
        check(have, value, limit, name)
    assert (dx_wide[:, :2] == 7).all() and (dx_wide[:, 2 + cols:] == 7).all()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("cols,x_gap,r_gap,y_gap", [(64, (0, 16), (8, 8), (16, 0)), (64, (1, 2), (0, 0), (3, 8)),
                                                    (129, (0, 0), (5, 6), (2, 1)), (8, (8, 0), (0, 8), (0, 24))])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout_into_rows_that_lie_differently(kind, cols, x_gap, r_gap, y_gap, residual):
    rows, p, seed, offset = 61, 0.3, 12345678901234567890, 77
    _, x = cut(normal(51, rows, cols, dtype=TYPES[kind]), *x_gap)
    _, add = cut(normal(52, rows, cols, dtype=TYPES[kind]), *r_gap)
    wide, out = cut(torch.zeros_like(x), *y_gap)
    y = sequence.dropout(x, p, seed, offset, residual=add if residual else None, out=out)
    keep = mask(rows * cols, p, seed, offset).view(rows, cols).cuda()
    want = torch.where(keep, x.double() * (65536 / (65536 - round(p * 65536))), 0.0)
    bound = 2 * U32 * want.abs()
    if residual:
        want = want + add.double()
        bound = bound + U32 * want.abs()
    check(y, want, bound, "y")
    assert (wide[:, :y_gap[0]] == 7).all() and (wide[:, y_gap[0] + cols:] == 7).all()


@pytest.mark.parametrize("dim", [64, 128])
def test_more_pieces_than_the_join_keeps_in_registers(dim):
    # above 128 pieces of four key tiles at least
    nq, nk = [1, 1], [100001, 5]
    q, k, v, _ = inputs(nq, nk, 2, 1, dim, seed=330)
    compare(run(q, k, v, None, nq, nk, True), q, k, v, None, nq, nk, True)


@pytest.mark.parametrize("group,dim", [(1, 64), (3, 128), (4, 24)])
@pytest.mark.parametrize("causal", [False, True])
def test_heads_before_tokens_in_every_tensor(group, dim, causal):
    nq, nk = [150, 31, 0, 200], [150, 300, 7, 64]
    q, k, v, grad = (t.transpose(0, 1).contiguous().transpose(0, 1)
                     for t in inputs(nq, nk, 2 * group, 2, dim, seed=340))
    places = [torch.full_like(t.transpose(0, 1), 7.0).transpose(0, 1) for t in (q, q, k, v)]
    out, lse = sequence.attention_forward(q, k, v, offsets(nq), offsets(nk), causal=causal,
                                          out=places[0])
    sequence.attention_backward(grad, q, k, v, out, lse, offsets(nq), offsets(nk), causal=causal,
                                grads=places[1:])
    compare([out, lse, *places[1:]], q, k, v, grad, nq, nk, causal)


@pytest.mark.parametrize("nq", [1, 7])
@pytest.mark.parametrize("group,dim", [(1, 64), (4, 128), (3, 40)])
def test_a_training_pass_of_few_queries_over_long_keys(nq, group, dim):
    nq, nk = [nq] * 6, [3000, 1, 900, 0, 2049, 1500]
    q, k, v, grad = inputs(nq, nk, 2 * group, 2, dim, seed=350)
    compare(run(q, k, v, grad, nq, nk, True), q, k, v, grad, nq, nk, True)
