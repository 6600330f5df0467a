"""Attention over packed sequences where operands are infinite or NaN: what a row
sees reaches it, what it does not see does not, and neither costs much more than
a clean call."""
import math

import pytest
import torch

from paper_2207_10731_gb300 import sequence
from tests.seq_util import check
from tests.test_gpu_attention import NAMES, inputs, offsets, reference, run

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


BAD = [float("nan"), math.inf, -math.inf]


def answers(q, k, v, grad, nq, nk, causal, status=False):
    """What the calls return, and reference() on inputs whose bad values are zeros:
    right wherever nothing bad is seen."""
    got = run(q, k, v, grad, nq, nk, causal, status=status)
    clean = [torch.where(x.isfinite(), x, 0.0) for x in (q, k, v, grad)]
    return got, reference(*clean[:3], nq, nk, causal, q.shape[2] ** -0.5, clean[3])


def check_where(mask, got, want, name):
    """check() at the places of the mask, which all are finite."""
    mask = mask.expand(got.shape)
    check(got[mask], want[0][mask], want[1][mask], name)


def rows(n, places, *more):
    """A mask over n rows, true at the places; further dimensions of size one."""
    m = torch.zeros(n, dtype=torch.bool, device="cuda")
    m[places] = True
    return m.view(n, *[1] * len(more)) if more else m


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("group,dim", [(1, 16), (2, 64), (3, 96), (4, 128), (70, 40)])
def test_rows_that_see_nothing_bad_are_right_element_by_element(bad, group, dim):
    # the last keys and queries of a causal sequence, and a whole neighbour, are bad
    n = [150, 90, 40]
    q, k, v, grad = inputs(n, n, 2 * group, 2, dim, seed=220)
    for x in (q, k, v, grad):
        x[145:240] = bad
    got, want = answers(q, k, v, grad, n, n, True)
    clean = list(range(145)) + list(range(240, 280))
    for i, name in enumerate(NAMES[:3]):
        check_where(rows(280, clean, *got[i].shape[1:]), got[i], want[i], name)
        assert not got[i][145:240].isfinite().all(-1).any(), name
    # a key before a bad query is seen by it
    for i, name in enumerate(NAMES[3:], 3):
        check_where(rows(280, slice(240, 280), 1, 1), got[i], want[i], name)
        assert not got[i][:240].isfinite().any(), name


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("group,dim", [(1, 64), (3, 128), (5, 24)])
def test_bad_sequences_among_short_ones(bad, causal, group, dim):
    # many to a tile, every third one bad in one of the operands
    n = [(7 * i) % 41 for i in range(60)]
    q, k, v, grad = inputs(n, n, 2 * group, 2, dim, seed=230)
    clean = torch.ones(sum(n), dtype=torch.bool, device="cuda")
    at = 0
    for i, m in enumerate(n):
        if i % 3 == 1:
            (q, k, v, grad)[i % 4][at:at + m] = bad
            clean[at:at + m] = False
        at += m
    got, want = answers(q, k, v, grad, n, n, causal)
    for name, x, y in zip(NAMES, got, want):
        check_where(clean.view(-1, *[1] * (x.dim() - 1)), x, y, name)


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("group,dim", [(1, 64), (2, 128), (3, 40)])
def test_one_bad_value_reaches_what_it_should_alone(bad, group, dim):
    n, at, c = [300], 170, 3
    heads = torch.arange(2 * group, device="cuda").view(1, -1, 1) // group   # their key head
    token = torch.arange(300, device="cuda").view(-1, 1, 1)
    column = torch.arange(dim, device="cuda")
    kv = torch.arange(2, device="cuda").view(1, -1, 1)
    # of v: column c of the rows that see it; dq and dk of those rows and what they see
    q, k, v, grad = inputs(n, n, 2 * group, 2, dim, seed=240)
    v[at, 1, c] = bad
    got, want = answers(q, k, v, grad, n, n, True)
    sees = (token >= at) & (heads == 1)
    check_where(~(sees & (column == c)), got[0], want[0], "out")
    assert not got[0][at:, group:, c].isfinite().any()
    check(got[1], *want[1], "lse")
    check_where(~sees, got[2], want[2], "dq")
    assert not got[2][at:, group:].isfinite().all(-1).any()
    check_where(kv == 0, got[3], want[3], "dk")
    # delta of a row that sees it is not finite, but p and grad are: dv stays
    check(got[4], *want[4], "dv")
    # of grad: its own dq, dk of the keys it sees, column c of their dv
    q, k, v, grad = inputs(n, n, 2 * group, 2, dim, seed=250)
    grad[at, 0, c] = bad
    got, want = answers(q, k, v, grad, n, n, True)
    check(got[0], *want[0], "out")
    own = (token == at) & (torch.arange(2 * group, device="cuda").view(1, -1, 1) == 0)
    check_where(~own, got[2], want[2], "dq")
    seen = (token <= at) & (kv == 0)
    check_where(~seen, got[3], want[3], "dk")
    assert not got[3][:at + 1, 0].isfinite().any()
    check_where(~(seen & (column == c)), got[4], want[4], "dv")
    assert not got[4][:at + 1, 0, c].isfinite().any()
    # of q: its own row everywhere, dk and dv of the keys it sees
    q, k, v, grad = inputs(n, n, 2 * group, 2, dim, seed=260)
    q[at, 0, c] = bad
    got, want = answers(q, k, v, grad, n, n, True)
    for i in (0, 2):
        check_where(~own, got[i], want[i], NAMES[i])
    check_where(~own[..., 0], got[1], want[1], "lse")
    for i in (3, 4):
        check_where(~seen, got[i], want[i], NAMES[i])


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 64), (8, 2, 128), (3, 1, 40)])
def test_bad_keys_behind_the_mask_of_a_split_range(bad, heads, kv_heads, dim):
    # the first query does not see the last key; the next sequence is all bad
    nq, nk = [2, 1, 1], [9001, 700, 3000]
    q, k, v, grad = inputs(nq, nk, heads, kv_heads, dim, seed=270)
    k[9000:9701], v[9000:9701] = bad, bad
    out, lse = run(q, k, v, None, nq, nk, True)
    (_, want) = answers(q, k, v, grad, nq, nk, True)
    for i, (name, x) in enumerate((("out", out), ("lse", lse))):
        check_where(rows(4, [0, 3], *x.shape[1:]), x, want[i], name)
    assert not out[1:3].isfinite().any()


def test_large_gradients_that_overflow_only_with_their_lift():
    # dK and dV are summed times 2^24: a gradient above 2^104 is summed again without
    n = [200]
    q, k, v, grad = inputs(n, n, 2, 1, 64, seed=280)
    grad = grad * 2.0 ** 110
    got, want = answers(q, k, v, grad, n, n, True)
    for name, x, y in zip(NAMES, got, want):
        check(x, *y, name)


@pytest.mark.parametrize("where", ["the last gradient", "everything"])
@pytest.mark.parametrize("dim", [64, 128])
def test_what_is_not_finite_does_not_hold_the_gpu(where, dim):
    # a NaN in a training step must not stall it: every row computed again runs on
    # the warps' products (an estimated tenth of the tiles' speed), so
    # 50 times a clean call is ample; a row and a key at a time would take over a thousand
    # (a million dependent steps a warp)
    n, heads = [8192], 4
    q, k, v, grad = inputs(n, n, heads, 1, dim, seed=290)
    off = offsets(n)

    def time():
        times = []
        for _ in range(3):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            out, lse = sequence.attention_forward(q, k, v, off)
            sequence.attention_backward(grad, q, k, v, out, lse, off)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return sorted(times)[1]
    clean = time()
    if where == "everything":
        for x in (q, k, v):
            x.fill_(float("nan"))
    grad[-1] = float("nan")
    odd = time()
    print(f"\ndim {dim}, {where}: clean {clean:.3f} ms, not finite {odd:.3f} ms")
    assert odd < 50 * clean


@pytest.mark.parametrize("group,dim", [(3, 64), (5, 128), (12, 128), (65, 40)])
def test_what_shared_memory_held_before_does_not_matter(group, dim):
    # tiles whose 128 rows the group does not divide: the rows over hold what the CTA
    # before left, here NaN
    n = [300, 20, 150]
    x = inputs(n, n, 2 * group, 2, dim, seed=295)
    want = run(*x, n, n, True, status=False)
    odd = [torch.full_like(y, float("nan")) for y in inputs([4096], [4096], 2 * 4, 2, dim)]
    off = offsets([4096])
    for _ in range(3):
        out, lse = sequence.attention_forward(*odd[:3], off)
        sequence.attention_backward(odd[3], *odd[:3], out, lse, off)
        got = run(*x, n, n, True, status=False)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
