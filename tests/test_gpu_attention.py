"""Attention over packed sequences against its definition in 64 bits, element by
element.

Bounds (u = 2^-24, b = 2^-8, one rounding to bf16).  A score scale q.k is off by
at most e = (dim + 16) u scale sum_c |q_c k_c| (fp32 products of bf16 values are
exact; sums in any order, the scaling and the exponential's argument take a few
u more), so a probability is off by 2 E + b of its size, E the row's largest e:
E for the exponential, E for the denominator, b for its rounding to bf16.
  out:  sum_j p_j |v_j| (2 E + b) and the sum's own (n + 16) u.
  lse:  E + 8 u |lse| + (n + 16) u
  delta = grad.out uses the rounded out: off by D = (dim u + b) sum_c |grad out|
    plus what out itself is off by.
  ds = p (dp - delta): |p| ((|dp| + |delta|) (3 E + b) + D + dim u sum_c |grad v|)
  dq, dk: the sums of those times |k| or |q|; dv: of p |grad| (3 E + b);
  each with the sum's own (n + 16) u on top.  All rounded once more to bf16.
"""
import math

import pytest
import torch

from tests.seq_util import UNIT, U32, check, normal

pytestmark = pytest.mark.gpu

B = UNIT[torch.bfloat16]


def ops():
    from paper_2207_10731_gb300 import sequence
    return sequence


def offsets(lens):
    return torch.tensor([0] + list(lens), dtype=torch.int64).cumsum(0).cuda()


def reference(q, k, v, nq, nk, causal, scale, grad=None, drop_masked=True):
    """[(value, bound)] of out, lse (and dq, dk, dv), in 64 bits."""
    group = q.shape[1] // k.shape[1]
    dim = q.shape[2]
    got = [[] for _ in range(5)]
    qi = ki = 0
    for n, m in zip(nq, nk):
        Q = q[qi:qi + n].double().transpose(0, 1)
        K, V = (x[ki:ki + m].double().transpose(0, 1).repeat_interleave(group, 0) for x in (k, v))
        seen = torch.ones(n, m, dtype=torch.bool, device=q.device)
        if causal:
            seen = seen.tril(m - n)
        S = (Q @ K.transpose(1, 2)) * scale
        S = torch.where(seen, S, -math.inf)
        size = torch.where(seen, Q.abs() @ K.abs().transpose(1, 2), 0.0)
        E = (dim + 16) * U32 * scale * (size.amax(2, keepdim=True) if m else size.new_zeros(1, n, 1))
        some = seen.any(1)[None, :, None]
        top = S.amax(2, keepdim=True) if m else S.new_full((1, n, 1), -math.inf)
        top = torch.where(some, top, 0.0)
        P = torch.where(seen, torch.exp(S - top), 0.0)
        total = P.sum(2, keepdim=True)
        lse = torch.where(some, top + total.log(), -math.inf)
        P = torch.where(some, P / total, 0.0)
        acc = (m + 16) * U32

        def rows(p, x):   # a masked value is not part of the sum, whatever it holds
            x = torch.where(torch.isfinite(x), x, 0.0)
            return p @ x
        O = rows(P, V)
        O_bound = rows(P, V.abs()) * (2 * E + B + acc)
        got[0].append((O.transpose(0, 1), O_bound.transpose(0, 1)))
        got[1].append((lse[..., 0].transpose(0, 1),
                       (E + 8 * U32 * lse.abs().nan_to_num(posinf=0) + acc)[..., 0].expand(lse.shape[:2]).transpose(0, 1)))
        if grad is not None:
            G = grad[qi:qi + n].double().transpose(0, 1)
            dP = G @ V.transpose(1, 2)
            delta = (G * O).sum(2, keepdim=True)
            D = (G.abs() * ((dim * U32 + B) * O.abs() + O_bound)).sum(2, keepdim=True)
            dS = P * (dP - delta)
            dS_bound = P * ((dP.abs() + delta.abs()) * (3 * E + B) + D +
                            dim * U32 * (G.abs() @ V.abs().transpose(1, 2)))
            acc_q = (n * group + 16) * U32

            def shared(x):
                return x.view(k.shape[1], group, m, dim).sum(1).transpose(0, 1)
            got[2].append((scale * (dS @ K).transpose(0, 1),
                           scale * ((dS_bound + acc * dS.abs()) @ K.abs()).transpose(0, 1)))
            dSt, dSb = dS.transpose(1, 2), dS_bound.transpose(1, 2)
            got[3].append((scale * shared(dSt @ Q), scale * shared((dSb + acc_q * dSt.abs()) @ Q.abs())))
            Pt, Eb = P.transpose(1, 2), (P * (3 * E + B + acc_q)).transpose(1, 2)
            got[4].append((shared(Pt @ G), shared(Eb @ G.abs())))
        qi, ki = qi + n, ki + m
    return [(torch.cat([x for x, _ in g]), torch.cat([x for _, x in g])) for g in got if g]


def inputs(nq, nk, heads, kv_heads, dim, seed=0):
    q = normal(seed, sum(nq), heads, dim, dtype=torch.bfloat16)
    k = normal(seed + 1, sum(nk), kv_heads, dim, dtype=torch.bfloat16)
    v = normal(seed + 2, sum(nk), kv_heads, dim, dtype=torch.bfloat16)
    grad = normal(seed + 3, sum(nq), heads, dim, dtype=torch.bfloat16)
    return q, k, v, grad


NAMES = ["out", "lse", "dq", "dk", "dv"]


def run(q, k, v, grad, nq, nk, causal, scale=None, status=True):
    st = torch.full((1,), 99, dtype=torch.int64, device="cuda") if status else None
    args = dict(causal=causal, scale=scale, status=st)
    qo, ko = offsets(nq), offsets(nk)
    out, lse = ops().attention_forward(q, k, v, qo, ko, **args)
    got = [out, lse]
    if status:
        assert st.item() == -1
        st.fill_(99)
    if grad is not None:
        got += ops().attention_backward(grad, q, k, v, out, lse, qo, ko, **args)
        if status:
            assert st.item() == -1
    return got


def compare(got, q, k, v, grad, nq, nk, causal, scale=None):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    want = reference(q, k, v, nq, nk, causal, scale, grad)
    for name, x, (y, bound) in zip(NAMES, got, want):
        check(x, y, bound, name)


LENS = {
    "one token": ([1], [1]),
    "one row": ([1, 1, 1], [1, 2, 129]),
    "short": ([5, 1, 17, 0, 64], [5, 1, 17, 0, 64]),
    "around a tile": ([127, 128, 129], [127, 128, 129]),
    "around two tiles": ([255, 256, 257], [255, 256, 257]),
    "long": ([700], [700]),
    "ragged": ([3, 0, 400, 1, 130, 0, 33], [3, 0, 400, 1, 130, 0, 33]),
    "many": ([(7 * i) % 41 for i in range(60)], [(7 * i) % 41 for i in range(60)]),
    "steps": ([1, 1, 1, 1, 1], [300, 1, 0, 1030, 128]),
    "few queries": ([7, 3, 0, 20], [500, 3, 70, 129]),
    "more queries than keys": ([40, 200, 5], [3, 130, 0]),
}


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 64), (4, 2, 128), (6, 2, 16)])
def test_lengths_and_masks(lens, causal, heads, kv_heads, dim):
    nq, nk = LENS[lens]
    q, k, v, grad = inputs(nq, nk, heads, kv_heads, dim)
    compare(run(q, k, v, grad, nq, nk, causal), q, k, v, grad, nq, nk, causal)


@pytest.mark.parametrize("lens", ["one token", "one row", "short", "around a tile", "more queries than keys"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 64), (6, 2, 128)])
def test_small_calls_without_a_status_word(lens, causal, heads, kv_heads, dim):
    # no work list is made for these: the same results, bit for bit
    nq, nk = LENS[lens]
    q, k, v, _ = inputs(nq, nk, heads, kv_heads, dim, seed=180)
    got = run(q, k, v, None, nq, nk, causal, status=False)
    compare(got, q, k, v, None, nq, nk, causal)
    listed = run(q, k, v, None, nq, nk, causal)
    assert torch.equal(got[0], listed[0]) and torch.equal(got[1], listed[1])


@pytest.mark.parametrize("dim", [8, 16, 24, 32, 40, 56, 64, 72, 80, 96, 112, 120, 128])
@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (5, 1)])
def test_dims(dim, heads, kv_heads):
    nq = nk = [150, 31]
    q, k, v, grad = inputs(nq, nk, heads, kv_heads, dim, seed=10)
    compare(run(q, k, v, grad, nq, nk, True), q, k, v, grad, nq, nk, True)


@pytest.mark.parametrize("group", [1, 2, 3, 4, 7, 8, 12, 16, 33, 65, 128])
def test_groups(group):
    nq, nk = [30, 1, 65], [30, 200, 65]
    q, k, v, grad = inputs(nq, nk, 2 * group, 2, 64, seed=20)
    for causal in (False, True):
        compare(run(q, k, v, grad, nq, nk, causal), q, k, v, grad, nq, nk, causal)


@pytest.mark.parametrize("keys,heads,kv_heads,dim", [(20000, 1, 1, 64), (9001, 8, 2, 128), (3001, 3, 1, 40)])
def test_one_query_over_a_long_sequence(keys, heads, kv_heads, dim):
    nq, nk = [1, 2], [keys, 77]
    q, k, v, grad = inputs(nq, nk, heads, kv_heads, dim, seed=30)
    compare(run(q, k, v, grad, nq, nk, True), q, k, v, grad, nq, nk, True)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("group,dim", [(1, 64), (2, 128), (3, 40), (1, 104)])
def test_as_many_tiles_as_fill_the_gpu(causal, group, dim):
    # long and short sequences, more keys than queries and fewer, an empty one
    nq, nk = [700, 300, 0, 513, 129, 257], [700, 450, 5, 513, 100, 0]
    kv_heads = 64 // group
    q, k, v, grad = inputs(nq, nk, kv_heads * group, kv_heads, dim, seed=140)
    compare(run(q, k, v, grad, nq, nk, causal), q, k, v, grad, nq, nk, causal)


def test_views_of_fused_buffers():
    nq = [100, 0, 37]
    heads, kv_heads, dim = 6, 2, 64
    rows = normal(40, sum(nq), heads + 2 * kv_heads, dim, dtype=torch.bfloat16)
    q, k, v = rows.split([heads, kv_heads, kv_heads], dim=1)
    to = torch.full_like(rows, 7.0)
    grads = to.split([heads, kv_heads, kv_heads], dim=1)
    # heads before tokens, as another layout of grad and out
    grad = normal(41, heads, sum(nq), dim, dtype=torch.bfloat16).transpose(0, 1)
    place = torch.zeros(heads, sum(nq), dim + 8, dtype=torch.bfloat16, device="cuda")
    off = offsets(nq)
    out, lse = ops().attention_forward(q, k, v, off, out=place[:, :, 8:].transpose(0, 1))
    assert (place[:, :, :8] == 0).all()
    ops().attention_backward(grad, q, k, v, out, lse, off, grads=grads)
    compare([out, lse, *grads], q, k, v, grad, nq, nq, True)


@pytest.mark.parametrize("scale", [1e-3, 1.0, 20.0])
def test_scales_and_large_scores(scale):
    nq = nk = [200]
    q, k, v, grad = inputs(nq, nk, 2, 1, 64, seed=50)
    # scores that rise and fall along the keys by far more than a tile's worth
    k = (k.float() * torch.linspace(0, 4, 200, device="cuda")[:, None, None]).bfloat16()
    compare(run(q, k, v, grad, nq, nk, True, scale), q, k, v, grad, nq, nk, True, scale)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -3.0e38])
@pytest.mark.parametrize("dim", [64, 128])
def test_masked_places_change_nothing(bad, dim):
    # the last keys and queries of a causal sequence, and a whole neighbour, are bad
    nq, n = [150, 90, 40], 150
    q, k, v, grad = inputs(nq, nq, 4, 2, dim, seed=60)
    clean = run(q, k, v, grad, nq, nq, True)
    k2, v2, q2, g2 = k.clone(), v.clone(), q.clone(), grad.clone()
    k2[n - 5:n + 90], v2[n - 5:n + 90] = bad, bad
    q2[n - 5:n + 90], g2[n - 5:n + 90] = bad, bad
    got = run(q2, k2, v2, g2, nq, nq, True)
    ok = [i for i in range(n - 5)] + [i for i in range(n + 90, sum(nq))]
    for name, x, y in zip(NAMES[:3], got[:3], clean[:3]):
        scale = y[ok].abs().float().amax()
        assert x[ok].isfinite().all(), name
        assert (x[ok].float() - y[ok].float()).abs().max() <= 4 * B * scale, name
    # a key before the bad queries is seen by them: its gradient is theirs too; the
    # third sequence has nothing to do with them
    ok = list(range(n + 90, sum(nq)))
    for name, x, y in zip(NAMES[3:], got[3:], clean[3:]):
        assert x[ok].isfinite().all(), name
        assert (x[ok].float() - y[ok].float()).abs().max() <= 4 * B * y[ok].abs().float().amax(), name


def test_bad_first_queries_leave_later_keys_alone():
    # query 0 sees key 0 only: the others' gradients hold nothing of it
    nq = [300]
    q, k, v, grad = inputs(nq, nq, 2, 2, 64, seed=70)
    clean = run(q, k, v, grad, nq, nq, True)
    q[0], grad[0] = float("nan"), float("inf")
    got = run(q, k, v, grad, nq, nq, True)
    assert got[0][0].isnan().all() and got[3][0].isnan().any()
    for name, x, y in zip(NAMES, got, clean):
        assert x[1:].isfinite().all(), name
        assert (x[1:].float() - y[1:].float()).abs().max() <= 4 * B * y[1:].abs().float().max(), name


def test_gradient_against_differences():
    nq, nk, heads, dim = [9, 30], [20, 30], 2, 16
    q, k, v, grad = inputs(nq, nk, heads, 1, dim, seed=80)
    got = run(q, k, v, grad, nq, nk, True)
    want = reference(q, k, v, nq, nk, True, dim ** -0.5, grad)
    # the formula's gradients against differences of the formula's forward, in 64 bits
    at = [x.double() for x in (q, k, v)]
    for i in range(3):
        d = normal(90 + i, *at[i].shape, dtype=torch.float64)
        values = []
        for sign in (1, -1):
            moved = list(at)
            moved[i] = moved[i] + sign * 1e-5 * d
            o = reference(*moved, nq, nk, True, dim ** -0.5)[0][0]
            values.append((o * grad.double()).sum())
        slope = (values[0] - values[1]) / 2e-5
        along = (want[2 + i][0] * d).sum()
        assert abs(slope - along) <= 1e-7 * (want[2 + i][0].abs() * d.abs()).sum()
        # and the kernel's along the same direction, within its element bounds
        mine = (got[2 + i].double() * d).sum()
        room = ((want[2 + i][1] + B * want[2 + i][0].abs()) * d.abs()).sum()
        assert abs(mine - slope) <= room


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_seen_bad_key_is_not_lost_in_a_split_range(bad):
    # one query over a long sequence, its keys split into pieces: a piece whose
    # sum is not finite must not pass for one that holds nothing
    q, k, v, _ = inputs([1, 1], [6000, 3000], 2, 1, 64, seed=150)
    clean, _ = run(q, k, v, None, [1, 1], [6000, 3000], True)
    k[4321] = bad
    out, lse = run(q, k, v, None, [1, 1], [6000, 3000], True)
    score = (q[0].double() @ k[4321, 0].double()) * 0.125
    for h in range(2):
        if score[h] == -math.inf:   # the key's weight is zero
            assert torch.isfinite(out[0, h]).all() and torch.isfinite(lse[0, h])
        else:
            assert out[0, h].isnan().all() and not torch.isfinite(lse[0, h])
    assert torch.equal(out[1], clean[1])
    # a value that is not finite, of a key with some weight
    k[4321] = 0
    v[4321, 0, 3] = bad
    out, _ = run(q, k, v, None, [1, 1], [6000, 3000], True)
    assert not torch.isfinite(out[0, :, 3]).any()
    assert torch.isfinite(out[0, :, 4]).all() and torch.equal(out[1], clean[1])


def test_tokens_outside_every_sequence_are_left_alone():
    n = 300
    q, k, v, grad = inputs([n], [n], 4, 2, 64, seed=160)
    off = torch.tensor([7, 40, 40, 190, 250], dtype=torch.int64, device="cuda")
    outside = torch.ones(n, dtype=torch.bool, device="cuda")
    outside[7:250] = False
    for t in (q, k, v, grad):   # what they hold does not matter
        t[outside] = float("nan")
    places = [torch.full_like(t, 7.0) for t in (q, q, k, v)]
    out, lse = ops().attention_forward(q, k, v, off, out=places[0])
    out[outside] = float("nan")
    lse[outside] = float("nan")
    ops().attention_backward(grad, q, k, v, out, lse, off, grads=places[1:])
    for p in places[1:]:
        assert (p[outside] == 7).all()
    lens = [33, 0, 150, 60]
    inner = [t[7:250] for t in (q, k, v, grad)]
    compare([t[7:250] for t in (out, lse, *places[1:])], *inner, lens, lens, True)


@pytest.mark.parametrize("heads,dim", [(1, 8), (2, 96)])
def test_thousands_of_sequences(heads, dim):
    # more than the planner keeps in shared memory, and more tiles (150 k tokens of
    # one head: 1170)
    lens = [(37 * i) % 101 for i in range(3000)]
    lens[1500] = 700
    if heads > 1:
        lens = [n % 7 for n in lens]
    q, k, v, grad = inputs(lens, lens, heads, 1, dim, seed=170)
    compare(run(q, k, v, grad, lens, lens, True), q, k, v, grad, lens, lens, True)


def test_equal_inputs_give_equal_bits_and_other_streams():
    nq = [400, 0, 3, 129, 700]
    q, k, v, grad = inputs(nq, nq, 8, 2, 64, seed=100)
    first = run(q, k, v, grad, nq, nq, True)
    assert all(torch.equal(x, y) for x, y in zip(first, run(q, k, v, grad, nq, nq, True)))
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in sides:
        with torch.cuda.stream(s):
            got.append(run(q, k, v, grad, nq, nq, True, status=False))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(x, y) for x, y in zip(first, g))
    off = offsets(nq)
    torch.cuda.synchronize()
    out, lse = ops().attention_forward(q, k, v, off, stream=sides[0])
    sides[0].synchronize()
    assert torch.equal(out, first[0]) and torch.equal(lse, first[1])


def test_rows_past_32_bit_offsets():
    # 34000 rows 131072 elements apart: the last one starts past 2^32 elements
    keys, dim = 34000, 64
    big = torch.empty(keys, 1, 131072, dtype=torch.bfloat16, device="cuda")
    k, v = big[:, :, :dim], big[:, :, 65536:65536 + dim]
    k.copy_(normal(110, keys, 1, dim, dtype=torch.bfloat16))
    v.copy_(normal(111, keys, 1, dim, dtype=torch.bfloat16))
    nq, nk = [3, 2], [200, keys - 200]
    q, grad = normal(112, 5, 2, dim, dtype=torch.bfloat16), normal(113, 5, 2, dim, dtype=torch.bfloat16)
    compare(run(q, k, v, grad, nq, nk, True), q, k, v, grad, nq, nk, True)


def test_malformed_offsets_are_reported_and_skipped():
    q, k, v, grad = inputs([60], [60], 2, 2, 64, seed=120)
    want = run(q[:20], k[:20], v[:20], None, [20], [20], True)
    for bad in ([0, 20, 10, 60], [0, 20, 61, 60], [0, 20, -5, 60], [0, 20, 2 ** 40, 60]):
        off = torch.tensor(bad, dtype=torch.int64, device="cuda")
        st = torch.zeros(1, dtype=torch.int64, device="cuda")
        out, lse = ops().attention_forward(q, k, v, off, status=st)
        assert st.item() == 1, bad
        assert torch.equal(out[:10], want[0][:10])
        st.zero_()
        ops().attention_backward(grad, q, k, v, out, lse, off, status=st)
        assert st.item() == 1


def test_offsets_that_overlap_stay_in_bounds():
    # back and forth: more rows in the sequences than there are; reported, and
    # nothing is written outside the tensors (the guard rows around them)
    guard = torch.full((3, 80, 2, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    q, k, v, grad = inputs([60], [60], 2, 2, 64, seed=130)
    off = torch.tensor([0, 60] * 40, dtype=torch.int64, device="cuda")
    st = torch.zeros(1, dtype=torch.int64, device="cuda")
    out, lse = ops().attention_forward(q, k, v, off, status=st, out=guard[0, 10:70])
    assert st.item() == 1
    ops().attention_backward(grad, q, k, v, out, lse, off, status=st, grads=(
        guard[1, 10:70], guard[2, 10:70], torch.empty_like(v)))
    assert st.item() == 1
    assert (guard[:, :10] == 3).all() and (guard[:, 70:] == 3).all()


def test_empty_batches():
    q, k, v, grad = inputs([0], [0], 2, 1, 64)
    for nq, nk in (([0], [0]), ([], []), ([0, 0], [0, 0])):
        out, lse = run(q, k, v, None, nq, nk, True)
        assert out.shape == (0, 2, 64) and lse.shape == (0, 2)
        assert all(x.numel() == 0 for x in run(q, k, v, grad, nq, nk, True)[2:])
    # queries without a key, and keys without a query
    q, k, v, grad = inputs([5], [0], 2, 1, 64)
    out, lse, dq, dk, dv = run(q, k, v, grad, [5], [0], False)
    assert (out == 0).all() and (lse == -math.inf).all() and (dq == 0).all()
    q, k, v, grad = inputs([0], [5], 2, 1, 64)
    out, lse, dq, dk, dv = run(q, k, v, grad, [0], [5], False)
    assert (dk == 0).all() and (dv == 0).all()


def test_refusals():
    from paper_2207_10731_gb300 import binding
    q, k, v, grad = inputs([8], [8], 4, 2, 64)
    off = offsets([8])
    fwd = ops().attention_forward
    with pytest.raises(TypeError):
        fwd(q.float(), k, v, off)
    with pytest.raises(TypeError):
        fwd(q.half(), k.half(), v.half(), off)
    with pytest.raises(TypeError):
        fwd(q, k, v, off.int())
    with pytest.raises(ValueError):
        fwd(q, k, v, off.cpu())
    with pytest.raises(ValueError):
        fwd(q.cpu(), k, v, off)
    with pytest.raises(ValueError):
        fwd(q, k, v[:7], off)
    with pytest.raises(ValueError):
        fwd(q, k[:, :, :32].contiguous(), v[:, :, :32].contiguous(), off)
    with pytest.raises(ValueError):
        fwd(q, k, v, off, offsets([8, 0]))
    with pytest.raises(ValueError):
        fwd(q.transpose(1, 2), k, v, off)
    lse = torch.empty(8, 4, device="cuda")
    with pytest.raises(ValueError):
        ops().attention_backward(grad, q, k, v, q, lse[:7], off)
    bad = [
        (q[:, :3], k, v, {}),                                     # heads not a multiple
        (q, k, v, dict(scale=0.0)), (q, k, v, dict(scale=-1.0)),
        (q, k, v, dict(scale=float("nan"))), (q, k, v, dict(scale=float("inf"))),
        (q[:, :, :60], k[:, :, :60], v[:, :, :60], {}),           # dim not a multiple of 8
        (q[:, :, 4:12], k[:, :, 4:12], v[:, :, 4:12], {}),        # not 16-byte aligned
        (q[:1].expand(8, 4, 64), k, v, {}),                       # overlapping rows
    ]
    wide = torch.zeros(8, 2, 136, dtype=torch.bfloat16, device="cuda")
    bad.append((wide, wide, wide, {}))                            # dim above 128
    odd = torch.zeros(8, 2, 68, dtype=torch.bfloat16, device="cuda")[:, :, :64]
    bad.append((odd, odd, odd, {}))                               # strides not multiples of 8
    for a, b, c, kw in bad:
        with pytest.raises(binding.PSSError) as e:
            fwd(a, b, c, off, **kw)
        assert e.value.status == binding.PSS_ERR_INVALID_ARG
