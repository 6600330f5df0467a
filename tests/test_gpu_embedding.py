"""Rows of a dense table by id and their gradient, against the definition in 64 bits.

Tolerances: forward, one product and one rounding.  Backward, a row's n gradients are
added in fp32 along at most 32 + 32 + 32 + 64 + 64 + n / 2048 + 256 additions (head, a piece,
tail, pieces on both sides of the large ones, these, and the groups' parts), each off by half
a unit of a partial sum that is at most sum |grad|; then the product with the scale and the last rounding."""
import pytest
import torch

from paper_2207_10731_gb300 import binding, sequence
from tests.seq_util import TYPES, U32, check, normal

pytestmark = pytest.mark.gpu


def ids_of(seed, n, rows, kind):
    gen = torch.Generator().manual_seed(seed)
    if kind == "one":
        ids = torch.full((n,), rows // 2)
    elif kind == "padded":
        ids = torch.randint(-2, rows + 2, (n,), generator=gen)
    else:   # popular ids first
        ids = (torch.rand(n, generator=gen, dtype=torch.float64) ** 4 * rows).long()
    return ids.cuda()


def first_outside(ids, rows):
    bad = ((ids < 0) | (ids >= rows)).view(-1).nonzero()
    return int(bad[0]) if bad.numel() else -1


def forward(weight, ids, scale):
    inside = (ids >= 0) & (ids < weight.shape[0])
    return weight.double()[ids.clamp(0, weight.shape[0] - 1)] * inside[..., None] * scale


def backward(grad, ids, rows, scale):
    """(gradient, its bound)."""
    ids, g = ids.view(-1), grad.reshape(ids.numel(), -1).double()
    inside = (ids >= 0) & (ids < rows)
    zero = torch.zeros(rows, g.shape[1], dtype=torch.float64, device="cuda")
    want = zero.index_add(0, ids[inside], g[inside]) * scale
    size = zero.index_add(0, ids[inside], g[inside].abs()) * abs(scale)
    n = torch.bincount(ids[inside], minlength=rows).double()
    depth = torch.minimum(n, 480 + n / 2048) + 2
    return want, depth[:, None] * U32 * size


CASES = [
    # tokens, rows, cols, kind, type, to
    (1, 1, 1, "one", "f32", "f32"),
    (26, 100, 128, "popular", "f32", "bf16"),
    (3, 5, 8, "padded", "bf16", "f32"),
    (63, 7, 16, "one", "f16", "f32"),
    (64, 7, 16, "one", "f16", "f16"),
    (65, 7, 24, "one", "bf16", "bf16"),
    (500, 40, 333, "padded", "f16", "f32"),
    (1000, 3000, 64, "popular", "bf16", "f16"),
    (4096, 600, 8, "popular", "f32", "f32"),
    (4097, 600, 12, "padded", "f32", "f32"),
    (4097, 1, 264, "one", "bf16", "f32"),
    (9001, 70000, 40, "popular", "f16", "f32"),
    (20000, 50, 129, "popular", "f32", "f16"),
    (70001, 3, 64, "popular", "bf16", "f32"),
    (300, 20, 1024, "popular", "bf16", "f32"),
    (3197, 839, 64, "popular", "f32", "bf16"),
    (8192, 300, 520, "popular", "bf16", "f32"),
    (8193, 4000, 8, "popular", "f16", "f32"),
    (60000, 700, 256, "popular", "f32", "f32"),
    (33, 9, 2056, "padded", "f32", "bf16"),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("gap", [0, 8, 3])
def test_against_the_definition(case, gap):
    n, rows, cols, kind, a, b = case
    ids = ids_of(n, n, rows, kind)
    scale = 2.75
    status = torch.full((1,), 77, device="cuda")
    weight = normal(1, rows, cols + gap, dtype=TYPES[a])[:, :cols]
    wide = torch.full((n, cols + gap), 9.0, dtype=TYPES[b], device="cuda")
    out = sequence.embedding_forward(weight, ids, scale=scale, out=wide[:, :cols], status=status)
    want = forward(weight, ids, scale)
    check(out, want, want.abs() * U32, "out")
    assert (wide[:, cols:] == 9).all() and int(status) == first_outside(ids, rows)
    grad = normal(2, n, cols + gap, dtype=TYPES[a])[:, :cols]
    wide = torch.full((rows, cols + gap), 9.0, dtype=TYPES[b], device="cuda")
    got = sequence.embedding_backward(grad, ids, rows, scale=scale, out=wide[:, :cols],
                                      status=status.fill_(77))
    check(got, *backward(grad, ids, rows, scale), "dweight")
    assert (wide[:, cols:] == 9).all() and int(status) == first_outside(ids, rows)
    again = sequence.embedding_backward(grad, ids, rows, scale=scale, out_dtype=TYPES[b])
    assert torch.equal(again, got)


def test_long_runs_and_large_tables():
    # runs of every length around the pieces' sizes, one after another
    rows = 400
    counts = torch.tensor([[1, 63, 64, 65, 127, 128, 129, 300][i % 8] for i in range(rows)])
    counts[7], counts[201] = 4096 * 2 + 5, 4096 * 3
    ids = torch.repeat_interleave(torch.arange(rows), counts)
    ids = ids[torch.randperm(ids.numel(), generator=torch.Generator().manual_seed(3))].cuda()
    grad = normal(4, ids.numel(), 72, dtype=torch.bfloat16)
    check(sequence.embedding_backward(grad, ids, rows), *backward(grad, ids, rows, 1.0), "dweight")
    # offsets past 32 bits on the table's side and on the tokens' side
    rows, cols = 4400001, 512
    weight = torch.zeros(rows, cols, dtype=torch.float16, device="cuda")
    ids = torch.tensor([rows - 1, 0, 4194304, 4194303, -1, rows], device="cuda")
    weight[ids[:4]] = normal(5, 4, cols, dtype=torch.float16)
    out = sequence.embedding_forward(weight, ids)
    assert torch.equal(out[:4], weight[ids[:4]]) and not out[4:].any()
    got = sequence.embedding_backward(out, ids, rows, out_dtype=torch.float16)
    assert torch.equal(got, weight)
    del got, weight
    n = 4400001
    ids = torch.arange(n, device="cuda") % 5
    ids[1:-1] = -1
    grad = torch.ones(n, cols, dtype=torch.float16, device="cuda")
    got = sequence.embedding_backward(grad, ids, 5)
    want = torch.zeros(5, cols, device="cuda")
    want[0] += 1
    want[(n - 1) % 5] += 1
    assert torch.equal(got, want)


def test_empty_sizes():
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    w = normal(1, 5, 8)
    assert sequence.embedding_forward(w, none).shape == (0, 8)
    assert sequence.embedding_forward(w, none.view(3, 0)).shape == (3, 0, 8)
    some = torch.tensor([0, -1], device="cuda")
    assert sequence.embedding_forward(w[:, :0], some).shape == (2, 0)
    status = torch.zeros(1, dtype=torch.int64, device="cuda")
    assert not sequence.embedding_forward(w[:0], some, status=status).any() and int(status) == 0
    assert not sequence.embedding_backward(w[:0], none, 7, status=status).any()
    assert int(status) == -1
    assert sequence.embedding_backward(w[:2], some, 0).shape == (0, 8)
    wide = torch.full((4, 11), 3.0, device="cuda")
    sequence.embedding_backward(w[:0], none, 4, out=wide[:, :8])
    assert not wide[:, :8].any() and (wide[:, 8:] == 3).all()


def test_values_that_are_not_finite_stay_in_their_rows():
    w = normal(1, 6, 40)
    w[2, 5], w[3, 6] = float("nan"), float("inf")
    ids = torch.tensor([0, 2, 3, -1, 5], device="cuda")
    assert torch.equal(sequence.embedding_forward(w, ids).nan_to_num(nan=7.0),
                       torch.cat([w[[0, 2, 3]], w[:1] * 0, w[5:]]).nan_to_num(nan=7.0))
    ids = torch.tensor([4] * 70 + [1, -1, 6] + [0] * 70, device="cuda")
    g = normal(2, ids.numel(), 40)
    g[3], g[71], g[72] = float("inf"), float("nan"), float("nan")
    got = sequence.embedding_backward(g, ids, 6, scale=-1.0)
    assert (got[4] == -float("inf")).all() and got[[0, 1]].isfinite().all() and not got[[2, 3, 5]].any()


def test_shapes_streams_and_graphs():
    ids = ids_of(1, 6000, 300, "padded").view(20, 300)
    w, g = normal(1, 300, 64), normal(2, 20, 300, 64)

    def calls():
        return sequence.embedding_forward(w, ids), sequence.embedding_backward(g, ids, 300)
    want = calls()
    assert want[0].shape == (20, 300, 64)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    got = (sequence.embedding_forward(w, ids, stream=side),
           sequence.embedding_backward(g, ids, 300, stream=side))
    side.synchronize()
    assert not torch.cuda.current_stream().query()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls()
    others = ids_of(2, 6000, 300, "popular").view(20, 300), normal(3, 300, 64), normal(4, 20, 300, 64)
    ids.copy_(others[0]), w.copy_(others[1]), g.copy_(others[2])
    for _ in range(2):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, calls()))


def test_refusals():
    w, ids = normal(1, 5, 8), torch.tensor([1, 2], device="cuda")
    f, b = sequence.embedding_forward, sequence.embedding_backward
    for error, call in [
            (TypeError, lambda: f(w.double(), ids)), (TypeError, lambda: f(w, ids.int())),
            (ValueError, lambda: f(w.cpu(), ids)), (ValueError, lambda: f(w, ids.cpu())),
            (ValueError, lambda: f(w[0], ids)), (ValueError, lambda: f(w.t(), ids)),
            (ValueError, lambda: f(w, ids, out=w)), (TypeError, lambda: f(w, ids, out_dtype=torch.int32)),
            (ValueError, lambda: f(w, torch.stack([ids, ids], 1)[:, 0])),
            (binding.PSSError, lambda: f(w, ids, scale=float("inf"))),
            (TypeError, lambda: f(w, ids, status=ids[:1].int())),
            (ValueError, lambda: b(w[:3], ids, 4)), (TypeError, lambda: b(w[:2], ids, 4, out=w, out_dtype=torch.float16)),
            (ValueError, lambda: b(w[:2], ids, 4, out=w)),
            (binding.PSSError, lambda: b(w[:2], ids, 4, scale=float("nan")))]:
        with pytest.raises(error):
            call()
