"""Products on rows that lie further apart than they are wide, on the 16-byte grid: read and written in
place, whatever lies between them, against the definition in 64 bits (the bounds of
test_gpu_linear)."""
import pytest
import torch

from paper_2207_10731_gb300 import sequence
from tests.seq_util import TYPES, check, normal
from tests.test_gpu_linear import backward, forward

pytestmark = pytest.mark.gpu


def apart(seed, rows, cols, stride, dtype, scale=1.0):
    """Rows from column 0 of wider ones, NaN between them."""
    t = torch.full((rows, stride), float("nan"), dtype=dtype, device="cuda")
    t[:, :cols] = normal(seed, rows, cols, dtype=dtype, scale=scale)
    return t[:, :cols]


def up(n, more):
    """The next multiple of 8 that leaves a gap, and `more` of them."""
    return n // 8 * 8 + 8 * more


CASES = [
    # tokens, in, out, type, activation, bias, residual, wide
    (7, 333, 129, "f16", "gelu", 1, 1, 0), (40, 517, 300, "bf16", None, 1, 1, 1), (129, 63, 65, "bf16", "relu", 1, 1, 0),
    (200, 333, 517, "bf16", "silu", 1, 1, 0), (513, 1025, 511, "f16", "gelu", 1, 1, 0), (1000, 512, 512, "bf16", "gelu", 1, 1, 0),
    (1500, 64, 2094, "bf16", "gelu", 1, 1, 0), (3620, 45, 705, "f16", None, 0, 1, 1), (2233, 72, 1645, "bf16", "relu", 1, 1, 0),
    (70, 4099, 44, "bf16", None, 1, 1, 0), (5000, 100, 121, "f16", "silu", 1, 0, 0), (9000, 128, 115, "bf16", None, 0, 0, 0),
    (1, 20, 12, "bf16", "gelu", 1, 1, 0), (2, 1, 3, "f16", "gelu", 1, 1, 0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("more", [1, 3])
@pytest.mark.parametrize("dense", ["out", "in"])
def test_rows_apart(case, more, dense):
    t, n, m, kind, name, bias, residual, wide = case
    kind = TYPES[kind]
    result = torch.float32 if wide else kind
    x = apart(1, t, n, up(n, more), kind)
    w = apart(2, n, m, up(m, more), kind, n ** -0.5) if dense == "out" else \
        apart(2, m, n, up(n, more), kind, n ** -0.5).t()
    bias = normal(3, m) if bias else None
    r = apart(4, t, m, up(m, more), result) if residual else None
    grad = apart(5, t, m, up(m, more), result)
    room = torch.full((t, up(m, more)), 9.0, dtype=result, device="cuda")
    status = torch.full((1,), 5, device="cuda")
    got = sequence.linear_forward(x, w, bias, name, r, keep=name is not None, out=room[:, :m], status=status)
    y, z = got if name else (got, None)
    (wy, by), (wz, bz) = forward(x, w, bias, name, r)
    check(y, wy, by, "y")
    if name:
        check(z, wz, bz, "z")
    assert (room[:, m:] == 9).all() and int(status) == -1
    if r is not None:   # in place, and what lies between the residual's rows stays
        kept = r._base.clone()
        assert sequence.linear_forward(x, w, bias, name, r, out=r) is r and torch.equal(r, y)
        assert r._base[:, m:].isnan().all() and kept[:, m:].isnan().all()
    room = torch.full((t, up(n, more)), 9.0, dtype=kind, device="cuda")
    rows, cols = (n, m) if dense == "out" else (m, n)
    for dtype in (kind, torch.float32):
        other = torch.full((rows, up(cols, more)), 9.0, dtype=dtype, device="cuda")
        dweight = other[:, :cols] if dense == "out" else other[:, :cols].t()
        zz = None if z is None else apart(6, t, m, up(m, more), kind).copy_(z)
        back = sequence.linear_backward(grad, x, w, zz, name, dx=room[:, :n], dweight=dweight,
                                        status=status.fill_(5))
        narrow = kind if name or wide else None
        for what, g, v in zip(("dx", "dweight", "dbias"), back, backward(grad, x, w, z, name, narrow)):
            check(g, v[0], v[1], what)
        assert (room[:, n:] == 9).all() and (other[:, cols:] == 9).all() and int(status) == -1
    back = sequence.linear_backward(grad, x, w, z, name)
    assert back[1].stride() == ((m, 1) if dense == "out" or m == 1 else (1, n))


@pytest.mark.parametrize("out", [66, 80, 96, 104, 112, 113, 120, 127, 128, 160, 192, 224, 320, 448])
@pytest.mark.parametrize("tokens", [300, 2500])
def test_weight_gradients_of_every_tile_width(out, tokens):
    """dweight's second operand lies across the contraction, in boxes of 64: widths around a pair's
    tiles of 160 to 256 columns and half of them."""
    for n in (129, 520, 4096):
        x, g = normal(1, tokens, n, dtype=torch.bfloat16), normal(2, tokens, out, dtype=torch.bfloat16)
        w = torch.empty(n, out, dtype=torch.bfloat16, device="cuda")
        _, dw, _ = sequence.linear_backward(g, x, w, dx=False, dbias=False)
        size = x.double().abs().t() @ g.double().abs()
        check(dw, x.double().t() @ g.double(), size * 2 * (tokens + 2) * 2.0 ** -24, "dweight")
        _, dw, _ = sequence.linear_backward(g, x, w.t().contiguous().t(), dx=False, dbias=False)
        check(dw, x.double().t() @ g.double(), size * 2 * (tokens + 2) * 2.0 ** -24, "dweight, in dense")


@pytest.mark.parametrize("tokens", [1, 40, 300, 5000])
@pytest.mark.parametrize("n", [1, 60, 333, 1024])
@pytest.mark.parametrize("strides", ["dense", "other stride", "row apart", "off the grid"])
def test_single_columns(tokens, n, strides):
    """A weight [n, 1], as a gate's, however its n values lie."""
    kind = torch.bfloat16
    whole = normal(2, 1, n * 8 + 8, dtype=kind, scale=n ** -0.5)[0]
    at, step, other = {"dense": (0, 1, 1), "other stride": (8, 1, n + 3), "row apart": (0, 8, 1),
                       "off the grid": (1, 1, 1)}[strides]
    w = whole.as_strided((n, 1), (step, other), at)
    x, bias, grad = normal(1, tokens, n, dtype=kind), normal(3, 1), normal(5, tokens, 1, dtype=kind)
    y = sequence.linear_forward(x, w, bias)
    check(y, *forward(x, w, bias, None, None)[0], "y")
    other = torch.full_like(whole, 9.0).as_strided(w.shape, w.stride(), at)
    for dweight in (True, other):
        back = sequence.linear_backward(grad, x, w, dweight=dweight)
        for what, g, v in zip(("dx", "dweight", "dbias"), back, backward(grad, x, w, None, None, None)):
            check(g, v[0], v[1], what)
    marks = torch.full_like(whole, 9.0)
    marks.as_strided(w.shape, w.stride(), at).copy_(other)
    assert torch.equal(other._base if other._base is not None else other, marks)
