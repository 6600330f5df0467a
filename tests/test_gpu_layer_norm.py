"""Layer norm against its definition in 64 bits, element by element.

Bounds (u = 2^-24, fp32): the kernels sum a row in a tree of depth below 32
(16 values a thread, 10 shuffle levels), so a mean of n values is off by at
most 32 u mean|x| (Higham, "Accuracy and Stability of Numerical Algorithms",
Sec. 4.2).  With m = mean|x| + |mean| of a row, x - mean is off by 33 u m, and
the rest of y = (x - mean) rstd w + b by a few u of its size: the variance's
relative error is at most 34 u + 2 * 33 u m * rstd (its terms' sizes are
1 / rstd on average), the square root halves it.  Together, with h = (x -
mean) rstd,  |dy| <= u (34 m rstd |w| (1 + |h|) + 40 |h w| + 4 |b|), and y is
rounded once more to its type.  The backward pass takes mean and rstd as given;
its row sums have the same depth.
"""
import pytest
import torch

from tests.seq_util import TYPES, U32, check, normal

pytestmark = pytest.mark.gpu

# 1 thread to a row up to a whole CTA, odd widths, every vector width and count
COLS = [1, 2, 3, 7, 8, 16, 31, 64, 100, 127, 128, 200, 256, 257, 333, 384, 400, 511, 512, 520, 1000,
        1024, 3328, 4097, 8192, 8200, 16383, 16384]


def reference(x, w, b, eps):
    x, w, b = x.double(), w.double(), b.double()
    mean = x.mean(-1, keepdim=True)
    rstd = ((x - mean).square().mean(-1, keepdim=True) + eps).rsqrt()
    h = (x - mean) * rstd
    m = x.abs().mean(-1, keepdim=True) + mean.abs()
    bound = U32 * (34 * m * rstd * w.abs() * (1 + h.abs()) + 40 * (h * w).abs() + 4 * b.abs())
    return h * w + b, mean[..., 0], rstd[..., 0], bound, (32 * U32 * m)[..., 0], \
        (rstd * U32 * (40 + 67 * m * rstd))[..., 0]


def backward_reference(g, x, w, mean, rstd):
    g, x, w = g.double(), x.double(), w.double()
    mean, rstd = mean.double()[..., None], rstd.double()[..., None]
    h = (x - mean) * rstd
    gw = g * w
    dx = rstd * (gw - gw.mean(-1, keepdim=True) - h * (gw * h).mean(-1, keepdim=True))
    size = gw.abs() + gw.abs().mean(-1, keepdim=True) + \
        h.abs() * (gw * h).abs().mean(-1, keepdim=True)
    # h itself carries the rounding of x - mean
    off = (x.abs() + mean.abs()) * rstd
    size = size + off * (gw * h).abs().mean(-1, keepdim=True) + \
        h.abs() * (gw * off).abs().mean(-1, keepdim=True)
    rows = g.reshape(-1, g.shape[-1])
    hr, offr = h.reshape(rows.shape), off.reshape(rows.shape)
    n = rows.shape[0]
    # a column's sum runs over at most n rows in sequence
    db_bound = n * U32 * rows.abs().sum(0)
    dw_bound = (n + 3) * U32 * (rows.abs() * (hr.abs() + offr)).sum(0)
    return dx, (rows * hr).sum(0), rows.sum(0), 40 * U32 * rstd * size, dw_bound, db_bound


def ops():
    from paper_2207_10731_gb300 import sequence
    return sequence


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("a,b", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("f16", "f32"),
                                 ("bf16", "f16")])
def test_forward_and_backward(cols, a, b):
    rows = max(3, min(700, 60000 // cols))
    x = (normal(cols, rows, cols) * 1.5 + normal(1, rows, 1)).to(TYPES[a])
    w, c = 1 + normal(2, cols, scale=0.3), normal(3, cols)
    y, mean, rstd = ops().layer_norm_forward(x, w, c, eps=1e-5, out_dtype=TYPES[b])
    ref, m, r, bound, m_bound, r_bound = reference(x, w, c, 1e-5)
    assert y.dtype == TYPES[b] and y.shape == x.shape
    check(mean, m, m_bound, "mean")
    check(rstd, r, r_bound, "rstd")
    check(y, ref, bound, "y")
    g = normal(4, rows, cols, dtype=TYPES[b])
    got = ops().layer_norm_backward(g, x, w, mean, rstd)
    dx, dw, db, x_bound, w_bound, b_bound = backward_reference(g, x, w, mean, rstd)
    assert got[0].dtype == x.dtype
    check(got[0], dx, x_bound, "dx")
    check(got[1], dw, w_bound, "dweight")
    check(got[2], db, b_bound, "dbias")


@pytest.mark.parametrize("rows", [0, 1, 2, 151, 40000])
def test_row_counts(rows):
    x, w, c = normal(5, rows, 128), normal(6, 128), normal(7, 128)
    y, mean, rstd = ops().layer_norm_forward(x, w, c)
    ref, m, r, bound, _, _ = reference(x, w, c, 1e-5)
    check(y, ref, bound, "y")
    dx, dw, db = ops().layer_norm_backward(x, x, w, mean, rstd)
    ref = backward_reference(x, x, w, mean, rstd)
    check(dx, ref[0], ref[3], "dx")
    check(dw, ref[1], ref[4], "dweight")
    check(db, ref[2], ref[5], "dbias")


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("cols", [128, 129])
def test_strided_rows_off_alignment_and_in_place(cols, shift):
    wide = normal(8, 40, 3, 160 + shift, dtype=torch.bfloat16)
    x = wide[:, :, shift:shift + cols]
    before = wide.clone()
    w, c = normal(9, cols), normal(10, cols)
    ref, _, _, bound, _, _ = reference(x, w, c, 1e-5)
    y, mean, rstd = ops().layer_norm_forward(x, w, c, out=x)
    assert y.data_ptr() == x.data_ptr()
    check(y, ref, bound, "y")
    wide[:, :, shift:shift + cols] = before[:, :, shift:shift + cols]
    assert torch.equal(wide, before), "written outside the rows"
    g = normal(11, 40, 3, 160 + shift, dtype=torch.bfloat16)[:, :, shift:shift + cols]
    want = backward_reference(g, x, w, mean, rstd)
    dx, dw, _ = ops().layer_norm_backward(g, x, w, mean, rstd, out=g)
    check(dx, want[0], want[3], "dx")
    check(dw, want[1], want[4], "dweight")


def test_rows_far_from_zero_and_constant_rows():
    x = normal(12, 64, 1024, scale=1e-2) + 1000.0
    x[7] = 3.25
    w, c = torch.ones(1024, device="cuda"), torch.zeros(1024, device="cuda")
    y, mean, rstd = ops().layer_norm_forward(x, w, c)
    ref, m, r, bound, m_bound, _ = reference(x, w, c, 1e-5)
    check(mean, m, m_bound, "mean")
    check(y, ref, bound, "y")
    assert (y[7] == 0).all()


def test_what_is_not_finite_stays_in_its_row():
    x, w, c = normal(13, 9, 96), normal(14, 96), normal(15, 96)
    clean, _, _ = ops().layer_norm_forward(x, w, c)
    x[4, 17] = float("inf")
    x[6, 3] = float("nan")
    y, _, _ = ops().layer_norm_forward(x, w, c)
    keep = torch.tensor([i for i in range(9) if i not in (4, 6)])
    assert torch.equal(y[keep], clean[keep])
    assert y[4].isnan().all() and y[6].isnan().all()


def test_gradient_against_differences():
    rows, cols, step = 6, 48, 1e-2
    x, w, c = normal(16, rows, cols), normal(17, cols), normal(18, cols)
    g = normal(19, rows, cols)

    def loss(x, w, c):
        return (ops().layer_norm_forward(x, w, c)[0].double() * g.double()).sum()

    _, mean, rstd = ops().layer_norm_forward(x, w, c)
    grads = ops().layer_norm_backward(g, x, w, mean, rstd)
    for i, (to, d) in enumerate(zip(grads, (normal(20, rows, cols), normal(21, cols),
                                            normal(22, cols)))):
        at = [x, w, c]
        values = []
        for sign in (1, -1):
            moved = list(at)
            moved[i] = moved[i] + sign * step * d
            values.append(loss(*moved))
        slope = (values[0] - values[1]) / (2 * step)
        along = (to.double() * d.double()).sum()
        # the third derivative along a unit-size direction over cubes of step, and
        # roundings of 2^-24 of the loss's terms over the step
        room = step ** 2 * 10 * to.double().norm() * d.double().norm() + \
            U32 * 10 / step * (g.abs() * 3).double().sum()
        assert abs(slope - along) <= room
        assert room < 0.2 * to.double().norm() * d.double().norm()


def test_equal_inputs_give_equal_bits():
    x, w, c = normal(23, 30000, 128, dtype=torch.bfloat16), normal(24, 128), normal(25, 128)
    _, mean, rstd = ops().layer_norm_forward(x, w, c)
    first = ops().layer_norm_backward(x, x, w, mean, rstd)
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in
                   zip(first, ops().layer_norm_backward(x, x, w, mean, rstd)))


def test_another_stream():
    x, w, c = normal(26, 20000, 256), normal(27, 256), normal(28, 256)
    want = ops().layer_norm_forward(x, w, c)
    want_back = ops().layer_norm_backward(x, x, w, want[1], want[2])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = ops().layer_norm_forward(x, w, c)
        got_back = ops().layer_norm_backward(x, x, w, got[1], got[2])
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want + want_back, got + got_back))


def test_refusals():
    from paper_2207_10731_gb300 import binding
    x, w = normal(29, 4, 32), normal(30, 32)
    fwd, back = ops().layer_norm_forward, ops().layer_norm_backward
    with pytest.raises(ValueError):
        fwd(x.cpu(), w, w)
    with pytest.raises(TypeError):
        fwd(x.double(), w, w)
    with pytest.raises(TypeError):
        fwd(x, w.half(), w)
    with pytest.raises(ValueError):
        fwd(x, w[:31], w)
    with pytest.raises(ValueError):
        fwd(x.t(), w[:4].contiguous(), w[:4].contiguous())
    with pytest.raises(ValueError):
        fwd(x, w, w, out=torch.empty(4, 31, device="cuda"))
    with pytest.raises(ValueError):
        fwd(x[:1].expand(4, 32), w, w)
    with pytest.raises(TypeError):
        back(x, x, w, w[:4].contiguous(), w[:4].contiguous(), out=x.half())
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(binding.PSSError) as e:
            fwd(x, w, w, eps=eps)
        assert e.value.status == binding.PSS_ERR_INVALID_ARG
    big = torch.zeros(1, 16385, device="cuda")
    with pytest.raises(binding.PSSError) as e:
        fwd(big, big[0], big[0])
    assert e.value.status == binding.PSS_ERR_UNSUPPORTED


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 5), (2, 3), (9, 13), (300, 333), (130, 1001), (40, 8191), (20, 12001)])
def test_odd_rows_read_nothing_of_their_neighbours(kind, rows, cols):
    # every row between NaN rows and NaN margins: only its own values may count
    wide = torch.full((2 * rows + 1, cols), float("nan"), dtype=TYPES[kind], device="cuda")
    x = wide[1::2]
    x.copy_(normal(31, rows, cols).to(TYPES[kind]))
    gwide = torch.full_like(wide, float("nan"))
    g = gwide[1::2]
    g.copy_(normal(32, rows, cols).to(TYPES[kind]))
    w, c = normal(33, cols), normal(34, cols)
    out = torch.full_like(wide, 5.0)
    y, mean, rstd = ops().layer_norm_forward(x, w, c, out=out[1::2])
    ref, _, _, bound, _, _ = reference(x, w, c, 1e-5)
    check(y, ref, bound, "y")
    assert (out[::2] == 5).all()
    want = backward_reference(g, x, w, mean, rstd)
    dx, dw, db = ops().layer_norm_backward(g, x, w, mean, rstd, out=out[1::2])
    check(dx, want[0], want[3], "dx")
    check(dw, want[1], want[4], "dweight")
    check(db, want[2], want[5], "dbias")
    assert (out[::2] == 5).all()
