"""Products with bias, activation and residual, and their gradients, against the definition in
64 bits.

Tolerances, U = 2^-24: a sum of k products is made in fp32, in any order, the tensor core
cutting where a sum is rounded: k * 2 U of the sum of the products' sizes S.  An activation passes
an error of z on with at most its largest slope (1.13) and adds its own: the exponential
2 + 1.2 |z| units in the last place (2 U each) and erfc and the quotient a few.  The gradient
through an activation enters the products with one rounding more, h = 2^-8 or 2^-11, of each
term: h S."""
import math

import pytest
import torch

from paper_2207_10731_gb300 import binding, sequence
from tests.seq_util import TYPES, U32, UNIT, check, normal

pytestmark = pytest.mark.gpu


def cut(seed, rows, cols, gap, dtype, scale=1.0):
    return normal(seed, rows, cols + gap, dtype=dtype, scale=scale)[:, gap // 2:cols + gap // 2]


def phi(z):
    """By erfc, which keeps its relative accuracy below zero (special.ndtr is 0 from -9 on, where
    Phi is 1.1e-19)."""
    return 0.5 * torch.special.erfc(-z * math.sqrt(0.5))


def act(z, name):
    return {None: lambda: z, "relu": lambda: z.clamp(min=0), "gelu": lambda: z * phi(z),
            "silu": lambda: z * torch.sigmoid(z)}[name]()


def slope(z, name):
    if name is None:
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return phi(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(z)
    return s + z * s * torch.sigmoid(-z)


def own_error(z, name):
    """Of an activation (or of its slope, over z): units in the last place of its parts."""
    return (24 + 4 * z.abs().clamp(max=128).square()) * U32 if name in ("gelu", "silu") else 0 * z


def forward(x, w, bias, name, residual):
    """((y, bound), (z, bound))."""
    x, w = x.double(), w.double()
    k = x.shape[-1]
    z, size = x @ w, x.abs() @ w.abs()
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    bz = 2 * (k + 2) * U32 * size
    y = act(z, name)
    by = (1.13 if name else 1.0) * bz + (y.abs() + z.abs() * U32) * own_error(z, name)
    if residual is not None:
        y = y + residual.double()
        by = by + U32 * y.abs() + U32 * residual.double().abs()
    return (y, by), (z, bz)


def backward(grad, x, w, z, name, narrow):
    """[(dx, bound), (dweight, bound), (dbias, bound)]; narrow: dz is rounded for the products."""
    g, x, w = grad.double(), x.double(), w.double()
    n, m = w.shape
    t = g.shape[0]
    bd = 0 * g
    if name:
        z = z.double()
        bd = g.abs() * (slope(z, name).abs() + z.abs() * torch.exp(-z * z / 8) + 2.0 ** -20) * own_error(z, name)
        g = g * slope(z, name)
    h = UNIT[x_type(narrow)] if narrow else 0.0
    each = bd + (g.abs() + bd) * (h + 2 * U32) + (2.0 ** -25 if narrow is torch.float16 else 0)
    dx = g @ w.t(), each @ w.abs().t() + 2 * (m + 2) * U32 * (g.abs() @ w.abs().t())
    dw = x.t() @ g, x.abs().t() @ each + 2 * (t + 2) * U32 * (x.abs().t() @ g.abs())
    db = g.sum(0), bd.sum(0) + (t + 64) * U32 * g.abs().sum(0)
    return [dx, dw, db]


def x_type(t):
    return t


CASES = [
    # tokens, in, out, type, activation, bias, residual, wide (result in fp32)
    (1, 1, 1, "bf16", None, 1, 0, 0), (1, 64, 128, "f16", "silu", 1, 1, 0), (1, 4096, 520, "bf16", "gelu", 1, 0, 1),
    (7, 333, 129, "f16", "gelu", 1, 1, 0), (32, 128, 64, "bf16", "relu", 0, 0, 0), (33, 72, 1000, "f16", None, 0, 1, 1),
    (64, 512, 257, "bf16", "silu", 1, 1, 0), (65, 512, 256, "bf16", "silu", 1, 1, 0), (127, 1000, 40, "f16", "gelu", 1, 0, 0),
    (129, 63, 65, "bf16", "relu", 1, 1, 1), (300, 16, 8, "bf16", "gelu", 0, 1, 0), (1000, 200, 300, "f16", "silu", 1, 1, 1),
    (2000, 8, 777, "bf16", None, 1, 1, 0), (513, 1025, 511, "bf16", "gelu", 1, 1, 0), (4097, 320, 96, "f16", "relu", 1, 0, 0),
    (3000, 256, 1024, "bf16", None, 0, 0, 0), (20000, 64, 64, "bf16", "gelu", 1, 0, 0), (257, 2048, 3, "f16", None, 1, 1, 0),
    # tiles of 192, 160 and 224 columns, whose last 32 go another way
    (1500, 64, 2096, "bf16", "gelu", 1, 1, 0), (3620, 48, 712, "f16", "silu", 1, 1, 0), (2233, 72, 1648, "bf16", None, 1, 1, 1),
    (2233, 72, 1648, "f16", "relu", 1, 0, 0), (1000, 1024, 4096, "bf16", None, 1, 0, 0),
]


def make(case, gap, dense):
    t, n, m, kind, name, bias, residual, wide = case
    kind = TYPES[kind]
    d = {"x": cut(1, t, n, gap, kind), "bias": normal(3, m) if bias else None,
         "residual": cut(4, t, m, gap, torch.float32 if wide else kind) if residual else None,
         "grad": cut(5, t, m, gap, torch.float32 if wide else kind)}
    w = cut(2, n, m, gap, kind, n ** -0.5) if dense == "out" else cut(2, m, n, gap, kind, n ** -0.5).t()
    return dict(d, weight=w, activation=name, out_dtype=torch.float32 if wide else kind)


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("gap", [0, 8, 6])
@pytest.mark.parametrize("dense", ["out", "in"])
def test_against_the_definition(case, gap, dense):
    d = make(case, gap, dense)
    t, n, m = case[:3]
    name, x, w = d["activation"], d["x"], d["weight"]
    status = torch.full((1,), 5, device="cuda")
    wide = torch.full((t, m + gap), 9.0, dtype=d["out_dtype"], device="cuda")
    got = sequence.linear_forward(x, w, d["bias"], name, d["residual"], keep=name is not None,
                                  out=wide[:, :m], status=status)
    y, z = got if name else (got, None)
    (wy, by), (wz, bz) = forward(x, w, d["bias"], name, d["residual"])
    check(y, wy, by, "y")
    if name:
        check(z, wz, bz, "z")
    assert (wide[:, m:] == 9).all() and int(status) == -1
    again = sequence.linear_forward(x, w, d["bias"], name, d["residual"], out_dtype=d["out_dtype"])
    assert torch.equal(again, y)
    narrow = x.dtype if name or d["grad"].dtype == torch.float32 else None
    want = backward(d["grad"], x, w, z, name, narrow)
    back = sequence.linear_backward(d["grad"], x, w, z, name, status=status.fill_(5))
    for what, g, v in zip(("dx", "dweight", "dbias"), back, want):
        check(g, v[0], v[1], what)
    assert int(status) == -1 and back[1].stride() == (w.stride() if gap == 0 else back[1].stride())
    back2 = sequence.linear_backward(d["grad"], x, w, z, name, dx=False, dbias=False,
                                     dweight_dtype=torch.float32)
    assert back2[0] is None and back2[2] is None
    check(back2[1], *want[1], "dweight in fp32")
    room = torch.full((t, n + gap), 9.0, dtype=x.dtype, device="cuda")
    back2 = sequence.linear_backward(d["grad"], x, w, z, name, dx=room[:, :n], dweight=False)
    assert torch.equal(back2[0], back[0]) and back2[1] is None and torch.equal(back2[2], back[2])
    assert (room[:, n:] == 9).all()


def test_long_contractions_and_large_results():
    x, w = normal(1, 200, 70000, dtype=torch.bfloat16), normal(2, 70000, 24, dtype=torch.bfloat16)
    (wy, by), _ = forward(x, w, None, None, None)
    check(sequence.linear_forward(x, w, out_dtype=torch.float32), wy, by, "y")
    # a result past 2^32 values: its first, last and some rows between
    x, w = normal(3, 1100001, 16, dtype=torch.bfloat16), normal(4, 16, 4096, dtype=torch.bfloat16)
    y = sequence.linear_forward(x, w)
    rows = torch.tensor([0, 1, 524287, 524288, 1048575, 1048576, 1048577, 1100000], device="cuda")
    (wy, by), _ = forward(x[rows], w, None, None, None)
    check(y[rows], wy, by, "y")
    _, dw, db = sequence.linear_backward(y, x, w, dx=False)
    want = torch.zeros(16, 4096, dtype=torch.float64, device="cuda")
    size, sums, sizes = want.clone(), want[0].clone(), want[0].clone()
    for i in range(0, x.shape[0], 65536):
        a, b = x[i:i + 65536].double(), y[i:i + 65536].double()
        want += a.t() @ b
        size += a.abs().t() @ b.abs()
        sums += b.sum(0)
        sizes += b.abs().sum(0)
    # parts of the contraction are joined by additions: at most all of their length in one part
    check(dw, want, size * 2 * x.shape[0] * U32, "dweight")
    check(db, sums, sizes * x.shape[0] * U32, "dbias")


def test_shapes_in_place_and_empty():
    x, w, b = normal(1, 3, 5, 96, dtype=torch.bfloat16), normal(2, 96, 40, dtype=torch.bfloat16), normal(3, 40)
    r = normal(4, 3, 5, 40, dtype=torch.bfloat16)
    want = sequence.linear_forward(x, w, b, "gelu", r)
    assert want.shape == (3, 5, 40)
    assert sequence.linear_forward(x, w, b, "gelu", r, out=r) is r and torch.equal(r, want)
    none = x[:0]
    y, z = sequence.linear_forward(none, w, b, "silu", keep=True)
    assert y.shape == z.shape == (0, 5, 40)
    for weight in (w, w.t().contiguous().t()):
        dx, dw, db = sequence.linear_backward(y, none, weight, z, "silu")
        assert dx.shape == none.shape and not dw.any() and not db.any() and dw.shape == w.shape


@pytest.mark.parametrize("name", [None, "relu", "gelu", "silu"])
@pytest.mark.parametrize("tokens", [4, 200])
def test_values_that_are_not_finite_stay_in_their_rows(name, tokens):
    x, w = normal(1, tokens, 128, dtype=torch.bfloat16), normal(2, 128, 192, dtype=torch.bfloat16)
    x[2, 5] = float("nan")
    y, z = sequence.linear_forward(x, w, None, name, keep=True) if name else \
        (sequence.linear_forward(x, w), None)
    fine = torch.arange(tokens, device="cuda") != 2
    assert y[2].isnan().all() and y[fine].isfinite().all()
    dx, dw, db = sequence.linear_backward(y, x, w, z, name)
    assert dx[2].isnan().all() and dx[fine].isfinite().all() and dw.isnan().all() and db.isnan().all()


@pytest.mark.parametrize("name", ["relu", "gelu", "silu"])
def test_activations_far_from_zero(name):
    # one product by one: z is the weight itself
    z = torch.cat([torch.linspace(-300, 300, 4001), torch.linspace(-14, 14, 4001)]).half().cuda()
    one = torch.ones(1, 1, dtype=torch.float16, device="cuda")
    y, kept = sequence.linear_forward(one, z[None], activation=name, keep=True, out_dtype=torch.float32)
    assert torch.equal(kept[0], z)
    w = z.double()
    want = act(w, name)
    # where Phi or the sigmoid is below the smallest normal number, it is held to 2^-149: times |z|
    low = w.abs() * 2.0 ** -148
    check(y[0], want, want.abs() * own_error(w, name) + low, "y")
    g = torch.ones(1, z.numel(), device="cuda")
    _, _, db = sequence.linear_backward(g, one, z[None], kept, name)
    want = slope(w, name)
    # the slope is a sum of two parts that cancel near its zero: the error is that of each part
    s = torch.sigmoid(w)
    part = {"relu": 0 * w, "gelu": phi(w) + w.abs() * torch.exp(-w * w / 2),
            "silu": s + w.abs() * s * torch.sigmoid(-w)}[name]
    if name == "gelu":   # exp(-z^2 / 2) below 2^-126 counts as zero: at most that, and |z| times that
        low = low + (1 + w.abs()) * 2.0 ** -126
    check(db, want, (want.abs() + part) * own_error(w, name) + low, "slope")


@pytest.mark.parametrize("name", ["relu", "gelu", "silu"])
def test_slopes_against_differences(name):
    z = torch.linspace(-6, 6, 1001, dtype=torch.float64) + 0.0003
    h = 1e-5
    assert ((act(z + h, name) - act(z - h, name)) / (2 * h) - slope(z, name)).abs().max() < 1e-8


def test_streams_threads_and_graphs():
    d = make((3000, 512, 768, "bf16", "gelu", 1, 1, 0), 0, "out")
    small = make((3, 1024, 768, "bf16", "gelu", 1, 1, 0), 0, "in")

    def calls(**kw):
        got = ()
        for v in (d, small):
            y, z = sequence.linear_forward(v["x"], v["weight"], v["bias"], "gelu", v["residual"], keep=True, **kw)
            got += (y, z) + sequence.linear_backward(v["grad"], v["x"], v["weight"], z, "gelu", **kw)
        return got
    want = calls()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    torch.cuda._sleep(300_000_000)
    got = calls(stream=side)
    side.synchronize()
    assert not torch.cuda.current_stream().query()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    import threading
    got = []
    threads = [threading.Thread(target=lambda: got.append(calls())) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert len(got) == 2 and all(torch.equal(a, b) for one in got for a, b in zip(one, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls()
    d["x"].copy_(normal(31, 3000, 512, dtype=torch.bfloat16))
    small["weight"].copy_(normal(32, 1024, 768, dtype=torch.bfloat16, scale=0.05))
    for t in got:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, calls()))


def test_refusals():
    x, w, b = normal(1, 6, 16, dtype=torch.bfloat16), normal(2, 16, 24, dtype=torch.bfloat16), normal(3, 24)
    y = sequence.linear_forward(x, w, b)
    f, g = sequence.linear_forward, sequence.linear_backward
    wide = normal(2, 16, 48, dtype=torch.bfloat16)
    for error, call in [
            (TypeError, lambda: f(x.float(), w)), (TypeError, lambda: f(x, w.half())),
            (ValueError, lambda: f(x[:, :8], w)), (ValueError, lambda: f(x, w[0])), (ValueError, lambda: f(x.t(), w)),
            (ValueError, lambda: f(x, w.cpu())), (ValueError, lambda: f(x, w, b[:3])), (TypeError, lambda: f(x, w, b.half())),
            (ValueError, lambda: f(x, w, b, "tanh")), (ValueError, lambda: f(x, w, b, keep=True)),
            (ValueError, lambda: f(x, w, residual=y[:3])), (TypeError, lambda: f(x, w, residual=y.float())),
            (TypeError, lambda: f(x, w, out_dtype=torch.float16)), (ValueError, lambda: f(x, w, out=x)),
            (binding.PSSError, lambda: f(x, wide[:, ::2])), (binding.PSSError, lambda: f(x, w[:1].expand(16, 24))),
            (binding.PSSError, lambda: f(x[:, :0], w[:0])),
            (ValueError, lambda: g(y, x, w, None, "gelu")), (TypeError, lambda: g(y.half(), x, w)),
            (ValueError, lambda: g(y[:, :8], x, w)), (TypeError, lambda: g(y, x, w, dweight_dtype=torch.float16)),
            (ValueError, lambda: g(y, x, w, dweight=w.t())), (ValueError, lambda: g(y, x, w, dx=y)),
            (ValueError, lambda: g(y, x, w, dbias=b[:2])), (TypeError, lambda: g(y, x, w, y.float(), "relu"))]:
        with pytest.raises(error):
            call()
