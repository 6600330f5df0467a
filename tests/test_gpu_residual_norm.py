"""The norms after and before a block with its gate and residual, against the definition
in 64 bits and against differences.

Tolerances, in units U = 2^-24: a row's sum runs along at most 16 additions of a thread and
11 between threads, so it is off by less than 32 U of the sum of its terms' sizes and r(v) by
20 U; sigmoid goes through one exponential (documented at 2 + 1.2 |g| units in the last place, 2 U
each) and a division (2 units): 12 + 2.4 |g| in U; a weight's sum over R rows, along at most R
additions and 64 between groups and CTAs."""
import pytest
import torch

from paper_2207_10731_gb300 import binding, sequence
from tests.seq_util import TYPES, U32, check, normal

pytestmark = pytest.mark.gpu

EPS = 1e-5
F32 = torch.float32


def rows_of(seed, rows, cols, gap, dtype, scale=1.0):
    """Rows cut out of wider ones; a gap of 5 leaves them off every 16-byte boundary."""
    return normal(seed, rows, cols + gap, dtype=dtype, scale=scale)[:, gap:] if gap else \
        normal(seed, rows, cols, dtype=dtype, scale=scale)


def inputs(rows, cols, kind, stream, post, pre, gates, gap):
    t, r = TYPES[kind], TYPES[stream]
    d = {"x": rows_of(1, rows, cols, gap, t, 1.5), "residual": rows_of(2, rows, cols, gap, r),
         "post": 1 + normal(3, cols, scale=0.3) if post else None,
         "pre": 1 + normal(4, cols, scale=0.3) if pre else None,
         "gate": {0: None, 1: rows_of(5, rows, 1, gap, t, 3.0),
                  2: rows_of(6, rows, cols, gap, t, 3.0)}[gates],
         "grad_total": rows_of(7, rows, cols, gap, r), "grad_y": None}
    if pre:
        d["grad_y"] = rows_of(8, rows, cols, gap, t)
    return d


def size(gate):
    """|gate| up to 128: past 104 the exponential is below the smallest fp32 number, so that the
    value is 0 or 1 (or its error at most the value itself, which check()'s floor covers), and a
    bound made from an infinite gate would be NaN."""
    return gate.abs().clamp(max=128)


def rstd_of(v):
    return (v.square().mean(-1, keepdim=True) + EPS) ** -0.5


def forward(d, scale):
    """[(name, value, bound)] of a forward call."""
    x = d["x"].double()
    u, err, answer = x, 0.0, []
    post = rstd_of(x)
    if d["post"] is not None:
        u, err = x * post * d["post"].double(), 24.0
    open_ = 1.0
    if d["gate"] is not None:
        g = d["gate"].double()
        open_, err = torch.sigmoid(g), err + 14 + 2.4 * size(g)
    r = d["residual"].double()
    add = scale * open_ * u
    total = r + add
    bt = U32 * ((err + 3) * add.abs() + total.abs())
    answer.append(("total", total, bt))
    pre = rstd_of(total)
    off = (bt.square().sum(-1, keepdim=True) / total.square().sum(-1, keepdim=True)).sqrt()
    if d["pre"] is not None:
        w = d["pre"].double()
        y = total * pre * w
        answer.append(("y", y, pre * w.abs() * bt + y.abs() * (off + 24 * U32)))
    else:
        answer.append(None)
    answer.append(("post_rstd", post[..., 0], post[..., 0] * 20 * U32) if d["post"] is not None else None)
    answer.append(("pre_rstd", pre[..., 0], pre[..., 0] * (20 * U32 + off[..., 0]))
                  if d["pre"] is not None else None)
    return answer


def backward(d, total, post, pre, scale):
    dt = d["grad_total"].double() if d["grad_total"] is not None else torch.zeros_like(total).double()
    dv, bd = dt, dt.abs() * U32
    dpre = dpost = dgate = None
    rows = total.shape[0]
    depth = (rows + 64) * U32
    mean = lambda v: v.mean(-1, keepdim=True)   # noqa: E731
    if d["pre"] is not None:
        r = pre.double()[:, None]
        that, gy = total.double() * r, d["grad_y"].double()
        g = gy * d["pre"].double()
        along = mean(g * that)
        dv = dt + (g - that * along) * r
        bd = U32 * (2 * dt.abs() + r * (6 * g.abs() + that.abs() * 44 * mean((g * that).abs())))
        dpre = ((gy * that).sum(0), ((gy * that).abs() * depth * 2).sum(0))
    x = d["x"].double()
    hat, w = x, 1.0
    if d["post"] is not None:
        hat, w = x * post.double()[:, None], d["post"].double()
    open_, slope, err = torch.ones_like(x[:, :1]), 0.0, 0.0
    e = scale * dv
    be = abs(scale) * bd + e.abs() * U32
    if d["gate"] is not None:
        gate = d["gate"].double()
        open_, err = torch.sigmoid(gate), (14 + 2.4 * size(gate)) * U32
        slope = open_ * torch.sigmoid(-gate)
        each = e * hat * w
        room = be * (hat * w).abs() + 4 * U32 * each.abs()
        if gate.shape[1] == 1 and x.shape[1] > 1 or x.shape[1] == 1:
            sum_, room = each.sum(-1, keepdim=True), (room + 40 * U32 * each.abs()).sum(-1, keepdim=True)
        else:
            sum_ = each
        dgate = (sum_ * slope, room * slope + (sum_ * slope).abs() * (2 * err + 8 * U32))
    be = be * open_ + (e * open_).abs() * (err + 2 * U32)
    e = e * open_
    dx, bx = e, be
    if d["post"] is not None:
        r = post.double()[:, None]
        h, bh = e * w, be * w.abs() + (e * w).abs() * U32
        along = mean(h * hat)
        dx = r * (h - hat * along)
        bx = r * (bh + hat.abs() * (mean(hat.abs() * bh) + 44 * U32 * mean((h * hat).abs()))) + \
            6 * U32 * r * (h.abs() + (hat * along).abs())
        dpost = ((e * hat).sum(0), (be * hat.abs() + (e * hat).abs() * depth * 2).sum(0))
    return [(dx, bx), (dv, bd), dgate, dpost, dpre]


CASES = [
    # rows, cols, type, stream, post, pre, gates
    (1, 1, "f32", "f32", 1, 1, 2), (3, 7, "bf16", "f32", 1, 1, 1), (8, 1024, "bf16", "bf16", 1, 1, 0),
    (37, 64, "f16", "f16", 1, 1, 2), (1000, 100, "f16", "f32", 1, 1, 2), (301, 129, "bf16", "bf16", 1, 1, 1),
    (77, 256, "f32", "f32", 1, 1, 2), (77, 257, "bf16", "f32", 1, 1, 2), (2000, 16, "bf16", "bf16", 1, 1, 2),
    (333, 512, "f16", "f32", 0, 1, 0), (333, 520, "f16", "f16", 1, 0, 2), (41, 1000, "bf16", "f32", 0, 0, 2),
    (41, 1001, "f32", "f32", 0, 1, 1), (700, 2048, "bf16", "bf16", 1, 1, 2), (19, 4096, "bf16", "f32", 1, 1, 2),
    (19, 4104, "f16", "f32", 1, 1, 2), (23, 5001, "bf16", "bf16", 1, 1, 1), (5, 8192, "f32", "f32", 1, 1, 2),
    (7, 16384, "bf16", "f32", 1, 1, 2), (6, 16381, "f16", "f16", 1, 1, 2), (50, 48, "f32", "f32", 0, 0, 0),
    (501, 505, "bf16", "bf16", 1, 1, 2), (501, 300, "f16", "f32", 1, 1, 1), (130, 512, "bf16", "bf16", 1, 1, 2),
]


def sames(got, want):
    return all((a is None) == (b is None) and (a is None or torch.equal(a, b)) for a, b in zip(got, want))


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("gap", [0, 8, 5])
def test_against_the_definition(case, gap):
    rows, cols, kind, stream, post, pre, gates = case
    d, scale = inputs(rows, cols, kind, stream, post, pre, gates, gap), 0.625
    more = dict(post_weight=d["post"], pre_weight=d["pre"], gate=d["gate"], scale=scale)
    got = sequence.residual_norm_forward(d["x"], d["residual"], eps=EPS, **more)
    for g, w in zip(got, forward(d, scale)):
        assert (g is None) == (w is None)
        if w is not None:
            check(g, w[1], w[2], w[0])
    total, _, post_rstd, pre_rstd = got
    back = sequence.residual_norm_backward(d["grad_total"], d["grad_y"], d["x"], total, post_rstd,
                                           pre_rstd, **more)
    want = backward(d, total, post_rstd, pre_rstd, scale)
    for name, g, w in zip(("dx", "dresidual", "dgate", "dpost", "dpre"), back, want):
        assert (g is None) == (w is None), name
        if w is not None:
            check(g, w[0], w[1], name)
    assert sames(back, sequence.residual_norm_backward(
        d["grad_total"], d["grad_y"], d["x"], total, post_rstd, pre_rstd, **more))
    if pre:   # nothing else reads the stream
        d["grad_total"] = None
        back = sequence.residual_norm_backward(None, d["grad_y"], d["x"], total, post_rstd, pre_rstd, **more)
        for name, g, w in zip(("dx", "dresidual", "dgate", "dpost", "dpre"), back,
                              backward(d, total, post_rstd, pre_rstd, scale)):
            if w is not None:
                check(g, w[0], w[1], name + " of y alone")


@pytest.mark.parametrize("gates", [0, 1, 2])
def test_gradients_against_differences(gates):
    """Of the 64-bit definition that the kernel's gradients are compared with above."""
    d = {k: v.double() if v is not None else None
         for k, v in inputs(6, 40, "f32", "f32", 1, 1, gates, 0).items()}
    scale = 0.75
    fw = forward(d, scale)
    total, post, pre = (fw[i][1] for i in (0, 2, 3))
    want = backward(d, total, post, pre, scale)
    names = ["x", "residual", "gate", "post", "pre"]

    def loss():
        got = forward(d, scale)
        return (got[0][1] * d["grad_total"]).sum() + (got[1][1] * d["grad_y"]).sum()
    for name, w in zip(names, want):
        if w is None:
            continue
        way = normal(9, *d[name].shape).double()
        at, h = d[name], 1e-6
        d[name] = at + h * way
        up = loss()
        d[name] = at - h * way
        down = loss()
        d[name] = at
        slope = (up - down) / (2 * h)
        # third derivative times h^2, and 2^-52 of the loss over h
        assert abs(slope - (w[0] * way).sum()) < 1e-6 * (1 + abs(slope)), name


@pytest.mark.parametrize("cols", [64, 333, 2048])
def test_in_place(cols):
    d = inputs(90, cols, "bf16", "bf16", 1, 1, 2, 0)
    more = dict(post_weight=d["post"], pre_weight=d["pre"], gate=d["gate"])
    want = sequence.residual_norm_forward(d["x"], d["residual"], **more)
    x, residual = d["x"].clone(), d["residual"].clone()
    got = sequence.residual_norm_forward(x, residual, total=residual, y=x, **more)
    assert got[0] is residual and got[1] is x and sames(got, want)
    total, _, a, b = want
    want = sequence.residual_norm_backward(d["grad_total"], d["grad_y"], d["x"], total, a, b, **more)
    gt, gy, gate = d["grad_total"].clone(), d["grad_y"].clone(), d["gate"].clone()
    more["gate"] = gate
    got = sequence.residual_norm_backward(gt, gy, d["x"], total, a, b, dx=gy, dresidual=gt, dgate=gate, **more)
    assert got[0] is gy and got[1] is gt and got[2] is gate and sames(got, want)


def test_large_gates_and_rows_that_are_not_finite():
    d = inputs(64, 96, "f32", "f32", 1, 1, 2, 0)
    d["gate"][0], d["gate"][1], d["gate"][2] = 60.0, -60.0, -200.0
    d["gate"][3], d["gate"][4] = float("inf"), -float("inf")
    d["x"][10, 3], d["residual"][11, 4], d["x"][12], d["residual"][13] = float("nan"), float("inf"), 0.0, 0.0
    d["x"][13] = 0.0
    more = dict(post_weight=d["post"], pre_weight=d["pre"], gate=d["gate"])
    total, y, a, b = sequence.residual_norm_forward(d["x"], d["residual"], **more)
    back = sequence.residual_norm_backward(d["grad_total"], d["grad_y"], d["x"], total, a, b, **more)
    fine = torch.ones(64, dtype=torch.bool, device="cuda")
    fine[[10, 11]] = False
    for t in (total, y, back[0], back[1], back[2]):
        assert t[fine].isfinite().all()
    assert total[10].isnan().all() and total[11, 4] == float("inf")
    assert torch.equal(total[[2, 4]], d["residual"][[2, 4]]) and not total[13].any() and not y[13].any()
    some = {k: v[fine] if v is not None and v.dim() == 2 else v for k, v in d.items()}
    want = backward(some, total[fine], a[fine], b[fine], 1.0)
    check(back[0][fine], *want[0], "dx")
    far = [3, 4]   # the slope of a gate at infinity
    assert not back[2][far].any()


def test_empty_streams_and_graphs():
    d = inputs(0, 24, "bf16", "f32", 1, 1, 2, 0)
    more = dict(post_weight=d["post"], pre_weight=d["pre"], gate=d["gate"])
    total, y, a, b = sequence.residual_norm_forward(d["x"], d["residual"], **more)
    back = sequence.residual_norm_backward(d["grad_total"], d["grad_y"], d["x"], total, a, b, **more)
    assert total.shape == y.shape == (0, 24) and not back[3].any() and not back[4].any()
    d = inputs(20000, 512, "bf16", "f32", 1, 1, 2, 0)
    more = dict(post_weight=d["post"], pre_weight=d["pre"], gate=d["gate"])

    def calls(**kw):
        got = sequence.residual_norm_forward(d["x"], d["residual"], **more, **kw)
        return got + sequence.residual_norm_backward(d["grad_total"], d["grad_y"], d["x"], got[0], *got[2:],
                                                     **more, **kw)
    want = calls()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    torch.cuda._sleep(300_000_000)
    got = calls(stream=side)
    side.synchronize()
    assert not torch.cuda.current_stream().query()
    torch.cuda.synchronize()
    assert sames(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls()
    d["x"].copy_(normal(21, 20000, 512, dtype=torch.bfloat16))
    graph.replay()
    torch.cuda.synchronize()
    assert sames(got, calls())


def test_refusals():
    d = inputs(4, 16, "bf16", "f32", 1, 1, 2, 0)
    x, r, w, g = d["x"], d["residual"], d["post"], d["gate"]
    f, b = sequence.residual_norm_forward, sequence.residual_norm_backward
    ones = torch.ones(4, device="cuda")
    for error, call in [
            (TypeError, lambda: f(x.double(), r)), (TypeError, lambda: f(x, r.half(), w, w)),
            (ValueError, lambda: f(x, r[:3], w, w)), (ValueError, lambda: f(x.cpu(), r, w, w)),
            (ValueError, lambda: f(x, r, w[:8], w)), (TypeError, lambda: f(x, r, w.half(), w)),
            (TypeError, lambda: f(x, r, w, w, g.float())), (ValueError, lambda: f(x, r, w, w, g[:, :3])),
            (ValueError, lambda: f(x, r, w, None, y=x)), (TypeError, lambda: f(x, r, w, w, total=x)),
            (binding.PSSError, lambda: f(x, r, w, w, eps=-1.0)),
            (binding.PSSError, lambda: f(x, r, w, w, scale=float("nan"))),
            (binding.PSSError, lambda: f(*(normal(1, 2, 16385) for _ in range(2)))),
            (ValueError, lambda: b(r, None, x, r, ones, ones, w, w)),
            (ValueError, lambda: b(r, x, x, r, ones, ones[:2], w, w)),
            (ValueError, lambda: b(r, x, x, r, ones, ones, w, w, dgate=g)),
            (TypeError, lambda: b(x, x, x, r, ones, ones, w, w)),
            (TypeError, lambda: b(r, x, x, r, ones, ones, w, w, dresidual=x))]:
        with pytest.raises(error):
            call()
