"""The norms' backward on rows of fp32 off the 16-byte grid, whose last 32 bytes hold four values or
fewer: nothing is copied for the other 16 bytes, and what lies between the rows reaches
nothing."""
import pytest
import torch

from paper_2207_10731_gb300 import sequence
from tests.seq_util import TYPES, check, normal
from tests.test_gpu_residual_norm import EPS, backward

pytestmark = pytest.mark.gpu


def rows_of(seed, rows, cols, gap, dtype):
    """Rows with NaN before and after them, none at a multiple of 8 values but every eighth."""
    t = torch.full((rows, cols + gap), float("nan"), dtype=dtype, device="cuda")
    t[:, 1:cols + 1] = normal(seed, rows, cols, dtype=dtype)
    return t[:, 1:cols + 1]


# a lane's vector, two, a CTA of up to 256 and of up to 512 threads to a row
@pytest.mark.parametrize("cols", [3, 34, 250, 252, 257, 331, 490, 1002, 2010, 2500, 4001])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_short_last_vectors(cols, kind):
    gap = 8 - (cols + 5) % 8 + 2          # rows an odd number of values apart
    gap += (cols + gap) % 2 == 0
    rows, kind, f32 = 41, TYPES[kind], torch.float32
    d = {"x": rows_of(1, rows, cols, gap, kind), "gate": rows_of(2, rows, cols, gap, kind),
         "post": normal(3, cols), "pre": normal(4, cols), "grad_y": rows_of(5, rows, cols, gap, kind),
         "grad_total": rows_of(6, rows, cols, gap, f32), "residual": rows_of(7, rows, cols, gap, f32)}
    total = torch.full((rows, cols + gap), float("nan"), device="cuda")[:, 1:cols + 1]
    outs = [torch.full((rows, cols + gap), 9.0, dtype=t, device="cuda") for t in (kind, f32, kind)]
    dx, dresidual, dgate = (t[:, 1:cols + 1] for t in outs)
    more = dict(post_weight=d["post"], pre_weight=d["pre"], gate=d["gate"], scale=0.625)
    _, _, post_rstd, pre_rstd = sequence.residual_norm_forward(d["x"], d["residual"], eps=EPS, total=total,
                                                               **more)
    back = sequence.residual_norm_backward(d["grad_total"], d["grad_y"], d["x"], total, post_rstd, pre_rstd,
                                           dx=dx, dresidual=dresidual, dgate=dgate, **more)
    want = backward(d, total, post_rstd, pre_rstd, 0.625)
    for name, g, w in zip(("dx", "dresidual", "dgate", "dpost", "dpre"), back, want):
        check(g, w[0], w[1], name)
    for t in outs:
        assert (t[:, 0] == 9).all() and (t[:, cols + 1:] == 9).all()
