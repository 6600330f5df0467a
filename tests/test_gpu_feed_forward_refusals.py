"""What is no tensor is refused as such, by its name, wherever the feed-forward half's calls take
one."""
import pytest
import torch

from paper_2207_10731_gb300 import sequence
from tests.seq_util import normal

pytestmark = pytest.mark.gpu


def calls():
    x, w = normal(1, 6, 16, dtype=torch.bfloat16), normal(2, 16, 16, dtype=torch.bfloat16)
    b, r = normal(3, 16), normal(4, 6)
    ids = torch.arange(6, device="cuda")
    f, g = sequence.linear_forward, sequence.linear_backward
    n, m = sequence.residual_norm_forward, sequence.residual_norm_backward
    e, d = sequence.embedding_forward, sequence.embedding_backward
    kind = torch.bfloat16
    return {
        "x": lambda v: f(v, w), "weight": lambda v: f(x, v), "bias": lambda v: f(x, w, v),
        "residual": lambda v: f(x, w, residual=v), "out": lambda v: f(x, w, out=v),
        "out ": lambda v: f(x, w, out=v, out_dtype=kind), "grad": lambda v: g(v, x, w),
        "z": lambda v: g(x, x, w, v, "gelu"), "dx": lambda v: g(x, x, w, dx=v),
        "dweight": lambda v: g(x, x, w, dweight=v), "dweight ": lambda v: g(x, x, w, dweight=v, dweight_dtype=kind),
        "dbias": lambda v: g(x, x, w, dbias=v), "status": lambda v: f(x, w, status=v),
        "residual ": lambda v: n(x, v, b, b), "post_weight": lambda v: n(x, x, v, b), "gate": lambda v: n(x, x, b, b, v),
        "total": lambda v: n(x, x, b, b, total=v), "y": lambda v: n(x, x, b, b, y=v),
        "grad_y": lambda v: m(x, v, x, x, r, r, b, b), "gate ": lambda v: m(x, x, x, x, r, r, b, b, v),
        "dgate": lambda v: m(x, x, x, x, r, r, b, b, x, dgate=v), "pre_rstd": lambda v: m(x, x, x, x, r, v, b, b),
        "weight ": lambda v: e(v, ids), "ids": lambda v: e(w, v), "out  ": lambda v: e(w, ids, out=v),
        "out   ": lambda v: e(w, ids, out=v, out_dtype=kind), "grad ": lambda v: d(v, ids, 16),
        "out    ": lambda v: d(x, ids, 16, out=v), "out     ": lambda v: d(x, ids, 16, out=v, out_dtype=kind),
    }


@pytest.mark.parametrize("value", [3.5, "x", (1, 2)], ids=str)
def test_what_is_no_tensor(value):
    for name, call in calls().items():
        with pytest.raises(TypeError, match=f"{name.strip()} must be a torch.Tensor"):
            call(value)
