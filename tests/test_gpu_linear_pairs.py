"""Products by pairs of CTAs between kernels that take their SMs at once: short contractions, whose
last loads, products and arrivals come close to the CTAs' end, give the bits that they give
alone."""
import pytest
import torch

from paper_2207_10731_gb300 import sequence
from tests.seq_util import normal
from tests.test_gpu_linear import check, forward

pytestmark = pytest.mark.gpu

# tokens, in, out: one to seven blocks of the contraction, tiles of 160 to 256 columns, fewer
# tiles than pairs and several to a pair
SHORT = [(1500, 64, 2096), (3620, 48, 712), (2233, 72, 1648), (9000, 16, 1024), (300, 8, 200),
         (5000, 448, 520), (20000, 128, 3328)]


def test_pairs_between_other_kernels():
    kind = torch.bfloat16
    calls = [(normal(i, t, n, dtype=kind), normal(50 + i, n, m, dtype=kind, scale=n ** -0.5))
             for i, (t, n, m) in enumerate(SHORT)]
    few = normal(90, 3, 512, dtype=kind), normal(91, 512, 264, dtype=kind)
    rows, ones = normal(92, 4000, 256), torch.ones(256, device="cuda")

    def others():
        return [sequence.linear_forward(*few),
                sequence.layer_norm_forward(rows, ones, ones, out_dtype=kind)[0]]
    alone = []
    for x, w in calls:
        y = sequence.linear_forward(x, w)
        torch.cuda.synchronize()
        dx, dw, _ = sequence.linear_backward(y, x, w, dbias=False)
        torch.cuda.synchronize()
        alone.append((y, dx, dw))
        (wy, by), _ = forward(x, w, None, None, None)
        check(y, wy, by, "y")
    want = others()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for turn in range(20):
        got, more = [], []
        for x, w in calls:
            y = sequence.linear_forward(x, w)
            more.append(sequence.linear_forward(x, w, stream=side))
            more += others()
            got.append((y, *sequence.linear_backward(y, x, w, dbias=False)[:2]))
        torch.cuda.synchronize()
        for a, b in zip(got, alone):
            assert all(torch.equal(p, q) for p, q in zip(a, b)), turn
        for i, (y, _, _) in enumerate(alone):
            assert torch.equal(more[3 * i], y) and torch.equal(more[3 * i + 1], want[0])
            assert torch.equal(more[3 * i + 2], want[1])
