"""The sequence operators called as programs call them: from a thread that has
not used the GPU before, and inside a captured CUDA graph.  The results are the
same kernels' on the same inputs, so they are compared bit by bit."""
import threading

import pytest
import torch

from paper_2207_10731_gb300 import sequence
from tests.seq_util import normal

pytestmark = pytest.mark.gpu

OFFSETS = [0, 1, 130, 130, 389, 700]


def _calls(x, w, b, q, k, v, g, off):
    """Every operator once; what they return, in a row."""
    y, mean, rstd = sequence.layer_norm_forward(x, w, b, out_dtype=torch.bfloat16)
    dx, dw, db = sequence.layer_norm_backward(x, x, w, mean, rstd)
    z = sequence.dropout(x, 0.25, 7, 3)
    out, lse = sequence.attention_forward(q, k, v, off)
    dq, dk, dv = sequence.attention_backward(g, q, k, v, out, lse, off)
    return y, mean, rstd, dx, dw, db, z, out, lse, dq, dk, dv


def _inputs(seed, dim):
    n = OFFSETS[-1]
    x = normal(seed, 77, 333)
    q, g = (normal(seed + i, n, 4, dim, dtype=torch.bfloat16) for i in (1, 2))
    k, v = (normal(seed + i, n, 2, dim, dtype=torch.bfloat16) for i in (3, 4))
    return (x, normal(seed + 5, 333), normal(seed + 6, 333), q, k, v, g,
            torch.tensor(OFFSETS, device="cuda"))


@pytest.mark.parametrize("dim", [64, 128])
def test_a_thread_that_has_not_used_the_gpu(dim):
    inputs = _inputs(11, dim)
    want = _calls(*inputs)
    torch.cuda.synchronize()
    got = []

    def run():
        try:
            got.append(_calls(*inputs))
        except Exception as error:
            got.append(error)

    thread = threading.Thread(target=run)
    thread.start()
    thread.join()
    torch.cuda.synchronize()
    if isinstance(got[0], Exception):
        raise got[0]
    assert all(torch.equal(a, b) for a, b in zip(got[0], want))


@pytest.mark.parametrize("dim", [64, 128])
def test_in_a_captured_graph(dim):
    inputs = _inputs(23, dim)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        _calls(*inputs)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _calls(*inputs)
    # other values, and sequences that end elsewhere, in the same memory
    others = _inputs(37, dim)
    others[-1].copy_(torch.tensor([0, 300, 301, 302, 650, 699]))
    for a, b in zip(inputs, others):
        a.copy_(b)
    for t in got:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    want = _calls(*others)
    inside = OFFSETS[-1] - 1   # the last token is in no sequence: its rows are left alone
    for a, b in zip(got, want):
        n = inside if a.shape[0] == OFFSETS[-1] else a.shape[0]
        assert torch.equal(a[:n], b[:n])
