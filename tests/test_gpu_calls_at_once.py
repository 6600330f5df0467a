"""Calls of one kernel with different amounts of shared memory, at once from two threads and one behind the
other in one captured graph: what one call asks for is no limit of another's."""
import sys
import threading

import pytest
import torch

from paper_2207_10731_gb300 import binding, sequence
from tests.seq_util import normal

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


class Call:
    """A call of the library alone, on tensors of its own, and the same by the Python function."""

    def __init__(self, name, args, made, python):
        self.at, self.args, self.made, self.python = getattr(binding.load_library(), name), args, made, python

    def again(self, stream, turns):
        """How many of these calls are refused."""
        at, args = self.at, (*self.args, stream.cuda_stream)
        return sum(at(*args) != 0 for _ in range(turns))


def like(*tensors):
    return [torch.empty_like(t) for t in tensors]


def residual_norm(cols, rows=8):
    x, r, w = normal(1, rows, cols, dtype=BF16), normal(2, rows, cols), normal(3, cols)
    rstd = torch.ones(rows, device="cuda")
    made = like(x, r, x, w, w)
    size = sequence._library().pss_residual_norm_workspace(rows, cols)
    work = torch.empty(size, dtype=torch.uint8, device="cuda")
    px, pr, pw, ps, *pm = (t.data_ptr() for t in (x, r, w, rstd, *made))
    args = (pr, cols, px, cols, px, 1, cols, pr, 0, cols, px, 2, cols, pw, pw, ps, ps, rows, cols, 1.0, pm[0], cols,
            pm[1], cols, pm[2], cols, pm[3], pm[4], work.data_ptr(), size)
    call = Call("pss_residual_norm_backward", args, made,
                lambda: sequence.residual_norm_backward(r, x, x, r, rstd, rstd, w, w, x))
    call.work = work
    return call


def layer_norm(cols, rows=8):
    x, w = normal(1, rows, cols, dtype=BF16), normal(3, cols)
    mean, rstd = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    made = like(x, w, w)
    size = sequence._library().pss_layer_norm_workspace(rows, cols)
    work = torch.empty(size, dtype=torch.uint8, device="cuda")
    px, pw, pmean, prstd, *pm = (t.data_ptr() for t in (x, w, mean, rstd, *made))
    args = (px, 1, cols, px, 1, cols, pw, pmean, prstd, rows, cols, pm[0], cols, pm[1], pm[2], work.data_ptr(), size)
    call = Call("pss_layer_norm_backward", args, made, lambda: sequence.layer_norm_backward(x, x, w, mean, rstd))
    call.work = work
    return call


def table(rows, tokens=9000):
    ids = (torch.arange(tokens, device="cuda") * 7919) % rows
    g, out = normal(4, tokens, 8), torch.empty(rows, 8, device="cuda")
    size = sequence._library().pss_embedding_workspace(tokens, rows, 8)
    work = torch.empty(size, dtype=torch.uint8, device="cuda")
    args = (g.data_ptr(), 0, 8, ids.data_ptr(), tokens, 1.0, rows, 8, out.data_ptr(), 0, 8, work.data_ptr(), size, None)
    call = Call("pss_embedding_backward", args, [out], lambda: (sequence.embedding_backward(g, ids, rows),))
    call.work = work
    return call


# the same kernel each: a row to a CTA, to a wide one, to a warp, off the 16-byte grid; digits of 11 bits
# and of 7
PAIRS = {
    "residual norm, a CTA": (residual_norm, 2048, 1536), "residual norm, wide": (residual_norm, 4096, 3584),
    "residual norm, a warp": (residual_norm, 512, 400), "residual norm, odd": (residual_norm, 2041, 1601),
    "layer norm": (layer_norm, 16384, 12288), "layer norm, odd": (layer_norm, 16001, 12291),
    "table": (table, 70000, 100),
}


def equal(got, want):
    return len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("name", PAIRS)
def test_in_one_graph(name):
    make, *sizes = PAIRS[name]
    calls = [make(s).python for s in sizes]
    want = [c() for c in calls]
    for order in ((0, 1), (1, 0)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = [calls[i]() for i in order]
        for _ in range(2):
            graph.replay()
            torch.cuda.synchronize()
            assert all(equal(g, want[i]) for g, i in zip(got, order))
            calls[1]()   # and a call between replays


@pytest.mark.parametrize("name", PAIRS)
def test_from_two_threads(name):
    make, *sizes = PAIRS[name]
    calls = [make(s) for s in sizes]
    want = [c.python() for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    refused, ready = [0, 0], threading.Barrier(2)
    often = sys.getswitchinterval()

    def run(i):
        ready.wait()
        for _ in range(100):
            refused[i] += calls[i].again(streams[i], 150)
            streams[i].synchronize()
    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    sys.setswitchinterval(1e-5)
    try:
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(often)
    assert refused == [0, 0]
    assert all(equal(c.made, w) for c, w in zip(calls, want))
