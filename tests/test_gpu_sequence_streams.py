"""The sequence operators on another stream than the current one, by their stream
keyword, and dropout in a captured graph."""
import pytest
import torch

from paper_2207_10731_gb300 import sequence
from tests.seq_util import normal

pytestmark = pytest.mark.gpu


def calls():
    """(name, call) of every operator, on inputs large enough to be still running
    when the call returns."""
    x, g = normal(1, 40000, 512), normal(2, 40000, 512)
    w, b = normal(3, 512), normal(4, 512)
    q, grad = (normal(s, 6000, 8, 64, dtype=torch.bfloat16) for s in (5, 6))
    k, v = (normal(s, 6000, 2, 64, dtype=torch.bfloat16) for s in (7, 8))
    off = torch.tensor([0, 2500, 2500, 6000], device="cuda")
    _, mean, rstd = sequence.layer_norm_forward(x, w, b)
    out, lse = sequence.attention_forward(q, k, v, off)
    torch.cuda.synchronize()
    return [
        ("layer_norm_forward", lambda **kw: sequence.layer_norm_forward(x, w, b, **kw)),
        ("layer_norm_backward", lambda **kw: sequence.layer_norm_backward(g, x, w, mean, rstd, **kw)),
        ("dropout", lambda **kw: sequence.dropout(x, 0.3, 5, 9, residual=g, **kw)),
        ("attention_forward", lambda **kw: sequence.attention_forward(q, k, v, off, **kw)),
        ("attention_backward",
         lambda **kw: sequence.attention_backward(grad, q, k, v, out, lse, off, **kw)),
    ]


def test_the_stream_keyword_of_every_operator():
    side = torch.cuda.Stream()
    for name, call in calls():
        want = call()
        torch.cuda.synchronize()
        # the current stream is busy; the call neither waits for it nor uses it
        torch.cuda._sleep(400_000_000)
        got = call(stream=side)
        side.synchronize()
        assert not torch.cuda.current_stream().query(), f"{name} waited for the current stream"
        got = got if isinstance(got, tuple) else (got,)
        with torch.cuda.stream(side):
            got = [t.clone() for t in got]
        torch.cuda.synchronize()
        want = want if isinstance(want, tuple) else (want,)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), name


def test_a_captured_graph_repeats_its_dropout_mask():
    x = normal(11, 300, 256)
    want = sequence.dropout(x, 0.4, 3, 7)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        sequence.dropout(x, 0.4, 3, 7)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = sequence.dropout(x, 0.4, 3, 7)
    for _ in range(2):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
