"""Workspaces of exactly the size asked for that start 16 bytes past a multiple of 32, as the contract
allows: the same bits as with one on a multiple of 512, and nothing written outside."""
import pytest
import torch

from paper_2207_10731_gb300 import sequence
from tests.seq_util import normal

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


class Shifted:
    """torch, but for byte tensors (the workspaces), which are cut out of larger ones."""

    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        return getattr(torch, name)

    def empty(self, *size, dtype=None, **kw):
        if dtype != torch.uint8:
            return torch.empty(*size, dtype=dtype, **kw)
        whole = torch.full((size[0] + 16 + 512,), 0xA5, dtype=torch.uint8, device="cuda")
        self.made.append(whole)
        assert whole.data_ptr() % 32 == 0
        return whole[16:16 + size[0]]


def product(tokens, n, m, gap=0):
    x = normal(1, tokens, n + gap, dtype=BF16)[:, :n]
    w, g = normal(2, n, m, dtype=BF16, scale=n ** -0.5), normal(3, tokens, m)

    def call():
        y, z = sequence.linear_forward(x, w, activation="gelu", keep=True)
        return (y, z, *sequence.linear_backward(g, x, w, z, "gelu"))
    return call


def table(tokens, rows, cols, dtype):
    ids = (torch.rand(tokens, generator=torch.Generator().manual_seed(4)) ** 3 * rows).long().cuda()
    g = normal(5, tokens, cols, dtype=dtype)
    return lambda: (sequence.embedding_backward(g, ids, rows),)


def attention(users, steps, keys, dim, odd=False):
    q = normal(6, users * steps, 4, dim, dtype=BF16)
    k, v = normal(7, users * keys, 2, dim, dtype=BF16), normal(8, users * keys, 2, dim, dtype=BF16)
    if odd:   # rows that are not finite go another way
        v[5, 0, 3] = float("inf")
    qo, ko = (torch.arange(users + 1, device="cuda") * n for n in (steps, keys))

    def call():
        out, lse = sequence.attention_forward(q, k, v, qo, ko)
        return (out, lse, *sequence.attention_backward(q, q, k, v, out, lse, qo, ko))
    return call


def norms(rows, cols):
    x, w = normal(9, rows, cols, dtype=BF16), normal(10, cols)

    def call():
        y, mean, rstd = sequence.layer_norm_forward(x, w, w)
        total, y2, a, b = sequence.residual_norm_forward(x, x, w, w)
        return (*sequence.layer_norm_backward(y, x, w, mean, rstd),
                *sequence.residual_norm_backward(total, y2, x, total, a, b, w, w))
    return call


CALLS = {
    "a product's parts": lambda: product(3, 4096, 768), "many tokens": lambda: product(3000, 520, 264),
    "off the grid": lambda: product(301, 333, 130, 1), "a long contraction": lambda: product(70000, 64, 72),
    "few tokens of a table": lambda: table(700, 40, 64, BF16), "pieces": lambda: table(5000, 3, 128, torch.float32),
    "large pieces": lambda: table(70001, 3, 64, BF16), "odd rows": lambda: table(9001, 50, 333, torch.float32),
    "split keys": lambda: attention(3, 1, 5000, 128), "split keys, small heads": lambda: attention(1, 3, 9000, 40),
    "split keys, not finite": lambda: attention(2, 2, 5000, 128, True), "prompts": lambda: attention(2, 300, 300, 64),
    "norms": lambda: norms(900, 520),
}


@pytest.mark.parametrize("name", CALLS)
def test_workspaces_off_the_grid_of_32_bytes(name, monkeypatch):
    call = CALLS[name]()
    want = [t for t in call() if t is not None]
    shifted = Shifted()
    monkeypatch.setattr(sequence, "torch", shifted)
    got = [t for t in call() if t is not None]
    torch.cuda.synchronize()
    assert shifted.made and len(got) == len(want)
    for a, b in zip(got, want):
        a, b = (t.view(torch.int32 if t.dtype == torch.float32 else torch.int16) for t in (a, b))
        assert torch.equal(a, b)
    for whole in shifted.made:
        assert (whole[:16] == 0xA5).all() and (whole[-512:] == 0xA5).all()
