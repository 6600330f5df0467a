"""The sequence operators together, in examples/history_encoder.py: a training
step's gradients against torch's autograd on the same formulas, learning, and
the serving step against the training forward."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "history_encoder.py")


def example():
    spec = importlib.util.spec_from_file_location("history_encoder", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_it_learns_and_serves_what_it_learned():
    ex = example()
    model = ex.HistoryEncoder(p=0.05)
    batches = [ex.histories(s, users=128, longest=40) for s in range(4)]
    first = sum(model.step(*b).item() for b in batches) / 4
    for _ in range(40):
        last = sum(model.step(*b) for b in batches).item() / 4
    # answering always with the labels' share costs about 0.69
    assert first > 0.5 and last < 0.75 * first
    ids, offsets, _ = batches[0]
    logits, _ = model.forward(ids, offsets, False)
    served = model.serve(ids, offsets)
    # the same sums over other tiles: the attention's output is rounded to bf16
    # either way (2^-8 of its size, twice), and so is the projection's
    assert (served - logits[offsets[1:] - 1]).abs().max() <= 0.05 * logits.abs().max()


def test_a_step_takes_the_formulas_gradient():
    # the whole chain against autograd in 64 bits, through the weights' first
    # Adagrad / Adam step: with zero moments its direction is the gradient's sign
    ex = example()
    model = ex.HistoryEncoder(p=0.0, seed=3)
    ids, offsets, labels = ex.histories(5, users=24, longest=20)
    w = {k: v.double().clone().requires_grad_() for k, v in model.w.items()}
    x = model.embed(ids, offsets).double()

    def norm(h, a, b):
        h = h - h.mean(1, keepdim=True)
        return h / (h.square().mean(1, keepdim=True) + 1e-5).sqrt() * a + b
    qkv = norm(x, w["norm"], w["norm_bias"]) @ w["qkv"]
    q, k, v = qkv.view(len(ids), -1, model.dim).split(
        [model.heads, model.kv_heads, model.kv_heads], 1)
    k, v = (t.repeat_interleave(model.heads // model.kv_heads, 1) for t in (k, v))
    user = torch.bucketize(torch.arange(len(ids), device="cuda"), offsets[1:], right=True)
    seen = (user[:, None] == user) & torch.ones(len(ids), len(ids), device="cuda").tril().bool()
    s = torch.einsum("ihd,jhd->hij", q, k) * model.dim ** -0.5
    s = s.masked_fill(~seen, -float("inf")).softmax(2)
    o = torch.einsum("hij,jhd->ihd", s, v).reshape(len(ids), -1) @ w["out"]
    z = norm(x + o, w["last"], w["last_bias"])
    loss = torch.nn.functional.binary_cross_entropy_with_logits(z @ w["head"], labels.double())
    loss.backward()
    got = model.step(ids, offsets, labels, lr=0.01)
    assert abs(got.item() - loss.item()) < 0.01 * loss.item()
    for name, (m, _) in model.moments.items():
        grad, want = m / 0.1, w[name].grad
        # bf16 operands: 2^-8 of each of a handful of factors
        assert (grad - want).norm() <= 0.03 * want.norm(), name


def test_an_empty_history_is_served_as_one():
    ex = example()
    model = ex.HistoryEncoder(seed=7)
    ids, offsets, _ = ex.histories(9, users=20, longest=30)
    want = model.serve(ids, offsets)
    # users without items first, between, last and in a row
    at = [0, 0, 5, 5, 11, 20]
    ends = offsets.tolist()
    with_empty, full = [0], []
    for user in range(20):
        for _ in range(at.count(user)):
            with_empty.append(ends[user])
            full.append(False)
        with_empty.append(ends[user + 1])
        full.append(True)
    with_empty.append(ends[-1])
    full.append(False)
    full = torch.tensor(full, device="cuda")
    got = model.serve(ids, torch.tensor(with_empty, device="cuda"))
    # nobody else's item answers for a user who has none
    assert got[~full].isnan().all()
    # the same rows through the same products, but other tiles and row counts
    assert (got[full] - want).abs().max() <= 0.05 * want.abs().max()
    # nobody has any
    none = torch.zeros(4, dtype=torch.int64, device="cuda")
    assert model.serve(ids[:0], none).isnan().all() and model.serve(ids[:0], none).shape == (3,)
