"""Lookup, norms between blocks and products with their epilogues together, in the larger model of
examples/history_encoder.py: all gradients of a step against torch's autograd in 64 bits on the
same formulas, the step captured in a CUDA graph, and the serving step."""
import pytest
import torch

from tests.test_gpu_history_encoder import example

pytestmark = pytest.mark.gpu


def reference(model, ids, offsets, labels):
    """(loss, gradients by name) in 64 bits; the items' rows are taken as they are."""
    w = {k: v.double().clone().requires_grad_() for k, v in model.w.items()}
    tokens = ids.numel()
    places = model.places(offsets, tokens)
    bags = torch.arange(tokens + 1, device="cuda")
    items = model.embedding.forward(ids, bags, tokens).view(tokens, model.d).double()
    h = items + model.scale * w["table"][places]

    def rms(v, weight):
        return v / (v.square().mean(1, keepdim=True) + 1e-5).sqrt() * weight
    y = h - h.mean(1, keepdim=True)
    y = y / (y.square().mean(1, keepdim=True) + 1e-5).sqrt() * w["norm"] + w["norm_bias"]
    q, k, v = (y @ w["qkv"]).view(tokens, -1, model.dim).split(
        [model.heads, model.kv_heads, model.kv_heads], 1)
    k, v = (t.repeat_interleave(model.heads // model.kv_heads, 1) for t in (k, v))
    user = torch.bucketize(torch.arange(tokens, device="cuda"), offsets[1:], right=True)
    seen = (user[:, None] == user) & torch.ones(tokens, tokens, device="cuda").tril().bool()
    s = torch.einsum("ihd,jhd->hij", q, k) * model.dim ** -0.5
    s = s.masked_fill(~seen, -float("inf")).softmax(2)
    o = torch.einsum("hij,jhd->ihd", s, v).reshape(tokens, -1) @ w["out"]
    total = h + rms(o, w["post"])
    n = rms(total, w["pre"])
    u = torch.nn.functional.gelu(n @ w["up"] + w["up_bias"])
    f = u @ w["down"] + w["down_bias"]
    total = total + 0.5 * torch.sigmoid(n @ w["gate"]) * rms(f, w["last_post"])
    logits = rms(total, w["last_pre"]) @ w["head"]
    loss = torch.nn.functional.binary_cross_entropy_with_logits(logits, labels.double())
    loss.backward()
    return loss.item(), {k: t.grad for k, t in w.items()}


def test_a_step_takes_the_formulas_gradients():
    ex = example()
    model = ex.FeedForwardEncoder(p=0.0, seed=3)
    ids, offsets, labels = ex.histories(5, users=24, longest=20)
    loss, want = reference(model, ids, offsets, labels)
    got, grads = model.gradients(ids, offsets, labels)
    assert abs(got.item() - loss) < 0.01 * loss and set(grads) == set(want) == set(model.w)
    for name, grad in grads.items():
        # bf16 operands and results: 2^-8 of each of some ten factors along the chain
        assert grad.shape == want[name].shape, name
        assert (grad - want[name]).norm() <= 0.04 * want[name].norm(), name


def test_steps_run_and_serve():
    ex = example()
    model = ex.FeedForwardEncoder(p=0.1, seed=5)
    ids, offsets, labels = ex.histories(2, users=40, longest=30)
    assert all(model.step(ids, offsets, labels).isfinite() for _ in range(3))
    logits, _ = model.forward(ids, offsets, False)
    served = model.serve(ids, offsets)
    assert (served - logits[offsets[1:] - 1]).abs().max() <= 0.05 * logits.abs().max()
    none = torch.zeros(4, dtype=torch.int64, device="cuda")
    assert model.serve(ids[:0], none).isnan().all()


def test_the_block_in_a_captured_graph():
    ex = example()
    model = ex.FeedForwardEncoder(p=0.0, seed=9)
    o = torch.randn(300, model.d, device="cuda").bfloat16()
    h = torch.randn(300, model.d, device="cuda")
    model.block(o, h)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, _ = model.block(o, h)
    for seed in (1, 2):
        o.copy_(torch.randn(300, model.d, device="cuda", generator=torch.Generator("cuda").manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, model.block(o, h)[0])
