"""The forward kernel that takes two query tiles to a CTA, which only long batches
reach: sizes follow from the GPU's SM count, and each test asks the plan first.
Bounds as in test_gpu_attention.py."""
import math

import pytest
import torch

from paper_2207_10731_gb300 import binding, sequence
from tests.seq_util import check
from tests.test_gpu_attention import compare, inputs, offsets, reference, run

pytestmark = pytest.mark.gpu


def many_heads(nq, group):
    """Key heads that make eight CTAs an SM of these queries' tiles."""
    tiles = -(-sum(nq) // (128 // group))
    return -(-8 * torch.cuda.get_device_properties(0).multi_processor_count // tiles)


def listed_items(sequences, nq, nk, heads, kv_heads, dim):
    """The workspace of a forward call; only the list's length depends on the
    number of sequences."""
    where = sequence._structs((sequences, 0, 0, sum(nq), sum(nk), heads, kv_heads, dim, 1, 0.125))
    return binding.load_library().pss_attention_workspace(where[0], 0)


def assert_two_tiles(nq, nk, heads, kv_heads, dim):
    # a great many sequences of the same tokens would be short ones: one tile an item.
    # (Lists of up to eight items take the same room; the rule goes by the number of
    # tiles times heads, which many_heads makes the same for all.)
    if -(-sum(nq) // (128 // (heads // kv_heads))) > 8:
        assert listed_items(len(nq), nq, nk, heads, kv_heads, dim) < \
            listed_items(1 << 20, nq, nk, heads, kv_heads, dim)


LENS = {
    "even tiles": ([768], [768]),
    "odd tiles": ([640], [640]),
    "a last tile of one token": ([641], [641]),
    "a last pair of one token": ([769], [769]),
    "more keys": ([600], [905]),
    "more queries": ([905], [300]),
    "no keys": ([600, 700], [600, 0]),
    "two sequences": ([701, 400], [701, 400]),
    "with short ones": ([0, 1700, 3, 1], [5, 1300, 3, 130]),
}


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("group,dim", [(1, 64), (3, 64), (1, 128), (3, 128), (2, 40), (5, 104)])
def test_two_tiles_to_a_cta(lens, causal, group, dim):
    nq, nk = LENS[lens]
    if sum(nq) < 512 * len(nq):
        nq = [nq[0], nq[1] + 512 * len(nq) - sum(nq)] + nq[2:]
    kv_heads = many_heads(nq, group)
    assert_two_tiles(nq, nk, kv_heads * group, kv_heads, dim)
    q, k, v, _ = inputs(nq, nk, kv_heads * group, kv_heads, dim, seed=300)
    compare(run(q, k, v, None, nq, nk, causal), q, k, v, None, nq, nk, causal)


@pytest.mark.parametrize("group,nq", [(2, [900, 333]), (1, [2177])])
def test_two_tiles_in_a_training_pass(group, nq):
    kv_heads = many_heads(nq, group)
    assert_two_tiles(nq, nq, group * kv_heads, kv_heads, 64)
    q, k, v, grad = inputs(nq, nq, group * kv_heads, kv_heads, 64, seed=310)
    compare(run(q, k, v, grad, nq, nq, True), q, k, v, grad, nq, nq, True)


@pytest.mark.parametrize("bad", [float("nan"), math.inf, -3.0e38])
@pytest.mark.parametrize("at", [100, 127, 128, 600, 767])
@pytest.mark.parametrize("group,dim", [(1, 64), (3, 128)])
def test_masked_values_in_a_pair_of_tiles(bad, at, group, dim):
    nq = [768]
    kv_heads = many_heads(nq, group)
    assert_two_tiles(nq, nq, kv_heads * group, kv_heads, dim)
    q, k, v, _ = inputs(nq, nq, kv_heads * group, kv_heads, dim, seed=320)
    want = reference(q[:at], k[:at], v[:at], [at], [at], True, dim ** -0.5)
    k[at:], v[at:] = bad, bad
    off = offsets(nq)
    out, lse = sequence.attention_forward(q, k, v, off)
    check(out[:at], *want[0], "out")
    check(lse[:at], *want[1], "lse")
    if bad != -3.0e38:
        assert not out[at:].isfinite().any()
