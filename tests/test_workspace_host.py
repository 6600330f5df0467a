"""Sizes of workspaces, without a GPU.  A workspace is aligned to 16 bytes by contract, but its parts hold
fp32 values that are moved 32 bytes at a time: these start at its first multiple of 32, up to 16
bytes in, for which the size has to have room."""
import pytest

from paper_2207_10731_gb300 import binding, build, sequence


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def parts(*sizes):
    """Each part's bytes end at a multiple of 256."""
    return sum(-(-s // 256) * 256 for s in sizes)


@pytest.mark.parametrize("tokens,cols", [(100, 8), (5000, 64), (8192, 333)])
def test_tables(lib, tokens, cols):
    # the count, a flag, the sorted places, sums of 32 places and of 2048, in rows of multiples of 8
    wide = -(-cols // 8) * 8 * 4
    least = parts(16, 4, 8 * tokens, tokens // 32 * wide, tokens // 2048 * wide)
    assert lib.pss_embedding_workspace(tokens, 40, cols) >= least + 16


def test_products(lib):
    # x off the 16-byte grid: its copy, and no parts of a contraction of 8
    def forward(x):
        at = sequence._packed(sequence._FORWARD, 100, 8, 16, x, 8, 4096, 16, 1, 0, 0, 16, 4096, 16, 0, 16,
                              1, 1, 0, 0)
        return lib.pss_linear_forward_workspace(at)
    assert forward(4096) == 0
    assert forward(4098) >= parts(100 * 8 * 2) + 16
    # the bias's sums alone: two parts of 32 tokens or more
    at = sequence._packed(sequence._BACKWARD, 64, 8, 16, 4096, 16, 4096, 8, 4096, 16, 1, 0, 16, 0, 8,
                          0, 16, 1, 4096, 1, 1, 1, 0)
    assert lib.pss_linear_backward_workspace(at) >= parts(16 * 4) + 16


def test_attention(lib):
    # one query over long keys: the keys' pieces leave sums
    def size(keys):
        where = sequence._structs((1, 0, 0, 1, keys, 1, 1, 128, 1, 0.125))
        return lib.pss_attention_workspace(where[0], 0)
    assert size(100000) > size(128)
    # (every part but the room itself ends at a multiple of 256)
    assert size(128) % 256 >= 16 and size(100000) % 256 >= 16
