"""How products are dealt out, without a GPU: what the sizes of workspaces say of it."""
import pytest

from paper_2207_10731_gb300 import binding, build, sequence


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def weight_gradient(lib, tokens, n=8, m=8):
    """Bytes of the parts of dweight alone, [n, m] in bf16."""
    at = sequence._packed(sequence._BACKWARD, tokens, n, m, 4096, m, 4096, n, 4096, m, 1, 0, m, 0, n,
                          4096, m, 1, 0, 1, 1, 1, 0)
    return lib.pss_linear_backward_workspace(at)


@pytest.mark.parametrize("tokens", [10 ** 7, 10 ** 8, 440 * 10 ** 6, 550 * 10 ** 6, 10 ** 9, 2 ** 31 - 1025])
def test_long_contractions_are_split(lib, tokens):
    # one tile: its contraction is dealt out to as many CTAs as ten million tokens are, and more
    # tokens change nothing
    assert weight_gradient(lib, tokens) == weight_gradient(lib, 10 ** 6) > 0


@pytest.mark.parametrize("n", [8, 60, 1024])
def test_a_dense_column_is_read_in_place(lib, n):
    """A weight [n, 1], as a gate's: neither direction has a copy of it to make."""
    def forward(w, wi, wo):
        return lib.pss_linear_forward_workspace(sequence._packed(
            sequence._FORWARD, 1000, n, 1, 4096, up, w, wi, wo, 0, 0, 1, 4096, 1, 0, 1, 1, 1, 0, 0))

    def backward(w, wi, wo):   # dx alone, with the upstream gradient on the grid
        return lib.pss_linear_backward_workspace(sequence._packed(
            sequence._BACKWARD, 1000, n, 1, 4096, 8, 4096, up, w, wi, wo, 0, 1, 4096, n, 0, 1, 1, 0,
            1, 1, 1, 0))
    up = -(-n // 8) * 8
    for call in (forward, backward):
        rows = call(4096, 8, 1)                 # rows of one value, each on the grid
        assert call(4096, 1, 1) <= rows         # a dense column
        assert call(4096, 1, n) <= rows         # its other stride is free
        assert call(4098, 1, 1) >= rows + -(-n * 2 // 256) * 256   # off the grid: copied
