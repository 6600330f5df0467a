"""The status word of the table's calls where no value is read or written."""
import pytest
import torch

from paper_2207_10731_gb300 import sequence

pytestmark = pytest.mark.gpu


def calls(ids, rows, cols):
    """The status after the forward and after the backward call."""
    status = torch.full((1,), 77, device="cuda")
    sequence.embedding_forward(torch.ones(rows, cols, device="cuda"), ids, status=status)
    forward = int(status)
    sequence.embedding_backward(torch.ones(*ids.shape, cols, device="cuda"), ids, rows, status=status.fill_(77))
    return forward, int(status)


@pytest.mark.parametrize("tokens", [1, 700, 20000])
def test_tables_without_rows_or_columns(tokens):
    ids = torch.arange(tokens, device="cuda") % 5
    for cols in (0, 1, 16):
        assert calls(ids, 0, cols) == (0, 0)            # every id is outside
        assert calls(ids[:0], 0, cols) == (-1, -1)      # there is none
    assert calls(ids, 5, 0) == (-1, -1)
    ids[tokens - 1] = 5
    assert calls(ids, 5, 0) == calls(ids, 5, 8) == (tokens - 1, tokens - 1)
    ids[tokens // 2] = -1
    assert calls(ids, 5, 0) == calls(ids, 5, 8) == (tokens // 2, tokens // 2)


def test_without_a_status():
    ids = torch.zeros(9, dtype=torch.int64, device="cuda")
    assert sequence.embedding_forward(torch.ones(0, 4, device="cuda"), ids).shape == (9, 4)
    assert sequence.embedding_backward(torch.ones(9, 4, device="cuda"), ids, 0).shape == (0, 4)
    assert sequence.embedding_backward(torch.ones(9, 0, device="cuda"), ids, 3).shape == (3, 0)
