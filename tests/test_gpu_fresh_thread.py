"""Small calls whose first work in a thread is a tensor map: the driver's encoder wants the
device's context bound to the thread, which nothing has done before."""
import threading

import pytest
import torch

from paper_2207_10731_gb300 import sequence
from tests.seq_util import normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128])
def test_attention_without_a_work_list(dim):
    q, k, v = (normal(s, 40, 4, dim, dtype=torch.bfloat16) for s in (1, 2, 3))
    off = torch.tensor([0, 40], device="cuda")
    want, lse = sequence.attention_forward(q, k, v, off)
    got = []

    def run():
        try:
            got.append(sequence.attention_forward(q, k, v, off))
        except Exception as error:
            got.append(error)

    torch.cuda.synchronize()
    thread = threading.Thread(target=run)
    thread.start()
    thread.join()
    torch.cuda.synchronize()
    if isinstance(got[0], Exception):
        raise got[0]
    assert torch.equal(got[0][0], want) and torch.equal(got[0][1], lse)
