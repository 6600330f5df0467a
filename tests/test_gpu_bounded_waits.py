"""The attention kernels' waits end: a barrier at which nothing arrives makes a wait
give up after its limit, and the CTA's other waits at once.  The waits are compiled
into a small kernel of their own, since no call of the library makes one run out."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2207_10731_gb300 import build

pytestmark = pytest.mark.gpu

SOURCE = r"""
#include "seq/tc.cuh"
using namespace pss::seq;

// [0]: the wait for an arrival that came, [1]: for one that does not, [2]: another
// wait after it, [3]: nanoseconds of [1], [4]: of [2]
__global__ void k_waits(unsigned long long* out, unsigned long long* status) {
    __shared__ uint64_t came, missing;
    __shared__ volatile int stop;
    if (threadIdx.x != 0) return;
    stop = 0;
    bar_init(&came, 1);
    bar_init(&missing, 1);
    bar_init_done();
    bar_arrive(&came);
    out[0] = bar_wait(&came, 0, &stop);
    const uint64_t a = now_ns();
    out[1] = bar_wait(&missing, 0, &stop);
    const uint64_t b = now_ns();
    out[2] = bar_wait(&missing, 0, &stop);
    out[3] = b - a;
    out[4] = now_ns() - b;
    if (stop) report_stop(status);
}

extern "C" int run_waits(void* out, void* status) {
    k_waits<<<1, 32>>>((unsigned long long*)out, (unsigned long long*)status);
    return (int)cudaGetLastError();
}
"""


def test_a_wait_that_nothing_ends_gives_up(tmp_path):
    src, lib = tmp_path / "waits.cu", tmp_path / "waits.so"
    src.write_text(SOURCE)
    made = subprocess.run([build.nvcc_path(), *build._flags(), "-shared", str(src), "-o", str(lib)],
                          capture_output=True, text=True)
    assert made.returncode == 0, made.stderr
    out = torch.full((5,), 7, dtype=torch.int64, device="cuda")
    status = torch.full((1,), -1, dtype=torch.int64, device="cuda")
    torch.cuda.synchronize()
    run = ctypes.CDLL(os.fspath(lib)).run_waits
    assert run(ctypes.c_void_p(out.data_ptr()), ctypes.c_void_p(status.data_ptr())) == 0
    torch.cuda.synchronize()
    came, missing, after, waited, next_waited = out.tolist()
    assert came == 1 and missing == 0 and after == 0
    assert 2.0e9 <= waited < 3.0e9      # the limit is 2 s
    assert next_waited < 0.1e9          # told by the first
    assert status.item() == -2
    # the context is as usable as before
    assert torch.ones(1000, device="cuda").sum().item() == 1000
