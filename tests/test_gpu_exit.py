"""The exit of a cluster's CTA when a bounded wait ran out for some of its warps and not for the others."""
import pytest
import torch

import gpu_util as G
from paper_2310_08041_b200 import binding as B

pytestmark = pytest.mark.gpu


def test_one_warp_whose_wait_ran_out_takes_the_others_along():
    """Every warp of both CTAs leaves, the status word says why, once, and the next call of the kernel that has this exit is right."""
    assert B.qllm_poll_status() == B.QLLM_OK
    left = torch.zeros(2, dtype=torch.int32, device=G.DEV)
    for times in (1, 2, 3):
        B.qllm_debug_exit_expiry(left)
        assert B.qllm_poll_status() == B.QLLM_ERR_TIMEOUT
        assert left.tolist() == [4 * times, 4 * times]
    assert B.qllm_poll_status() == B.QLLM_OK
    # rank 72, few rows: the tensor-core kernel in clusters.  Sums of eight ones times one half: exact
    top, K, N, rows = 72, 256, 512, 3
    A, Bm = torch.zeros(1, top, K, device=G.DEV), torch.zeros(1, N, top, device=G.DEV)
    A[0, :, :8], Bm[0, :, :4] = 1, 0.5
    ad = B.Adapters(A.bfloat16(), Bm.bfloat16(), torch.ones(1, device=G.DEV))
    x, out = torch.ones(rows, K, device=G.DEV).bfloat16(), torch.empty(rows, N, device=G.DEV).bfloat16()
    ints = lambda *a: torch.tensor(a, dtype=torch.int32, device=G.DEV)  # noqa: E731
    B.qllm_adapters_add(ad, x, None, out, ints(0, rows), ints(0))
    assert (out == 16).all() and B.qllm_poll_status() == B.QLLM_OK
