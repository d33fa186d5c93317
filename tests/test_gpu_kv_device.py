"""The 4-bit cache's calls refuse handles and tensors that are not on the current device, where their kernels would run."""
import numpy as np
import pytest
import torch

import gpu_util as G
from paper_2310_08041_b200 import binding as B
from test_gpu_kv import ints, random_cache

pytestmark = pytest.mark.gpu


def calls(cache, pool, batch):
    x = torch.zeros(3, 2, 64, device=G.DEV)
    q, out, ws = torch.zeros(3, 4, 64, device=G.DEV), torch.zeros(3, 4, 64, device=G.DEV), torch.empty(1 << 22, dtype=torch.uint8, device=G.DEV)
    one, many = ints([0]), ints([0] * 8)
    return [lambda: B.qllm_kv_append(cache, 0, x, x, batch), lambda: B.qllm_kv_read(cache, 0, x, x, batch),
            lambda: B.qllm_kv_attention(cache, 0, q, out, 0.1, batch, ws), lambda: B.qllm_kv_pages_extend(cache, pool, ints([0, 0])),
            lambda: B.qllm_kv_pages_fork(cache, pool, one, ints([1])), lambda: B.qllm_kv_pages_compact(cache, pool, many),
            lambda: B.qllm_kv_pages_copy(cache, one, ints([1])), lambda: B.qllm_kv_pages_free(pool, one)]


def handles():
    cache, pool = random_cache(91, 1, 8, 2, 16, 64), B.KvPool.empty(8, 2, 4)
    batch = B.KvBatch(ints(np.array([[0, 1]])), ints([20]), ints([0, 3]), 3, 3)
    return cache, pool, batch


def refused(fn):
    before = B.qllm_launch_count()
    with pytest.raises(AssertionError):
        fn()
    assert B.qllm_launch_count() == before


def test_another_device_is_current(monkeypatch):
    """One GPU stands in for two: the binding asks for the current device in one place."""
    todo = calls(*handles())
    for fn in todo:
        fn()
    torch.cuda.synchronize()
    monkeypatch.setattr(B, "_current_device", lambda: 1)
    for fn in todo:
        refused(fn)


@pytest.mark.parametrize("which", range(3))
def test_a_handle_of_another_device(which):
    h = handles()
    todo = calls(*h)
    h[which].device = 1
    uses = [[0, 1, 2, 3, 4, 5, 6], [3, 4, 5, 7], [0, 1, 2]][which]
    for i in uses:
        refused(todo[i])


def test_tensors_that_are_not_on_the_device():
    cache, pool, batch = handles()
    x, there = torch.zeros(3, 2, 64), torch.zeros(3, 2, 64, device=G.DEV)
    q, ws = torch.zeros(3, 4, 64, device=G.DEV), torch.empty(1 << 22, dtype=torch.uint8, device=G.DEV)
    refused(lambda: B.qllm_kv_append(cache, 0, x, there, batch))
    refused(lambda: B.qllm_kv_read(cache, 0, there, x, batch))
    refused(lambda: B.qllm_kv_attention(cache, 0, q, q.clone(), 0.1, batch, ws.cpu()))
    refused(lambda: B.qllm_kv_attention(cache, 0, q, q.clone(), 0.1, batch, ws, lse=torch.zeros(3, 4)))
    refused(lambda: B.qllm_kv_pages_free(pool, torch.zeros(1, dtype=torch.int32)))
    refused(lambda: B.KvCache(cache.k_codes, cache.k_param.cpu(), cache.v_codes, cache.v_param))
    refused(lambda: B.KvBatch(batch.table, batch.seq_lens.cpu(), batch.q_start, 3, 3))
