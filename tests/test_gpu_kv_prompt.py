"""The tensor-core attention kernel of the 4-bit cache under bounds that follow its roundings (kv_bounds, which test_kv_bounds.py
tries on the CPU)."""
import numpy as np
import pytest
import torch

import gpu_util as G
import kv_bounds
from paper_2310_08041_b200 import binding as B
from test_gpu_kv import attend, batch_of, ints, make_table, random_cache

pytestmark = pytest.mark.gpu


def layer_of(cache, layer=0):
    return tuple(t[layer] for t in (cache.k_codes, cache.k_param, cache.v_codes, cache.v_param))


def queries(seed, *shape):
    g = torch.Generator(device=G.DEV); g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device=G.DEV).bfloat16()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,page,heads,group", [(128, 64, 2, 4), (64, 16, 3, 2), (128, 256, 1, 7), (64, 32, 2, 8)])
@pytest.mark.parametrize("lens,news", [([257], [257]), ([700, 90], [130, 90]), ([3000], [70]), ([513, 300], [70, 100]), ([1000, 520], [600, 515])])
def test_errors_are_those_of_the_roundings(lens, news, d, page, heads, group, causal):
    table = make_table(np.random.RandomState(51), lens, page, sum(-(-n // page) for n in lens) + 2)
    cache = random_cache(51, 1, sum(-(-n // page) for n in lens) + 2, heads, page, d)
    batch, start = batch_of(table, lens, news)
    q = queries(52, batch.rows, heads * group, d)
    assert max(news) * group > 96                            # the tensor-core kernel's, whatever the sequence
    want = kv_bounds.expect(layer_of(cache), table, lens, start, q, d ** -0.5, causal)
    got, lse = attend(cache, 0, q, batch, d ** -0.5, causal)
    kv_bounds.check(got, lse, want)
    assert B.qllm_poll_status() == B.QLLM_OK


@pytest.mark.parametrize("news", [[200], [130, 150, 0]])
def test_a_graph_writes_logarithms_and_outputs_within_the_bounds(news):
    """Captured with its keys cut into parts (few rows) and replayed while lengths, pages and queries change."""
    heads, group, page, d = 1, 4, 16, 128
    top = [1500] * len(news)
    cache = random_cache(53, 1, 300, heads, page, d)
    batch, start = batch_of(make_table(np.random.RandomState(53), top, page, 300), top, news)
    q = queries(54, batch.rows, heads * group, d)
    out, lse, st = torch.empty_like(q), torch.empty(batch.rows, heads * group, device=G.DEV), torch.cuda.Stream()
    ws = torch.full((B.qllm_kv_attention_workspace(cache, heads * group, q, batch),), 0xFF, dtype=torch.uint8, device=G.DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        B.qllm_kv_attention(cache, 0, q, out, 0.09, batch, ws, lse=lse, stream=st)
    st.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        B.qllm_kv_attention(cache, 0, q, out, 0.09, batch, ws, lse=lse, stream=st)
    for lens in ([1500] * len(news), [200, 170, 0][:len(news)], [911, 151, 64][:len(news)]):
        table = make_table(np.random.RandomState(lens[0]), top, page, 300)
        batch.seq_lens.copy_(ints(lens))
        batch.table.copy_(ints(table))
        q.copy_(queries(lens[0], *q.shape))
        lse.fill_(7.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            g.replay()
        torch.cuda.synchronize()
        kv_bounds.check(out, lse, kv_bounds.expect(layer_of(cache), table, lens, start, q, 0.09, True))
    assert B.qllm_poll_status() == B.QLLM_OK
