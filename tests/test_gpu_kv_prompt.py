"""The tensor-core attention kernel of the 4-bit cache under bounds that follow its roundings (kv_bounds, which test_kv_bounds.py
tries on the CPU)."""
import numpy as np
import pytest
import torch

import gpu_util as G
import kv_bounds
import kv_ref
from paper_2310_08041_b200 import binding as B
from test_gpu_kv import DT, attend, batch_of, check_attention, host, ints, make_table, random_cache, store_of

pytestmark = pytest.mark.gpu


def layer_of(cache, layer=0):
    return tuple(t[layer] for t in (cache.k_codes, cache.k_param, cache.v_codes, cache.v_param))


def queries(seed, *shape):
    g = torch.Generator(device=G.DEV); g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device=G.DEV).bfloat16()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_graph_of_the_streaming_kernel_writes_logarithms(dtype):
    """Few new tokens: captured, replayed while lengths, pages and queries change, against 64-bit logarithms."""
    heads, group, page, d, news = 2, 4, 16, 128, [1, 3, 0, 2]
    top = [1500] * len(news)
    cache = random_cache(55, 1, 400, heads, page, d)
    batch, start = batch_of(make_table(np.random.RandomState(55), top, page, 400), top, news)
    q = queries(56, batch.rows, heads * group, d).to(DT[dtype])
    out, lse, st = torch.empty_like(q), torch.empty(batch.rows, heads * group, device=G.DEV), torch.cuda.Stream()
    ws = torch.full((B.qllm_kv_attention_workspace(cache, heads * group, q, batch),), 0xFF, dtype=torch.uint8, device=G.DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        B.qllm_kv_attention(cache, 0, q, out, 0.09, batch, ws, lse=lse, stream=st)
    st.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        B.qllm_kv_attention(cache, 0, q, out, 0.09, batch, ws, lse=lse, stream=st)
    for lens in ([1500] * 4, [1, 2, 0, 17], [911, 151, 64, 1]):
        table = make_table(np.random.RandomState(lens[1]), top, page, 400)
        batch.seq_lens.copy_(ints(lens))
        batch.table.copy_(ints(table))
        q.copy_(queries(lens[0], *q.shape))
        lse.fill_(7.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            g.replay()
        torch.cuda.synchronize()
        check_attention(out, lse, kv_ref.attention(store_of(cache, 0), table, lens, start, host(q), 0.09, True), DT[dtype])
    assert B.qllm_poll_status() == B.QLLM_OK


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


@pytest.mark.parametrize("seed", range(30))
def test_random_shapes_and_ranges(seed):
    """Calls of every shape that the tensor-core kernel takes, keys cut into parts or not, over scales that spread by up to 2^36 and
    zero-points up to +-1200, so that its tiles take every path."""
    rng, g = np.random.RandomState(900 + seed), torch.Generator(device=G.DEV)
    g.manual_seed(seed)
    d, page = int(rng.choice([64, 128])), int(rng.choice([16, 32, 64, 128, 256]))
    heads, group, seqs = int(rng.choice([1, 2, 8])), int(rng.choice([1, 2, 3, 5, 8])), int(rng.randint(1, 4))
    first = 96 // group + 1 + int(rng.randint(0, 200))
    news = [first] + [int(rng.randint(1, first + 1)) for _ in range(seqs - 1)]
    lens = [n + int(rng.choice([0, 1, 130, 700])) for n in news]
    table = make_table(rng, lens, page, sum(-(-n // page) for n in lens) + 2)
    cache = random_cache(seed, 1, sum(-(-n // page) for n in lens) + 2, heads, page, d)
    spread = lambda t, by: t * 2.0 ** (by * (torch.rand(t.shape, generator=g, device=G.DEV) - 1))  # noqa: E731
    keys, vals, far = rng.choice([0, 8, 16, 36], 3)
    cache.k_param[..., 0] = spread(cache.k_param[..., 0], float(keys))
    cache.v_param[..., 0] = spread(cache.v_param[..., 0], float(vals))
    if far >= 16:
        cache.v_param[..., 1] = torch.randint(-1200, 1201, cache.v_param.shape[:-1], generator=g, device=G.DEV).float()
    if far == 36:
        cache.k_param[..., 1] = torch.randint(-1200, 1201, cache.k_param.shape[:-1], generator=g, device=G.DEV).float()
    batch, start = batch_of(table, lens, news, max_new=first)
    q, scale, causal = queries(seed, batch.rows, heads * group, d), float(rng.choice([0.001, 0.09, -0.3])), bool(rng.rand() < 0.7)
    want = kv_bounds.expect(layer_of(cache), table, lens, start, q, scale, causal)
    got, lse = attend(cache, 0, q, batch, scale, causal)
    took = [s for s in range(seqs) if news[s] * group > 96]   # shorter ones are the streaming kernel's
    rows = torch.cat([torch.arange(int(start[s]), int(start[s + 1])) for s in took]).to(G.DEV)
    kv_bounds.check(got, lse, want, rows)
    assert torch.isfinite(got.float()).all() and B.qllm_poll_status() == B.QLLM_OK
