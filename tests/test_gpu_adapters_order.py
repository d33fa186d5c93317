"""qllm_adapters_add: a row's result does not depend on where in the batch its sequence stands."""
import numpy as np
import pytest
import torch

import gpu_util as G
from paper_2310_08041_b200 import binding as B

pytestmark = pytest.mark.gpu


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=G.DEV)


def interleaved(rng, adapter, slots):
    """An order of the sequences that keeps those of one adapter in their order and mixes the adapters."""
    left = [[s for s, a in enumerate(adapter) if a == g] for g in range(-1, slots)]
    order = []
    while any(left):
        pick = rng.choice([g for g in range(len(left)) if left[g]])
        order.append(left[pick].pop(0))
    return order


# single tokens, some rows, prompts; ranks on both sides of the border between the kernels
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("top", [16, 32, 64, 72, 128])
@pytest.mark.parametrize("news", [[1, 1, 2, 1, 0, 1, 3, 1, 1, 1, 2, 1], [40, 1, 30, 70, 5, 9], [500, 1, 300, 129, 700, 1, 64]], ids=["step", "some", "prompts"])
def test_sequences_moved_elsewhere(dtype, top, news):
    """Bit for bit, the same batch in other orders: an adapter's rows stay in their order."""
    K, N, slots = 1032, 520, 3
    torch.manual_seed(top)
    rng = np.random.RandomState(top + len(news))
    adapter = [s % (slots + 1) - 1 for s in range(len(news))]
    ad = B.Adapters(torch.randn(slots, top, K, device=G.DEV).bfloat16(), torch.randn(slots, N, top, device=G.DEV).bfloat16(), torch.rand(slots, device=G.DEV),
                    ints([top, top - 3, max(1, top // 2)]))
    start = np.concatenate([[0], np.cumsum(news)])
    x, base = torch.randn(start[-1], K, device=G.DEV).to(dtype), torch.randn(start[-1], N, device=G.DEV).to(dtype)
    bits = torch.int16 if dtype == torch.bfloat16 else torch.int32
    first = torch.empty_like(base)
    B.qllm_adapters_add(ad, x, base, first, ints(start), ints(adapter))
    moved = 0
    for _ in range(4):
        order = interleaved(rng, adapter, slots)
        rows = torch.from_numpy(np.concatenate([np.arange(start[s], start[s + 1]) for s in order])).to(G.DEV)
        out = torch.empty_like(base)
        B.qllm_adapters_add(ad, x[rows].contiguous(), base[rows].contiguous(), out, ints(np.concatenate([[0], np.cumsum([news[s] for s in order])])),
                            ints([adapter[s] for s in order]))
        assert torch.equal(out.view(bits), first[rows].view(bits))
        moved += order != list(range(len(news)))
    assert moved and B.qllm_poll_status() == B.QLLM_OK
