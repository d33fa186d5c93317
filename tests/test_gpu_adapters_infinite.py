"""qllm_adapters_add: rows of bf16 with an infinity come out as the formula has them, infinite or NaN, number by number."""
import numpy as np
import pytest
import torch

import gpu_util as G
from paper_2310_08041_b200 import binding as B

pytestmark = pytest.mark.gpu


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=G.DEV)


@pytest.mark.parametrize("top", [8, 16, 32, 40, 64, 72, 128])
@pytest.mark.parametrize("news", [[1] * 30, [1], [50, 3], [300, 170], [1200, 100]], ids=["step", "token", "some", "prompts", "long"])
@pytest.mark.parametrize("use", ["one", "few", "all"])
def test_an_infinity_among_ordinary_numbers(top, news, use):
    """In every fifth row one infinity: each sum over K is one too, and an output is an infinity where its terms agree in sign."""
    K, N, slots = 136, 264, 2
    torch.manual_seed(top + len(news))
    rank = {"one": 1, "few": 3, "all": top}[use]
    A, Bm = torch.randn(slots, top, K, device=G.DEV).bfloat16(), torch.randn(slots, N, top, device=G.DEV).bfloat16()
    assert (A != 0).all() and (Bm != 0).all()
    scale = torch.rand(slots, device=G.DEV) + 0.25
    start, adapter = np.concatenate([[0], np.cumsum(news)]), [s % slots for s in range(len(news))]
    rows = int(start[-1])
    who = torch.from_numpy(np.repeat(adapter, news)).to(G.DEV)
    x, base = torch.randn(rows, K, device=G.DEV).bfloat16(), torch.randn(rows, N, device=G.DEV).bfloat16()
    odd = torch.arange(0, rows, 5, device=G.DEV)
    at = torch.randint(0, K, (len(odd),), device=G.DEV)
    sign = torch.randint(0, 2, (len(odd),), device=G.DEV) * 2.0 - 1
    x[odd, at] = (float("inf") * sign).bfloat16()
    out = torch.empty_like(base)
    B.qllm_adapters_add(B.Adapters(A, Bm, scale, ints([rank] * slots)), x, base, out, ints(start), ints(adapter))
    # terms of an output: their signs are those of a, b and the infinity
    up = (A[who[odd], :rank, at].double().sign() * sign.double()[:, None])[:, None] * Bm[who[odd], :, :rank].double().sign()
    want = torch.where((up > 0).all(2), float("inf"), torch.where((up < 0).all(2), -float("inf"), float("nan")))
    got = out[odd].double()
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got[~want.isnan()], want[~want.isnan()])
    rest = torch.ones(rows, dtype=torch.bool, device=G.DEV)
    rest[odd] = False
    assert out[rest].isfinite().all()
