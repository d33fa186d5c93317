"""qllm_adapters_add: the sums over K enter the product with B with all of their bits.

Every row of x has one number and every adapter one row of A, so a sum over K is one product a x, and out = base + s a x b has one term.  base takes
away that term rounded to bf16: what is left of it are the bits behind the eighth, and those are compared.

Bound, in units of the term t = s a x b.  a x: exact for bf16 x; float32 x goes in as three parts, whose products are summed in float32 (two
additions; an MMA's may be truncated: 2^-23 each, one more for a result that is rounded on its way).  s (a x): 2^-24.  Its three parts hold 24 bits;
their products with b are exact and summed in float32 (three additions, 2^-23 each).  Then base is added (2^-24 of what comes out) and the result rounded
to its type."""
import numpy as np
import pytest
import torch

import gpu_util as G
from paper_2310_08041_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=G.DEV)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("top", [8, 16, 24, 32, 40, 64, 72, 128])
@pytest.mark.parametrize("news", [[1] * 40, [1], [37, 20, 11], [200, 150, 90], [900, 200, 130]], ids=["step", "token", "some", "prompts", "long"])
def test_what_base_leaves_of_a_term(dtype, top, news):
    K, N, slots = 72, 264, 3
    gen = torch.Generator(device=G.DEV)
    gen.manual_seed(top + len(news))
    normal = lambda *s: torch.randn(*s, generator=gen, device=G.DEV)  # noqa: E731
    at = [0, top // 2, top - 1]                            # the row of each adapter
    A, Bm = torch.zeros(slots, top, K, device=G.DEV), normal(slots, N, top).bfloat16()
    for a, r in enumerate(at):
        A[a, r] = normal(K)
    A = A.bfloat16()
    scale = 0.5 + torch.rand(slots, generator=gen, device=G.DEV)
    start, adapter = np.concatenate([[0], np.cumsum(news)]), [s % slots for s in range(len(news))]
    rows = int(start[-1])
    who = torch.from_numpy(np.repeat(adapter, news)).to(G.DEV)
    col = torch.randint(0, K, (rows,), generator=gen, device=G.DEV)
    x = torch.zeros(rows, K, device=G.DEV).to(DT[dtype])
    x[torch.arange(rows), col] = normal(rows).to(DT[dtype])
    row = torch.tensor(at, device=G.DEV)[who]
    term = (scale.double()[who] * A.double()[who, row, col] * x.double().sum(1))[:, None] * Bm.double()[who, :, row]
    base = -term.bfloat16().to(DT[dtype])
    want = base.double() + term
    out = torch.empty(rows, N, device=G.DEV).to(DT[dtype])
    B.qllm_adapters_add(B.Adapters(A, Bm, scale), x, base, out, ints(start), ints(adapter))
    tol = ((0 if dtype == "bf16" else 3) * 2.0 ** -23 + 2.0 ** -24 + 3 * 2.0 ** -23) * term.abs() + (2.0 ** -24 + torch.finfo(DT[dtype]).eps / 2) * want.abs() + 2.0 ** -120
    off = (out.double() - want).abs()
    assert (off <= tol).all(), "%d of %d beyond the bound, worst %.3g times" % ((off > tol).sum(), off.numel(), (off / tol).max())
    assert B.qllm_poll_status() == B.QLLM_OK
