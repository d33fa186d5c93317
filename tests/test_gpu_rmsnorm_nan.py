"""qllm_rmsnorm_quant: a row whose only number that is not zero is a NaN or an infinity keeps it."""
import pytest
import torch

import gpu_util as G
from paper_2310_08041_b200 import binding as B

pytestmark = pytest.mark.gpu


def one_each(C, drop=None):
    """A map that takes every channel as it is, but for `drop`, in whose place the next one comes twice."""
    src = torch.arange(C, dtype=torch.int32, device=G.DEV)
    if drop is not None:
        src[drop] = (drop + 1) % C
    return torch.arange(C + 1, dtype=torch.int32, device=G.DEV), src, torch.ones(C, device=G.DEV)


# one row and many (other kernels), channels in registers, in more of them, in shared memory
@pytest.mark.parametrize("M", [3, 400])
@pytest.mark.parametrize("C", [24, 1004, 2048, 4096, 8192, 8200, 16384])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("which", ["plain", "map", "dropped"])
def test_among_zeros(M, C, dtype, which):
    at, odd, last = C // 3, M // 2, M - 1
    x, r = torch.zeros(M, C, device=G.DEV, dtype=dtype), torch.zeros(M, C, device=G.DEV, dtype=dtype)
    (x if C % 16 else r)[odd, at] = float("nan")
    x[last, at] = float("inf")
    gamma = torch.full((C,), 1.25, device=G.DEV)
    csr = None if which == "plain" else one_each(C, at if which == "dropped" else None)
    for bits in (4, 8):
        codes = torch.empty(M, C // 2 if bits == 4 else C, dtype=torch.uint8, device=G.DEV)
        scale, zero, values, y = torch.empty(M, device=G.DEV), torch.empty(M, device=G.DEV), torch.empty_like(x), torch.empty_like(x)
        B.qllm_rmsnorm_quant(x, gamma, bits, codes, scale, zero, residual=r, y=y, map=csr)
        B.qllm_dequantize_rows(codes, scale, zero, bits, values)
        assert scale[odd].isnan() and values[odd].isnan().all() and y[odd].isnan().all()
        # the factor of a row with an infinity is 0
        assert scale[last].isnan() or scale[last] == 0
        others = [m for m in range(M) if m not in (odd, last)]
        assert (scale[others] == 1).all() and (values[others] == 0).all() and (y[others] == 0).all()
