"""The norm, the adapters and the rotating append refuse handles and tensors that are not on the current device; a call captured before any
other call of its kind has run."""
import subprocess
import sys

import pytest
import torch

import gpu_util as G
from paper_2310_08041_b200 import binding as B
from test_gpu_kv import ints, random_cache

pytestmark = pytest.mark.gpu


def operands():
    x, y = torch.randn(3, 128, device=G.DEV), torch.empty(3, 128, device=G.DEV)
    codes, s, z = torch.empty(3, 128, dtype=torch.uint8, device=G.DEV), torch.empty(3, device=G.DEV), torch.empty(3, device=G.DEV)
    ad = B.Adapters(torch.zeros(2, 8, 128, device=G.DEV).bfloat16(), torch.zeros(2, 128, 8, device=G.DEV).bfloat16(), torch.ones(2, device=G.DEV))
    rot, cache = B.Rotary(torch.zeros(8, 32, 2, device=G.DEV)), random_cache(3, 1, 4, 2, 16, 64)
    batch = B.KvBatch(ints([[0]]), ints([3]), ints([0, 3]), 3, 3)
    return x, y, codes, s, z, ad, rot, cache, batch


def calls(x, y, codes, s, z, ad, rot, cache, batch):
    g, q, kv = torch.ones(128, device=G.DEV), torch.zeros(3, 4, 64, device=G.DEV), torch.zeros(3, 2, 64, device=G.DEV)
    start, which = ints([0, 3]), ints([0])
    return [lambda: B.qllm_rmsnorm_quant(x, g, 8, codes, s, z), lambda: B.qllm_dequantize_rows(codes, s, z, 8, y),
            lambda: B.qllm_adapters_add(ad, x, x, y, start, which), lambda: B.qllm_rotary_table(rot.table),
            lambda: B.qllm_kv_rotate_append(cache, 0, q, q, kv, kv, rot, batch)]


def refused(fn):
    before = B.qllm_launch_count()
    with pytest.raises(AssertionError):
        fn()
    assert B.qllm_launch_count() == before


def test_another_device_is_current(monkeypatch):
    """One GPU stands in for two: the binding asks for the current device in one place."""
    todo = calls(*operands())
    for fn in todo:
        fn()
    torch.cuda.synchronize()
    monkeypatch.setattr(B, "_current_device", lambda: 1)
    for fn in todo:
        refused(fn)


@pytest.mark.parametrize("which,uses", [(5, [2]), (6, [4]), (7, [4]), (8, [4])])
def test_a_handle_of_another_device(which, uses):
    o = operands()
    todo = calls(*o)
    o[which].device = 1
    for i in uses:
        refused(todo[i])


CAPTURE = """
import sys, torch
sys.path[:0] = %r
import test_gpu_block_device as D
from paper_2310_08041_b200 import binding as B
todo = D.calls(*D.operands())
torch.cuda.synchronize()
g, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
fn = todo[int(sys.argv[1])]
with torch.cuda.graph(g, stream=st):
    fn()
g.replay()
torch.cuda.synchronize()
assert B.qllm_poll_status() == B.QLLM_OK
"""


@pytest.mark.parametrize("i", range(5))
def test_captured_without_a_call_before(i):
    """In a process of its own."""
    r = subprocess.run([sys.executable, "-c", CAPTURE % sys.path, str(i)], capture_output=True, text=True, timeout=240)
    assert r.returncode == 0, r.stderr[-1500:]


CAPTURE_TILES = """
import sys, torch
sys.path[:0] = %r
from paper_2310_08041_b200 import binding as B
top, rows = int(sys.argv[1]), int(sys.argv[2])
ad = B.Adapters(torch.ones(2, top, 256, device="cuda").bfloat16(), torch.ones(2, 128, top, device="cuda").bfloat16(), torch.ones(2, device="cuda"))
x, out = torch.ones(rows, 256, device="cuda").bfloat16(), torch.zeros(rows, 128, device="cuda").bfloat16()
start, which = torch.tensor([0, rows], dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
torch.cuda.synchronize()
g, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
with torch.cuda.graph(g, stream=st):
    B.qllm_adapters_add(ad, x, None, out, start, which)
g.replay()
torch.cuda.synchronize()
assert B.qllm_poll_status() == B.QLLM_OK and (out == 256.0 * top).all()
"""


@pytest.mark.parametrize("top,rows", [(16, 3), (128, 3), (40, 200), (16, 2000)])
def test_adapters_captured_without_a_call_before(top, rows):
    """Every kind of launch asks the device what it holds; 256 * rank is a bf16 number."""
    r = subprocess.run([sys.executable, "-c", CAPTURE_TILES % sys.path, str(top), str(rows)], capture_output=True, text=True, timeout=240)
    assert r.returncode == 0, r.stderr[-1500:]
