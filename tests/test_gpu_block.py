"""The norm, the adapters and the rotating append as a decoder block uses them, around a quantized QKV and output projection and
the 4-bit cache: a prompt of several requests with adapters of their own, then steps, eager and from a graph."""
import numpy as np
import pytest
import torch

import block_ref
import gpu_util as G
import kv_ref
from paper_2310_08041_b200 import binding as B
from test_gpu_kv import DT, attend, check_attention, host, ints, store_of

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def seeded():
    torch.manual_seed(7)


class Projection:
    """A quantized projection (4-bit weights of plain Eq. 2 per output channel) behind 8-bit activations."""

    def __init__(self, K, N):
        w = torch.randn(N, K, device=G.DEV) * K ** -0.5
        self.codes = torch.empty(N, K // 2, dtype=torch.uint8, device=G.DEV)
        self.scale, self.zero, self.colsum = torch.empty(N, device=G.DEV), torch.empty(N, device=G.DEV), torch.empty(N, dtype=torch.int32, device=G.DEV)
        B.qllm_quantize_rows(w, 4, self.codes, self.scale, self.zero, self.colsum)
        self.K, self.N = K, N
        self.values = torch.empty(N, K, device=G.DEV)
        B.qllm_dequantize_rows(self.codes, self.scale, self.zero, 4, self.values)

    def __call__(self, a, out):
        B.qllm_qgemm(a.codes, a.scale, a.zero, self.codes, self.scale, self.zero, self.colsum, None, out, out.shape[0], self.N, self.K, 8, 4, a_rowsum=a.rowsum)


class Codes:
    def __init__(self, M, C):
        self.codes = torch.empty(M, C, dtype=torch.uint8, device=G.DEV)
        self.scale, self.zero, self.rowsum = torch.empty(M, device=G.DEV), torch.empty(M, device=G.DEV), torch.empty(M, dtype=torch.int32, device=G.DEV)

    def values(self):
        return (self.codes.double() - self.zero.double()[:, None]) * self.scale.double()[:, None]


class Block:
    """Attention half of a decoder block: norm, QKV with adapters, rotation into the cache, attention, output with adapters, norm."""

    def __init__(self, C, heads, q_heads, d, slots, top):
        self.C, self.heads, self.q_heads, self.d = C, heads, q_heads, d
        self.gamma, self.gamma2 = (1 + 0.1 * torch.randn(C, device=G.DEV) for _ in range(2))
        self.qkv, self.o = Projection(C, (q_heads + 2 * heads) * d), Projection(q_heads * d, C)
        ranks = ints([top, top // 2, top - 1][:slots])
        make = lambda K, N: B.Adapters((torch.randn(slots, top, K, device=G.DEV) * K ** -0.5).bfloat16(), (0.3 * torch.randn(slots, N, top, device=G.DEV)).bfloat16(),  # noqa: E731
                                       torch.rand(slots, device=G.DEV) + 0.5, ranks)
        self.ad_qkv, self.ad_o = make(C, self.qkv.N), make(q_heads * d, C)
        self.rotary = B.Rotary.make(300, d)

    def buffers(self, M):
        e = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=G.DEV)  # noqa: E731
        return dict(h=e(M, self.C), y=e(M, self.C), a=Codes(M, self.C), qkv=e(M, self.qkv.N), att=e(M, self.q_heads, self.d), b=Codes(M, self.q_heads * self.d),
                    o=e(M, self.C), h2=e(M, self.C), c=Codes(M, self.C), base=e(M, self.qkv.N), base_o=e(M, self.C), turned=e(M, self.q_heads, self.d))

    def __call__(self, x, residual, t, cache, layer, batch, adapter, workspace):
        """x: the layer before's output, residual: the stream.  Keeps what the checks need."""
        M, H, Hk, d = x.shape[0], self.q_heads, self.heads, self.d
        B.qllm_rmsnorm_quant(x, self.gamma, 8, t["a"].codes, t["a"].scale, t["a"].zero, t["a"].rowsum, residual=residual, h=t["h"], y=t["y"])
        self.qkv(t["a"], t["base"])
        B.qllm_adapters_add(self.ad_qkv, t["y"], t["base"], t["qkv"], batch.q_start, adapter)
        rows = t["qkv"].view(M, H + 2 * Hk, d)
        B.qllm_kv_rotate_append(cache, layer, rows[:, :H], t["turned"], rows[:, H:H + Hk], rows[:, H + Hk:], self.rotary, batch)
        B.qllm_kv_attention(cache, layer, t["turned"], t["att"], d ** -0.5, batch, workspace)
        flat = t["att"].view(M, H * d)
        B.qllm_quantize_rows(flat, 8, t["b"].codes, t["b"].scale, t["b"].zero, t["b"].rowsum)
        self.o(t["b"], t["base_o"])
        B.qllm_adapters_add(self.ad_o, flat, t["base_o"], t["o"], batch.q_start, adapter)
        B.qllm_rmsnorm_quant(t["o"], self.gamma2, 8, t["c"].codes, t["c"].scale, t["c"].zero, t["c"].rowsum, residual=t["h"], h=t["h2"])

    def check(self, x, residual, t, cache, layer, batch, adapter):
        """Every step against 64 bits on what it was given."""
        half = 2.0 ** -9 * (1 + 2.0 ** -7)                   # bf16's rounding, and float32's behind it
        M, H, Hk, d = x.shape[0], self.q_heads, self.heads, self.d
        start, lens, table = batch.q_start.tolist(), batch.seq_lens.tolist(), batch.table.cpu().numpy()
        f = lambda v: v.float().cpu().numpy()  # noqa: E731
        hh, y, factor, codes, zero, alpha, _ = block_ref.norm(f(x), f(residual), f(self.gamma), 1e-5, None, 8)
        assert np.array_equal(t["a"].codes.cpu().numpy(), codes) and np.allclose(f(t["y"]), y, rtol=2 * half, atol=0)
        base = t["a"].values() @ self.qkv.values.double().T
        mag = t["a"].values().abs() @ self.qkv.values.double().abs().T
        # (the product of the values as stored: float32 products of scales, and the GEMM's rounding)
        assert ((t["base"].double() - base).abs() <= 2 * half * base.abs() + 2.0 ** -22 * mag).all()
        for ad, src, b, out in ((self.ad_qkv, t["y"], t["base"], t["qkv"]), (self.ad_o, t["att"].view(M, H * d), t["base_o"], t["o"])):
            want, first, second = block_ref.adapters(ad.A, ad.B, ad.scale, ad.rank.tolist(), src, b, start, adapter.tolist())
            assert ((out.double() - want).abs() <= 2 * half * want.abs() + (ad.K / 16 + 32) * 2.0 ** -23 * first + 2.0 ** -15 * second).all()
        pos = np.concatenate([np.arange(n - (e - s), n) for n, s, e in zip(lens, start[:-1], start[1:])])
        cs = f(self.rotary.table)[pos]
        rows = f(t["qkv"]).reshape(M, H + 2 * Hk, d)
        turned = block_ref.turned(rows, cs[..., 0], cs[..., 1], d, False)
        assert torch.equal(t["turned"].cpu(), torch.from_numpy(turned[:, :H]).bfloat16())
        st, seq = store_of(cache, layer), np.repeat(np.arange(len(lens)), np.diff(start))
        pg, at = table[seq, pos // st.page], pos % st.page
        assert np.array_equal(st.kc[pg, :, at], kv_ref.quantize(turned[:, H:H + Hk])[0]) and np.array_equal(st.vc[pg, :, at], kv_ref.quantize(rows[:, H + Hk:])[0])
        ref = kv_ref.attention(st, table, lens, start, host(t["turned"]), d ** -0.5, True)
        check_attention(t["att"], torch.from_numpy(ref[1]).float(), ref, torch.bfloat16, prompt=batch.max_new * H // Hk > 96)
        _, _, _, codes, _, _, _ = block_ref.norm(f(t["o"]), f(t["h"]), f(self.gamma2), 1e-5, None, 8)
        assert np.array_equal(t["c"].codes.cpu().numpy(), codes)


@pytest.mark.parametrize("C,heads,q_heads,d,top", [(512, 2, 4, 64, 16), (1024, 1, 8, 128, 40)])
def test_block(C, heads, q_heads, d, top):
    block, page, seqs = Block(C, heads, q_heads, d, 3, top), 16, 4
    cache, pool = B.KvCache.empty(2, 40, heads, page, d), B.KvPool.empty(40, seqs, 12)
    adapter = ints([1, -1, 0, 1])
    B.qllm_kv_pages_extend(cache, pool, ints([37, 1, 90, 12]))
    start = [0, 37, 38, 128, 140]
    batch = B.KvBatch(pool.table, pool.seq_lens, ints(start), 140, 90)
    x, residual = torch.randn(140, C, device=G.DEV).bfloat16(), (2 * torch.randn(140, C, device=G.DEV)).bfloat16()
    t = block.buffers(140)
    ws = torch.empty(max(16, B.qllm_kv_attention_workspace(cache, q_heads, t["turned"], batch)), dtype=torch.uint8, device=G.DEV)
    block(x, residual, t, cache, 1, batch, adapter, ws)
    block.check(x, residual, t, cache, 1, batch, adapter)

    # single tokens, first eager, then from a graph that also takes the new tokens' pages
    one = ints([1] * seqs)
    batch = B.KvBatch(pool.table, pool.seq_lens, ints([0, 1, 2, 3, 4]), seqs, 1)
    x, residual, t = x[:seqs].clone(), residual[:seqs].clone(), block.buffers(seqs)
    ws = torch.empty(max(16, B.qllm_kv_attention_workspace(cache, q_heads, t["turned"], batch)), dtype=torch.uint8, device=G.DEV)
    side = torch.cuda.Stream()

    def step():
        B.qllm_kv_pages_extend(cache, pool, one)
        block(x, residual, t, cache, 1, batch, adapter, ws)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    block.check(x, residual, t, cache, 1, batch, adapter)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for new in ([1, -1, 0, 1], [2, 0, -1, -1], [0, 0, 0, 0]):
        x.normal_(); residual.normal_()
        adapter.copy_(ints(new))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        block.check(x, residual, t, cache, 1, batch, adapter)
    assert B.qllm_poll_status() == B.QLLM_OK and pool.seq_lens.tolist() == [41, 5, 94, 16]


def test_nothing_takes_device_memory():
    """Every call a second time: free memory as before."""
    block = Block(512, 2, 4, 64, 2, 16)
    cache, table = B.KvCache.empty(1, 8, 2, 16, 64), ints([[0, 1, 2], [3, 4, 5]])
    batch = B.KvBatch(table, ints([20, 30]), ints([0, 20, 50]), 50, 30)
    x, r, t = torch.randn(50, 512, device=G.DEV).bfloat16(), torch.randn(50, 512, device=G.DEV).bfloat16(), block.buffers(50)
    ws = torch.empty(max(16, B.qllm_kv_attention_workspace(cache, 4, t["turned"], batch)), dtype=torch.uint8, device=G.DEV)
    values, adapter = torch.empty(50, 512, device=G.DEV), ints([0, 1])

    def calls():
        block(x, r, t, cache, 0, batch, adapter, ws)
        B.qllm_dequantize_rows(t["a"].codes, t["a"].scale, t["a"].zero, 8, values)
        B.qllm_rotary_table(block.rotary.table)
    calls()
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    for _ in range(3):
        calls()
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free


def test_two_streams_at_once():
    """The same calls on two streams with operands of their own, many times: no result depends on the other stream."""
    sides = []
    for i in range(2):
        torch.manual_seed(i)
        block = Block(1024, 2, 8, 128, 3, 32)
        cache, table = B.KvCache.empty(1, 40, 2, 16, 128), ints(np.arange(36).reshape(3, 12))
        lens, start = [180, 31, 5], [0, 180, 181, 183]
        batch = B.KvBatch(table, ints(lens), ints(start), 183, 180)
        x, r, t = torch.randn(183, 1024, device=G.DEV).bfloat16(), torch.randn(183, 1024, device=G.DEV).bfloat16(), block.buffers(183)
        ws = torch.empty(max(16, B.qllm_kv_attention_workspace(cache, 8, t["turned"], batch)), dtype=torch.uint8, device=G.DEV)
        sides.append((block, x, r, t, cache, batch, ints([0, 2, 1]), ws, torch.cuda.Stream()))
    torch.cuda.synchronize()
    first = []
    for block, x, r, t, cache, batch, adapter, ws, st in sides:
        with torch.cuda.stream(st):
            block(x, r, t, cache, 0, batch, adapter, ws)
        st.synchronize()
        first.append([t["qkv"].clone(), t["turned"].clone(), t["c"].codes.clone(), t["o"].clone()])
    torch.cuda.synchronize()
    for _ in range(30):
        for block, x, r, t, cache, batch, adapter, ws, st in sides:
            with torch.cuda.stream(st):
                block(x, r, t, cache, 0, batch, adapter, ws)
    torch.cuda.synchronize()
    for want, (block, x, r, t, *_) in zip(first, sides):
        for a, b in zip(want, (t["qkv"], t["turned"], t["c"].codes, t["o"])):
            assert torch.equal(a, b)
    assert B.qllm_poll_status() == B.QLLM_OK
