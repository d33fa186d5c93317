"""qllm_rmsnorm_quant and qllm_dequantize_rows on the GPU against plain statements of them (block_ref).

Codes, zero-points and code sums are decided by float32 operations that do not depend on an order, so they have to be equal.  h is one float32
addition and one rounding: equal too.  What depends on the sum of squares has a bound: at most 96 terms of one sign per thread in order
and ten levels of a tree, half a step 2^-24 each; the factor takes the root, half of that; division by C, eps, root, reciprocal and the product
with alpha (itself two roundings) or u (two) add 8 roundings at most."""
import numpy as np
import pytest
import torch

import block_ref
import gpu_util as G
from paper_2310_08041_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
FACTOR = ((96 + 10) / 2 + 8) * 2.0 ** -24


def rounded(a, dtype):
    """float64 array -> the nearest values of dtype, through float32 as the kernels' results go."""
    return torch.from_numpy(np.asarray(a, np.float32)).to(dtype)


def run(x, residual, gamma, eps, csr, bits, want_y=True, want_h=True, inplace=None, stream=None):
    """Every output between canaries.  x, residual: device tensors."""
    M, C = x.shape
    g = dict(codes=G.Guarded((M, C // 2 if bits == 4 else C), torch.uint8, 0xAB), scale=G.Guarded((M,), torch.float32, -1.0),
             zero=G.Guarded((M,), torch.float32, -1e9), rowsum=G.Guarded((M,), torch.int32, -7), values=G.Guarded((M, C), x.dtype, 3.0))
    if want_y:
        g["y"] = G.Guarded((M, C), x.dtype, 3.0)
    if want_h and inplace is None:
        g["h"] = G.Guarded((M, C), x.dtype, 3.0)
    h = inplace if inplace is not None else g["h"].t if want_h else None
    B.qllm_rmsnorm_quant(x, gamma, bits, g["codes"].t, g["scale"].t, g["zero"].t, g["rowsum"].t, residual=residual, h=h, y=g["y"].t if want_y else None,
                         map=csr, eps=eps, stream=stream)
    B.qllm_dequantize_rows(g["codes"].t, g["scale"].t, g["zero"].t, bits, g["values"].t, stream=stream)
    torch.cuda.synchronize()
    for k, v in g.items():
        v.check(k)
    out = {k: v.t for k, v in g.items()}
    if h is not None:
        out["h"] = h
    return out


def check(got, x, residual, gamma, eps, csr, bits):
    """x, residual: as they were before the call."""
    host = lambda t: None if t is None else t.float().cpu().numpy()  # noqa: E731
    csr_np = None if csr is None else [t.cpu().numpy() for t in csr]
    h, y, factor, codes, zero, alpha, _ = block_ref.norm(host(x), host(residual), host(gamma), eps, csr_np, bits)
    dtype, eps_t = x.dtype, torch.finfo(x.dtype).eps / 2
    have = block_ref.unpack(got["codes"].cpu().numpy(), bits)
    assert np.array_equal(have, codes), "%d codes differ" % (have != codes).sum()
    assert np.array_equal(got["zero"].cpu().numpy(), zero[:, 0])
    assert np.array_equal(got["rowsum"].cpu().numpy(), codes.sum(1))
    flat = (codes == zero).all(1) & (zero[:, 0] == 0) & (alpha[:, 0] == 1)      # rows of zeros: scale 1
    scale = np.where(flat, 1.0, (alpha * factor)[:, 0])
    s = got["scale"].cpu().numpy().astype(np.float64)
    assert (np.abs(s - scale) <= FACTOR * np.abs(scale)).all(), (np.abs(s - scale) / scale).max() / FACTOR
    if "h" in got:
        assert torch.equal(got["h"].cpu(), rounded(h, dtype))
    if "y" in got:
        bad = np.abs(host(got["y"]) - y) > (FACTOR + eps_t) * np.abs(y) + 2.0 ** -140
        assert not bad.any(), bad.sum()
    back = (codes - zero) * s[:, None]                      # two float32 roundings and the type's
    assert (np.abs(host(got["values"]) - back) <= (2 * 2.0 ** -24 + eps_t) * np.abs(back) + 2.0 ** -140).all()


def inputs(seed, M, C, dtype, with_residual):
    gen = torch.Generator(device=G.DEV); gen.manual_seed(seed)
    x = torch.randn(M, C, generator=gen, device=G.DEV)
    x[:, torch.randint(0, C, (max(1, C // 100),), generator=gen, device=G.DEV)] *= 25
    r = (2 * torch.randn(M, C, generator=gen, device=G.DEV)).to(DT[dtype]) if with_residual else None
    return x.to(DT[dtype]), r, 1 + 0.1 * torch.randn(C, generator=gen, device=G.DEV)


CASES = [(1, 8), (3, 24), (2, 100), (5, 1000), (300, 512), (4, 1028), (1, 2048), (700, 4096), (9, 4104), (61, 5120), (310, 5120), (2, 8192), (333, 8192),
         (3, 8200), (2, 12000), (297, 16384), (2, 16392), (2, 20002), (1, 49152)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,C", CASES)
@pytest.mark.parametrize("residual,bits", [(True, 8), (False, 4), (True, 4), (True, 6)])
def test_norm(dtype, M, C, residual, bits):
    x, r, g = inputs(M + C + bits, M, C, dtype, residual)
    check(run(x, r, g, 1e-5, None, bits), x, r, g, 1e-5, None, bits)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,C", [(1, 64), (5, 1000), (2, 1026), (297, 2048), (1, 4096), (7, 4096), (301, 4096), (3, 5120), (299, 8192), (2, 8200), (2, 12000)])
@pytest.mark.parametrize("residual,bits", [(True, 8), (False, 4), (True, 6)])
def test_norm_with_a_map(dtype, M, C, residual, bits):
    x, r, g = inputs(M + C + bits, M, C, dtype, residual)
    csr = [G.dev(a) for a in block_ref.random_map(np.random.RandomState(C + bits), C)]
    check(run(x, r, g, 1e-5, csr, bits), x, r, g, 1e-5, csr, bits)


@pytest.mark.parametrize("C", [40, 1004, 4096, 8192])
def test_norm_alone(C):
    """Without codes, and with y or h alone."""
    x, r, g = inputs(C, 70, C, "bf16", True)
    both = run(x, r, g, 1e-6, None, 8)
    y, h = G.Guarded((70, C), x.dtype, 3.0), G.Guarded((70, C), x.dtype, 3.0)
    B.qllm_rmsnorm_quant(x, g, 8, None, None, None, residual=r, y=y.t, eps=1e-6)
    B.qllm_rmsnorm_quant(x, g, 8, None, None, None, residual=r, h=h.t, eps=1e-6)
    torch.cuda.synchronize()
    y.check("y"); h.check("h")
    assert torch.equal(y.t, both["y"]) and torch.equal(h.t, both["h"])


def test_odd_channel_counts_in_8_bits():
    x, r, g = inputs(5, 6, 1001, "f32", True)
    check(run(x, r, g, 1e-5, None, 8), x, r, g, 1e-5, None, 8)


@pytest.mark.parametrize("which", ["residual", "x"])
@pytest.mark.parametrize("dtype,M,C", [("bf16", 350, 4096), ("f32", 2, 1004), ("bf16", 1, 8192)])
def test_residual_stream_in_place(which, dtype, M, C):
    x, r, g = inputs(M, M, C, dtype, True)
    x0, r0 = x.clone(), r.clone()
    check(run(x, r, g, 1e-5, None, 8, inplace=r if which == "residual" else x), x0, r0, g, 1e-5, None, 8)


@pytest.mark.parametrize("C", [16, 1004, 4096, 16384])
@pytest.mark.parametrize("with_map", [False, True])
def test_rows_of_every_size(C, with_map):
    """Rows whose squares pass float32 or vanish in it, next to ordinary ones; eps small enough to leave them alone."""
    sizes = [1e-38, 1e-30, 1e-19, 1e-12, 1.0, 1e12, 1e19, 1e30, 1e37]
    x, _, g = inputs(3, len(sizes), C, "f32", False)
    x = (x / x.abs().amax(1, keepdim=True) * torch.tensor(sizes, device=G.DEV)[:, None]).contiguous()
    csr = [G.dev(a) for a in block_ref.random_map(np.random.RandomState(C), C)] if with_map else None
    got = run(x, None, g, 0.0, csr, 8)
    csr_np = None if csr is None else [t.cpu().numpy() for t in csr]
    for i, size in enumerate(sizes):
        # every row is an ordinary one times a power of two, exactly: that one's codes, and its scale, for eps = 0
        by = 2.0 ** -np.floor(np.log2(size))
        row = (x[i:i + 1].double() * by).float()
        assert torch.equal(row.double() / by, x[i:i + 1].double())
        _, y, factor, codes, zero, alpha, _ = block_ref.norm(row.cpu().numpy(), None, g.cpu().numpy(), 0.0, csr_np, 8)
        assert np.array_equal(got["codes"][i].cpu().numpy(), codes[0]) and got["zero"][i].item() == zero[0, 0], size
        assert abs(got["scale"][i].item() / (alpha * factor).item() - 1) <= FACTOR, size
        assert (np.abs(got["y"][i].cpu().numpy() - y[0]) <= (FACTOR + 2.0 ** -24) * np.abs(y[0]) + 2.0 ** -100).all(), size


@pytest.mark.parametrize("C", [24, 1004, 4096])
def test_zeros_constants_infinities_and_nan(C):
    x, _, g = inputs(4, 6, C, "f32", False)
    g.fill_(1.0)
    x[0] = 0
    x[1] = 3.5
    x[2, 1] = float("nan")
    x[3, 2] = float("inf")
    x[4] = 1000 + 1e-3 * x[4].sign()                         # far from zero, next to no range
    for eps in (1e-5, 0.0):
        got = run(x, None, g, eps, None, 8)
        v, s = got["values"], got["scale"]
        assert (v[0] == 0).all() and s[0] == 1 and (got["y"][0] == 0).all()
        assert ((v[1] - 1).abs() < 1e-5).all() and (got["rowsum"][1] == got["codes"][1].int().sum()).all()
        assert s[2].isnan() and v[2].isnan().all() and got["y"][2].isnan().all()
        assert not s[3].isfinite() or s[3] == 0
        assert got["y"][3, 2].isnan() and (got["y"][3, 3:] == 0).all()           # inf / inf, finite / inf
        check({k: t[4:] for k, t in got.items()}, x[4:], None, g, eps, None, 8)


def test_no_rows():
    x = torch.empty(0, 64, device=G.DEV)
    z = torch.empty(0, device=G.DEV)
    B.qllm_rmsnorm_quant(x, torch.ones(64, device=G.DEV), 8, torch.empty(0, 64, dtype=torch.uint8, device=G.DEV), z, z)
    B.qllm_dequantize_rows(torch.empty(0, 64, dtype=torch.uint8, device=G.DEV), z, z, 8, x)


@pytest.mark.parametrize("bits", [4, 6, 8])
@pytest.mark.parametrize("C", [2, 34, 1000, 4096, 4112])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_dequantize_rows_of_the_row_quantizer(bits, C, dtype):
    """What qllm_quantize_rows writes, read back."""
    M = 37
    x, _, _ = inputs(bits, M, C, dtype, False)
    codes, s, z = torch.empty(M, C // 2 if bits == 4 else C, dtype=torch.uint8, device=G.DEV), torch.empty(M, device=G.DEV), torch.empty(M, device=G.DEV)
    B.qllm_quantize_rows(x, bits, codes, s, z)
    out = G.Guarded((M, C), DT[dtype], 3.0)
    B.qllm_dequantize_rows(codes, s, z, bits, out.t)
    torch.cuda.synchronize()
    out.check()
    diff = block_ref.unpack(codes.cpu().numpy(), bits).astype(np.float32) - z.cpu().numpy()[:, None]     # exact: both are small integers
    assert torch.equal(out.t.cpu(), rounded(diff * s.cpu().numpy()[:, None], DT[dtype]))


def test_codes_do_not_depend_on_the_batch():
    """A row alone and among others (other kernels) has the same codes."""
    x, r, g = inputs(9, 400, 4096, "bf16", True)
    csr = [G.dev(a) for a in block_ref.random_map(np.random.RandomState(2), 4096)]
    for m in (None, csr):
        whole, one = run(x, r, g, 1e-5, m, 4), run(x[123:124].clone(), r[123:124].clone(), g, 1e-5, m, 4)
        assert torch.equal(whole["codes"][123:124], one["codes"]) and torch.equal(whole["rowsum"][123:124], one["rowsum"])


def test_stream_and_graph():
    """Captured on a side stream and replayed with other contents; feeds the integer GEMM as qllm_reassemble_quant's output does."""
    M, C, N, bits = 20, 512, 256, 8
    x, r, g = inputs(11, M, C, "bf16", True)
    qw = torch.randint(0, 16, (N, C), device=G.DEV, dtype=torch.uint8)
    packed = (qw[:, 0::2] | (qw[:, 1::2] << 4)).contiguous()
    ws, wz = torch.rand(N, device=G.DEV) * 0.01, torch.full((N,), 8.0, device=G.DEV)
    colsum = qw.int().sum(1, dtype=torch.int32)
    codes, s, z, rs = torch.empty(M, C, dtype=torch.uint8, device=G.DEV), torch.empty(M, device=G.DEV), torch.empty(M, device=G.DEV), torch.empty(M, dtype=torch.int32, device=G.DEV)
    h, out = torch.empty_like(x), torch.empty(M, N, device=G.DEV)
    st = torch.cuda.Stream()

    def step():
        B.qllm_rmsnorm_quant(x, g, bits, codes, s, z, rs, residual=r, h=h, stream=st)
        B.qllm_qgemm(codes, s, z, packed, ws, wz, colsum, None, out, M, N, C, bits, 4, a_rowsum=rs, stream=st)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        step()
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        step()
    for seed in (1, 2):
        x2, r2, _ = inputs(seed, M, C, "bf16", True)
        x.copy_(x2); r.copy_(r2); out.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            graph.replay()
        torch.cuda.synchronize()
        _, _, factor, c, zero, alpha, _ = block_ref.norm(x.float().cpu().numpy(), r.float().cpu().numpy(), g.cpu().numpy(), 1e-5, None, bits)
        assert np.array_equal(codes.cpu().numpy(), c)
        whole = torch.from_numpy(c - zero).to(G.DEV) @ (qw.double() - 8).T       # integers: exact, also where they cancel
        want = whole * torch.from_numpy(alpha * factor).to(G.DEV) * ws.double()
        # a_scale's error, the epilogue's two products and the sum's rounding to float32
        assert ((out - want).abs() <= (FACTOR + 4 * 2.0 ** -24) * want.abs() + 1e-30).all()


def test_wrong_tensors_are_refused():
    x, r, g = inputs(1, 4, 64, "bf16", True)
    codes, s, z = torch.empty(4, 64, dtype=torch.uint8, device=G.DEV), torch.empty(4, device=G.DEV), torch.empty(4, device=G.DEV)
    before = B.qllm_launch_count()
    for fn, e in [(lambda: B.qllm_rmsnorm_quant(x, g, 4, codes, s, z), "SHAPE"), (lambda: B.qllm_rmsnorm_quant(x, g[:32], 8, codes, s, z), "SHAPE"),
                  (lambda: B.qllm_rmsnorm_quant(x, g, 8, codes, s[:3], z), "SHAPE"), (lambda: B.qllm_rmsnorm_quant(x, g, 8, codes, s, z, residual=r.float()), "DTYPE"),
                  (lambda: B.qllm_rmsnorm_quant(x, g, 8, codes, s, z, h=torch.empty_like(x)[:2]), "SHAPE"),
                  (lambda: B.qllm_rmsnorm_quant(x, g, 8, None, s, z, y=torch.empty_like(x)), "SHAPE"),
                  (lambda: B.qllm_rmsnorm_quant(x.half(), g, 8, codes, s, z), "DTYPE"), (lambda: B.qllm_dequantize_rows(codes, s, z, 4, x), "SHAPE"),
                  (lambda: B.qllm_dequantize_rows(codes, s, z, 8, x.half()), "DTYPE")]:
        with pytest.raises(B.QllmError) as ei:
            fn()
        assert ei.value.status == getattr(B, "QLLM_ERR_" + e)
    for fn in (lambda: B.qllm_rmsnorm_quant(x, g.cpu(), 8, codes, s, z), lambda: B.qllm_rmsnorm_quant(x, g, 8, codes, s.cpu(), z),
               lambda: B.qllm_dequantize_rows(codes.cpu(), s, z, 8, x), lambda: B.qllm_rmsnorm_quant(x[:, :32], g[:32].clone(), 8, codes[:, :32].contiguous(), s, z)):
        with pytest.raises(AssertionError):
            fn()
    assert B.qllm_launch_count() == before
