"""qllm_adapters_add on the GPU against its statement in 64 bits (block_ref.adapters).

Bound.  A x: products of exact operands, summed in float32 by 16-term MMAs, eight warps and up to eight CTAs: at most K / 16 + 32
additions in a row with a relative error of 2^-23 each (an MMA's own additions may be truncated), of what the terms come to without
signs; that error goes through B.  The sums enter the second product with 16 bits for bf16 (a truncated and a rounded part: 2^-16),
24 for float32.  The second product: max_rank / 16 x parts MMA steps.  Then base is added (a float32 rounding) and the result rounded to
its type."""
import numpy as np
import pytest
import torch

import block_ref
import gpu_util as G
from paper_2310_08041_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(autouse=True)
def seeded():
    torch.manual_seed(7)


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=G.DEV)


def make(slots, top, K, N, ranks, junk=float("nan")):
    """Random adapters; what lies behind a slot's rank is `junk`."""
    A, Bm = torch.randn(slots, top, K, device=G.DEV) * K ** -0.5, torch.randn(slots, N, top, device=G.DEV)
    for a, r in enumerate(ranks):
        A[a, r:] = junk
        Bm[a, :, r:] = junk
    return B.Adapters(A.bfloat16(), Bm.bfloat16(), torch.rand(slots, device=G.DEV) + 0.25, ints(ranks))


def check(got, ad, ranks, x, base, start, adapter):
    want, first, second = block_ref.adapters(ad.A, ad.B, ad.scale, ranks, x, base, start, adapter)
    half = torch.finfo(got.dtype).eps / 2
    split = 2.0 ** -16 if got.dtype == torch.bfloat16 else 2.0 ** -23
    tol = (ad.K / 16 + 32) * 2.0 ** -23 * first + (split + (ad.max_rank / 16 * 3 + 4) * 2.0 ** -23) * second + (half + 2.0 ** -24) * want.abs() + 2.0 ** -130
    off = (got.double() - want).abs()
    assert (off <= tol).all(), "%d of %d beyond the bound, worst %.3g times" % ((off > tol).sum(), off.numel(), (off / tol).nan_to_num(1e30).max())


def run(ad, x, base, start, adapter, inplace=False, pad=(0, 0, 0), **kw):
    """out between canaries, rows and gaps that nobody owns keep their contents."""
    rows, N = x.shape[0], ad.N
    out = G.Guarded((max(rows, 1), N + pad[2]), x.dtype, 3.0)
    view = out.t[:rows, :N]
    if inplace:
        view.copy_(base)
    before = out.t.clone()

    def strided(t, extra):
        wide = torch.full((t.shape[0], t.shape[1] + extra), float("nan"), dtype=t.dtype, device=t.device)
        wide[:, :t.shape[1]] = t
        return wide[:, :t.shape[1]]
    b = view if inplace else None if base is None else strided(base, pad[1])
    B.qllm_adapters_add(ad, strided(x, pad[0]), b, view, ints(start), ints(adapter), **kw)
    torch.cuda.synchronize()
    out.check()
    mine = torch.zeros(rows, dtype=torch.bool, device=G.DEV)
    for s, a in enumerate(adapter):
        mine[start[s]:start[s + 1]] = True
    same = out.t.view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32) == before.view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32)
    assert same[:rows][~mine].all() and same[:, N:].all(), "rows or gaps of nobody were written"
    return view, mine


def case(dtype, K, N, top, ranks, news, adapter, lead=0, tail=0, **kw):
    start = (np.concatenate([[0], np.cumsum(news)]) + lead).tolist()
    rows = start[-1] + tail
    ad = make(len(ranks), top, K, N, ranks)
    x, base = torch.randn(rows, K, device=G.DEV).to(DT[dtype]), torch.randn(rows, N, device=G.DEV).to(DT[dtype])
    x[:, 5] *= 20
    got, mine = run(ad, x, base, start, adapter, **kw)
    check(got[mine], ad, ranks, x[mine], base[mine], (np.array(start) - lead).tolist(), adapter)
    assert B.qllm_poll_status() == B.QLLM_OK


SIZES = [(8, 8), (40, 72), (256, 1000), (1032, 264), (4096, 4096), (5120, 1288)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K,N", SIZES)
@pytest.mark.parametrize("top", [8, 16, 24, 32, 64, 128])
def test_one_token(dtype, K, N, top):
    case(dtype, K, N, top, [top, 1, top - 3], [1], [2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K,N", SIZES)
@pytest.mark.parametrize("top", [8, 16, 40, 64, 120])
def test_a_step_of_many_requests(dtype, K, N, top):
    """Single tokens of 70 requests on 6 adapters of different ranks (one of rank 0), some without one, some sequences without tokens."""
    rng = np.random.RandomState(K + N + top)
    news = rng.choice([0, 1, 1, 1], 70)
    case(dtype, K, N, top, [top, 0, 1, top // 2, top - 1, top], news, rng.randint(-1, 6, 70), lead=3, tail=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K,N", [(40, 72), (1032, 264), (4096, 1000)])
@pytest.mark.parametrize("top", [8, 16, 32, 56, 64, 128])
def test_prompts_and_tokens(dtype, K, N, top):
    """Runs of rows longer and shorter than a tile, the same adapter in sequences far apart."""
    case(dtype, K, N, top, [top, top // 2, top - 1], [130, 1, 64, 0, 17, 300, 1, 65, 16], [0, 1, 2, 0, 0, 1, -1, 2, 1], lead=1, tail=5)


@pytest.mark.parametrize("K,N,top,slots", [(8192, 10240, 64, 14), (8200, 10248, 40, 18), (8136, 10120, 56, 15), (1032, 264, 128, 13), (40, 72, 72, 30), (4096, 1288, 120, 20)])
@pytest.mark.parametrize("rows", ["ones", "some"])
def test_steps_of_large_adapters(K, N, top, slots, rows):
    """Few rows for each of many large adapters, ranks from 0 to all, groups of 1 to 30 rows."""
    rng = np.random.RandomState(K + top)
    seqs = 40 if rows == "ones" else 25
    news = np.ones(seqs, int) if rows == "ones" else rng.choice([0, 1, 3, 9], seqs)
    ranks = [top, 0, 1, top - 1, top // 2] + [int(r) for r in rng.randint(1, top + 1, slots - 5)]
    case("bf16", K, N, top, ranks, news, rng.randint(-1, slots, seqs), lead=2, tail=1)
    case("bf16", K, N, top, ranks, news, rng.randint(-1, slots, seqs), inplace=True)


@pytest.mark.parametrize("K,N", [(40, 72), (1032, 264), (4104, 2056)])
@pytest.mark.parametrize("top", [8, 16, 24, 32, 40, 64, 72, 128])
def test_long_prompts(K, N, top):
    """Tiles of 64 and 128 rows, full and ragged, all of one adapter or cut by others; strided, in place, without a base."""
    case("bf16", K, N, top, [top, max(1, top - 5)], [513, 1, 700], [0, 1, 1], pad=(8, 16, 24))
    case("bf16", K, N, top, [top], [1111], [0], inplace=True, pad=(0, 0, 8))
    start, adapter = [0, 600, 640, 1300], [0, -1, 0]
    x = torch.randn(1300, K, device=G.DEV).bfloat16()
    ad = make(1, top, K, N, [top])
    got, _ = run(ad, x, None, start, adapter)
    check(got, ad, [top], x, torch.zeros_like(got), start, adapter)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news", [[1, 1, 2], [100, 40, 3]])
def test_in_place_and_strided(dtype, news):
    case(dtype, 256, 520, 16, [16, 9], news, [1, -1, 0], inplace=True, pad=(0, 0, 8))
    case(dtype, 256, 520, 16, [16, 9], news, [1, -1, 0], pad=(16, 24, 8), lead=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_base_and_ranks(dtype):
    """base = None counts as zeros, also for rows without an adapter; rank = None as max_rank."""
    start, adapter = [0, 3, 60, 61], [0, -1, 1]
    x = torch.randn(61, 512, device=G.DEV).to(DT[dtype])
    ad = make(2, 32, 512, 256, [32, 32])
    got, mine = run(B.Adapters(ad.A, ad.B, ad.scale), x, None, start, adapter)
    assert mine.all()
    check(got, ad, [32, 32], x, torch.zeros_like(got), start, adapter)
    assert (got[3:60] == 0).all()


def test_part_of_a_fused_projection():
    """Queries' and values' columns of one buffer, each with adapters of its own; the keys' columns stay as they are."""
    x = torch.randn(50, 512, device=G.DEV).bfloat16()
    out = torch.randn(50, 3 * 256, device=G.DEV).bfloat16()
    before, start, adapter = out.clone(), [0, 1, 30, 50], [1, 0, 1]
    for part in (0, 2):
        ad = make(2, 16, 512, 256, [16, 8])
        cols = slice(256 * part, 256 * part + 256)
        B.qllm_adapters_add(ad, x, out[:, cols], out[:, cols], ints(start), ints(adapter))
        check(out[:, cols], ad, [16, 8], x, before[:, cols], start, adapter)
    assert torch.equal(out[:, 256:512], before[:, 256:512])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("seqs,slots,top", [(257, 3, 8), (1000, 700, 8), (3000, 8192, 8), (5000, 1, 8), (700, 900, 72), (1500, 8192, 72), (2000, 2, 40)])
def test_more_sequences_and_slots_than_threads(dtype, seqs, slots, top):
    rng = np.random.RandomState(seqs)
    K, N = 64, 40
    A, Bm = torch.randn(slots, top, K, device=G.DEV).bfloat16(), torch.randn(slots, N, top, device=G.DEV).bfloat16()
    ad = B.Adapters(A, Bm, torch.rand(slots, device=G.DEV), ints(rng.randint(0, top + 1, slots)))
    news, adapter = rng.choice([0, 1, 1, 2, 5], seqs), rng.randint(-1, slots, seqs)
    start = np.concatenate([[0], np.cumsum(news)]).tolist()
    x, base = torch.randn(start[-1], K, device=G.DEV).to(DT[dtype]), torch.randn(start[-1], N, device=G.DEV).to(DT[dtype])
    got, _ = run(ad, x, base, start, adapter)
    row_ad = torch.from_numpy(np.repeat(adapter, news)).to(G.DEV)
    rank = ad.rank[row_ad.clamp(min=0)]
    live = (torch.arange(top, device=G.DEV)[None] < rank[:, None]) & (row_ad >= 0)[:, None]
    aa, bb = A[row_ad.clamp(min=0)].double() * live[:, :, None], Bm[row_ad.clamp(min=0)].double() * live[:, None]
    sc = ad.scale[row_ad.clamp(min=0)].double()
    mid = torch.einsum("mk,mrk->mr", x.double(), aa)
    want = base + sc[:, None] * torch.einsum("mr,mnr->mn", mid, bb)
    first = sc[:, None] * torch.einsum("mr,mnr->mn", torch.einsum("mk,mrk->mr", x.double().abs(), aa.abs()), bb.abs())
    second = sc[:, None] * torch.einsum("mr,mnr->mn", mid.abs(), bb.abs())
    half, split = torch.finfo(DT[dtype]).eps / 2, 2.0 ** -16 if dtype == "bf16" else 2.0 ** -23
    assert ((got - want).abs() <= (K / 16 + 32) * 2.0 ** -23 * first + (split + (top / 16 * 3 + 4) * 2.0 ** -23) * second + (half + 2.0 ** -24) * want.abs()).all()
    assert B.qllm_poll_status() == B.QLLM_OK


@pytest.mark.parametrize("dtype,top,news", [("bf16", 16, [20000]), ("bf16", 40, [9000, 1, 12000]), ("bf16", 128, [10000, 7000]), ("bf16", 128, [1] * 700), ("f32", 16, [9000, 3000])])
def test_more_tiles_than_run_at_once(dtype, top, news):
    slots = min(len(news), 500)
    case(dtype, 64, 136, top, [top] * slots, news, [i % slots for i in range(len(news))])


@pytest.mark.parametrize("seed", range(16))
def test_random_shapes(seed):
    r = np.random.RandomState(500 + seed)
    top, slots = 8 * r.randint(1, 17), r.randint(1, 30)
    K, N = 8 * r.randint(1, 400), 8 * r.randint(1, 400)
    seqs = r.randint(1, 50)
    news = [int(x) for x in (r.randint(0, 4, seqs) if seed % 3 else r.randint(0, 90, seqs))]
    ranks = [int(x) for x in r.randint(0, top + 1, slots)]
    case(["bf16", "f32"][seed % 2], K, N, top, ranks, news, r.randint(-1, slots, seqs), lead=r.randint(0, 3), tail=r.randint(0, 3),
         pad=tuple(8 * int(v) for v in r.randint(0, 3, 3)))


@pytest.mark.parametrize("dtype,top", [("f32", 16), ("bf16", 16), ("bf16", 72)])
def test_contents_out_of_range_are_reported_and_harmless(dtype, top):
    """Slots that do not exist count as none, ranks are cut, row ranges are cut to the tensors; the other sequences are served."""
    K, N, rows = 256, 128, 40
    x, base = torch.randn(rows, K, device=G.DEV).to(DT[dtype]), torch.randn(rows, N, device=G.DEV).to(DT[dtype])
    good = dict(start=[0, 10, 20, 30, 40], adapter=[0, 1, 0, -1], ranks=[16, 12])
    for change in (dict(adapter=[0, 2, 0, -1]), dict(adapter=[0, 2 ** 30, 0, -1]), dict(ranks=[16, top + 1]), dict(ranks=[16, -5]), dict(start=[0, 10, 20, 30, 1000]),
                   dict(start=[-7, 10, 20, 30, 40]), dict(start=[0, 10, 2 ** 31 - 1, 30, 40]), dict(start=[0, 10, -2 ** 31, 30, 40])):
        c = dict(good, **change)
        ad = make(2, top, K, N, good["ranks"], junk=0.0)
        ad.rank.copy_(ints(c["ranks"]))
        out = G.Guarded((rows, N), DT[dtype], 3.0)
        B.qllm_adapters_add(ad, x, base, out.t, ints(c["start"]), ints(c["adapter"]))
        assert B.qllm_poll_status() == B.QLLM_ERR_PAGE, change
        out.check()
        # the first ten rows and rows 30 .. 39 are named rightly in every variant
        same = [16 if c["ranks"][0] == 16 else 0]
        check(out.t[:10], ad, same + [0], x[:10], base[:10], [0, 10], [0])
        assert torch.equal(out.t[30:], base[30:]) or change.get("start", [0] * 5)[2] in (2 ** 31 - 1,)
        if "adapter" in change:
            assert torch.equal(out.t[10:20], base[10:20])
        if "ranks" in change:
            check(out.t[10:20], ad, [16, min(max(change["ranks"][1], 0), top)], x[10:20], base[10:20], [0, 10], [1])
    assert B.qllm_poll_status() == B.QLLM_OK


@pytest.mark.parametrize("seqs,rows,top", [(40000, 200000, 16), (200, 1 << 25, 16), (40000, 200000, 72), (200, 1 << 25, 72)])
def test_decreasing_ranges_that_would_pass_31_bits(seqs, rows, top):
    """Every second range is the whole tensor: the rows of one adapter add up to 2^31 and more."""
    ad = make(2, top, 8, 8, [8, 8])
    x, base = torch.ones(rows, 8, device=G.DEV).bfloat16(), torch.ones(rows, 8, device=G.DEV).bfloat16()
    out = G.Guarded((rows, 8), torch.bfloat16, 3.0)
    B.qllm_adapters_add(ad, x, base, out.t, ints([rows * (s % 2) for s in range(seqs + 1)]), ints([1] * seqs))
    assert B.qllm_poll_status() == B.QLLM_ERR_PAGE
    out.check()
    assert (out.t == 3.0).all()
    # the same sizes with ranges that increase
    cut = [rows * s // seqs for s in range(seqs + 1)]
    B.qllm_adapters_add(ad, x, base, out.t, ints(cut), ints([s % 2 for s in range(seqs)]))
    assert B.qllm_poll_status() == B.QLLM_OK
    for s in (0, 1, 2, 77, seqs - 2, seqs - 1):
        lo, hi = cut[s], min(cut[s] + 40, cut[s + 1])
        check(out.t[lo:hi], ad, [8, 8], x[lo:hi], base[lo:hi], [0, hi - lo], [s % 2])


def test_rows_with_nan_and_infinities_stay_by_themselves():
    for dtype, top in (("bf16", 16), ("f32", 16), ("bf16", 72)):
        ad = make(1, top, 256, 128, [16])
        x, base = torch.randn(40, 256, device=G.DEV).to(DT[dtype]), torch.randn(40, 128, device=G.DEV).to(DT[dtype])
        x[3, 7], x[20, 9] = float("nan"), float("inf")
        out = torch.empty_like(base)
        B.qllm_adapters_add(ad, x, base, out, ints([0, 40]), ints([0]))
        keep = [i for i in range(40) if i not in (3, 20)]
        assert out[3].isnan().all() and not out[20].isfinite().any()
        check(out[keep], ad, [16], x[keep], base[keep], [0, 38], [0])


def test_float32_over_its_range():
    """Large and small activations: exact parts, nothing passes bf16's range on the way."""
    ad = make(1, 8, 64, 32, [8])
    x = torch.randn(9, 64, device=G.DEV) * torch.tensor([1e-30, 1e-20, 1e-10, 1e-3, 1.0, 1e3, 1e10, 1e30, 3e36], device=G.DEV)[:, None]
    base = torch.zeros(9, 32, device=G.DEV)
    out = torch.empty_like(base)
    B.qllm_adapters_add(ad, x, base, out, ints([0, 9]), ints([0]))
    for i in range(9):
        check(out[i:i + 1], ad, [8], x[i:i + 1], base[i:i + 1], [0, 1], [0])


def test_results_do_not_depend_on_the_run_or_the_order_of_sequences():
    """Bit for bit; rows of a sequence moved elsewhere in the batch, its adapter's other rows staying in their order."""
    ad = make(3, 32, 1024, 512, [32, 20, 7])
    news, adapter = [40, 1, 30, 70, 5], [0, 1, 2, 0, 1]
    start = np.concatenate([[0], np.cumsum(news)]).tolist()
    x, base = torch.randn(146, 1024, device=G.DEV).bfloat16(), torch.randn(146, 512, device=G.DEV).bfloat16()
    a, b = torch.empty_like(base), torch.empty_like(base)
    for o in (a, b):
        B.qllm_adapters_add(ad, x, base, o, ints(start), ints(adapter))
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_stream_and_graph():
    """A captured call follows the contents of row ranges, adapters, ranks, scales and weights."""
    slots, top, K, N, rows = 4, 16, 512, 384, 24
    ad = make(slots, top, K, N, [16, 16, 16, 16], junk=0.0)
    x, base, out = torch.randn(rows, K, device=G.DEV).bfloat16(), torch.randn(rows, N, device=G.DEV).bfloat16(), torch.empty(rows, N, device=G.DEV).bfloat16()
    start, adapter, st = ints([0, 1, 2, 24]), ints([0, 1, 2]), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        B.qllm_adapters_add(ad, x, base, out, start, adapter, stream=st)
    st.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        B.qllm_adapters_add(ad, x, base, out, start, adapter, stream=st)
    rng = np.random.RandomState(5)
    for _ in range(4):
        cut = sorted(rng.randint(0, rows + 1, 2).tolist())
        s, a, r = [0] + cut + [rows], rng.randint(-1, slots, 3).tolist(), rng.randint(1, 17, slots).tolist()
        start.copy_(ints(s)); adapter.copy_(ints(a)); ad.rank.copy_(ints(r)); ad.scale.uniform_(); ad.A.normal_(); x.normal_()
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            g.replay()
        torch.cuda.synchronize()
        check(out, ad, r, x, base, s, a)


def test_wrong_tensors_are_refused():
    ad = make(2, 16, 256, 128, [16, 9])
    x, base, out = torch.randn(4, 256, device=G.DEV), torch.randn(4, 128, device=G.DEV), torch.empty(4, 128, device=G.DEV)
    s, a = ints([0, 2, 4]), ints([0, 1])
    before = B.qllm_launch_count()
    for fn, e in [(lambda: B.qllm_adapters_add(ad, x[:, :248], base, out, s, a), "SHAPE"), (lambda: B.qllm_adapters_add(ad, x, base[:3], out, s, a), "SHAPE"),
                  (lambda: B.qllm_adapters_add(ad, x, base, out.bfloat16(), s, a), "SHAPE"), (lambda: B.qllm_adapters_add(ad, x, base, out, s, a[:1]), "SHAPE"),
                  (lambda: B.qllm_adapters_add(ad, x.half(), base.half(), out.half(), s, a), "DTYPE"), (lambda: B.qllm_adapters_add(ad, x, base, out, s.long(), a), "DTYPE"),
                  (lambda: B.qllm_adapters_add(ad, x, base, torch.empty(4, 132, device=G.DEV)[:, 2:130], s, a), "ALIGN"),
                  (lambda: B.Adapters(ad.A.float(), ad.B, ad.scale), "DTYPE"), (lambda: B.Adapters(ad.A, ad.B[:, :, :8], ad.scale), "SHAPE"),
                  (lambda: B.Adapters(ad.A, ad.B, ad.scale[:1]), "SHAPE"), (lambda: B.Adapters(ad.A, ad.B, ad.scale, ad.rank[:1]), "SHAPE")]:
        with pytest.raises(B.QllmError) as ei:
            fn()
        assert ei.value.status == getattr(B, "QLLM_ERR_" + e)
    for fn in (lambda: B.qllm_adapters_add(ad, x.cpu(), base, out, s, a), lambda: B.qllm_adapters_add(ad, x, base, out, s.cpu(), a),
               lambda: B.Adapters(ad.A, ad.B.cpu(), ad.scale)):
        with pytest.raises(AssertionError):
            fn()
    assert B.qllm_launch_count() == before
