"""The 4-bit key/value cache on the GPU against plain 64-bit statements of it (kv_ref): storing and reading, attention over
it, its pages, and a run of them behind a quantized layer."""
import numpy as np
import pytest
import torch

import gpu_util as G
import kv_ref
from paper_2310_08041_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(autouse=True)
def seeded():
    torch.manual_seed(7)


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=G.DEV)


def make_table(rng, lens, page, pages, width=None):
    used = [-(-n // page) for n in lens]
    width = width or max(max(used), 1)
    table = np.full((len(lens), width), -1, np.int32)
    order = rng.permutation(pages)[:sum(used)]
    at = 0
    for s, n in enumerate(used):
        table[s, :n] = order[at:at + n]
        at += n
    return table


def random_cache(seed, layers, pages, heads, page, d, zeros=(3, 13)):
    """Random codes; scales about 0.1 .. 0.4, integer zero-points."""
    g = torch.Generator(device=G.DEV); g.manual_seed(seed)
    shape = (layers, pages, heads, page)
    c = []
    for _ in range(2):
        c.append(torch.randint(0, 256, shape + (d // 2,), generator=g, device=G.DEV, dtype=torch.uint8))
        p = torch.empty(shape + (2,), device=G.DEV).uniform_(0.1, 0.4, generator=g)
        p[..., 1].random_(*zeros, generator=g)
        c.append(p)
    return B.KvCache(*c)


def store_of(cache, layer):
    return kv_ref.Store(*[t[layer].cpu().numpy() for t in (cache.k_codes, cache.k_param, cache.v_codes, cache.v_param)])


def batch_of(table, lens, news, rows=None, max_new=None):
    start = np.concatenate([[0], np.cumsum(news)])
    return B.KvBatch(ints(table), ints(lens), ints(start), int(start[-1]) if rows is None else rows,
                     max(list(news) + [0]) if max_new is None else max_new), start


def attend(cache, layer, q, batch, scale, causal, fill=7.0, workspace=None):
    """(out, lse) with canaries around both."""
    out = G.Guarded(tuple(q.shape), q.dtype, fill)
    lse = G.Guarded((q.shape[0], q.shape[1]), torch.float32, fill)
    if workspace is None:
        n = B.qllm_kv_attention_workspace(cache, q.shape[1], q, batch)
        workspace = torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device=G.DEV)      # NaN patterns: nothing of it may be relied on
    B.qllm_kv_attention(cache, layer, q, out.t, scale, batch, workspace, causal=causal, lse=lse.t)
    torch.cuda.synchronize()
    out.check("out"); lse.check("lse")
    return out.t, lse.t


def check_attention(got, lse, ref, dtype, rounded_codes=False, prompt=False):
    """|error| <= rounding of the output + what the weights' and scores' errors can move.

    Weights: a bf16 call rounds each weight p_j vs_j once to 11 bits (fp16, half a step 2^-11 relative, or 2^-25 of the largest
    weight where it is small: at most `seen` 2^-25 in all); a float32 call to 22 bits.  Scores: sums of head_dim + 1 products
    in float32, each of at most |mag| with at most 2^-23 relative error per addition, so (256 + 8) 2^-23 mag < 2^-14.9 mag in the
    worst order; every kernel adds them in groups of 16 at least, whose error is at most (16 + 16) 2^-23 mag = 2^-18 mag.  A
    relative change of every weight by e moves out by at most 2 e spread.  exp and the running rescalings: 2^-20.
    prompt (bf16, more than 96 query rows per key head): the prompt kernel also rounds the value scale and the value it
    multiplies to 11 bits, 2^-11 of the value each, which is at most the spread's term of its token; and likewise the key's scale
    and product, 2^-11 of |key| each, which moves a score by at most 2^-10 scale sum |q| |key| <= 2^-10 mag.
    rounded_codes: the prompt kernel stores (code - zero) of rows far from zero in 11 bits, moving a score by 2^-11 mag and a
    value by 2^-11 of itself.  Sums over the keys: `seen` terms of one sign (the weights) or of at most the spread in all, added
    in float32 in any order, are off by at most seen 2^-24 of that sum; a logarithm turns a relative error into the same
    absolute one."""
    out, ref_lse, spread, mag, seen = ref
    w = 2.0 ** -11 + seen * 2.0 ** -25 if dtype == torch.bfloat16 else 2.0 ** -22 + seen * 2.0 ** -36
    w = w + 2 * seen * 2.0 ** -24                            # numerator and denominator
    w = w + (2 * 2.0 ** -11 if prompt else 0)
    e = 2.0 ** -18 * mag + 2.0 ** -20 + (2.0 ** -10 * mag if prompt else 0) + (2.0 ** -11 * (mag + 1) if rounded_codes else 0)
    tol = (w + 2 * e)[..., None] * spread + np.abs(out) * torch.finfo(dtype).eps / 2 + 1e-30
    a = host(got)
    bad = ~(np.abs(a - out) <= tol)
    assert not bad.any(), "%d of %d beyond the bound, worst %.3g times" % (bad.sum(), bad.size, (np.abs(a - out) / tol).max())
    b = host(lse)
    assert np.array_equal(np.isneginf(b), np.isneginf(ref_lse))
    fin = np.isfinite(ref_lse)
    assert (np.abs(b[fin] - ref_lse[fin]) <= (e * 2 + seen * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(ref_lse)))[fin]).all()


def run_case(seed, dtype, d, page, heads, group, lens, news, causal, scale=None, layers=2, zeros=(3, 13), stride_pad=0, max_new=None, rounded_codes=False):
    rng = np.random.RandomState(seed)
    pages = sum(-(-n // page) for n in lens) + 3
    table = make_table(rng, lens, page, pages)
    cache = random_cache(seed, layers, pages, heads, page, d, zeros)
    batch, start = batch_of(table, lens, news, max_new=max_new)
    gen = torch.Generator(device=G.DEV); gen.manual_seed(seed + 1)
    wide = torch.randn(max(batch.rows, 1), heads * group * d + stride_pad, generator=gen, device=G.DEV).to(DT[dtype])
    q = wide[:batch.rows, :heads * group * d].unflatten(1, (heads * group, d))
    scale = d ** -0.5 if scale is None else scale
    got, lse = attend(cache, layers - 1, q, batch, scale, causal)
    ref = kv_ref.attention(store_of(cache, layers - 1), table, lens, start, host(q), scale, causal)
    hint = (max(news) if max_new is None else max_new) * group
    check_attention(got, lse, ref, DT[dtype], rounded_codes, prompt=dtype == "bf16" and hint > 96)
    assert B.qllm_poll_status() == B.QLLM_OK
    return got


# ------------------------------------------------------------------------------------------------ append and read
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page,heads", [(64, 16, 1), (128, 64, 3), (256, 32, 2), (128, 256, 8), (64, 128, 5)])
def test_append_is_the_row_quantizer(dtype, d, page, heads):
    rng = np.random.RandomState(d + page)
    lens, news = [70, 5, 0, 300, 1, 33], [70, 2, 0, 1, 1, 20]
    pages = 40
    table = make_table(rng, lens, page, pages, width=20)
    cache = random_cache(5, 3, pages, heads, page, d)
    before = [t.clone() for t in (cache.k_codes, cache.k_param, cache.v_codes, cache.v_param)]
    batch, start = batch_of(table, lens, news)
    rows = batch.rows
    x = torch.randn(rows, 2 * heads * d + 16, device=G.DEV)
    x[3] *= 1000
    x[4] = 0.0                                               # constant rows: 0 and not 0
    x[5] = -2.5
    x[6] = 4096.0 + 0.001 * x[6]                             # far from zero for its range
    x = x.to(DT[dtype])
    k, v = x[:, :heads * d].unflatten(1, (heads, d)), x[:, heads * d:2 * heads * d].unflatten(1, (heads, d))
    B.qllm_kv_append(cache, 1, k, v, batch)
    want = [t.clone() for t in before]
    for t, (codes, param) in ((k, (0, 1)), (v, (2, 3))):
        flat = t.reshape(rows * heads, d).contiguous()
        c, s, z = (torch.from_numpy(a).to(G.DEV) for a in kv_ref.quantize(flat.float().cpu().numpy()))
        if d == 256:                                         # the row quantizer's one-pass kernels: the same bits
            c2, s2, z2 = torch.empty_like(c), torch.empty_like(s), torch.empty_like(z)
            B.qllm_quantize_rows(flat, 4, c2, s2, z2)
            assert torch.equal(c, c2) and torch.equal(s, s2) and torch.equal(z, z2)
        for q in range(len(lens)):
            for i in range(news[q]):
                pos, r = lens[q] - news[q] + i, (start[q] + i) * heads
                want[codes][1, table[q, pos // page], :, pos % page] = c[r:r + heads]
                want[param][1, table[q, pos // page], :, pos % page, 0] = s[r:r + heads]
                want[param][1, table[q, pos // page], :, pos % page, 1] = z[r:r + heads]
    torch.cuda.synchronize()
    for a, b in zip((cache.k_codes, cache.k_param, cache.v_codes, cache.v_param), want):
        assert torch.equal(a, b)                             # every other place of the cache as it was
    # read back: the values in the call's type, other rows untouched
    k_out, v_out = G.Guarded((rows, heads, d), DT[dtype], 3.0), G.Guarded((rows, heads, d), DT[dtype], 3.0)
    B.qllm_kv_read(cache, 1, k_out.t, v_out.t, batch)
    st = store_of(cache, 1)
    k_out.check(); v_out.check()
    for q in range(len(lens)):
        kc, kp, vc, vp = st.rows(table[q], lens[q] - news[q], lens[q])
        for got, c, p in ((k_out.t, kc, kp), (v_out.t, vc, vp)):
            f32 = (c.astype(np.float32) - p[..., 1:2].astype(np.float32)) * p[..., 0:1].astype(np.float32)
            assert torch.equal(got[start[q]:start[q + 1]].cpu(), torch.from_numpy(f32).to(DT[dtype]))
    assert B.qllm_poll_status() == B.QLLM_OK


def test_append_many_rows_and_rows_that_are_nobodys():
    """Enough rows for the four-row kernels; rows in front of the first sequence and behind the last stay as they are."""
    rng = np.random.RandomState(3)
    heads, d, page = 8, 128, 64
    lens, news = [2500, 1800], [2500, 1700]
    table = make_table(rng, lens, page, 80)
    cache = random_cache(1, 1, 80, heads, page, d)
    start = [5, 2505, 4205]
    batch = B.KvBatch(ints(table), ints(lens), ints(start), 4300, 2500)
    x = torch.randn(4300, 2, heads, d, device=G.DEV).bfloat16()
    B.qllm_kv_append(cache, 0, x[:, 0], x[:, 1], batch)
    out = torch.full((2, 4300, heads, d), 9.0, device=G.DEV).bfloat16()
    B.qllm_kv_read(cache, 0, out[0], out[1], batch)
    assert (out[:, :5] == 9).all() and (out[:, 4205:] == 9).all()
    # half a step of a row's scale, and the rounding of the value to bf16
    for i in range(2):
        x32 = x[5:4205, i].float()
        step = (x32.amax(-1) - x32.amin(-1)) / 15
        assert ((out[i, 5:4205].float() - x32).abs() <= step[..., None] * (0.5 + 1e-5) + x32.abs() * 2.0 ** -8 + step[..., None] * 2.0 ** -8).all()
    assert B.qllm_poll_status() == B.QLLM_OK


def test_more_new_tokens_than_length():
    cache = random_cache(2, 1, 4, 2, 16, 64)
    before = cache.k_codes.clone()
    batch = B.KvBatch(ints([[2, 1]]), ints([3]), ints([0, 5]), 5, 5)
    x = torch.randn(5, 2, 64, device=G.DEV)
    B.qllm_kv_append(cache, 0, x, x, batch)
    changed = (cache.k_codes != before).any(-1)[0]
    assert changed.nonzero()[:, 0].unique().tolist() == [2] and changed[2, :, 3:].sum() == 0
    k, v = torch.full((5, 2, 64), 8.0, device=G.DEV), torch.full((5, 2, 64), 8.0, device=G.DEV)
    B.qllm_kv_read(cache, 0, k, v, batch)
    assert (k[:2] == 0).all() and (v[:2] == 0).all() and (k[2:] != 8).all()
    got, lse = attend(cache, 0, x, batch, 0.1, True)
    assert (got[:2] == 0).all() and torch.isneginf(lse[:2]).all() and torch.isfinite(lse[2:]).all()
    assert B.qllm_poll_status() == B.QLLM_OK


# ------------------------------------------------------------------------------------------------ attention
LENS = {
    "one": ([1], [1]),
    "tile edges": ([15, 16, 17, 63, 64, 65, 127, 128, 129], [1] * 9),
    "empty and idle": ([0, 40, 0, 7, 0], [1, 0, 0, 1, 0]),
    "long": ([4099], [1]),
    "ragged": ([1, 700, 33, 2048, 5, 130, 1000, 64], [1] * 8),
    "several new": ([9, 200, 64, 1000, 3], [9, 5, 1, 12, 3]),
    "prompt": ([257], [257]),
    "chunk": ([700, 90], [130, 90]),
    "blocks": ([1000, 3000, 520], [600, 257, 515]),
    "long chunk": ([9000], [70]),
    "mixed": ([300, 513, 1, 129, 1030], [300, 1, 1, 129, 2]),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", list(LENS))
@pytest.mark.parametrize("d,page,heads,group", [(128, 64, 2, 4), (64, 16, 3, 1), (128, 32, 1, 8), (256, 16, 1, 5)])
def test_attention(dtype, what, d, page, heads, group):
    lens, news = LENS[what]
    run_case(11, dtype, d, page, heads, group, lens, news, True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [2, 3, 7, 9, 16, 20, 33])
def test_attention_groups(dtype, group):
    run_case(12, dtype, 128, 64, 2, group, [200, 31], [1, 3], True)
    run_case(13, dtype, 64, 128, 1, group, [150, 290], [150, 40], True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", ["ragged", "several new", "chunk", "empty and idle"])
def test_attention_without_causality(dtype, what):
    lens, news = LENS[what]
    run_case(14, dtype, 128, 128, 2, 3, lens, news, False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news", [[1, 1], [70, 300]])
def test_attention_strides_scales_and_hints(dtype, news):
    run_case(15, dtype, 128, 256, 2, 4, [513, 300], news, True, stride_pad=24)
    run_case(16, dtype, 64, 32, 2, 4, [513, 300], news, True, scale=1.7)
    run_case(17, dtype, 64, 32, 2, 4, [513, 300], news, True, scale=-0.3)
    run_case(18, dtype, 128, 32, 2, 4, [513, 300], news, True, scale=0.0)
    for hint in (0, 1, 5000):                                # max_new selects kernels, results do not depend on it
        run_case(19, dtype, 128, 64, 2, 4, [513, 300], news, True, max_new=hint)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news", [[1, 1, 1], [80, 200, 65]])
def test_attention_rows_far_from_zero(dtype, news):
    """Zero-points as a row far from zero for its range has them, up to beyond what 16 bits hold."""
    run_case(20, dtype, 128, 64, 2, 4, [300, 200, 65], news, True, scale=0.001, zeros=(-300, 300))
    run_case(21, dtype, 128, 64, 2, 4, [300, 200, 65], news, True, scale=1e-5, zeros=(-5000, 5000), rounded_codes=True)
    run_case(22, dtype, 64, 64, 2, 4, [300, 200, 65], news, True, scale=1e-8, zeros=(-4000000, 4000000), rounded_codes=True)


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news", [[1, 1], [150, 70]])
def test_attention_scales_of_every_size(dtype, news, seed):
    """Value scales from 1e-12 to 1e12 between tokens, key scales such that weights run over many decades; query rows of very
    different size."""
    lens, page, d, heads, group = [500, 130], 64, 128, 2, 4
    rng = np.random.RandomState(23)
    torch.manual_seed(seed)
    table = make_table(rng, lens, page, 12)
    cache = random_cache(23, 1, 12, heads, page, d)
    cache.v_param[..., 0] *= 10.0 ** torch.randint(-12, 13, cache.v_param.shape[:-1], device=G.DEV).float()
    cache.k_param[..., 0] *= 10.0 ** torch.randint(-4, 1, cache.k_param.shape[:-1], device=G.DEV).float()
    batch, start = batch_of(table, lens, news)
    q = torch.randn(batch.rows, heads * group, d, device=G.DEV)
    q *= 10.0 ** torch.randint(-20, 1, (batch.rows, heads * group, 1), device=G.DEV).float()
    q = q.to(DT[dtype])
    got, lse = attend(cache, 0, q, batch, 0.09, True)
    ref = kv_ref.attention(store_of(cache, 0), table, lens, start, host(q), 0.09, True)
    check_attention(got, lse, ref, DT[dtype], prompt=dtype == "bf16" and max(news) * group > 96)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news", [[1, 1, 1], [33, 80, 1], [66, 129, 1]])
def test_attention_ignores_what_lies_behind_a_sequence(dtype, news):
    """Places behind a sequence's end, and pages nobody's table names, hold NaN and infinite parameters: same bits as with
    clean ones."""
    lens, page, d, heads, group = [67, 130, 1], 64, 128, 2, 4
    rng = np.random.RandomState(24)
    table = make_table(rng, lens, page, 9)
    cache = random_cache(24, 1, 9, heads, page, d)
    batch, start = batch_of(table, lens, news)
    q = torch.randn(batch.rows, heads * group, d, device=G.DEV).to(DT[dtype])
    want = attend(cache, 0, q, batch, 0.09, True)
    used = np.zeros((9, page), bool)
    for s, n in enumerate(lens):
        for j in range(n):
            used[table[s, j // page], j % page] = True
    hole = torch.from_numpy(~used).to(G.DEV)[:, None, :].expand(9, heads, page)
    bad = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38], device=G.DEV)
    for p in (cache.k_param, cache.v_param):
        noise = bad[torch.randint(0, 4, p[0].shape, device=G.DEV)]
        p[0] = torch.where(hole[..., None], noise, p[0])
    cache.k_codes[0][hole] = 255
    cache.v_codes[0][hole] = 255
    got = attend(cache, 0, q, batch, 0.09, True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # keys behind a causal row's own position, which other rows of the call do see, are as harmless: the last token's
    # parameters turn to NaN, and only the last row of its sequence notices
    if news[1] > 1:
        at = lens[1] - 1
        cache.k_param[0, table[1, at // page], :, at % page] = float("nan")
        cache.v_param[0, table[1, at // page], :, at % page] = float("nan")
        got = attend(cache, 0, q, batch, 0.09, True)
        last = start[2] - 1
        keep = [r for r in range(batch.rows) if r != last]
        assert torch.equal(got[0][keep], want[0][keep]) and torch.isnan(got[0][last].float()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_infinite_query_stays_in_its_row(dtype):
    lens, news = [100, 300], [1, 140]
    rng = np.random.RandomState(25)
    table = make_table(rng, lens, 64, 9)
    cache = random_cache(25, 1, 9, 2, 64, 128)
    batch, start = batch_of(table, lens, news)
    q = torch.randn(batch.rows, 4, 128, device=G.DEV).to(DT[dtype])
    want, _ = attend(cache, 0, q, batch, 0.09, True)
    q[50, 1, 7] = float("nan")
    q[51, 1, 7] = float("inf")
    got, _ = attend(cache, 0, q, batch, 0.09, True)
    assert torch.isnan(got[50, 1].float()).all() and not torch.isfinite(got[51, 1].float()).any()
    q_rows = torch.ones(batch.rows, 4, dtype=torch.bool, device=G.DEV)
    q_rows[50, 1] = q_rows[51, 1] = False
    assert torch.equal(got[q_rows], want[q_rows])


@pytest.mark.parametrize("news", [[1, 1], [100, 70]])
def test_indices_out_of_range_are_reported_and_harmless(news):
    """Checked in plain code before this runs: the kernels cut lengths and rows to what exists and skip pages that do not."""
    lens, page, heads, d = [100, 130], 16, 2, 128
    rng = np.random.RandomState(26)
    table = make_table(rng, lens, page, 20)
    cache = random_cache(26, 1, 20, heads, page, d)
    q = torch.randn(sum(news), 8, d, device=G.DEV).bfloat16()
    x = torch.randn(sum(news), heads, d, device=G.DEV).bfloat16()
    bad = table.copy()
    bad[0, 2], bad[1, 3] = 20, -5
    batch, start = batch_of(bad, lens, news)
    got, lse = attend(cache, 0, q, batch, 0.09, True)
    assert B.qllm_poll_status() == B.QLLM_ERR_PAGE and B.qllm_poll_status() == B.QLLM_OK
    # the same as sequences without those pages' tokens: weights of absent tokens are 0
    st = store_of(cache, 0)
    for s, j in ((0, 2), (1, 3)):
        t2, dead = table.copy(), slice(j * page, (j + 1) * page)
        kc, kp, vc, vp = st.rows(t2[s], 0, lens[s])
        for i in range(news[s]):
            keys = np.arange(lens[s] - news[s] + i + 1)
            keys = keys[(keys < dead.start) | (keys >= dead.stop)]
            qq = host(q[start[s] + i])
            for h in range(8):
                sc = 0.09 * kp[keys, h // 4, 0] * (kc[keys, h // 4] @ qq[h] - kp[keys, h // 4, 1] * qq[h].sum())
                if len(keys) == 0:
                    assert (got[start[s] + i, h] == 0).all()
                    continue
                w = np.exp(sc - sc.max()); w /= w.sum()
                v = (vc[keys, h // 4] - vp[keys, h // 4, 1:2]) * vp[keys, h // 4, 0:1]
                assert np.abs(host(got[start[s] + i, h]) - w @ v).max() < 0.05
    B.qllm_kv_append(cache, 0, x, x, batch)
    B.qllm_kv_read(cache, 0, x.clone(), x.clone(), batch)
    expected = any(bad[s, (lens[s] - news[s] + i) // page] in (20, -5) for s in range(2) for i in range(news[s]))
    assert B.qllm_poll_status() == (B.QLLM_ERR_PAGE if expected else B.QLLM_OK)
    # lengths beyond the table, negative lengths, rows that decrease or lie beyond the tensors
    for lens2, start2 in (([100000, 130], start), ([-3, 130], start), (lens, [0, news[0] + 50, news[0] + 20]), (lens, [0, -4, 10 ** 6])):
        b2 = B.KvBatch(ints(table), ints(lens2), ints(start2), sum(news), max(news))
        attend(cache, 0, q, b2, 0.09, True)
        assert B.qllm_poll_status() == B.QLLM_ERR_PAGE
        B.qllm_kv_append(cache, 0, x, x, b2)
        assert B.qllm_poll_status() == B.QLLM_ERR_PAGE


@pytest.mark.parametrize("news", [[1], [200]])
def test_offsets_beyond_32_bits(news):
    """Layer 1 of a cache whose layer 0 alone takes 4.3 GB of codes: an offset cut to 32 bits would read layer 0."""
    heads, page, d = 8, 256, 128
    pages = 33000
    c = [torch.zeros(2, pages, heads, page, d // 2, dtype=torch.uint8, device=G.DEV) for _ in range(2)]
    p = [torch.ones(2, pages, heads, page, 2, device=G.DEV) for _ in range(2)]
    cache = B.KvCache(c[0], p[0], c[1], p[1])
    lens = [700]
    table = np.array([[pages - 1, pages - 2, pages - 3]], np.int32)
    batch, start = batch_of(table, lens, news)
    x = torch.randn(sum(news), 2, heads, d, device=G.DEV).bfloat16()
    sub = random_cache(27, 1, 3, heads, page, d)
    for dst, src in zip(c + p, (sub.k_codes, sub.v_codes, sub.k_param, sub.v_param)):
        dst[1, pages - 3:] = src[0]
    B.qllm_kv_append(cache, 1, x[:, 0], x[:, 1], batch)
    out = torch.empty(2, sum(news), heads, d, device=G.DEV).bfloat16()
    B.qllm_kv_read(cache, 1, out[0], out[1], batch)
    assert ((out[0].float() - x[:, 0].float()).abs().amax() < 0.6) and not c[0][0].any()
    q = torch.randn(sum(news), 16, d, device=G.DEV).bfloat16()
    got, lse = attend(cache, 1, q, batch, 0.09, True)
    st = kv_ref.Store(*[t[1, pages - 3:].cpu().numpy() for t in (c[0], p[0], c[1], p[1])])
    ref = kv_ref.attention(st, np.array([[2, 1, 0]]), lens, start, host(q), 0.09, True)
    check_attention(got, lse, ref, torch.bfloat16, prompt=news[0] * 2 > 96)


def test_streams_and_graphs():
    """Two captured steps with a workspace each, replayed on two streams at once while lengths and tables change between
    replays: the graphs follow the batch's contents."""
    heads, group, page, d, top = 4, 4, 64, 128, 900
    rng = np.random.RandomState(28)
    sides = []
    for i in range(2):
        lens = [top, top, top]
        table = make_table(rng, lens, page, 50)
        cache = random_cache(28 + i, 1, 50, heads, page, d)
        batch, start = batch_of(table, lens, [1, 1, 1])
        q = torch.randn(3, heads * group, d, device=G.DEV).bfloat16()
        kv = torch.randn(3, 2, heads, d, device=G.DEV).bfloat16()
        out = torch.empty_like(q)
        ws = torch.empty(max(16, B.qllm_kv_attention_workspace(cache, heads * group, q, batch)), dtype=torch.uint8, device=G.DEV)
        st = torch.cuda.Stream()

        def step():
            B.qllm_kv_append(cache, 0, kv[:, 0], kv[:, 1], batch, stream=st)
            B.qllm_kv_attention(cache, 0, q, out, 0.09, batch, ws, stream=st)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            step()
        st.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            step()
        sides.append((table, cache, batch, start, q, kv, out, st, g))
    for lens in ([1, 64, 65], [900, 2, 511], [700, 899, 1]):
        for table, cache, batch, start, q, kv, out, st, g in sides:
            batch.seq_lens.copy_(ints(lens))
            q.normal_(); kv.normal_()
        torch.cuda.synchronize()
        for _ in range(3):
            for side in sides:
                with torch.cuda.stream(side[7]):
                    side[8].replay()
        torch.cuda.synchronize()
        for table, cache, batch, start, q, kv, out, st, g in sides:
            ref = kv_ref.attention(store_of(cache, 0), table, lens, start, host(q), 0.09, True)
            # (the lse of the check is this one's own)
            check_attention(out, torch.from_numpy(ref[1]).float(), ref, torch.bfloat16)
    assert B.qllm_poll_status() == B.QLLM_OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news", [[1, 2], [120, 1], [130, 130]])
def test_attention_leaves_other_rows_and_the_gaps_of_strided_outputs(dtype, news):
    heads, group, page, d = 2, 4, 32, 64
    rng = np.random.RandomState(41)
    lens = [150, 400]
    table = make_table(rng, lens, page, 20)
    cache = random_cache(41, 1, 20, heads, page, d)
    start = [6, 6 + news[0], 6 + sum(news)]
    rows = start[-1] + 9
    batch = B.KvBatch(ints(table), ints(lens), ints(start), rows, max(news))
    q = torch.randn(rows, heads * group, d, device=G.DEV).to(DT[dtype])
    wide = torch.full((rows, heads * group * d + 32), 5.0, device=G.DEV, dtype=DT[dtype])
    out = wide[:, 16:-16].unflatten(1, (heads * group, d))
    lse = torch.full((rows, heads * group), 5.0, device=G.DEV)
    ws = torch.empty(max(16, B.qllm_kv_attention_workspace(cache, heads * group, q, batch)), dtype=torch.uint8, device=G.DEV)
    B.qllm_kv_attention(cache, 0, q, out, 0.1, batch, ws, lse=lse)
    assert (wide[:, :16] == 5).all() and (wide[:, -16:] == 5).all()
    for a, b in ((0, 6), (start[-1], rows)):
        assert (wide[a:b] == 5).all() and (lse[a:b] == 5).all()
    ref = kv_ref.attention(store_of(cache, 0), table, lens, start, host(q), 0.1, True)
    cut = tuple(r[6:start[-1]] for r in ref)
    check_attention(out[6:start[-1]], lse[6:start[-1]], cut, DT[dtype], prompt=dtype == "bf16" and max(news) * group > 96)
    assert B.qllm_poll_status() == B.QLLM_OK


@pytest.mark.parametrize("news", [[200], [130, 1, 0]])
def test_prompt_kernels_in_a_graph(news):
    """The tensor-core kernel with its keys cut into parts (few rows), alone and together with the streaming one, captured on a
    stream of its own and replayed while lengths and pages change."""
    heads, group, page, d = 1, 4, 16, 128
    rng = np.random.RandomState(42)
    top = [1500] * len(news)
    table = make_table(rng, top, page, 300)
    cache = random_cache(42, 1, 300, heads, page, d)
    batch, start = batch_of(table, top, news)
    q = torch.randn(batch.rows, heads * group, d, device=G.DEV).bfloat16()
    out, st = torch.empty_like(q), torch.cuda.Stream()
    ws = torch.full((B.qllm_kv_attention_workspace(cache, heads * group, q, batch),), 0xFF, dtype=torch.uint8, device=G.DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        B.qllm_kv_attention(cache, 0, q, out, 0.09, batch, ws, stream=st)
    st.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        B.qllm_kv_attention(cache, 0, q, out, 0.09, batch, ws, stream=st)
    for lens in ([1500] * len(news), [200, 17, 0][:len(news)], [911, 1, 64][:len(news)]):
        other = make_table(np.random.RandomState(lens[0]), top, page, 300)
        batch.seq_lens.copy_(ints(lens))
        batch.table.copy_(ints(other))
        q.normal_()
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            g.replay()
        torch.cuda.synchronize()
        ref = kv_ref.attention(store_of(cache, 0), other, lens, start, host(q), 0.09, True)
        check_attention(out, torch.from_numpy(ref[1]).float(), ref, torch.bfloat16, prompt=True)
    assert B.qllm_poll_status() == B.QLLM_OK


@pytest.mark.parametrize("seed", range(40))
def test_attention_random_shapes(seed):
    rng = np.random.RandomState(1000 + seed)
    d, page, dtype = int(rng.choice([64, 128, 256])), int(rng.choice([16, 32, 64, 128, 256])), ["bf16", "f32"][rng.randint(2)]
    heads, group, seqs = rng.randint(1, 4), rng.randint(1, 12), rng.randint(1, 7)
    lens = [int(x) for x in np.exp(rng.uniform(0, np.log(1500), seqs))]
    news = [int(min(n, max(0, rng.choice([0, 1, 1, 3, 17, n // 2, n])))) for n in lens]
    if sum(news) == 0:
        news[0] = 1
    run_case(seed, dtype, d, page, heads, group, lens, news, bool(rng.rand() < 0.8), stride_pad=8 * rng.randint(0, 3),
             max_new=int(rng.choice([max(news), max(news), 1, 4000])))


def test_read_of_a_page_that_does_not_exist_is_zero():
    cache = random_cache(40, 1, 4, 2, 16, 64)
    k, v = torch.full((40, 2, 64), 5.0, device=G.DEV), torch.full((40, 2, 64), 5.0, device=G.DEV)
    B.qllm_kv_read(cache, 0, k, v, B.KvBatch(ints([[1, 9, 2]]), ints([40]), ints([0, 40]), 40, 40))
    assert (k[16:32] == 0).all() and (v[16:32] == 0).all() and (k[:16] != 0).any() and (k[32:] != 0).any()
    assert B.qllm_poll_status() == B.QLLM_ERR_PAGE


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_sequences_than_threads(dtype):
    """The kernels share out the work of all sequences: more of them than a CTA has threads, many without new tokens, a few with
    enough for the prompt kernel."""
    rng = np.random.RandomState(31)
    lens = rng.randint(0, 90, 1500)
    news = np.where(rng.rand(1500) < 0.6, 1, 0)
    news[[3, 700, 1499]] = [70, 1, 66]
    lens[[3, 700, 1499]] = [80, 2500, 300]
    run_case(31, dtype, 64, 16, 1, 2, lens.tolist(), news.tolist(), True)


@pytest.mark.parametrize("dtype,news", [("bf16", [300]), ("bf16", [1]), ("f32", [5])])
def test_one_sequence_out_of_range_is_reported(dtype, news):
    cache = random_cache(32, 1, 8, 2, 64, 128)
    q = torch.randn(news[0], 8, 128, device=G.DEV).to(DT[dtype])
    for lens in ([-1], [100000]):
        attend(cache, 0, q, B.KvBatch(ints([[0, 1, 2, 3, 4, 5]]), ints(lens), ints([0, news[0]]), news[0], news[0]), 0.1, True)
        assert B.qllm_poll_status() == B.QLLM_ERR_PAGE
    attend(cache, 0, q, B.KvBatch(ints([[0, 1, 2, 3, 4, 5]]), ints([384]), ints([0, news[0]]), news[0], news[0]), 0.1, True)
    assert B.qllm_poll_status() == B.QLLM_OK


def test_calls_take_no_memory():
    """Device memory in use, as the driver counts it, is the same before and after calls of every kind (allocated by nobody)."""
    cache, pool = random_cache(33, 2, 40, 2, 64, 128), B.KvPool.empty(40, 4, 8)
    q = torch.randn(400, 8, 128, device=G.DEV).bfloat16()
    out = torch.empty_like(q)
    one, prompt = ints([1, 1, 1, 1]), ints([300, 1, 1, 98])
    parent, child, fresh, remap, gone = ints([0]), ints([3]), ints([0]), torch.empty(40, dtype=torch.int32, device=G.DEV), ints([3])
    B.qllm_kv_pages_extend(cache, pool, prompt)
    batches = [(B.KvBatch(pool.table, pool.seq_lens, ints([0, 300, 301, 302, 400]), 400, 300), q, out),
               (B.KvBatch(pool.table, pool.seq_lens, ints([0, 1, 2, 3, 4]), 4, 1), q[:4], out[:4])]
    ws = torch.empty(max(B.qllm_kv_attention_workspace(cache, 8, a, b) for b, a, _ in batches), dtype=torch.uint8, device=G.DEV)
    src, dst = ints([0, 1]), ints([38, 39])

    def everything():
        for b, a, o in batches:
            B.qllm_kv_append(cache, 1, a[:, :2], a[:, 2:4], b)
            B.qllm_kv_read(cache, 1, o[:, :2], o[:, 2:4], b)
            B.qllm_kv_attention(cache, 1, a, o, 0.1, b, ws)
        B.qllm_kv_pages_free(pool, gone)
        B.qllm_kv_pages_fork(cache, pool, parent, child, fresh)
        B.qllm_kv_pages_extend(cache, pool, one)
        B.qllm_kv_pages_copy(cache, src, dst)
        B.qllm_kv_pages_compact(cache, pool, remap)
    everything()
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    for _ in range(3):
        everything()
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == before
    B.qllm_poll_status()


def test_results_do_not_depend_on_the_run():
    lens, news = [1, 700, 33, 4048, 5, 130, 1000, 64], [1, 1, 33, 1, 1, 130, 1, 64]
    a = run_case(30, "bf16", 128, 64, 2, 4, lens, news, True)
    for _ in range(3):
        assert torch.equal(a, run_case(30, "bf16", 128, 64, 2, 4, lens, news, True))


# ------------------------------------------------------------------------------------------------ pages
def pool_state(pool):
    return [t.cpu().numpy() for t in (pool.refs, pool.table, pool.seq_lens)]


def assert_pool(pool, model, what):
    for name, a, b in zip(("refs", "table", "lens"), pool_state(pool), (model.refs, model.table, model.lens)):
        assert np.array_equal(a, b), (what, name)


@pytest.mark.parametrize("seed,pages,seqs,width,page,layers,heads,d", [
    (1, 40, 9, 8, 16, 3, 2, 64), (2, 300, 33, 20, 64, 1, 1, 128), (3, 5000, 40, 70, 16, 2, 1, 64), (4, 12, 16, 5, 32, 4, 3, 256)])
def test_pool_against_its_rules(seed, pages, seqs, width, page, layers, heads, d):
    """Random calls, indices out of range and duplicates among them, against the rules applied entry by entry; every page's
    contents are followed through copies and moves."""
    rng = np.random.RandomState(seed)
    cache = random_cache(seed, layers, pages, heads, page, d)
    arrays = (cache.k_codes, cache.k_param, cache.v_codes, cache.v_param)
    content = [t.cpu().numpy().copy() for t in arrays]
    pool, model = B.KvPool.empty(pages, seqs, width), kv_ref.Pool(pages, seqs, width, page)
    B.qllm_poll_status()
    for turn in range(40):
        kind = rng.choice(["extend", "fork", "free", "compact"], p=[0.4, 0.25, 0.2, 0.15])
        model.failed, model.copies = False, []
        if kind == "extend":
            add = rng.randint(0, 3 * page, seqs) * (rng.rand(seqs) < 0.4)
            if rng.rand() < 0.2:
                add[rng.randint(seqs)] = rng.choice([-1, 10 ** 9, 2 ** 31 - 1])
            model.extend(add)
            B.qllm_kv_pages_extend(cache, pool, ints(add))
        elif kind == "fork":
            n = rng.randint(1, seqs)
            parent = rng.randint(0, seqs, n)
            child = rng.randint(-1, seqs + 1, n) if rng.rand() < 0.5 else rng.permutation(seqs)[:n]
            fresh = model.fork(parent.tolist(), child.tolist())
            got = B.qllm_kv_pages_fork(cache, pool, ints(parent), ints(child))
            assert got.tolist() == fresh
        elif kind == "free":
            gone = rng.randint(0, seqs, rng.randint(1, 5)).tolist()
            gone += [gone[0]] + ([-1, seqs] if rng.rand() < 0.3 else [])
            model.free(gone)
            B.qllm_kv_pages_free(pool, ints(gone))
        else:
            remap = torch.full((pages,), -9, dtype=torch.int32, device=G.DEV)
            want = model.compact()
            B.qllm_kv_pages_compact(cache, pool, remap)
            assert np.array_equal(remap.cpu().numpy(), want)
        assert_pool(pool, model, (turn, kind))
        assert B.qllm_poll_status() == (B.QLLM_ERR_PAGE if model.failed else B.QLLM_OK), (turn, kind)
        for c, t in zip(content, arrays):
            old = c.copy()
            for a, b in model.copies:
                c[:, b] = old[:, a]
            assert np.array_equal(c, t.cpu().numpy()), (turn, kind)


def test_page_copies():
    cache = random_cache(31, 5, 30, 3, 32, 128)
    arrays = (cache.k_codes, cache.k_param, cache.v_codes, cache.v_param)
    want = [t.clone() for t in arrays]
    src, dst = [3, 3, 7, 29, 40, 2, 5], [10, 0, 28, 1, 4, -1, 5]     # one page twice; two that do not exist; one onto itself
    for a, b in zip(src, dst):
        if 0 <= a < 30 and 0 <= b < 30:
            for t in want:
                t[:, b] = t[:, a]
    B.qllm_kv_pages_copy(cache, ints(src), ints(dst))
    for a, b in zip(arrays, want):
        assert torch.equal(a, b)
    assert B.qllm_poll_status() == B.QLLM_ERR_PAGE
    B.qllm_kv_pages_copy(cache, ints([]), ints([]))
    assert B.qllm_poll_status() == B.QLLM_OK


def test_pool_in_a_graph():
    """A captured decode step: room for one more token of every sequence, then append and attention, replayed over page
    boundaries; against a cache that was filled in one go."""
    heads, group, page, d, steps, seqs = 2, 4, 16, 64, 40, 3
    cache, pool = B.KvCache.empty(1, 20, heads, page, d), B.KvPool.empty(20, seqs, 4)
    x = torch.randn(steps, seqs, 2, heads, d, device=G.DEV).bfloat16()
    q = torch.randn(steps, seqs, heads * group, d, device=G.DEV).bfloat16()
    kv, qq = x[0].clone(), q[0].clone()
    one = ints([1] * seqs)
    batch = B.KvBatch(pool.table, pool.seq_lens, ints(range(seqs + 1)), seqs, 1)
    out = torch.empty_like(qq)
    ws = torch.empty(max(16, B.qllm_kv_attention_workspace(cache, heads * group, qq, batch)), dtype=torch.uint8, device=G.DEV)

    def step():
        B.qllm_kv_pages_extend(cache, pool, one)
        B.qllm_kv_append(cache, 0, kv[:, 0], kv[:, 1], batch)
        B.qllm_kv_attention(cache, 0, qq, out, d ** -0.5, batch, ws)
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    B.qllm_kv_pages_free(pool, ints(range(seqs)))
    outs = []
    for i in range(steps):
        kv.copy_(x[i]); qq.copy_(q[i])
        g.replay()
        outs.append(out.clone())
    assert B.qllm_poll_status() == B.QLLM_OK and pool.seq_lens.tolist() == [steps] * seqs
    whole, lens = B.KvCache.empty(1, 9, heads, page, d), [steps] * seqs
    table = np.arange(9, dtype=np.int32).reshape(3, 3)
    b2, start = batch_of(table, lens, [steps] * seqs)
    flat = x.transpose(0, 1).reshape(steps * seqs, 2, heads, d)
    B.qllm_kv_append(whole, 0, flat[:, 0], flat[:, 1], b2)
    ref = kv_ref.attention(store_of(whole, 0), table, lens, start, host(q.transpose(0, 1).reshape(steps * seqs, heads * group, d)), d ** -0.5, True)
    got = torch.stack(outs, 1).reshape(steps * seqs, heads * group, d)
    check_attention(got, torch.from_numpy(ref[1]).float(), ref, torch.bfloat16)


# ------------------------------------------------------------------------------------------------ as they are used
@pytest.mark.parametrize("out_dtype", ["bf16", "f32"])
def test_behind_a_quantized_layer(out_dtype):
    """A quantized QKV layer's rows go into the cache as they lie (three strided parts), a prompt first, then forked
    sequences token by token; every step against 64-bit attention over what the cache holds."""
    import parity
    from paper_2310_08041_b200 import synth
    heads, group, d, page = 1, 2, 64, 16                    # 2 query heads, 1 key and 1 value head: 256 outputs
    cfg = synth.CONFIGS["c1"].scaled(M=64, N=(group + 2) * heads * d)
    L = parity.oracle_layer(cfg)
    h = B.qllm_build_reassembly(L["absmax"], L["theta"], L["W"], L["lrA"], L["lrB"], cfg.w_bits)
    layer = B.Layer(h, L["gamma"], L["beta"], cfg.ln_eps, None, cfg.a_bits, B.QLLM_F32, B.QLLM_BF16 if out_dtype == "bf16" else B.QLLM_F32, max_M=64)
    x = G.dev_x(synth.activations(cfg))
    cache, pool = B.KvCache.empty(2, 24, heads, page, d), B.KvPool.empty(24, 4, 6)

    def split(t):
        t = t.view(t.shape[0], (group + 2) * heads, d)
        return t[:, :group * heads], t[:, group * heads:(group + 1) * heads], t[:, (group + 1) * heads:]

    def step(rows, batch, start):
        out = torch.empty(rows.shape[0], cfg.N, device=G.DEV, dtype=DT[out_dtype])
        layer.forward(rows, out)
        q, k, v = split(out)
        B.qllm_kv_append(cache, 1, k, v, batch)
        got, lse = attend(cache, 1, q, batch, d ** -0.5, True)
        ref = kv_ref.attention(store_of(cache, 1), batch.table.cpu().numpy(), batch.seq_lens.tolist(), start, host(q), d ** -0.5, True)
        check_attention(got, lse, ref, DT[out_dtype], prompt=out_dtype == "bf16" and batch.max_new * group > 96)

    B.qllm_kv_pages_extend(cache, pool, ints([41, 0, 0, 0]))
    start = [0, 41, 41, 41, 41]
    step(x[:41].contiguous(), B.KvBatch(pool.table, pool.seq_lens, ints(start), 41, 41), start)
    B.qllm_kv_pages_fork(cache, pool, ints([0, 0]), ints([2, 3]))
    for i in range(9):                                       # the three siblings go on with tokens of their own
        B.qllm_kv_pages_extend(cache, pool, ints([1, 0, 1, 1]))
        start = [0, 1, 1, 2, 3]
        rows = x[[41 + i, 50 + i, 20 + i]].contiguous()
        step(rows, B.KvBatch(pool.table, pool.seq_lens, ints(start), 3, 1), start)
    B.qllm_kv_pages_free(pool, ints([0]))
    B.qllm_kv_pages_compact(cache, pool, torch.empty(24, dtype=torch.int32, device=G.DEV))
    B.qllm_kv_pages_extend(cache, pool, ints([0, 0, 3, 2]))
    start = [0, 0, 0, 3, 5]
    step(x[59:64].contiguous(), B.KvBatch(pool.table, pool.seq_lens, ints(start), 5, 3), start)
    assert B.qllm_poll_status() == B.QLLM_OK and pool.seq_lens.tolist() == [0, 0, 53, 52]
    layer.destroy()
