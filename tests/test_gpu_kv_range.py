"""The 4-bit cache where its numbers lie far apart: keys and values of very different size in one tile, rows without a range, rows
that are no numbers, queries near the end of their type."""
import numpy as np
import pytest
import torch

import gpu_util as G
import kv_bounds
import kv_ref
from paper_2310_08041_b200 import binding as B
from test_gpu_kv import DT, attend, batch_of, check_attention, host, ints, make_table, random_cache, store_of
from test_gpu_kv_prompt import layer_of, queries

pytestmark = pytest.mark.gpu


def place(table, s, position, page):
    return int(table[s, position // page]), position % page


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("power", [8, 12, 14, 16, 20, 24, 33, 60])
@pytest.mark.parametrize("where", ["behind the rows", "seen and turned away from", "far from zero"])
def test_a_loud_key_leaves_the_others_their_bits(where, power, d):
    """One key 2^power times the others, in a tile of the tensor-core kernel: behind the rows that are looked at (causal), or in front of
    them with a score so low that it has no weight.  The others' scores decide every row and keep their precision; so they do where all
    keys lie far from zero."""
    lens, news, page, heads, group = [300, 150], [150, 100], 64, 2, 4
    table = make_table(np.random.RandomState(61), lens, page, 9)
    cache = random_cache(61, 1, 9, heads, page, d)
    batch, start = batch_of(table, lens, news)
    q, scale = queries(62, batch.rows, heads * group, d), d ** -0.5
    if where == "far from zero":
        cache.k_param[..., 1] = torch.randint(-4000, 4000, cache.k_param.shape[:-1], device=G.DEV).float()
        scale /= 300
    for s, n in enumerate(lens):
        at = n - 1 if where != "seen and turned away from" else 70 + s
        p, i = place(table, s, at, page)
        cache.k_param[0, p, :, i, 0] *= 2.0 ** power
        if where == "seen and turned away from":
            cache.k_param[0, p, :, i, 1] = 16.0              # code - zero < 0 in every channel
            q = q.abs()
    want = kv_bounds.expect(layer_of(cache), table, lens, start, q, scale, True)
    got, lse = attend(cache, 0, q, batch, scale, True)
    rows = [r for r in range(batch.rows) if r + 1 not in start] if where != "seen and turned away from" else None
    kv_bounds.check(got, lse, want, rows)
    assert B.qllm_poll_status() == B.QLLM_OK


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_keys_of_every_size(causal, d):
    """Key scales spread evenly over 2^-40 .. 1 in every tile, and queries large enough for the small ones to matter too."""
    lens, news, page, heads, group = [500, 130], [200, 130], 32, 2, 2
    table = make_table(np.random.RandomState(63), lens, page, 25)
    cache = random_cache(63, 1, 25, heads, page, d)
    g = torch.Generator(device=G.DEV); g.manual_seed(63)
    cache.k_param[..., 0] = 2.0 ** (torch.rand(cache.k_param.shape[:-1], generator=g, device=G.DEV) * -40)
    cache.k_param[..., 1] = 16.0                             # with queries above zero every score is negative: the small ones lead
    batch, start = batch_of(table, lens, news)
    q = queries(64, batch.rows, heads * group, d).abs() * 2.0 ** torch.randint(0, 30, (batch.rows, heads * group, 1), generator=g, device=G.DEV)
    q = q.bfloat16()
    want = kv_bounds.expect(layer_of(cache), table, lens, start, q, d ** -0.5, causal)
    got, lse = attend(cache, 0, q, batch, d ** -0.5, causal)
    kv_bounds.check(got, lse, want)
    # a key without a scale, as in a cache that was never written, scores zero
    cache.k_param[:, ::2, :, ::3, 0] = 0.0
    want = kv_bounds.expect(layer_of(cache), table, lens, start, q, d ** -0.5, causal)
    got, lse = attend(cache, 0, q, batch, d ** -0.5, causal)
    kv_bounds.check(got, lse, want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("zero", [3, 60, 200, 400, 800, 899])
@pytest.mark.parametrize("apart", [1.02, 1.9, 8.0, 100.0])
def test_quiet_values_far_from_zero_beside_loud_ones(apart, zero, d):
    """Values up to nearly 2^11 apart in one tile of the tensor-core kernel, zero-points up to where it takes them as they are: rows whose
    weight lies on quiet tokens have their values with the bits that a scale has in fp16.  The quiet scale lies between two
    subnormal fp16 numbers when it is counted in the loud values' power of two."""
    lens, news, page, heads, group = [400, 150], [150, 100], 64, 2, 4
    table = make_table(np.random.RandomState(65), lens, page, 11)
    cache = random_cache(65, 1, 11, heads, page, d)
    batch, start = batch_of(table, lens, news)
    g = torch.Generator(device=G.DEV); g.manual_seed(65)
    cache.v_param[..., 1] = -zero
    loud = torch.rand(cache.v_param.shape[:-1], generator=g, device=G.DEV) < 0.2
    power = int(np.floor(np.log2(zero + 15)))                # of the loudest value: their scale is 1
    quiet = (np.floor(apart * 16384 / (zero + 15)) + 0.45) * 2.0 ** (power - 24)
    cache.v_param[..., 0] = torch.where(loud, 1.0, quiet)
    cache.k_param[..., 1] = torch.where(loud, 20.0, cache.k_param[..., 1])   # queries above zero turn away from the loud tokens
    q = queries(66, batch.rows, heads * group, d).abs()
    want = kv_bounds.expect(layer_of(cache), table, lens, start, q, d ** -0.5, True)
    got, lse = attend(cache, 0, q, batch, d ** -0.5, True)
    kv_bounds.check(got, lse, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_a_row_with_nan_reads_back_as_nan(dtype, d):
    """One NaN anywhere in a key or value row, and the row is NaN when it is read and in the attention of every token that sees it; rows
    beside it, of the same token too, are as without it."""
    heads, page, n = 2, 16, 40
    cache = B.KvCache.empty(1, 4, heads, page, d)
    batch, start = batch_of(np.array([[2, 0, 3]]), [n], [n])
    g = torch.Generator(device=G.DEV); g.manual_seed(71)
    x = torch.randn(n, 2, heads, d, generator=g, device=G.DEV).to(DT[dtype])
    B.qllm_kv_append(cache, 0, x[:, 0], x[:, 1], batch)
    clean = torch.empty_like(x)
    B.qllm_kv_read(cache, 0, clean[:, 0], clean[:, 1], batch)
    bad = torch.zeros(n, 2, heads, dtype=torch.bool, device=G.DEV)
    for i, (t, kv, h) in enumerate([(0, 0, 0), (7, 1, 1), (21, 0, 1), (21, 1, 0), (39, 1, 0)]):
        x[t, kv, h, (17 * i + d - 1) % d] = float("nan") if i % 2 else -float("nan")
        bad[t, kv, h] = True
    B.qllm_kv_append(cache, 0, x[:, 0], x[:, 1], batch)
    back = torch.empty_like(x)
    B.qllm_kv_read(cache, 0, back[:, 0], back[:, 1], batch)
    assert torch.isnan(back[bad]).all() and torch.equal(back[~bad], clean[~bad])
    q = torch.randn(n, 2 * heads, d, generator=g, device=G.DEV).to(DT[dtype])
    got, lse = attend(cache, 0, q, batch, 0.1, True)
    first = torch.where(bad.any(1), torch.arange(n, device=G.DEV)[:, None], n).amin(0)          # per key head
    sees = torch.arange(n, device=G.DEV)[:, None] >= first[None]
    sees = sees.repeat_interleave(2, 1)
    assert torch.isnan(got[sees].float()).all() and torch.isfinite(got[~sees].float()).all()


TINY = 2.0 ** -127


def tiny_rows(d):
    """Rows whose range, or whose only value, is too small for a float32 reciprocal; some far from zero for it, some at its border."""
    g = torch.Generator().manual_seed(72)
    u = torch.rand(16, d, generator=g, dtype=torch.float64)
    rows = [u[0] * 1e-39, u[1] * 1e-39 - 5e-40, -u[2] * 1e-39, torch.full((d,), 1e-40), torch.full((d,), -1e-40), torch.full((d,), 2.0 ** -149),
            (u[3] < 0.5) * 2.0 ** -149, 1e-37 + u[4] * 2e-38, 1e-33 + (u[5] < 0.1) * 1e-40, -1e-31 - (u[6] < 0.1) * 1e-38, u[7] * 15 * TINY,
            u[8] * 14.9 * 2 * TINY, u[9] * 1e-30, torch.zeros(d), torch.full((d,), 2.0 ** -126), torch.full((d,), -3e-38)]
    return torch.stack([r.double() for r in rows]).float()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_rows_whose_range_has_no_reciprocal(dtype, d):
    """Underflowed rows are finite data: they read back within half a step, a step being a fifteenth of the range or 2^-127 where that
    is larger, and attention over them is finite."""
    x = tiny_rows(d).to(DT[dtype]).to(G.DEV)
    n, heads, page = x.shape[0], 1, 16
    cache = B.KvCache.empty(1, 3, heads, page, d)
    batch, start = batch_of(np.array([[1]]), [n], [n])
    rows = x[:, None].contiguous()
    B.qllm_kv_append(cache, 0, rows, rows.flip(0).contiguous(), batch)
    k, v = torch.empty_like(rows, dtype=torch.float32), torch.empty_like(rows, dtype=torch.float32)
    B.qllm_kv_read(cache, 0, k, v, batch)
    x64 = x.double()
    # half a step; the zero-point and the quotient are float32 numbers, off by 2^-23 of a row far from zero each, as is the range's step
    step = ((x64.amax(-1) - x64.amin(-1)) / 15).clamp(min=TINY)[:, None]
    step = torch.where((x64.amax(-1) == x64.amin(-1))[:, None], TINY, step)                     # a constant row is its own scale
    tol = step * (0.5 + 2.0 ** -20) + 2.0 ** -21 * x64.abs() + 2.0 ** -148
    assert torch.isfinite(k).all() and ((k[:, 0].double() - x64).abs() <= tol).all()
    assert torch.equal(v, k.flip(0))
    q = torch.randn(n, 4 * heads, d, device=G.DEV).to(DT[dtype])
    got, lse = attend(cache, 0, q, batch, 0.1, True)
    ref = kv_ref.attention(store_of(cache, 0), np.array([[1]]), [n], start, host(q), 0.1, True)
    # all values lie below 2e-31, and weights of values so far below the row of zeros, whose scale is 1, may count as nothing
    assert (np.abs(host(got) - ref[0]) <= 1e-30).all() and np.abs(host(lse) - ref[1]).max() < 1e-4


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_rows_whose_range_passes_the_largest_float(dtype, d):
    """hi - lo beyond float32 is still finite data: its fifteenth is a float32 number, and the row reads back within half of it."""
    g = torch.Generator(device=G.DEV); g.manual_seed(73)
    n, page = 12, 16
    x = (torch.rand(n, 1, d, generator=g, device=G.DEV) * 2 - 1) * 3.3e38
    x[:, 0, 0], x[:, 0, d - 1] = 3.3e38, -3.3e38
    x[1] = x[1].sign() * 3.3e38
    x[2, 0, 0] = 1e38                                        # -3.3e38 .. 3.3e38 at one end only
    x[3, 0] = torch.where(x[3, 0] < 0, -3.38e38, 0.5e38)
    x = x.to(DT[dtype])
    cache = B.KvCache.empty(1, 3, 1, page, d)
    batch, start = batch_of(np.array([[2]]), [n], [n])
    B.qllm_kv_append(cache, 0, x, x, batch)
    k, v = torch.empty(n, 1, d, device=G.DEV), torch.empty(n, 1, d, device=G.DEV)
    B.qllm_kv_read(cache, 0, k, v, batch)
    x64 = x.double()
    step = (x64.amax(-1, keepdim=True) - x64.amin(-1, keepdim=True)) / 15
    # the values themselves may pass the largest float32 by the rounding of their step: no infinity may come out of that
    assert torch.isfinite(k).all() and torch.equal(k, v)
    assert ((k.double() - x64).abs() <= step * (0.5 + 2.0 ** -20) + 2.0 ** -21 * x64.abs()).all()
    # an infinity still has no finite scale
    x[5, 0, 3] = float("inf")
    B.qllm_kv_append(cache, 0, x, x, batch)
    B.qllm_kv_read(cache, 0, k, v, batch)
    assert not torch.isfinite(k[5]).any() and torch.isfinite(k[4]).all() and torch.isfinite(k[6]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_beside_the_largest_float(dtype):
    """Rows that lie at one end of float32, far from zero for their range or not: finite, within half a step."""
    g = torch.Generator(device=G.DEV); g.manual_seed(74)
    ends = [(3.0e38, 3.38e38), (-3.38e38, -3.0e38), (2.0e38, 3.38e38), (-3.38e38, 1e30), (-1e38, 3.38e38), (3.3e38, 3.38e38), (-3.38e38, 3.1e38), (0.0, 3.38e38)]
    n, d = len(ends), 128
    x = torch.rand(n, 1, d, generator=g, device=G.DEV)
    for i, (lo, hi) in enumerate(ends):
        x[i] = lo * (1 - x[i]) + hi * x[i]
        x[i, 0, 5], x[i, 0, 77] = lo, hi
    x = x.to(DT[dtype])
    cache = B.KvCache.empty(1, 3, 1, 16, d)
    batch, start = batch_of(np.array([[1]]), [n], [n])
    B.qllm_kv_append(cache, 0, x, x, batch)
    k, v = torch.empty_like(x), torch.empty_like(x)
    B.qllm_kv_read(cache, 0, k, v, batch)
    x64 = x.double()
    step = (x64.amax(-1, keepdim=True) - x64.amin(-1, keepdim=True)) / 15
    assert torch.isfinite(k).all() and torch.equal(k, v)
    # half a step, float32 roundings of scale, zero-point and value, and the value's rounding to the type
    tol = step * (0.5 + 2.0 ** -20) + x64.abs() * (2.0 ** -20 + torch.finfo(x.dtype).eps) + step * torch.finfo(x.dtype).eps
    assert ((k.double() - x64).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news", [[1, 1], [5, 2], [70, 130]])
@pytest.mark.parametrize("power", [100, 114, 115, 116, 117, 120, 125, 127])
def test_queries_near_the_end_of_their_type(power, news, dtype):
    """Finite queries of up to 2^128 against keys so small that the scores are ordinary; beside them, in the same calls, rows of ordinary
    size, whose scores vanish."""
    lens, page, heads, group, d = [300, 140], 64, 2, 4, 128
    table = make_table(np.random.RandomState(75), lens, page, 9)
    cache = random_cache(75, 1, 9, heads, page, d)
    cache.k_param[..., 0] *= 2.0 ** -(power - 1)
    batch, start = batch_of(table, lens, news)
    q = torch.randn(batch.rows, heads * group, d, device=G.DEV).clamp(-3.9, 3.9)
    q[:, 1::2] *= 2.0 ** (power - 2)
    q = q.to(DT[dtype])
    got, lse = attend(cache, 0, q, batch, 0.09, True)
    ref = kv_ref.attention(store_of(cache, 0), table, lens, start, host(q), 0.09, True)
    check_attention(got, lse, ref, DT[dtype], prompt=dtype == "bf16" and max(news) * group > 96)
    assert B.qllm_poll_status() == B.QLLM_OK


def one_in_front(power, sign, page, lens, table, cache, at):
    """Keys of one sequence all alike and one of twice their size: scores sign 2^power and, at position `at`, twice (a half, when they
    are negative) that, for queries of ones."""
    heads, d = cache.kv_heads, cache.head_dim
    for s, n in enumerate(lens):
        cache.k_codes[0] = 0x11                              # every code 1: code - zero = 1 - zero = +-1
        cache.k_param[0, ..., 1] = 0.0 if sign > 0 else 2.0
        cache.k_param[0, ..., 0] = 2.0 ** power / d
        for s, n in enumerate(lens):
            p, i = place(table, s, at % n, page)
            cache.k_param[0, p, :, i, 0] *= 2.0 if sign > 0 else 0.5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news", [[1, 1], [9, 3], [70, 130]])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("power", [6, 14, 20, 22, 24, 25, 26, 27, 28, 30, 36, 60, 90])
def test_scores_of_every_size(power, sign, news, dtype):
    """Scores whose float32 numbers lie far apart: with one key in front of the others its value comes out, with all keys alike the mean
    of all values.  The scale's mantissa is no power of two, so no product of it is exact."""
    lens, page, heads, group, d, scale = [700, 400], 64, 2, 4, 128, 0.7
    table = make_table(np.random.RandomState(77), lens, page, 20)
    cache = random_cache(77, 1, 20, heads, page, d)
    batch, start = batch_of(table, lens, news)
    q = torch.ones(batch.rows, heads * group, d, device=G.DEV, dtype=DT[dtype])
    st = store_of(cache, 0)
    eps = torch.finfo(DT[dtype]).eps
    for at in (0, 133, 299):                                 # in front of every causal row's limit
        one_in_front(power, sign, page, lens, table, cache, at)
        got, lse = attend(cache, 0, q, batch, scale, False)
        best = scale * sign * 2.0 ** power * (2 if sign > 0 else 0.5)
        for s, n in enumerate(lens):
            kc, kp, vc, vp = st.rows(table[s], at % n, at % n + 1)
            v = np.repeat((vc[0] - vp[0, :, 1:2]) * vp[0, :, 0:1], group, 0)
            rows = slice(int(start[s]), int(start[s + 1]))
            a = host(got[rows])
            # the weights beside it are below 2^-21 together; the value's scale and products carry 11 bits at least
            assert np.abs(a - v[None]).max() <= (eps + 2 * 2.0 ** -11 if dtype == "bf16" else 2.0 ** -20) * np.abs(v).max(), (at, s)
            assert np.abs(host(lse[rows]) / best - 1).max() < (2.0 ** -9 if dtype == "bf16" else 2.0 ** -20)
    cache.k_param[0, ..., 0] = 2.0 ** power / d
    for causal in (True, False):
        got, lse = attend(cache, 0, q, batch, scale, causal)
        st = store_of(cache, 0)
        for s, n in enumerate(lens):
            kc, kp, vc, vp = st.rows(table[s], 0, n)
            v = np.repeat((vc - vp[..., 1:2]) * vp[..., 0:1], group, 1)
            for i in range(news[s]):
                m = n - news[s] + i + 1 if causal else n
                a, want = host(got[int(start[s]) + i]), v[:m].mean(0)
                spread = np.abs(v[:m]).mean(0)
                assert (np.abs(a - want) <= np.abs(want) * eps + spread * (2.0 ** -9 if dtype == "bf16" else 2.0 ** -18)).all(), (causal, s, i)
    assert B.qllm_poll_status() == B.QLLM_OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news", [[1, 1], [70, 130]])
@pytest.mark.parametrize("power", [-135, -127, -126, -100, 60, 120])
def test_scales_near_the_ends_of_float32(power, news, dtype):
    """Scales of 2^power times 0.7, subnormal ones among them, against queries and keys that make ordinary scores of them."""
    lens, page, heads, group, d = [300, 140], 64, 2, 4, 128
    table = make_table(np.random.RandomState(79), lens, page, 9)
    cache = random_cache(79, 1, 9, heads, page, d)
    there = -power // 2 - 2                                  # half of it on the keys, half on the queries
    cache.k_param[..., 0] *= 2.0 ** there
    batch, start = batch_of(table, lens, news)
    q = (torch.randn(batch.rows, heads * group, d, device=G.DEV) * 2.0 ** (-power - there - 3)).to(DT[dtype])
    scale = 0.7 * 2.0 ** power
    got, lse = attend(cache, 0, q, batch, scale, True)
    ref = kv_ref.attention(store_of(cache, 0), table, lens, start, host(q), float(np.float32(scale)), True)
    check_attention(got, lse, ref, DT[dtype], prompt=dtype == "bf16" and max(news) * group > 96)
    assert B.qllm_poll_status() == B.QLLM_OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news", [[1, 3], [70, 130]])
def test_zero_points_that_are_no_integers(news, dtype):
    """As append stores them for rows near the end of float32, here at ordinary scales."""
    lens, page, heads, group, d = [300, 140], 64, 2, 4, 128
    table = make_table(np.random.RandomState(80), lens, page, 9)
    cache = random_cache(80, 1, 9, heads, page, d)
    g = torch.Generator(device=G.DEV); g.manual_seed(80)
    for p in (cache.k_param, cache.v_param):
        some = torch.rand(p.shape[:-1], generator=g, device=G.DEV) < 0.5
        p[..., 1] += torch.where(some, torch.rand(p.shape[:-1], generator=g, device=G.DEV), 0.0)
    batch, start = batch_of(table, lens, news)
    q = torch.randn(batch.rows, heads * group, d, device=G.DEV).to(DT[dtype])
    got, lse = attend(cache, 0, q, batch, 0.09, True)
    ref = kv_ref.attention(store_of(cache, 0), table, lens, start, host(q), 0.09, True)
    prompt = dtype == "bf16" and max(news) * group > 96
    check_attention(got, lse, ref, DT[dtype], prompt=prompt)
    if prompt:
        kv_bounds.check(got, lse, kv_bounds.expect(layer_of(cache), table, lens, start, q, 0.09, True))
