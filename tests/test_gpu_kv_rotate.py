"""qllm_kv_rotate_append and qllm_rotary_table on the GPU.  The rotation is a product, a product and a sum, each rounded to float32, so what
comes out has to be equal to the same operations in numpy: queries after their one rounding, keys as codes and parameters."""
import numpy as np
import pytest
import torch

import block_ref
import gpu_util as G
import kv_ref
from paper_2310_08041_b200 import binding as B
from test_gpu_kv import DT, batch_of, host, ints, make_table, random_cache, store_of

pytestmark = pytest.mark.gpu


def f32(t):
    return t.float().cpu().numpy()


def qkv_rows(seed, rows, q_heads, heads, d, dtype, pad=0):
    """The three parts of one projection's rows, as they lie."""
    g = torch.Generator(device=G.DEV); g.manual_seed(seed)
    wide = torch.randn(max(rows, 1), (q_heads + 2 * heads) * d + pad, generator=g, device=G.DEV)
    wide[:, 3::17] *= 6
    t = wide.to(DT[dtype])[:rows, :(q_heads + 2 * heads) * d].unflatten(1, (q_heads + 2 * heads, d))
    return t[:, :q_heads], t[:, q_heads:q_heads + heads], t[:, q_heads + heads:]


def positions(lens, start):
    """Of every row of the batch's sequences; negative: none."""
    return np.concatenate([np.arange(n - (b - a), n) for n, a, b in zip(lens, start[:-1], start[1:])])


def check(cache, layer, before, q, k, v, q_out, table, lens, start, ang, rot_dim, inter, present=None):
    """before: the layer's arrays as they were.  present: rows that have a place (default: position >= 0)."""
    pos = positions(lens, start)
    seq = np.repeat(np.arange(len(lens)), np.diff(start))
    rows = np.arange(start[0], start[-1])
    cs = f32(ang)[np.clip(pos, 0, ang.shape[0] - 1)]
    can = (pos >= 0) & (pos < ang.shape[0])
    turn = lambda x: block_ref.turned(f32(x)[rows], cs[..., 0], cs[..., 1], rot_dim, inter)  # noqa: E731
    if q is not None:
        want = torch.from_numpy(np.where(can[:, None, None], turn(q), 0)).to(q_out.dtype)
        assert torch.equal(q_out[rows[0]:rows[-1] + 1].cpu(), want)
    st, page = store_of(cache, layer), cache.page_size
    want = [t.copy() for t in before]
    for i, x in ((0, turn(k)), (2, f32(v)[rows])):
        codes, scale, zero = kv_ref.quantize(x)
        for r in np.nonzero(can if present is None else present)[0]:
            pg, at = table[seq[r]][pos[r] // page], pos[r] % page
            want[i][pg, :, at] = codes[r]
            want[i + 1][pg, :, at, 0], want[i + 1][pg, :, at, 1] = scale[r], zero[r]
    for name, a, b in zip(("k_codes", "k_param", "v_codes", "v_param"), (st.kc, st.kp, st.vc, st.vp), want):
        assert np.array_equal(a, b), "%s: %d values differ" % (name, (a != b).sum())


def layer_arrays(cache, layer):
    s = store_of(cache, layer)
    return [s.kc.copy(), s.kp.copy(), s.vc.copy(), s.vp.copy()]


def run_case(seed, dtype, d, rot_dim, inter, page, heads, q_heads, lens, news, pad=0, inplace=False, layers=2, gap=(0, 0)):
    rng = np.random.RandomState(seed)
    pages = sum(-(-n // page) for n in lens) + 3
    table = make_table(rng, lens, page, pages)
    cache = random_cache(seed, layers, pages, heads, page, d)
    batch, start = batch_of(table, lens, news)
    if gap != (0, 0):
        start = start + gap[0]
        batch = B.KvBatch(batch.table, batch.seq_lens, ints(start), int(start[-1]) + gap[1], max(news))
    q, k, v = qkv_rows(seed, batch.rows, q_heads, heads, d, dtype, pad)
    rot = B.Rotary.make(max(max(lens), 1), rot_dim, interleaved=inter)
    guard = None
    if q_heads == 0:
        q = q_out = None
    elif inplace:
        q_out, q = q, q.clone()
    else:
        guard = G.Guarded((batch.rows, q_heads, d), DT[dtype], 3.0)
        q_out = guard.t
    before, other = layer_arrays(cache, layers - 1), layer_arrays(cache, 0)
    B.qllm_kv_rotate_append(cache, layers - 1, q_out if inplace else q, q_out, k, v, rot, batch)
    assert B.qllm_poll_status() == B.QLLM_OK
    if guard is not None:
        guard.check("q_out")
        assert (q_out[:start[0]] == 3).all() and (q_out[start[-1]:] == 3).all()
    check(cache, layers - 1, before, q, k, v, q_out, table, lens, start, rot.table, rot_dim, inter)
    if layers > 1:
        assert all(np.array_equal(a, b) for a, b in zip(layer_arrays(cache, 0), other))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rot_dim", [(64, 64), (64, 16), (128, 128), (128, 96), (128, 16), (256, 256), (256, 48), (256, 128)])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("heads,q_heads,page", [(1, 8, 16), (4, 5, 64), (8, 64, 32)])
def test_rotate_append(dtype, d, rot_dim, inter, heads, q_heads, page):
    run_case(d + rot_dim + heads, dtype, d, rot_dim, inter, page, heads, q_heads, [70, 1, 33, 0, 200], [1, 1, 5, 0, 40])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_shapes(dtype):
    run_case(1, dtype, 128, 128, False, 16, 32, 32, [517], [1])                       # one token
    run_case(2, dtype, 128, 128, False, 64, 8, 64, [300, 5, 900], [300, 5, 900], pad=64)   # prompts, strided
    run_case(3, dtype, 128, 64, True, 64, 8, 8, [100] * 300, [1] * 300, layers=1)     # more sequences than a warp counts
    run_case(4, dtype, 64, 64, False, 16, 3, 0, [40, 3], [9, 3])                      # keys and values only
    run_case(5, dtype, 128, 128, False, 128, 2, 6, [80, 30], [20, 30], inplace=True, pad=32)
    run_case(6, dtype, 128, 128, False, 128, 2, 6, [80, 30], [20, 30], gap=(5, 7))
    run_case(7, dtype, 256, 256, True, 256, 1, 3, [80, 3000], [20, 1])
    run_case(8, dtype, 64, 32, False, 32, 1, 1, [1], [1])
    run_case(9, dtype, 128, 128, True, 16, 1024, 8, [3], [3], layers=1)               # more rows to a token than a CTA holds


@pytest.mark.parametrize("seed", range(6))
def test_random_shapes(seed):
    r = np.random.RandomState(100 + seed)
    d = int(r.choice([64, 128, 256]))
    lens = [int(x) for x in r.randint(0, 400, r.randint(1, 40))]
    news = [int(r.randint(0, n + 1)) if r.rand() < 0.3 else min(n, 1) for n in lens]
    run_case(seed, ["bf16", "f32"][seed % 2], d, 16 * r.randint(1, d // 16 + 1), bool(r.randint(2)), int(r.choice([16, 32, 64, 128, 256])),
             int(r.randint(1, 9)), int(r.randint(0, 20)), lens, news, inplace=bool(r.randint(2)))


def test_angle_zero_is_append():
    """With cosine 1 and sine 0 everywhere the cache is qllm_kv_append's, bit for bit, and queries come back as they were."""
    lens, news = [70, 9], [30, 9]
    table = make_table(np.random.RandomState(1), lens, 16, 12)
    a, b = random_cache(5, 1, 12, 4, 16, 128), random_cache(5, 1, 12, 4, 16, 128)
    batch, _ = batch_of(table, lens, news)
    q, k, v = qkv_rows(3, 39, 8, 4, 128, "bf16")
    ang = torch.zeros(70, 64, 2, device=G.DEV)
    ang[..., 0] = 1
    q_out = torch.empty(39, 8, 128, device=G.DEV, dtype=torch.bfloat16)
    B.qllm_kv_rotate_append(a, 0, q, q_out, k, v, B.Rotary(ang), batch)
    B.qllm_kv_append(b, 0, k, v, batch)
    for x, y in zip((a.k_codes, a.k_param, a.v_codes, a.v_param), (b.k_codes, b.k_param, b.v_codes, b.v_param)):
        assert torch.equal(x, y)
    assert torch.equal(q_out, q)


def test_more_new_tokens_than_length_and_positions_beyond_the_table():
    """Tokens without a position: queries 0, nothing stored.  Beyond the table: the same, and reported."""
    lens, news, page = [3, 40], [5, 10], 16
    table = make_table(np.random.RandomState(2), lens, page, 9)
    cache = random_cache(6, 1, 9, 2, page, 64)
    batch, start = batch_of(table, lens, news)
    q, k, v = qkv_rows(4, 15, 4, 2, 64, "f32")
    for top, status in ((40, B.QLLM_OK), (36, B.QLLM_ERR_PAGE)):
        rot = B.Rotary.make(top, 64)
        before, q_out = layer_arrays(cache, 0), torch.full((15, 4, 64), 3.0, device=G.DEV)
        B.qllm_kv_rotate_append(cache, 0, q, q_out, k, v, rot, batch)
        assert B.qllm_poll_status() == status
        check(cache, 0, before, q, k, v, q_out, table, lens, start, rot.table, 64, False)
        assert (q_out[:2] == 0).all() and ((q_out[start[1] + 6:] == 0).all() == (top == 36))


def test_bad_pages_and_lengths_are_reported_and_harmless():
    """A token whose page does not exist is not stored, its queries are turned; a length beyond the table row is cut."""
    lens, news, page = [20, 40, 5], [20, 3, 5], 16
    table = make_table(np.random.RandomState(3), lens, page, 9)
    q, k, v = qkv_rows(5, 28, 4, 2, 64, "f32")
    for bad in (-1, 9, 2 ** 31 - 1, -2 ** 31):
        t = table.copy()
        t[0, 1] = bad                                        # positions 16 .. 19 of sequence 0
        cache = random_cache(7, 1, 9, 2, page, 64)
        batch, start = batch_of(t, lens, news)
        rot = B.Rotary.make(64, 64)
        before, q_out = layer_arrays(cache, 0), torch.full((28, 4, 64), 3.0, device=G.DEV)
        B.qllm_kv_rotate_append(cache, 0, q, q_out, k, v, rot, batch)
        assert B.qllm_poll_status() == B.QLLM_ERR_PAGE
        pos = positions(lens, start)
        present = ~((np.repeat([0, 1, 2], news) == 0) & (pos >= 16))
        check(cache, 0, before, q, k, v, q_out, t, lens, start, rot.table, 64, False, present)
    cache = random_cache(7, 1, 9, 2, page, 64)
    before = layer_arrays(cache, 0)
    cut = [20, 3 * page, 5]                                  # the table is three pages wide
    full = table.copy()
    full[1] = [p for p in range(9) if p not in (table[0, 0], table[0, 1], table[2, 0])][:3]
    batch, start = batch_of(full, [20, 10 ** 6, 5], news)
    q_out = torch.empty(28, 4, 64, device=G.DEV)
    B.qllm_kv_rotate_append(cache, 0, q, q_out, k, v, rot, batch)
    assert B.qllm_poll_status() == B.QLLM_ERR_PAGE
    check(cache, 0, before, q, k, v, q_out, full, cut, start, rot.table, 64, False)


def test_nan_and_infinity_stay_in_their_rows():
    lens = news = [8]
    table = make_table(np.random.RandomState(4), lens, 16, 2)
    cache = random_cache(8, 1, 2, 2, 16, 64)
    batch, start = batch_of(table, lens, news)
    q, k, v = (t.clone() for t in qkv_rows(6, 8, 2, 2, 64, "f32"))
    q[1, 0, 3], k[2, 1, 5], k[3, 0, 60], v[4, 0, 7] = float("inf"), float("nan"), float("inf"), float("nan")
    q_out, k2, v2 = (torch.empty_like(t) for t in (q, k, v))
    B.qllm_kv_rotate_append(cache, 0, q, q_out, k, v, B.Rotary.make(8, 64), batch)
    B.qllm_kv_read(cache, 0, k2, v2, batch)
    assert not k2[2, 1].isfinite().any() and not k2[3, 0].isfinite().any() and not v2[4, 0].isfinite().any()
    bad = torch.zeros(8, 2, dtype=torch.bool, device=G.DEV)
    bad[2, 1] = bad[3, 0] = True
    assert k2[~bad].isfinite().all() and q_out[1, 0, [3, 35]].isfinite().sum() == 0 and q_out.isfinite().sum() == q_out.numel() - 2
    bad.zero_(); bad[4, 0] = True
    assert v2[~bad].isfinite().all()


@pytest.mark.parametrize("positions_,rot_dim,base,divisor", [(1, 16, 10000.0, 1.0), (5000, 128, 10000.0, 1.0), (200000, 64, 500000.0, 1.0), (3000, 48, 10000.0, 8.0)])
def test_table(positions_, rot_dim, base, divisor):
    """Half a step of float32, and what 64 bits lose: three roundings of the angle (2^-52 of up to 2^18 each)."""
    t = G.Guarded((positions_, rot_dim // 2, 2), torch.float32, 3.0)
    B.qllm_rotary_table(t.t, base, divisor)
    torch.cuda.synchronize()
    t.check()
    p = np.arange(rot_dim // 2, dtype=np.float64)
    angle = np.arange(positions_, dtype=np.float64)[:, None] / divisor * base ** (-2 * p / rot_dim)[None]
    got = t.t.cpu().numpy()
    for i, want in ((0, np.cos(angle)), (1, np.sin(angle))):
        assert (np.abs(got[..., i] - want) <= 2.0 ** -24 * np.abs(want) + 4 * 2.0 ** -52 * (1 + angle)).all()


def test_scores_depend_on_distance_only():
    """The formula: the product of a turned query and a turned key is that of the unturned ones at the angle of their distance."""
    d, n = 64, 50
    rot = B.Rotary.make(n, d)
    cache, batch = B.KvCache.empty(1, 4, 1, 16, d), B.KvBatch(ints([[0, 1, 2, 3]]), ints([n]), ints([0, n]), n, n)
    q = torch.randn(1, 1, d, device=G.DEV).expand(n, 1, d).contiguous()
    out = torch.empty_like(q)
    B.qllm_kv_rotate_append(cache, 0, q, out, q, q, rot, batch)
    s = (out[:, 0].double() @ out[:, 0].double().T).cpu()
    for dist in (1, 7, 30):
        along = torch.diagonal(s, dist)
        assert ((along - along[0]).abs() <= 64 * 8 * 2.0 ** -24 * float((q[0] ** 2).sum())).all()    # eight roundings a product


def test_stream_and_graph():
    """Two captured decode steps replayed on two streams at once: each follows its batch's lengths."""
    heads, q_heads, d, page = 4, 8, 128, 16
    rot, sides = B.Rotary.make(200, d), []
    for i in range(2):
        lens = [1, 100, 37]
        table = make_table(np.random.RandomState(i), [200, 200, 200], page, 45)
        cache = random_cache(i, 1, 45, heads, page, d)
        batch, start = batch_of(table, lens, [1, 1, 1])
        q, k, v = (t.clone() for t in qkv_rows(i, 3, q_heads, heads, d, "bf16"))
        q_out, st = torch.empty_like(q), torch.cuda.Stream()
        torch.cuda.synchronize()

        def step():
            B.qllm_kv_rotate_append(cache, 0, q, q_out, k, v, rot, batch, stream=st)
        with torch.cuda.stream(st):
            step()
        st.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            step()
        sides.append((table, cache, batch, start, q, k, v, q_out, st, g))
    for lens in ([1, 200, 17], [16, 64, 199]):
        befores = []
        for table, cache, batch, start, q, k, v, q_out, st, g in sides:
            batch.seq_lens.copy_(ints(lens))
            q.normal_(); k.normal_(); v.normal_()
            befores.append(layer_arrays(cache, 0))
        torch.cuda.synchronize()
        for side in sides:
            with torch.cuda.stream(side[8]):
                side[9].replay()
        torch.cuda.synchronize()
        for before, (table, cache, batch, start, q, k, v, q_out, st, g) in zip(befores, sides):
            check(cache, 0, before, q, k, v, q_out, table, lens, start, rot.table, d, False)


def test_offsets_beyond_32_bits():
    """A layer behind 4.3 GB of codes and positions far into a long table."""
    heads, d, page = 8, 128, 256
    pages = 33000                                            # a layer: 4.3 GB of key codes
    cache = B.KvCache(*(torch.empty(2, pages, heads, page, w, dtype=t, device=G.DEV) for w, t in ((d // 2, torch.uint8), (2, torch.float32)) * 2))
    lens, table = [page * 3 - 1], np.array([[pages - 1, 0, pages - 2]])
    batch, start = batch_of(table, lens, [4])
    q, k, v = qkv_rows(1, 4, 8, heads, d, "bf16")
    q_out, k2, v2 = torch.empty(4, 8, d, device=G.DEV, dtype=torch.bfloat16), torch.empty_like(k), torch.empty_like(v)
    rot = B.Rotary.make(lens[0], d)
    B.qllm_kv_rotate_append(cache, 1, q, q_out, k, v, rot, batch)
    pos = positions(lens, start)
    cs = f32(rot.table)[pos]
    codes, scale, zero = kv_ref.quantize(block_ref.turned(f32(k), cs[..., 0], cs[..., 1], d, False))
    at = ints(pos % page).long()
    assert np.array_equal(cache.k_codes[1, pages - 2][:, at].transpose(0, 1).cpu().numpy(), codes)
    assert np.array_equal(cache.k_param[1, pages - 2][:, at].transpose(0, 1).cpu().numpy()[..., 0], scale)


def test_wrong_tensors_are_refused():
    cache = random_cache(1, 1, 4, 2, 16, 64)
    batch, _ = batch_of(np.array([[0, 1]]), [20], [3])
    q, k, v = (t.clone() for t in qkv_rows(1, 3, 4, 2, 64, "f32"))
    rot, o = B.Rotary.make(32, 64), torch.empty(3, 4, 64, device=G.DEV)
    before = B.qllm_launch_count()
    for fn, e in [(lambda: B.qllm_kv_rotate_append(cache, 0, q, o[:2], k, v, rot, batch), "SHAPE"), (lambda: B.qllm_kv_rotate_append(cache, 0, q, None, k, v, rot, batch), "SHAPE"),
                  (lambda: B.qllm_kv_rotate_append(cache, 0, q.bfloat16(), o, k, v, rot, batch), "SHAPE"), (lambda: B.qllm_kv_rotate_append(cache, 0, q, o, k[:, :1], v, rot, batch), "SHAPE"),
                  (lambda: B.qllm_kv_rotate_append(cache, 0, q.half(), o.half(), k.half(), v.half(), rot, batch), "DTYPE"),
                  (lambda: B.Rotary(rot.table.double()), "DTYPE"), (lambda: B.Rotary(rot.table[:, :, 0]), "SHAPE"), (lambda: B.Rotary.make(10, 24), "UNSUPPORTED")]:
        with pytest.raises(B.QllmError) as ei:
            fn()
        assert ei.value.status == getattr(B, "QLLM_ERR_" + e)
    for fn in (lambda: B.qllm_kv_rotate_append(cache, 0, q.cpu(), o, k, v, rot, batch), lambda: B.Rotary(rot.table[:, ::2])):
        with pytest.raises(AssertionError):
            fn()
    assert B.qllm_launch_count() == before
