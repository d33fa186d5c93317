"""Argument checks of the 4-bit key/value cache's entry points: status codes before anything is launched (no GPU needed)."""
import ctypes

import numpy as np
import pytest

import kv_ref
from paper_2310_08041_b200 import binding as B

ONE = 16            # not null, 16-byte aligned; never dereferenced on these paths
L = B._lib


def cache(**kw):
    d = dict(k_codes=ONE, k_param=ONE, v_codes=ONE, v_param=ONE, layers=2, pages=10, kv_heads=4, page_size=64, head_dim=128)
    d.update(kw)
    return B._KvCacheStruct(*[d[n] for n, _ in B._KvCacheStruct._fields_])


def batch(**kw):
    d = dict(table=ONE, seq_lens=ONE, q_start=ONE, seqs=3, table_width=5, rows=7, max_new=4)
    d.update(kw)
    return B._KvBatchStruct(*[d[n] for n, _ in B._KvBatchStruct._fields_])


def pool(**kw):
    d = dict(refs=ONE, table=ONE, seq_lens=ONE, pages=10, seqs=3, table_width=5)
    d.update(kw)
    return B._KvPoolStruct(*[d[n] for n, _ in B._KvPoolStruct._fields_])


def p(s):
    return None if s is None else ctypes.addressof(s)


def tokens(fn, c, b, layer=0, k=ONE, ks=512, v=ONE, vs=512, dtype=1):
    return fn(p(c), layer, k, ks, v, vs, dtype, p(b), None)


def attention(c, b, layer=0, q=ONE, qs=1024, out=ONE, os=1024, dtype=1, heads=8, scale=0.1, lse=None, ws=ONE, bytes_=1 << 40):
    return L.qllm_kv_attention(p(c), layer, q, qs, out, os, dtype, heads, scale, 1, lse, p(b), ws, bytes_, None)


CACHES = [(dict(layers=0), "SHAPE"), (dict(pages=0), "SHAPE"), (dict(kv_heads=-1), "SHAPE"), (dict(page_size=48), "UNSUPPORTED"),
          (dict(page_size=8), "UNSUPPORTED"), (dict(page_size=512), "UNSUPPORTED"), (dict(head_dim=96), "UNSUPPORTED"), (dict(kv_heads=1025), "UNSUPPORTED"),
          (dict(head_dim=0), "SHAPE"), (dict(k_codes=None), "NULL"), (dict(v_param=None), "NULL"), (dict(v_codes=8), "ALIGN"),
          (dict(k_param=4), "ALIGN")]
BATCHES = [(dict(seqs=-1), "SHAPE"), (dict(table_width=0), "SHAPE"), (dict(rows=-1), "SHAPE"), (dict(max_new=-1), "SHAPE"),
           (dict(rows=(1 << 30) + 1), "UNSUPPORTED"), (dict(seqs=(1 << 20) + 1), "UNSUPPORTED"), (dict(table=None), "NULL"),
           (dict(seq_lens=None), "NULL"), (dict(q_start=None), "NULL")]


def err(name):
    return getattr(B, "QLLM_ERR_" + name)


@pytest.mark.parametrize("kw,e", CACHES)
def test_caches_refused(kw, e):
    c = cache(**kw)
    for fn in (L.qllm_kv_append, L.qllm_kv_read):
        assert tokens(fn, c, batch()) == err(e)
    assert attention(c, batch()) == err(e)
    assert L.qllm_kv_attention_workspace(p(c), 8, 1, p(batch())) == err(e)
    assert L.qllm_kv_pages_extend(p(c), p(pool()), ONE, None) == err(e)
    assert L.qllm_kv_pages_fork(p(c), p(pool()), ONE, ONE, 2, ONE, None) == err(e)
    assert L.qllm_kv_pages_compact(p(c), p(pool()), ONE, None) == err(e)
    assert L.qllm_kv_pages_copy(p(c), ONE, ONE, 2, None) == err(e)


@pytest.mark.parametrize("kw,e", BATCHES)
def test_batches_refused(kw, e):
    b = batch(**kw)
    for fn in (L.qllm_kv_append, L.qllm_kv_read):
        assert tokens(fn, cache(), b) == err(e)
    assert attention(cache(), b) == err(e)
    assert L.qllm_kv_attention_workspace(p(cache()), 8, 1, p(b)) == err(e)


def test_positions_counted_in_30_bits():
    b = batch(table_width=(1 << 22) + 1)
    c = cache(page_size=256)
    for fn in (L.qllm_kv_append, L.qllm_kv_read):
        assert tokens(fn, c, b) == B.QLLM_ERR_UNSUPPORTED
    assert attention(c, b) == B.QLLM_ERR_UNSUPPORTED
    assert L.qllm_kv_pages_extend(p(c), p(pool(table_width=(1 << 22) + 1)), ONE, None) == B.QLLM_ERR_UNSUPPORTED
    assert attention(cache(), batch(rows=1 << 29)) == B.QLLM_ERR_UNSUPPORTED          # query rows in 31 bits


def test_tensors_refused():
    for fn in (L.qllm_kv_append, L.qllm_kv_read):
        assert tokens(fn, cache(), batch(), dtype=2) == B.QLLM_ERR_DTYPE
        assert tokens(fn, None, batch()) == B.QLLM_ERR_NULL
        assert tokens(fn, cache(), None) == B.QLLM_ERR_NULL
        assert tokens(fn, cache(), batch(), layer=2) == B.QLLM_ERR_SHAPE
        assert tokens(fn, cache(), batch(), layer=-1) == B.QLLM_ERR_SHAPE
        assert tokens(fn, cache(), batch(), k=None) == B.QLLM_ERR_NULL
        assert tokens(fn, cache(), batch(), v=None) == B.QLLM_ERR_NULL
        assert tokens(fn, cache(), batch(), v=24) == B.QLLM_ERR_ALIGN
        assert tokens(fn, cache(), batch(), ks=511) == B.QLLM_ERR_SHAPE
        assert tokens(fn, cache(), batch(), ks=516) == B.QLLM_ERR_ALIGN
        assert tokens(fn, cache(), batch(), vs=514, dtype=0) == B.QLLM_ERR_ALIGN
        assert tokens(fn, cache(), batch(rows=0), k=None) == B.QLLM_OK
        assert tokens(fn, cache(), batch(seqs=0, table=None), k=None) == B.QLLM_OK
    assert attention(cache(), batch(), dtype=-1) == B.QLLM_ERR_DTYPE
    assert attention(cache(), batch(), heads=6) == B.QLLM_ERR_SHAPE
    assert attention(cache(), batch(), heads=0) == B.QLLM_ERR_SHAPE
    assert attention(cache(), batch(), layer=5) == B.QLLM_ERR_SHAPE
    assert attention(cache(), batch(), scale=float("nan")) == B.QLLM_ERR_SHAPE
    assert attention(cache(), batch(), scale=float("inf")) == B.QLLM_ERR_SHAPE
    assert attention(cache(), batch(), q=None) == B.QLLM_ERR_NULL
    assert attention(cache(), batch(), out=None) == B.QLLM_ERR_NULL
    assert attention(cache(), batch(), out=8) == B.QLLM_ERR_ALIGN
    assert attention(cache(), batch(), qs=1000) == B.QLLM_ERR_SHAPE
    assert attention(cache(), batch(), os=1028) == B.QLLM_ERR_ALIGN
    assert attention(cache(), batch(rows=0), q=None) == B.QLLM_OK
    assert attention(None, batch()) == B.QLLM_ERR_NULL


def test_workspace():
    """The size depends on the arguments only (148 SMs are assumed without a device); smaller, missing and unaligned ones are refused."""
    for dtype, b in ((0, batch()), (1, batch()), (1, batch(rows=4000, max_new=2000)), (1, batch(seqs=1, rows=300, max_new=300))):
        n = L.qllm_kv_attention_workspace(p(cache()), 8, dtype, p(b))
        assert n >= 0 and n == L.qllm_kv_attention_workspace(p(cache()), 8, dtype, p(b))
        if n:
            kw = dict(dtype=dtype)
            assert attention(cache(), b, ws=None, **kw) == B.QLLM_ERR_NULL
            assert attention(cache(), b, bytes_=n - 1, **kw) == B.QLLM_ERR_SHAPE
            assert attention(cache(), b, ws=8, **kw) == B.QLLM_ERR_ALIGN
    assert L.qllm_kv_attention_workspace(p(cache()), 8, 1, p(batch(rows=0))) == 0
    assert L.qllm_kv_attention_workspace(p(cache()), 6, 1, p(batch())) == B.QLLM_ERR_SHAPE
    assert B.qllm_status_string(B.QLLM_ERR_PAGE) not in ("ok", "unknown status")


def test_pools_refused():
    for kw, e in [(dict(pages=0), "SHAPE"), (dict(seqs=0), "SHAPE"), (dict(table_width=0), "SHAPE"), (dict(seqs=8193), "UNSUPPORTED"),
                  (dict(refs=None), "NULL"), (dict(table=None), "NULL"), (dict(seq_lens=None), "NULL")]:
        q = pool(**kw)
        assert L.qllm_kv_pages_extend(p(cache()), p(q), ONE, None) == err(e)
        assert L.qllm_kv_pages_fork(p(cache()), p(q), ONE, ONE, 2, ONE, None) == err(e)
        assert L.qllm_kv_pages_free(p(q), ONE, 2, None) == err(e)
        assert L.qllm_kv_pages_compact(p(cache()), p(q), ONE, None) == err(e)
    other = pool(pages=11)
    assert L.qllm_kv_pages_extend(p(cache()), p(other), ONE, None) == B.QLLM_ERR_SHAPE
    assert L.qllm_kv_pages_fork(p(cache()), p(other), ONE, ONE, 2, ONE, None) == B.QLLM_ERR_SHAPE
    assert L.qllm_kv_pages_compact(p(cache()), p(other), ONE, None) == B.QLLM_ERR_SHAPE
    assert L.qllm_kv_pages_extend(p(cache()), None, ONE, None) == B.QLLM_ERR_NULL
    assert L.qllm_kv_pages_extend(p(cache()), p(pool()), None, None) == B.QLLM_ERR_NULL
    for n, e in ((-1, B.QLLM_ERR_SHAPE), (8193, B.QLLM_ERR_UNSUPPORTED), (0, B.QLLM_OK)):
        assert L.qllm_kv_pages_fork(p(cache()), p(pool()), ONE, ONE, n, ONE, None) == e
        assert L.qllm_kv_pages_free(p(pool()), ONE, n, None) == e
    assert L.qllm_kv_pages_fork(p(cache()), p(pool()), ONE, ONE, 2, None, None) == B.QLLM_ERR_NULL
    assert L.qllm_kv_pages_free(p(pool()), None, 2, None) == B.QLLM_ERR_NULL
    assert L.qllm_kv_pages_compact(p(cache()), p(pool()), None, None) == B.QLLM_ERR_NULL
    assert L.qllm_kv_pages_copy(p(cache()), ONE, ONE, -1, None) == B.QLLM_ERR_SHAPE
    assert L.qllm_kv_pages_copy(p(cache()), None, ONE, 1, None) == B.QLLM_ERR_NULL
    assert L.qllm_kv_pages_copy(p(cache()), None, None, 0, None) == B.QLLM_OK


def test_reference_attention_by_hand():
    """The 64-bit statement the GPU tests compare with, on a case small enough to do by hand: two keys with equal scores average
    their values, a row whose keys are all hidden gives zeros."""
    kc = np.zeros((1, 1, 16, 32), np.uint8)
    kp = np.ones((1, 1, 16, 2), np.float32)
    vc = kc.copy()
    vc[0, 0, 0], vc[0, 0, 1] = 0x31, 0x75                    # channels 1, 3, 1, 3 .. and 5, 7, 5, 7 ..
    vp = kp.copy()
    vp[..., 1] = 2.0
    st = kv_ref.Store(kc, kp, vc, vp)
    out, lse, _, _, seen = kv_ref.attention(st, np.array([[0]]), [2], [0, 3], np.ones((3, 1, 64)), 0.5, True)
    assert (out[0] == 0).all() and np.isneginf(lse[0, 0]) and seen[:, 0].tolist() == [0, 1, 2]
    assert np.allclose(out[1, 0, :2], [-1, 1]) and np.allclose(out[2, 0, :2], [1, 3])
    assert np.isclose(lse[2, 0], 0.5 * -64 + np.log(2))


def test_reference_pool_by_hand():
    m = kv_ref.Pool(5, 3, 3, 16)
    m.extend([20, 0, 0])
    assert m.table[0].tolist() == [0, 1, -1] and m.refs.tolist() == [1, 1, 0, 0, 0]
    assert m.fork([0], [2]) == [2] and m.table[2].tolist() == [0, 2, -1] and m.refs.tolist() == [2, 1, 1, 0, 0]
    m.free([0, 0])
    assert m.refs.tolist() == [1, 0, 1, 0, 0] and m.lens.tolist() == [0, 0, 20]
    assert m.compact().tolist() == [0, -1, 1, -1, -1] and m.table[2].tolist() == [0, 1, -1] and m.copies[-1] == (2, 1)
