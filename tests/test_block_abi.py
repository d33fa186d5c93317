"""Argument checks of the norm, the adapters and the rotating append: status codes before anything is launched (no GPU needed)."""
import ctypes

import numpy as np
import pytest

import block_ref
from paper_2310_08041_b200 import binding as B
from test_kv_abi import BATCHES, CACHES, ONE, batch, cache, err, p

L = B._lib


def norm(x=ONE, res=ONE, dtype=1, M=4, C=64, gamma=ONE, eps=1e-5, ptr=None, src=None, coef=None, bits=8, h=ONE, y=ONE, codes=ONE, s=ONE, z=ONE, r=ONE):
    return L.qllm_rmsnorm_quant(x, res, dtype, M, C, gamma, eps, ptr, src, coef, bits, h, y, codes, s, z, r, None)


@pytest.mark.parametrize("kw,e", [
    (dict(bits=5), "BITS"), (dict(bits=0), "BITS"), (dict(dtype=2), "DTYPE"), (dict(M=-1), "SHAPE"), (dict(C=0), "SHAPE"), (dict(C=63, bits=4), "SHAPE"),
    (dict(eps=-1e-9), "SHAPE"), (dict(eps=float("nan")), "SHAPE"), (dict(eps=float("inf")), "SHAPE"), (dict(C=49153), "UNSUPPORTED"), (dict(x=None), "NULL"),
    (dict(gamma=None), "NULL"), (dict(s=None), "NULL"), (dict(z=None), "NULL"), (dict(ptr=ONE), "NULL"), (dict(ptr=ONE, src=ONE), "NULL"),
    (dict(codes=None, h=None, y=None), "NULL"), (dict(codes=None, ptr=ONE, src=ONE, coef=ONE), "NULL"), (dict(x=8), "ALIGN"), (dict(res=4), "ALIGN"),
    (dict(h=8), "ALIGN"), (dict(y=8), "ALIGN"), (dict(codes=1), "ALIGN")])
def test_norm_refused(kw, e):
    assert norm(**kw) == err(e)


def test_norm_without_rows_is_fine():
    assert norm(M=0, x=None, codes=None, h=None, y=None) == B.QLLM_OK


def deq(codes=ONE, s=ONE, z=ONE, M=4, C=64, bits=8, out=ONE, dtype=1):
    return L.qllm_dequantize_rows(codes, s, z, M, C, bits, out, dtype, None)


@pytest.mark.parametrize("kw,e", [(dict(bits=7), "BITS"), (dict(dtype=-1), "DTYPE"), (dict(M=-1), "SHAPE"), (dict(C=0), "SHAPE"), (dict(C=7, bits=4), "SHAPE"),
                                  (dict(codes=None), "NULL"), (dict(s=None), "NULL"), (dict(z=None), "NULL"), (dict(out=None), "NULL"), (dict(codes=8), "ALIGN"),
                                  (dict(out=8), "ALIGN")])
def test_dequantize_refused(kw, e):
    assert deq(**kw) == err(e)
    assert deq(M=0, codes=None) == B.QLLM_OK


def add(x=ONE, xs=256, base=ONE, bs=512, out=ONE, os=512, dtype=1, start=ONE, adapter=ONE, seqs=3, rows=7, **kw):
    d = dict(A=ONE, B=ONE, scale=ONE, rank=ONE, slots=4, max_rank=16, K=256, N=512)
    d.update(kw)
    a = B._AdaptersStruct(*[d[n] for n, _ in B._AdaptersStruct._fields_])
    return L.qllm_adapters_add(p(a), x, xs, base, bs, out, os, dtype, start, adapter, seqs, rows, None)


@pytest.mark.parametrize("kw,e", [
    (dict(dtype=3), "DTYPE"), (dict(slots=0), "SHAPE"), (dict(max_rank=0), "SHAPE"), (dict(K=0), "SHAPE"), (dict(N=-8), "SHAPE"), (dict(seqs=-1), "SHAPE"),
    (dict(rows=-1), "SHAPE"), (dict(slots=8193), "UNSUPPORTED"), (dict(max_rank=136), "UNSUPPORTED"), (dict(max_rank=12), "UNSUPPORTED"),
    (dict(K=252), "UNSUPPORTED"), (dict(N=508), "UNSUPPORTED"), (dict(seqs=(1 << 20) + 1), "UNSUPPORTED"), (dict(rows=(1 << 30) + 1), "UNSUPPORTED"),
    (dict(A=None), "NULL"), (dict(B=None), "NULL"), (dict(scale=None), "NULL"), (dict(x=None), "NULL"), (dict(out=None), "NULL"), (dict(start=None), "NULL"),
    (dict(adapter=None), "NULL"), (dict(A=8), "ALIGN"), (dict(B=8), "ALIGN"), (dict(x=8), "ALIGN"), (dict(base=8), "ALIGN"), (dict(out=24), "ALIGN"),
    (dict(xs=255), "SHAPE"), (dict(bs=511), "SHAPE"), (dict(os=504), "SHAPE"), (dict(xs=260), "ALIGN"), (dict(bs=516, base=32), "ALIGN"), (dict(os=516), "ALIGN"),
    (dict(xs=258, dtype=0), "ALIGN"), (dict(K=(1 << 20) + 8, xs=1 << 21), "UNSUPPORTED"),
    (dict(N=(1 << 20) + 8, bs=1 << 21, os=1 << 21), "UNSUPPORTED"), (dict(os=520), "SHAPE")])
def test_adapters_refused(kw, e):
    """(the last one: base is out, with another stride)"""
    assert add(**kw) == err(e)


def test_adapters_without_rows_are_fine():
    assert add(rows=0, x=None) == B.QLLM_OK and add(seqs=0, start=None) == B.QLLM_OK
    assert L.qllm_adapters_add(None, ONE, 8, ONE, 8, ONE, 8, 1, ONE, ONE, 1, 1, None) == B.QLLM_ERR_NULL


def rotate(c=None, b=None, layer=0, q=ONE, qs=1024, o=ONE, os=1024, heads=8, k=ONE, ks=512, v=ONE, vs=512, dtype=1, rot=True, **kw):
    d = dict(table=ONE, positions=100, rot_dim=128, interleaved=0)
    d.update(kw)
    r, c, b = B._RotaryStruct(*[d[n] for n, _ in B._RotaryStruct._fields_]), c or cache(), b or batch()
    return L.qllm_kv_rotate_append(p(c), layer, q, qs, o, os, heads, k, ks, v, vs, dtype, p(r) if rot else None, p(b), None)


@pytest.mark.parametrize("kw,e", [
    (dict(dtype=2), "DTYPE"), (dict(layer=2), "SHAPE"), (dict(layer=-1), "SHAPE"), (dict(heads=-1), "SHAPE"), (dict(heads=8193, qs=1 << 21, os=1 << 21), "UNSUPPORTED"),
    (dict(rot=False), "NULL"), (dict(table=None), "NULL"), (dict(table=8), "ALIGN"), (dict(positions=0), "SHAPE"), (dict(rot_dim=0), "SHAPE"),
    (dict(rot_dim=144), "SHAPE"), (dict(rot_dim=24), "UNSUPPORTED"), (dict(rot_dim=8), "UNSUPPORTED"), (dict(q=None), "NULL"), (dict(o=None), "NULL"),
    (dict(k=None), "NULL"), (dict(v=None), "NULL"), (dict(qs=1016), "SHAPE"), (dict(os=1023), "SHAPE"), (dict(ks=511), "SHAPE"), (dict(vs=500), "SHAPE"),
    (dict(q=8), "ALIGN"), (dict(o=24), "ALIGN"), (dict(qs=1028, o=32), "ALIGN"), (dict(ks=516), "ALIGN"), (dict(os=1032), "SHAPE")])
def test_rotate_refused(kw, e):
    """(the last one: queries in place with another stride)"""
    assert rotate(**kw) == err(e)


@pytest.mark.parametrize("kw,e", CACHES)
def test_rotate_refuses_caches(kw, e):
    assert rotate(c=cache(**kw)) == err(e)


@pytest.mark.parametrize("kw,e", BATCHES)
def test_rotate_refuses_batches(kw, e):
    assert rotate(b=batch(**kw)) == err(e)


def test_rotate_without_rows_is_fine():
    assert rotate(b=batch(rows=0), q=None) == B.QLLM_OK and rotate(b=batch(seqs=0, table=None), k=None) == B.QLLM_OK


@pytest.mark.parametrize("kw,e", [(dict(base=0.0), "SHAPE"), (dict(base=float("nan")), "SHAPE"), (dict(div=0.0), "SHAPE"), (dict(div=float("inf")), "SHAPE"),
                                  (dict(pos=0), "SHAPE"), (dict(rot=-16), "SHAPE"), (dict(rot=40), "UNSUPPORTED"), (dict(rot=272), "UNSUPPORTED"),
                                  (dict(table=None), "NULL"), (dict(table=4), "ALIGN")])
def test_table_refused(kw, e):
    d = dict(table=ONE, pos=10, rot=64, base=1e4, div=1.0)
    d.update(kw)
    assert L.qllm_rotary_table(d["table"], d["pos"], d["rot"], ctypes.c_double(d["base"]), ctypes.c_double(d["div"]), None) == err(e)


def test_reference_norm_by_hand():
    x, g = np.array([[3.0, -4.0]], np.float32), np.array([1.0, 2.0], np.float32)
    h, y, f, codes, zero, alpha, u = block_ref.norm(x, np.array([[0.0, 0.0]], np.float32), g, 0.0, None, 4)
    assert np.allclose(f, 1 / np.sqrt(12.5)) and np.allclose(y, [[3 / np.sqrt(12.5), -8 / np.sqrt(12.5)]])
    assert codes.tolist() == [[15.0, 0.0]] and zero.item() == 11 and np.isclose(alpha.item(), 11 / 15)


def test_reference_rotation_by_hand():
    x = np.arange(1.0, 5.0).reshape(1, 1, 4)
    quarter = (np.zeros((1, 2)), np.ones((1, 2)))
    assert block_ref.turned(x, *quarter, 4, False).tolist() == [[[-3, -4, 1, 2]]]
    assert block_ref.turned(x, *quarter, 4, True).tolist() == [[[-2, 1, -4, 3]]]
    assert block_ref.turned(x, quarter[0][:, :1], quarter[1][:, :1], 2, False).tolist() == [[[-2, 1, 3, 4]]]


def test_reference_map_is_one():
    ptr, src, coef = block_ref.random_map(np.random.RandomState(1), 1200)
    assert B.qllm_validate_map(ptr, src, 1200) == B.QLLM_OK and len(np.diff(ptr)) == 1200 and (np.diff(ptr) > 4).any() and (np.diff(ptr) == 2).any()
    assert np.isclose(coef[(np.diff(ptr) > 1).repeat(np.diff(ptr))].sum(), (np.diff(ptr) > 1).sum())
