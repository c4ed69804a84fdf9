"""What the page calls refuse.  Nothing reaches a GPU; addresses are made up and every
check fails first."""

import ctypes as C

import pytest
import torch

import paper_2608_01821_amd as dv

EINVAL, ESHAPE, EDTYPE, ENOMEM = -1, -2, -3, -4
A = 1 << 20
i32 = lambda v: None if v is None else (C.c_int32 * len(v))(*v)


def _cache(**kw):
    f = dict(k=A, v=A << 4, page_table=A << 6, max_pages=1 << 16, n_pages=32,
             page_size=64, n_kv_heads=2, head_dim=64, dtype=dv.DAVET_F16)
    f.update(kw)
    return C.byref(dv.KvCacheT(*f.values()))


def _bounds(cu=(0, 3), kv=(10,), bounds=A << 1, **cache):
    return dv.raw().davet_cache_page_bounds(_cache(**cache), len(kv), i32(cu), i32(kv),
                                            bounds, None)


@pytest.mark.parametrize("kw,status", [
    (dict(bounds=None), EINVAL), (dict(bounds=A + 8), EINVAL), (dict(k=None), EINVAL),
    (dict(cu=(0, 11)), ESHAPE), (dict(cu=(1, 3)), ESHAPE), (dict(dtype=3), EDTYPE),
    (dict(max_pages=0), ESHAPE), (dict(cu=None), EINVAL),
])
def test_bounds_refusals(kw, status):
    assert _bounds(**kw) == status


def test_no_new_tokens_have_no_bounds():
    assert _bounds(cu=(0, 0)) == 0
    assert _bounds(cu=(0, 0), v=None) == 0


def _select(cu=(0, 3), kv=(10,), heads=4, q=A << 1, ldq=256, block=0, bounds=A << 2,
            first=0, last=0, top=4, pages=A << 3, **cache):
    return dv.raw().davet_cache_page_select(
        _cache(**cache), len(kv), i32(cu), i32(kv), q, ldq, heads, block, bounds, first,
        last, top, pages, None)


@pytest.mark.parametrize("kw,status", [
    (dict(top=0), ESHAPE), (dict(top=32769), ESHAPE), (dict(first=3, last=2), ESHAPE),
    (dict(first=2 ** 31 - 1, last=2 ** 31 - 1), ESHAPE), (dict(first=-1), EINVAL),
    (dict(last=-1), EINVAL), (dict(block=-1), EINVAL), (dict(heads=5), ESHAPE),
    (dict(kv=(32768 * 64 + 1,)), ESHAPE), (dict(bounds=None), EINVAL),
    (dict(bounds=A + 4), EINVAL), (dict(pages=None), EINVAL), (dict(pages=A + 2), EINVAL),
    (dict(q=None), EINVAL), (dict(ldq=255), EINVAL), (dict(ldq=248), ESHAPE),
])
def test_select_refusals(kw, status):
    assert _select(**kw) == status


def test_nothing_to_select():
    assert _select(cu=(0, 0), q=None, bounds=None, pages=None) == 0
    # a sequence without new tokens may be as long as it likes
    assert _select(cu=(0, 0), kv=(32768 * 64 + 1,), q=None) == 0


def _attend(cu=(0, 3), kv=(10,), heads=4, scale=0.0, block=0, pages=A << 5, top=4,
            q=A << 1, ldq=256, out=A << 2, ldo=256, lse=None, ws=A << 3, nb=1 << 30,
            **cache):
    return dv.raw().davet_cache_page_attention(
        _cache(**cache), len(kv), i32(cu), i32(kv), q, ldq, heads, scale, block, pages,
        top, out, ldo, lse, ws, nb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(pages=None), EINVAL), (dict(pages=A + 2), EINVAL), (dict(top=0), ESHAPE),
    (dict(top=(1 << 26) + 1), ESHAPE), (dict(block=-1), EINVAL), (dict(heads=3), ESHAPE),
    (dict(cu=(0, 11)), ESHAPE), (dict(out=A << 1), EINVAL), (dict(ws=None), ENOMEM),
    (dict(nb=1000), ENOMEM), (dict(scale=1e31), EINVAL), (dict(lse=A + 2), EINVAL),
    (dict(v=None), EINVAL),
])
def test_attention_refusals(kw, status):
    assert _attend(**kw) == status


def test_binding_refusals():
    k = torch.zeros(4, 2, 16, 64, dtype=torch.float16)
    c = dv.KvCache(k, k, torch.zeros(2, 3, dtype=torch.int32), dv.DAVET_F16)
    q = torch.zeros(3, 256, dtype=torch.float16)
    b = torch.zeros(4, 2, 2, 64, dtype=torch.float16)
    p = torch.zeros(3, 2, 2, dtype=torch.int32)
    one = ([0, 3], [3])
    for call in (lambda: dv.davet_cache_page_bounds(c, *one, b.float()),
                 lambda: dv.davet_cache_page_select(c, *one, q.float(), 4, b, p),
                 lambda: dv.davet_cache_page_select(c, *one, q, 4, b.float(), p),
                 lambda: dv.davet_cache_page_select(c, *one, q, 4, b, p.float()),
                 lambda: dv.davet_cache_page_attention(c, *one, q, 4, p.float(), q)):
        with pytest.raises(ValueError, match="is of torch"):
            call()
    for call in (lambda: dv.davet_cache_page_bounds(c, *one, b[:3]),
                 lambda: dv.davet_cache_page_select(c, *one, q, 4, b, p[:2]),
                 lambda: dv.davet_cache_page_select(c, *one, q, 4, b, p[:, :1]),
                 lambda: dv.davet_cache_page_select(c, *one, q, 4, b, p[0]),
                 lambda: dv.davet_cache_page_attention(c, *one, q, 4, p[:, :, :1], q),
                 lambda: dv.davet_cache_page_attention(c, *one, q, 4, p.view(3, 4), q)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: dv.davet_cache_page_select(c, *one, q, 4, b, p, first=2 ** 32),
                 lambda: dv.davet_cache_page_select(c, *one, q, 4, b, p, last=2 ** 32),
                 lambda: dv.davet_cache_page_select(c, *one, q, 4, b, p, block=2 ** 32),
                 lambda: dv.davet_cache_page_attention(c, *one, q, 4, p, q,
                                                       block=2 ** 32)):
        with pytest.raises(ValueError, match="32-bit"):
            call()
    with pytest.raises(ValueError, match="on a GPU"):
        dv.davet_cache_page_bounds(c, *one, b)
