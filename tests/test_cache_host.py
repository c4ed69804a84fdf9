"""Refusals and host arithmetic of the cache and log-probability entry points;
nothing reaches a GPU.  Addresses are made up: every check fails first."""

import ctypes as C

import numpy as np
import pytest
import torch

import paper_2608_01821_amd as dv

EINVAL, ESHAPE, EDTYPE, ENOMEM = -1, -2, -3, -4
A = 1 << 20                                    # an aligned made-up address


def _cache(**kw):
    f = dict(k=A, v=A << 4, page_table=A << 8, max_pages=8, n_pages=32,
             page_size=16, n_kv_heads=2, head_dim=64, dtype=dv.DAVET_F16)
    f.update(kw)
    return dv.KvCacheT(*[f[n] for n, _ in dv.KvCacheT._fields_])


def _i(*v):
    return (C.c_int32 * len(v))(*v)


def _append(cache=None, n=1, cu=(0, 3), kv=(10,), qkv=A << 1, ldx=512, heads=4,
            norm=0, eps=1e-6, theta=1e4, q=A << 2, ldq=256, gq=None, gk=None):
    c = cache if cache is not None else _cache()
    return dv.raw().davet_cache_append(
        C.byref(c), n, _i(*cu) if cu else None, _i(*kv) if kv else None, qkv, ldx,
        heads, None, norm, gq, gk, eps, theta, q, ldq, None)


def _attend(cache=None, n=1, cu=(0, 3), kv=(10,), q=A << 1, ldq=256, heads=4,
            scale=0.0, block=0, out=A << 2, ldo=256, ws=A << 3, nb=1 << 30):
    c = cache if cache is not None else _cache()
    return dv.raw().davet_cache_attention(
        C.byref(c), n, _i(*cu) if cu else None, _i(*kv) if kv else None, q, ldq,
        heads, scale, block, out, ldo, None, ws, nb, None)


def _weigh(cache=None, n=1, cu=(0, 3), kv=(10,), q=A << 1, ldq=256, heads=4,
           scale=0.0, block=0, lse=A << 2, w=A << 5, ldw=16, ws=A << 3, nb=1 << 30):
    c = cache if cache is not None else _cache()
    return dv.raw().davet_cache_weights(
        C.byref(c), n, _i(*cu), _i(*kv), q, ldq, heads, scale, block, lse, None, w,
        ldw, ws, nb, None)


@pytest.mark.parametrize("call", [_append, _attend, _weigh])
def test_cache_and_chunk_are_checked(call):
    for bad, status in [(dict(dtype=7), EDTYPE), (dict(k=None), EINVAL),
                        (dict(page_table=None), EINVAL), (dict(k=A + 8), EINVAL),
                        (dict(head_dim=96), ESHAPE), (dict(page_size=24), ESHAPE),
                        (dict(page_size=8), ESHAPE), (dict(page_size=512), ESHAPE),
                        (dict(n_kv_heads=0), ESHAPE), (dict(n_pages=0), ESHAPE),
                        (dict(max_pages=0), ESHAPE), (dict(n_kv_heads=3), ESHAPE)]:
        assert call(cache=_cache(**bad)) == status, bad
    for kw, status in [(dict(n=0), ESHAPE), (dict(n=65), ESHAPE),
                       (dict(cu=(1, 3)), ESHAPE), (dict(cu=(0, -1)), ESHAPE),
                       (dict(kv=(2,)), ESHAPE), (dict(kv=(129,)), ESHAPE),
                       (dict(heads=0), ESHAPE), (dict(heads=5), ESHAPE),
                       (dict(heads=2048), ESHAPE)]:
        assert call(**kw) == status, kw
    assert b"" != dv.raw().davet_last_error()


def test_append_refusals():
    assert _append(cache=_cache(v=None)) == EINVAL
    assert _append(cu=None) == EINVAL and _append(kv=None) == EINVAL
    assert _append(qkv=None) == EINVAL and _append(qkv=A + 2) == EINVAL
    assert _append(ldx=511) == EINVAL and _append(ldx=504) == ESHAPE
    assert _append(q=None) == EINVAL and _append(ldq=248) == ESHAPE
    assert _append(norm=2) == EINVAL and _append(theta=0.0) == EINVAL
    assert _append(theta=float("inf")) == EINVAL
    assert _append(norm=1, eps=-1.0) == EINVAL
    assert _append(norm=1, gq=A + 4) == EINVAL and _append(gk=A + 8) == EINVAL
    # q_out inside qkv at another stride or place
    assert _append(qkv=A << 1, q=A << 1, ldq=256) == EINVAL
    assert _append(qkv=A << 1, q=(A << 1) + 512, ldq=512) == EINVAL
    # no new token: nothing to do, nothing launched
    assert _append(cu=(0, 0), kv=(0,), qkv=None, q=None) == 0


def test_attention_and_weights_refusals():
    assert _attend(cache=_cache(v=None)) == EINVAL
    for kw in (dict(scale=-1.0), dict(scale=float("nan")), dict(block=-1),
               dict(scale=1e-38), dict(scale=float("inf")),
               dict(q=None), dict(out=None), dict(q=A + 8), dict(ldq=260),
               dict(out=A << 1)):
        assert _attend(**kw) == EINVAL, kw
    assert _attend(ldq=128) == ESHAPE and _attend(ldo=128) == ESHAPE
    need = dv.davet_cache_workspace_bytes(4, 64, 3)
    for kw in (dict(ws=None), dict(ws=A + 64), dict(nb=1000)):
        assert _attend(**kw) == ENOMEM, kw
        assert _weigh(**kw) == ENOMEM, kw
    assert _attend(cu=(0, 0), kv=(5,), q=None, out=None, ws=None) == 0
    assert need > 1000
    assert _weigh(lse=None) == EINVAL and _weigh(w=None) == EINVAL
    assert _weigh(ldw=9) == ESHAPE
    assert _weigh(scale=float("inf")) == EINVAL and _weigh(block=-3) == EINVAL


def test_workspace_bounds_grow():
    """Enough for every chunk up to max_q."""
    for heads, dim in ((1, 64), (32, 128), (1024, 128)):
        last = 0
        for q in (1, 2, 3, 31, 64, 65, 1000, 4096, 4097, 100000):
            b = dv.davet_cache_workspace_bytes(heads, dim, q)
            assert b >= last and b % 256 == 0
            last = b
        assert last <= (1 << 17) * (dim + 2) * 4 + 256
    out = C.c_size_t()
    f = dv.raw().davet_cache_workspace_bytes
    assert f(32, 96, 1, C.byref(out)) == ESHAPE
    assert f(0, 64, 1, C.byref(out)) == ESHAPE
    assert f(4, 64, 0, C.byref(out)) == ESHAPE
    assert f(4, 64, 1, None) == EINVAL


def _select(n=1, ns=(10,), keep=(4,), w=A, ldw=16, first=0, last=0, kept=A << 1,
            ldk=8, out=A << 2, ldo=8):
    return dv.raw().davet_evict_select(n, _i(*ns), _i(*keep), w, ldw, first, last,
                                       kept, ldk, out, ldo, None)


def test_select_and_gather_refusals():
    for kw in (dict(n=0), dict(n=65), dict(ns=(-1,)), dict(keep=(11,)),
               dict(keep=(-1,)), dict(first=3, last=2), dict(ldw=9), dict(ldk=3),
               dict(ldo=3)):
        assert _select(**kw) == ESHAPE, kw
    for kw in (dict(w=None), dict(kept=None), dict(first=-1), dict(last=-1),
               dict(out=A)):
        assert _select(**kw) == EINVAL, kw
    assert _select(keep=(0,), first=9, last=9) == 0      # nothing stays

    def gather(cache=None, n=1, keep=(4,), kept=A << 1, ldk=8, dst=A << 2, mp=2):
        c = cache if cache is not None else _cache()
        return dv.raw().davet_cache_gather(C.byref(c), n, _i(*keep), kept, ldk,
                                           dst, mp, None)
    assert gather(cache=_cache(v=None)) == EINVAL
    assert gather(cache=_cache(page_size=20)) == ESHAPE
    assert gather(kept=None) == EINVAL and gather(dst=None) == EINVAL
    assert gather(n=0) == ESHAPE and gather(keep=(9,)) == ESHAPE
    assert gather(keep=(-1,)) == ESHAPE
    assert gather(keep=(40,), ldk=64, mp=2) == ESHAPE
    assert gather(keep=(0,)) == 0


def test_logprobs_refusals():
    def f(rows=2, vocab=100, x=A, dt=dv.DAVET_F16, ld=100, tgt=A, lp=A, top=2,
          tl=A, ti=A, ws=A, nb=1 << 20):
        return dv.raw().davet_token_logprobs(rows, vocab, x, dt, ld, -1, tgt, lp,
                                             None, top, tl, ti, ws, nb, None)
    assert f(dt=9) == EDTYPE
    for kw in (dict(rows=-1), dict(vocab=0), dict(ld=99), dict(top=65),
               dict(top=-1)):
        assert f(**kw) == ESHAPE, kw
    for kw in (dict(x=None), dict(tgt=None), dict(tl=None), dict(ti=None),
               dict(x=A + 1)):
        assert f(**kw) == EINVAL, kw
    assert f(vocab=50000, ld=50000, ws=None) == ENOMEM
    assert f(vocab=50000, ld=50000, nb=10) == ENOMEM
    assert f(vocab=50000, ld=50000, ws=A + 8) == ENOMEM
    assert f(rows=0) == 0
    assert dv.davet_logprobs_workspace_bytes(2, 100, 5) == 0
    assert dv.davet_logprobs_workspace_bytes(2, 126464, 5) > 0
    assert dv.davet_logprobs_workspace_bytes(4096, 126464, 5) == 0


def test_binding_checks_sizes():
    """Tensors that are too small, overlapping or of another width are refused
    before their addresses are taken."""
    k = torch.zeros(4, 2, 16, 64, dtype=torch.float16)
    table = torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(ValueError):
        dv.KvCache(k, k[:2], table, dv.DAVET_F16)
    with pytest.raises(ValueError):
        dv.KvCache(k, k, table, dv.DAVET_F32)
    with pytest.raises(ValueError):
        dv.KvCache(k, k, table.long(), dv.DAVET_F16)
    with pytest.raises(ValueError):
        dv.KvCache(k.transpose(1, 2), k.transpose(1, 2), table, dv.DAVET_F16)
    c = dv.KvCache(k, k, table, dv.DAVET_F16)
    q = torch.zeros(3, 256, dtype=torch.float16)
    small = torch.zeros(2, 256, dtype=torch.float16)
    for args in ((c, [0, 3], [3, 4], q, 4, q), (c, [0, 3], [3], small, 4, q),
                 (c, [0, 3], [3], q, 4, small), (c, [0, 3], [3], q.float(), 4, q),
                 (c, [0, 3], [3], q[:, ::2], 2, q),
                 (c, [0, 1, 1, 1], [3, 3, 3], q, 4, q)):
        with pytest.raises(ValueError):
            dv.davet_cache_attention(*args)
    with pytest.raises(ValueError):
        dv.davet_cache_attention(c, [0, 3], [3], q, 4, q, lse=torch.zeros(11))
    w = torch.zeros(1, 4)
    with pytest.raises(ValueError):
        dv.davet_evict_select([5], [2], w, torch.zeros(1, 4, dtype=torch.int32))
    with pytest.raises(ValueError):
        dv.davet_token_logprobs(torch.zeros(2, 9), dv.DAVET_F32,
                                top_ids=torch.zeros(2, 3, dtype=torch.int32))
    with pytest.raises(ValueError):
        dv.davet_token_logprobs(torch.zeros(2, 9), dv.DAVET_F16)
