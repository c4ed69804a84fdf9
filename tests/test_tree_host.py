"""What the tree calls refuse.  Nothing reaches a GPU; addresses are made up and every
check fails first."""

import ctypes as C

import pytest
import torch

import paper_2608_01821_amd as dv

EINVAL, ESHAPE, EDTYPE, ENOMEM = -1, -2, -3, -4
A = 1 << 20
i32 = lambda v: None if v is None else (C.c_int32 * len(v))(*v)


def _plan(n=2, cu=(0, 3, 5), kv=(10, 5), first=None, parent=A, pos=A << 1, mask=A << 2):
    return dv.raw().davet_tree_plan(n, i32(cu), i32(kv), i32(first), parent, pos, mask,
                                    None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), ESHAPE), (dict(n=65), ESHAPE), (dict(cu=None), EINVAL),
    (dict(kv=None), EINVAL), (dict(cu=(1, 3, 5)), ESHAPE), (dict(cu=(0, 5, 3)), ESHAPE),
    (dict(cu=(0, 257, 258), kv=(300, 300)), ESHAPE), (dict(kv=(2, 5)), ESHAPE),
    (dict(first=(2 ** 31 - 200, 0)), ESHAPE), (dict(parent=None), EINVAL),
    (dict(pos=None, mask=None), EINVAL), (dict(parent=A + 2), EINVAL),
    (dict(pos=A + 2), EINVAL), (dict(mask=A + 2), EINVAL),
])
def test_plan_refusals(kw, status):
    assert _plan(**kw) == status


def test_nothing_to_plan():
    assert _plan(cu=(0, 0, 0), parent=None, pos=None, mask=None) == 0


def _attend(cu=(0, 3), kv=(10,), heads=4, scale=0.0, mask=A << 5, q=A << 1, ldq=256,
            out=A << 2, ldo=256, lse=None, ws=A << 3, nb=1 << 30, **cache):
    f = dict(k=A, v=A << 4, page_table=A << 6, max_pages=8, n_pages=32, page_size=64,
             n_kv_heads=2, head_dim=64, dtype=dv.DAVET_F16)
    f.update(cache)
    c = dv.KvCacheT(*f.values())
    return dv.raw().davet_cache_tree_attention(
        C.byref(c), len(kv), i32(cu), i32(kv), q, ldq, heads, scale, mask, out, ldo, lse,
        ws, nb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(mask=None), EINVAL), (dict(mask=A + 2), EINVAL),
    (dict(cu=(0, 257), kv=(300,)), ESHAPE), (dict(cu=(0, 11)), ESHAPE),
    (dict(kv=(513,)), ESHAPE), (dict(heads=3), ESHAPE), (dict(ldq=248), ESHAPE),
    (dict(ldo=260), EINVAL), (dict(q=None), EINVAL), (dict(q=A + 8), EINVAL),
    (dict(out=A << 1), EINVAL), (dict(lse=A + 2), EINVAL), (dict(scale=-1.0), EINVAL),
    (dict(ws=None), ENOMEM), (dict(ws=A + 16), ENOMEM), (dict(nb=1000), ENOMEM),
    (dict(dtype=5), EDTYPE), (dict(v=None), EINVAL), (dict(page_size=24), ESHAPE),
    (dict(head_dim=96), ESHAPE),
])
def test_attention_refusals(kw, status):
    assert _attend(**kw) == status
    if status == ENOMEM:
        assert "davet_cache_tree_attention" in dv.raw().davet_last_error().decode()


def test_no_rows_is_fine():
    assert _attend(cu=(0, 0), mask=None, q=None, out=None, ws=None) == 0


def test_binding_refusals():
    k = torch.zeros(4, 2, 16, 64, dtype=torch.float16)
    c = dv.KvCache(k, k, torch.zeros(2, 3, dtype=torch.int32), dv.DAVET_F16)
    q = torch.zeros(3, 256, dtype=torch.float16)
    I, F = torch.zeros(3, 8, dtype=torch.int32), torch.zeros(3, 8)
    p = torch.zeros(3, dtype=torch.int32)
    for call in (lambda: dv.davet_tree_plan([0, 3], [3], F[:, 0].contiguous(), pos=p),
                 lambda: dv.davet_tree_plan([0, 3], [3], p, pos=F),
                 lambda: dv.davet_tree_plan([0, 3], [3], p, mask=F),
                 lambda: dv.davet_cache_tree_attention(c, [0, 3], [3], q, 4, F, q),
                 lambda: dv.davet_cache_tree_attention(c, [0, 3], [3], q, 4, I, q,
                                                       lse=I)):
        with pytest.raises(ValueError, match="is of torch"):
            call()
    for call in (lambda: dv.davet_tree_plan([0, 3], [3, 3], p, pos=p),
                 lambda: dv.davet_tree_plan([0], [], p, pos=p),
                 lambda: dv.davet_tree_plan([0, 3], None, p, pos=p),
                 lambda: dv.davet_tree_plan([0, 3], [3], p, mask=I[:2]),
                 lambda: dv.davet_tree_plan([0, 3], [3], p[:2], pos=p),
                 lambda: dv.davet_cache_tree_attention(c, [0, 3], [3], q, 4, I[:, :4],
                                                       q)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError, match="32-bit"):
        dv.davet_tree_plan([0, 3], [2 ** 32 + 3], p, pos=p)
    with pytest.raises(ValueError, match="32-bit"):
        dv.davet_cache_tree_attention(c, [0, 3], [3], q, 2 ** 32 + 4, I, q)
    with pytest.raises(ValueError, match="on a GPU"):
        dv.davet_tree_plan([0, 3], [3], p, pos=p, mask=I)
