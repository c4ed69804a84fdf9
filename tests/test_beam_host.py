"""What the beam calls promise and refuse.  Nothing reaches a GPU; addresses are made up
and every check fails first."""

import ctypes as C

import pytest
import torch

import paper_2608_01821_amd as dv

EINVAL, ESHAPE, EDTYPE, ENOMEM = -1, -2, -3, -4
A = 1 << 20
i32 = lambda v: None if v is None else (C.c_int32 * len(v))(*v)


def _select(groups=2, beams=4, vocab=1000, logits=A, dtype=dv.DAVET_F16, ld=1000,
            exclude=-1, scores=A, done=None, pad=0, top=4, osc=A, orow=A, otok=A, ws=A,
            nb=1 << 20):
    return dv.raw().davet_beam_select(groups, beams, vocab, logits, dtype, ld, exclude,
                                      scores, done, pad, top, osc, orow, otok, ws, nb,
                                      None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=4), EDTYPE), (dict(groups=-1), ESHAPE), (dict(beams=0), ESHAPE),
    (dict(beams=65), ESHAPE), (dict(groups=1 << 21), ESHAPE), (dict(vocab=0), ESHAPE),
    (dict(top=0), ESHAPE), (dict(top=65), ESHAPE), (dict(ld=999), ESHAPE),
    (dict(ld=1 << 40), ESHAPE), (dict(logits=None), EINVAL), (dict(scores=None), EINVAL),
    (dict(osc=None), EINVAL), (dict(orow=None), EINVAL), (dict(otok=None), EINVAL),
    (dict(logits=A + 1), EINVAL), (dict(scores=A + 2), EINVAL), (dict(done=A + 2), EINVAL),
    (dict(osc=A + 2), EINVAL), (dict(orow=A + 2), EINVAL), (dict(otok=A + 2), EINVAL),
    (dict(ws=None), ENOMEM), (dict(ws=A + 64), ENOMEM), (dict(nb=255), ENOMEM),
    (dict(top=3), EINVAL), (dict(osc=A + 4), EINVAL), (dict(osc=A - 4), EINVAL),
])
def test_select_refusals(kw, status):
    assert _select(**kw) == status


def test_nothing_to_select():
    assert _select(groups=0, logits=None, scores=None, ws=None) == 0
    assert dv.davet_beam_workspace_bytes(0, 4, 1000, 4) == 0


@pytest.mark.parametrize("top", [1, 8, 64])
@pytest.mark.parametrize("vocab", [300, 32003, 126464, 1 << 24])
def test_a_workspace_for_every_count_of_requests(vocab, top):
    """The header's bound, though fewer requests may need more."""
    most = 0
    for beams in (1, 4, 7):
        for groups in range(1, 300):
            most = dv.davet_beam_workspace_bytes(groups, beams, vocab, top)
            for fewer in (1, groups // 2 or 1, groups):
                need = dv.davet_beam_workspace_bytes(fewer, beams, vocab, top)
                assert need <= (groups * beams + 255) * (8 * top + 12) + 255


def _reorder(kv=(40, 40), parent=A, fresh=A, dst=A << 2, dst_max=8, n=None, **cache):
    f = dict(k=A, v=A << 4, page_table=A << 6, max_pages=8, n_pages=32, page_size=16,
             n_kv_heads=2, head_dim=64, dtype=dv.DAVET_F16)
    f.update(cache)
    return dv.raw().davet_cache_reorder(C.byref(dv.KvCacheT(*f.values())),
                                        len(kv) if n is None else n, i32(kv), parent,
                                        fresh, dst, dst_max, None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), ESHAPE), (dict(n=65, kv=(1,) * 65), ESHAPE), (dict(kv=(-1, 0)), ESHAPE),
    (dict(kv=(129, 1)), ESHAPE), (dict(kv=(40, 40), dst_max=2), ESHAPE),
    (dict(parent=None), EINVAL), (dict(fresh=None), EINVAL), (dict(dst=None), EINVAL),
    (dict(parent=A + 2), EINVAL), (dict(fresh=A + 2), EINVAL), (dict(dst=A + 2), EINVAL),
    (dict(dst=A << 6), EINVAL), (dict(dst=(A << 6) + 60), EINVAL),
    (dict(dst=(A << 6) - 4), EINVAL), (dict(kv=(0, 0), dst_max=-1), ESHAPE),
    (dict(v=None), EINVAL), (dict(dtype=3), EDTYPE),
])
def test_reorder_refusals(kw, status):
    assert _reorder(**kw) == status


def test_binding_refusals():
    x, f = torch.zeros(4, 100), torch.zeros(4)
    o, i = torch.zeros(2, 3), torch.zeros(2, 3, dtype=torch.int32)
    call = dv.davet_beam_select
    for args, kw in (((x.half(), dv.DAVET_F32, f, 2, o, i, i), {}),
                     ((x, dv.DAVET_F32, f.double(), 2, o, i, i), {}),
                     ((x, dv.DAVET_F32, f, 2, i, i, i), {}),
                     ((x, dv.DAVET_F32, f, 2, o, o, i), {}),
                     ((x, dv.DAVET_F32, f, 2, o, i, o), {}),
                     ((x, dv.DAVET_F32, f, 2, o, i, i), dict(done=f))):
        with pytest.raises(ValueError, match="is of torch"):
            call(*args, **kw)
    for args in ((x, dv.DAVET_F32, f, 3, o, i, i), (x, dv.DAVET_F32, f, 0, o, i, i),
                 (x, dv.DAVET_F32, f[:3], 2, o, i, i),
                 (x, dv.DAVET_F32, f, 2, o[:1], i, i),
                 (x, dv.DAVET_F32, f, 2, o, i[:, :2], i),
                 (x, dv.DAVET_F32, f, 1, o, i, i)):
        with pytest.raises(ValueError):
            call(*args)
    for kw in (dict(exclude=2 ** 32), dict(pad=2 ** 32)):
        with pytest.raises(ValueError, match="32-bit"):
            call(x, dv.DAVET_F32, f, 2, o, i, i, **kw)
    with pytest.raises(ValueError, match="on a GPU"):
        call(x, dv.DAVET_F32, f, 2, o, i, i)
    k = torch.zeros(4, 2, 16, 64, dtype=torch.float16)
    t = torch.zeros(2, 3, dtype=torch.int32)
    c, one = dv.KvCache(k, k, t, dv.DAVET_F16), torch.zeros(2, dtype=torch.int32)
    for args in (([1], one, one, t), ([], one, one, t), ([1, 1], one[:1], one, t),
                 ([1, 1], one, one[:1], t), ([1, 1], one, one, t[:1]),
                 ([1, 1], one.float(), one, t), ([1, 1], one, one, t.float()),
                 ([1, 2 ** 32], one, one, t), ([1, 1], one, one, t.clone())):
        with pytest.raises(ValueError):
            dv.davet_cache_reorder(c, *args)
