"""davet_rotary_turns against the formula, and what the rotary calls refuse.
Nothing reaches a GPU; addresses are made up and every check fails first."""

import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2608_01821_amd as dv
from oracle import rotary as orot

EINVAL, ESHAPE, EDTYPE = -1, -2, -3
A = 1 << 20
NAMES = {"plain": dv.DAVET_ROTARY_PLAIN, "linear": dv.DAVET_ROTARY_LINEAR,
         "base": dv.DAVET_ROTARY_BASE, "ramp": dv.DAVET_ROTARY_RAMP}


@pytest.mark.parametrize("scaling", list(NAMES))
@pytest.mark.parametrize("dim", [2, 4, 32, 62, 128, 512])
@pytest.mark.parametrize("theta", [1.0, 1e4, 5e5, 1e6])
def test_turns(scaling, dim, theta):
    kw = dict(factor=8.0, trained=8192.0, fast=32.0, slow=1.0)
    got = dv.davet_rotary_turns(dim, theta, NAMES[scaling], **kw)
    ref = orot.turns(dim, theta, scaling, **kw)
    # powers, a quotient and a sum in float64: a few of its roundings
    assert np.allclose(got, ref, rtol=64 * 2.0 ** -53, atol=0)


def test_turns_at_the_ends():
    """The stretched base keeps the fastest pair and slows the last by `factor`; the
    ramp keeps pairs of `fast` turns and more and slows those of `slow` and fewer."""
    plain = dv.davet_rotary_turns(128, 1e4)
    base = dv.davet_rotary_turns(128, 1e4, dv.DAVET_ROTARY_BASE, factor=4.0)
    assert base[0] == plain[0] and math.isclose(base[-1], plain[-1] / 4, rel_tol=1e-13)
    ramp = dv.davet_rotary_turns(128, 1e4, dv.DAVET_ROTARY_RAMP, factor=4.0,
                                 trained=4096, fast=32, slow=1)
    for r, p in zip(ramp, plain):
        if p * 4096 >= 32:
            assert r == p
        elif p * 4096 <= 1:
            assert r == p / 4
        else:
            assert p / 4 < r < p
    assert dv.davet_rotary_turns(128, 1e4, dv.DAVET_ROTARY_LINEAR, factor=1.0) == plain


@pytest.mark.parametrize("args,status", [
    ((0, 1e4), ESHAPE), ((3, 1e4), ESHAPE), ((514, 1e4), ESHAPE), ((-2, 1e4), ESHAPE),
    ((64, 0.5), EINVAL), ((64, math.inf), EINVAL), ((64, math.nan), EINVAL),
    ((64, 1e4, 4), EINVAL), ((64, 1e4, -1), EINVAL),
    ((64, 1e4, 1, 0.5), EINVAL), ((64, 1e4, 2, math.nan), EINVAL),
    ((64, 1e4, 3, 2.0, 0.0, 32, 1), EINVAL), ((64, 1e4, 3, 2.0, 4096, 1, 1), EINVAL),
    ((64, 1e4, 3, 2.0, 4096, 32, -1), EINVAL), ((64, 1e4, 3, 2.0, math.inf, 32, 1),
                                                EINVAL),
])
def test_turns_refusals(args, status):
    with pytest.raises(dv.DavetError) as e:
        dv.davet_rotary_turns(*args)
    assert e.value.status == status


def _call(rows=3, heads=2, width=64, dim=64, layout=0, x=A, ldx=128, out=A << 1,
          ldo=128, dtype=dv.DAVET_F16, pos=None, turns=A << 2, gain=1.0, inverse=0):
    return dv.raw().davet_rotary(rows, heads, width, dim, layout, x, ldx, out, ldo,
                                 dtype, pos, turns, gain, inverse, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), EDTYPE), (dict(layout=2), EINVAL), (dict(layout=-1), EINVAL),
    (dict(inverse=2), EINVAL), (dict(gain=math.inf), EINVAL),
    (dict(gain=math.nan), EINVAL),
    (dict(rows=-1), ESHAPE), (dict(rows=(1 << 24) + 1), ESHAPE), (dict(heads=0), ESHAPE),
    (dict(heads=4097), ESHAPE), (dict(width=65, dim=64), ESHAPE),
    (dict(width=514), ESHAPE), (dict(dim=66), ESHAPE), (dict(dim=63), ESHAPE),
    (dict(dim=0), ESHAPE), (dict(ldx=127), ESHAPE), (dict(ldo=127), ESHAPE),
    (dict(ldx=1 << 31), ESHAPE), (dict(ldx=-128), ESHAPE),
    (dict(x=None), EINVAL), (dict(out=None), EINVAL), (dict(turns=None), EINVAL),
    (dict(x=A + 1), EINVAL), (dict(out=(A << 1) + 1), EINVAL),
    (dict(turns=(A << 2) + 4), EINVAL), (dict(pos=A + 2), EINVAL),
    # shared memory other than in place
    (dict(out=A + 2), EINVAL), (dict(out=A, ldo=136), EINVAL),
    (dict(out=A + 256), EINVAL), (dict(out=A - 2), EINVAL),
    (dict(out=A + 254, ldx=256, ldo=256), EINVAL),
])
def test_refusals(kw, status):
    assert _call(**kw) == status


def test_nothing_to_do():
    assert _call(rows=0, x=None, out=None, turns=None) == 0


def test_binding_refusals():
    x, f = torch.zeros(3, 128, dtype=torch.float16), torch.zeros(3, 128)
    t = torch.zeros(32, dtype=torch.float64)
    call = dv.davet_rotary
    for args, kw in (((f, 2, 64, t, x, dv.DAVET_F16), {}),
                     ((x, 2, 64, t, f, dv.DAVET_F16), {}),
                     ((x, 2, 64, f[0], x, dv.DAVET_F16), {}),
                     ((x, 2, 64, t, x, dv.DAVET_F16), dict(pos=f[0]))):
        with pytest.raises(ValueError, match="is of torch"):
            call(*args, **kw)
    for args in ((x, 3, 64, t, x), (x[0], 2, 64, t, x), (x, 2, 64, t, x[:2]),
                 (x[:, ::2], 1, 64, t, x), (x, 2, 64, t[::2], x)):
        with pytest.raises(ValueError):
            call(*args, dv.DAVET_F16)
    with pytest.raises(ValueError, match="32-bit"):
        call(x, 2 + 2 ** 32, 64, t, x, dv.DAVET_F16)
    with pytest.raises(ValueError, match="32-bit"):
        call(x, 2, 64, t, x, dv.DAVET_F16, layout=2 ** 32)
    with pytest.raises(ValueError, match="on a GPU"):
        call(x, 2, 64, t, x, dv.DAVET_F16)
