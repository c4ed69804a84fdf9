"""Scores and values that are not finite, chunks split over many workgroups, and
single rows: davet_cache_append, davet_cache_attention and davet_cache_weights
against float64."""

import numpy as np
import pytest
import torch

import paper_2608_01821_amd as dv
from cache_util import TORCH, Setup, check_attention, f64
from oracle import cache as oc

pytestmark = pytest.mark.gpu


def received(t, lse, block=0, scale=0.0, prev=None):
    """davet_cache_weights of a Setup, float64."""
    w = torch.zeros(len(t.kv), max(t.kv), device="cuda") if prev is None else prev
    dv.davet_cache_weights(t.device(), t.cu, t.kv, t.q.cuda(), t.heads,
                           torch.from_numpy(lse).float().cuda(), w, prev=prev,
                           scale=scale, block=block, workspace=t.workspace())
    torch.cuda.synchronize()
    return f64(w)


def put(t, name, s, js, dim, value):
    """Element `dim` of the keys or values of cache indices `js`, every head."""
    for j in js:
        page, off = oc.slot(t.host, s, j)
        getattr(t, name)[page, :, off, dim] = value


# ------------------------------------------------------------ scores of -inf --

@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("scale", [0.0, 0.2, 0.25])
def test_weights_of_scores_of_minus_infinity(dtype, dim, scale):
    """A key that scores -inf receives nothing, the others what they would have;
    a row with no other score (lse -inf) gives nothing.  (As a sum of two
    floats 0.2 log2(e) has a negative second one, and so has the default scale of
    128 dims; 0.25 log2(e) and that of 64 dims a positive one.)"""
    new, kv = 6, 70
    t = Setup(23, dtype, [new], [kv], 4, 2, dim, 16)
    q = t.q.view(new, 4, dim)
    q[:, :, 9] = -q[:, :, 9].abs() - 0.5
    low = list(range(kv - new + 1)) + [kv - 2]       # all that row 0 sees, one more
    put(t, "k", 0, low, 9, np.inf)
    ref = oc.attention(t.host, t.cu, t.kv, f64(t.q), 4, scale=scale, block=1)
    assert np.isneginf(ref["lse"][0]).all() and np.isfinite(ref["lse"][1:]).all()
    want = oc.weights(t.host, t.cu, t.kv, f64(t.q), 4, f64(torch.from_numpy(
        ref["lse"]).float()), scale=scale, block=1)
    assert np.all(want[0, low] == 0)
    prev = torch.full((1, kv), 0.5, device="cuda")
    plain = received(t, ref["lse"], 1, scale)
    added = received(t, ref["lse"], 1, scale, prev)
    # a term's error as in the weights tests, of scores without the infinity
    top = (scale or dim ** -0.5) * np.abs(f64(t.q)).max() * 5 * dim
    rel = (dim + 8) * 2.0 ** -24 * (top + np.abs(ref["lse"][1:]).max() + 1) + \
        (new * 4 + 8) * 2.0 ** -24
    assert np.all(plain[0, low] == 0) and np.all(added[0, low] == 0.5)
    assert np.all(np.abs(plain - want) <= rel * want)
    assert np.all(np.abs(added - want - 0.5) <= rel * (want + 0.5))
    lse = t.attend(block=1, scale=scale)[1]
    assert np.isneginf(lse[0]).all() and np.isfinite(lse[1:]).all()


# --------------------------------------------------------------- single rows --

@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("spare", [0, 5])
def test_append_of_one_row_in_place(dtype, spare):
    """A tensor of exactly one row, its queries in place: what separate outputs
    give, bit for bit; columns past the query heads stay."""
    t = Setup(25, dtype, [1], [20], 4, 2, 64, 16)
    qkv = torch.from_numpy(t.rng.standard_normal((1, 8 * 64 + spare))).to(
        TORCH[dtype]).cuda()
    got, want = qkv.clone(), torch.zeros(1, 4 * 64, dtype=TORCH[dtype], device="cuda")
    k = []
    for x, out in ((qkv, want), (got, got)):
        cache = t.device()
        dv.davet_cache_append(cache, t.cu, t.kv, x, 4, out, norm=True)
        torch.cuda.synchronize()
        k.append(t.dk)
    assert torch.equal(got[:, :256], want) and torch.equal(got[:, 256:], qkv[:, 256:])
    assert torch.equal(k[0], k[1])


# ---------------------------------------------------- values of no importance --

@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("new,kv", [(3, 90), (3, 1300), (80, 200), (80, 1600)])
def test_rows_of_minus_infinity_are_zeros(dtype, new, kv):
    """A row whose every score is -inf gets zeros and lse -inf whatever the values
    it sees hold: in tiles that all rows see, in the last ones, in pieces."""
    t = Setup(27, dtype, [new], [kv], 2, 2, 64, 16)
    t.q.view(new, 2, 64)[:, :, 9] = -1.0
    put(t, "k", 0, range(kv - new + 2), 9, np.inf)   # all that rows 0 and 1 see
    put(t, "v", 0, (2, kv - new, kv - new + 1), 5, np.inf)
    put(t, "v", 0, (3, kv - new), 6, np.nan)
    out, lse = t.attend(block=1)
    assert np.isneginf(lse[:2]).all() and np.all(out[:2] == 0)
    assert np.isfinite(lse[2:]).all()
    rest = [d for d in range(64) if d not in (5, 6)]
    ref = oc.attention(t.host, t.cu, t.kv, f64(t.q), 2, block=1)
    ref["dot"] = np.full_like(ref["dot"], np.abs(f64(t.q)).max() * 5 * 64 ** 0.5)
    ref = {k: x[2:] if x.ndim == 2 else x[2:][..., rest] for k, x in ref.items()}
    check_attention((out[2:][..., rest], lse[2:]), ref, dtype, 64, kv)
