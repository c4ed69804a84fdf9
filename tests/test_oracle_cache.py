"""The cache oracle against the step oracle, closed forms and torch float64."""

import numpy as np
import pytest
import torch

from oracle import cache as oc
from oracle import model


def _cache(rng, kv, hk, page, dim, total=None):
    counts = [-(-n // page) for n in kv]
    total = total or sum(counts)
    order, at = rng.permutation(total), 0
    table = np.full((len(kv), max(counts)), -1, np.int32)
    for s, c in enumerate(counts):
        table[s, :c] = order[at:at + c]
        at += c
    shape = (total, hk, page, dim)
    return dict(k=rng.standard_normal(shape), v=rng.standard_normal(shape),
                table=table)


def test_append_then_attention_is_the_step_oracles_layer():
    """A whole sequence entered at once and attended in full: the rotary
    embedding and the bidirectional attention of the denoiser."""
    rng = np.random.default_rng(0)
    n, h, dim = 37, 3, 64
    c = _cache(rng, [n], h, 16, dim)
    qkv = rng.standard_normal((n, 3 * h * dim))
    q, k, v = oc.append(c, [0, n], [n], qkv, h, theta=10000.0)
    ang = model.rope_angles(n, dim, 10000.0)
    x = qkv.reshape(n, 3, h, dim)
    rq, rk = model.rope(x[:, 0], ang), model.rope(x[:, 1], ang)
    assert np.allclose(q, rq, atol=1e-12)
    r = oc.attention(dict(c, k=k, v=v), [0, n], [n], q, h)
    assert np.allclose(r["out"], model.attention(rq, rk, x[:, 2]), atol=1e-12)


def test_norm_is_rmsnorm_per_head():
    rng = np.random.default_rng(1)
    c = _cache(rng, [5], 1, 16, 64)
    qkv, gain = rng.standard_normal((5, 4 * 64)), rng.standard_normal(64)
    q, k, _ = oc.append(c, [0, 5], [5], qkv, 2, pos=[0] * 5, norm=True,
                        q_gain=gain, eps=1e-6)
    x = qkv.reshape(5, 4, 64)
    assert np.allclose(q, model.rmsnorm(x[:, :2], gain, 1e-6))
    assert np.allclose(k[c["table"][0, 0], 0, :5], model.rmsnorm(x[:, 2], None, 1e-6))


@pytest.mark.parametrize("block", [0, 1, 4, 100])
def test_masked_attention_against_torch(block):
    rng = np.random.default_rng(block)
    n, kv, h, hk, dim = 11, 53, 4, 2, 64
    c = _cache(rng, [kv], hk, 16, dim)
    c["table"][0, 1] = -1                       # a hole: indices 16 .. 31
    q = rng.standard_normal((n, h, dim))
    r = oc.attention(c, [0, n], [kv], q, h, block=block)
    k = np.stack([c["k"][max(0, c["table"][0, j // 16]), :, j % 16] for j in range(kv)])
    v = np.stack([c["v"][max(0, c["table"][0, j // 16]), :, j % 16] for j in range(kv)])
    i, j = np.arange(n)[:, None], np.arange(kv)[None]
    seen = j < (kv if block == 0 else kv - n + np.minimum(n, (i // block + 1) * block))
    seen = seen & (j // 16 != 1)
    kt, vt = (torch.from_numpy(x).repeat_interleave(2, 1) for x in (k, v))
    x = torch.einsum("ihd,jhd->hij", torch.from_numpy(q), kt) / 8.0
    x = x.masked_fill(~torch.from_numpy(seen), -np.inf)
    assert np.allclose(torch.logsumexp(x, 2).t().numpy(), r["lse"])
    o = torch.einsum("hij,jhd->ihd", torch.softmax(x, 2), vt)
    assert np.allclose(o.numpy(), r["out"])
    w = oc.weights(c, [0, n], [kv], q, h, r["lse"], block=block)
    assert np.allclose(w[0], torch.softmax(x, 2).sum((0, 1)).numpy())


def test_empty_rows_and_select_and_logprobs():
    rng = np.random.default_rng(3)
    c = _cache(rng, [8], 1, 16, 64)
    c["table"][:] = 99
    r = oc.attention(c, [0, 2], [8], rng.standard_normal((2, 1, 64)), 1)
    assert np.all(r["out"] == 0) and np.all(np.isneginf(r["lse"]))
    w = [3.0, np.nan, 3.0, -np.inf, 5.0, 0.0, -0.0, 1.0]
    assert oc.select(8, 3, w) == [0, 2, 4]
    assert oc.select(8, 2, w) == [0, 4]
    assert oc.select(8, 3, w, first=1, last=1) == [0, 4, 7]
    assert oc.select(8, 6, w) == [0, 2, 4, 5, 6, 7]
    assert oc.select(8, 0, w) == [] and oc.select(8, 8, w) == list(range(8))
    x = rng.standard_normal(40)
    lp, ent, top = oc.logprobs(x, 7, exclude=3, top=4)
    keep = np.delete(x, 3)
    p = np.exp(keep) / np.exp(keep).sum()
    assert np.isclose(lp, x[7] - np.log(np.exp(keep).sum()))
    assert np.isclose(ent, -(p * np.log(p)).sum())
    assert [j for j, _ in top] == [j for j in np.argsort(-x) if j != 3][:4]
    assert oc.logprobs(x, 3, exclude=3)[0] == -np.inf
    assert oc.logprobs([-np.inf] * 4, 1, top=2) == (-np.inf, 0.0, [])
