"""davet_evict_select, davet_cache_gather and davet_token_logprobs against the
float64 oracle."""

import numpy as np
import pytest
import torch

import paper_2608_01821_amd as dv
from cache_util import CODE, TORCH, f64, page_table, values
from oracle import cache as oc

pytestmark = pytest.mark.gpu


def _select(n, keep, w, first=0, last=0):
    w = torch.as_tensor(np.asarray(w, np.float32)).cuda()
    m = max(max(keep), 1)
    kept = torch.full((len(n), m + 3), -9, dtype=torch.int32, device="cuda")
    out = torch.full((len(n), m + 1), 7.0, device="cuda")
    dv.davet_evict_select(n, keep, w, kept, first=first, last=last, weights_out=out)
    torch.cuda.synchronize()
    return kept.cpu().numpy(), out.cpu().numpy(), w.cpu().numpy()


def _check_select(n, keep, w, first=0, last=0):
    kept, out, w = _select(n, keep, w, first, last)
    for s, (a, b) in enumerate(zip(n, keep)):
        want = oc.select(a, b, w[s], first, last)
        assert kept[s, :b].tolist() == want
        assert np.array_equal(out[s, :b], w[s, want], equal_nan=True)
        assert np.all(kept[s, b:] == -9) and np.all(out[s, b:] == 7)


@pytest.mark.parametrize("n,keep", [
    ([1], [1]), ([1], [0]), ([2, 0, 5], [1, 0, 5]), ([63, 64, 65], [30, 64, 1]),
    ([1000], [999]), ([1025], [512]), ([5000, 700], [77, 600]), ([70001], [35000])])
def test_select_random(n, keep):
    rng = np.random.default_rng(sum(n))
    w = np.exp(3 * rng.standard_normal((len(n), max(n))))
    _check_select(n, keep, w)
    f = min(2, min(k for k in keep if k) // 2) if any(keep) else 0
    _check_select(n, keep, w, first=f, last=f)


@pytest.mark.parametrize("kind", ["ties", "equal", "special", "few bits"])
def test_select_ties_and_specials(kind):
    rng = np.random.default_rng(1)
    n, keep = [3001, 200], [1234, 150]
    w = rng.integers(0, 4, (2, 3001)).astype(np.float32)
    if kind == "equal":
        w[:] = 0.25
    if kind == "special":
        pool = np.array([np.nan, np.inf, -np.inf, 0.0, -0.0, 1.0, -1.0, 3.4e38,
                         -3.4e38, 1e-45, -1e-45], np.float32)
        w = pool[rng.integers(0, len(pool), w.shape)]
    if kind == "few bits":
        w = 1.0 + rng.integers(0, 50, w.shape) * 2.0 ** -23
    _check_select(n, keep, w)
    _check_select(n, keep, w, first=7, last=100)
    _check_select(n, [n[0], 1], w)


@pytest.mark.parametrize("dtype,dim,page,hk", [("f16", 64, 16, 3), ("bf16", 128, 64, 2),
                                               ("f32", 128, 32, 1), ("f32", 64, 256, 2)])
def test_gather(dtype, dim, page, hk):
    rng = np.random.default_rng(dim + page)
    n, keep = [150, 40, 9, 1], [77, 40, 0, 1]
    total, table = page_table(rng, n, page, extra=0)
    ndst = [-(-k // page) for k in keep]
    dst = np.full((4, max(ndst) + 1), -1, np.int32)
    at = total
    for s, c in enumerate(ndst):
        dst[s, :c] = np.arange(at, at + c)
        at += c
    k, v = (values(rng, (at + 1, hk, page, dim), dtype) for _ in range(2))
    table[1, 0] = -3                               # a source hole: zeros
    kept = np.full((4, 80), 5, np.int32)
    for s, (a, b) in enumerate(zip(n, keep)):
        kept[s, :b] = np.sort(rng.permutation(a)[:b])
    kept[0, 76] = 10 ** 9                          # outside: zeros
    kept[0, 0] = -1
    if page == 16:
        dst[0, 1] = at + 5                         # a destination hole
    dk, dvv = k.cuda(), v.cuda()
    cache = dv.KvCache(dk, dvv, torch.from_numpy(table).cuda(), CODE[dtype])
    dv.davet_cache_gather(cache, torch.from_numpy(kept).cuda(), keep,
                          torch.from_numpy(dst).cuda())
    torch.cuda.synchronize()
    for got, x in ((dk.cpu(), k), (dvv.cpu(), v)):
        want = x.clone()
        for s, b in enumerate(keep):
            for j in range(b):
                d = dst[s, j // page]
                if not 0 <= d <= at:
                    continue
                i = int(kept[s, j])
                p = table[s, i // page] if 0 <= i < table.shape[1] * page else -1
                want[d, :, j % page] = x[p, :, i % page] if p >= 0 else 0
        assert torch.equal(got, want)


# ----------------------------------------------------------------- logprobs --

def _logprobs(x, dtype, targets, top, exclude=-1):
    rows, vocab = x.shape
    d = dict(device="cuda")
    lp, en = torch.full((rows,), 7.0, **d), torch.full((rows,), 7.0, **d)
    tl = torch.full((rows, top), 7.0, **d)
    ti = torch.full((rows, top), 7, dtype=torch.int32, **d)
    nb = dv.davet_logprobs_workspace_bytes(rows, vocab, top)
    dv.davet_token_logprobs(
        x, CODE[dtype], targets=torch.as_tensor(targets, dtype=torch.int32).cuda(),
        logp=lp, entropy=en, top_logp=tl, top_ids=ti, exclude=exclude,
        workspace=torch.empty(max(nb, 256), dtype=torch.uint8, **d))
    torch.cuda.synchronize()
    return f64(lp), f64(en), f64(tl), ti.cpu().numpy()


def _check_logprobs(x, dtype, targets, top, exclude=-1):
    got = _logprobs(x, dtype, targets, top, exclude)
    host = f64(x)
    for r in range(len(host)):
        lp, ent, best = oc.logprobs(host[r], int(targets[r]), exclude, top)
        fin = host[r][np.isfinite(host[r])]
        m = np.abs(fin).max() if len(fin) else 0.0
        spread = fin.max() - fin.min() if len(fin) else 0.0
        # a difference x - m and its logarithm's sum: roundings of m, x and
        # ln S; the sum of n exponentials in fp32 (at most 32 + n / 64 terms a
        # lane, then the tree), each off by 3 2^-24 of its argument (weights
        # beyond 88 below the maximum are 0)
        rel = (40 + len(host[r]) / 64 + 3 * min(spread, 88)) * 2.0 ** -24
        tol = 4 * 2.0 ** -24 * (m + 12) + rel
        assert got[0][r] == lp or abs(got[0][r] - lp) <= tol, (got[0][r], lp)
        assert abs(got[1][r] - ent) <= tol + rel * (ent + 12)
        ids = [j for j, _ in best] + [-1] * (top - len(best))
        assert got[3][r].tolist() == ids
        for i, (_, v) in enumerate(best):
            assert abs(got[2][r, i] - v) <= tol
        assert np.all(np.isneginf(got[2][r, len(best):]))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,vocab,top", [
    (1, 1, 1), (1, 5, 64), (3, 63, 5), (2, 1000, 0), (5, 4097, 20), (2, 32003, 64),
    (3, 126464, 5), (1030, 300, 3), (1, 20000, 1)])
def test_logprobs(dtype, rows, vocab, top):
    rng = np.random.default_rng(rows + vocab + top)
    x = values(rng, (rows, vocab), dtype, 3.0).cuda()
    t = rng.integers(0, vocab, rows)
    _check_logprobs(x, dtype, t, top, exclude=vocab // 2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [1, 3, 7])
def test_logprobs_rows_at_any_alignment(dtype, offset):
    """Odd strides and starts: the edges outside whole 16-byte pieces, with the
    largest values in them, and neighbours that must not be read into a row."""
    rng = np.random.default_rng(offset)
    big = values(rng, (6, 9000), dtype).cuda()
    x = big[:, offset:offset + 8191]
    big[:, :offset] = 100.0
    big[:, offset + 8191:] = 100.0
    x[0, 0], x[1, -1], x[2, 1], x[3, -2] = 9, 9, 9, 9
    flat = torch.empty(6 * 8191 + 8, dtype=TORCH[dtype], device="cuda")
    dense = flat[offset:offset + 6 * 8191].view(6, 8191)
    dense.copy_(x)
    for y in (x, dense):
        _check_logprobs(y, dtype, [0, 8190, 1, 8189, 5, 6], 6)


def test_logprobs_orders():
    """Ascending rows (every value enters the list), equal rows (lowest ids),
    quantised rows (ties across lanes, waves and slices)."""
    up = torch.linspace(-8, 8, 40000).repeat(3, 1)
    up[1] = up[1].flip(0)
    up[2] = 0.5
    _check_logprobs(up.cuda(), "f32", [0, 1, 39999], 64)
    rng = np.random.default_rng(8)
    q = torch.from_numpy(rng.integers(0, 6, (4, 50000)).astype(np.float32))
    _check_logprobs(q.cuda(), "f32", [1, 2, 3, 4], 33)
    _check_logprobs(q.half().cuda(), "f16", [1, 2, 3, 4], 33, exclude=0)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [1, 2, 63, 65, 512, 513, 1000, 1024, 1025, 1100])
def test_logprobs_short_rows(dtype, vocab):
    """Rows that one workgroup holds whole, and the first that it does not: random,
    equal, quantised, ascending, masked to one, to none; strided, any start."""
    rng = np.random.default_rng(vocab)
    big = values(rng, (7, vocab + 5), dtype, 3.0).cuda()
    x = big[:, 3:3 + vocab]
    x[1] = 0.25
    x[2] = torch.from_numpy(rng.integers(0, 4, vocab).astype(np.float32)).to(x.dtype)
    x[3] = torch.linspace(-6, 6, vocab).to(x.dtype)
    x[4] = -np.inf
    x[4, vocab // 2] = 1.0
    x[5] = -np.inf
    x[6, ::2] = torch.finfo(x.dtype).min
    big[:, :3], big[:, 3 + vocab:] = 100.0, 100.0
    last = vocab - 1
    for top in (0, 1, 33, 64):
        _check_logprobs(x, dtype, [last, 0, last // 2, 0, vocab // 2, 0, vocab], top)
    _check_logprobs(x, dtype, [last, 0, last // 2, 0, vocab // 2, 0, -1], 20,
                    exclude=vocab // 2)


def test_logprobs_masked_rows():
    """-inf, the type's lowest value, rows with nothing, targets out of range."""
    rng = np.random.default_rng(2)
    for dtype in ("f32", "f16"):
        lo = torch.finfo(TORCH[dtype]).min
        x = values(rng, (8, 9001), dtype).cuda()
        x[0] = -np.inf
        x[1, 7:] = -np.inf
        x[2] = lo
        x[3, 3:] = lo
        x[4] = -np.inf
        x[4, 77] = 2.0
        x[5] = -np.inf
        x[5, 5] = lo
        x[6, 100:8000] = -np.inf
        _check_logprobs(x, dtype, [3, 100, 8, 1, 77, 5, -1, 9001], 9)
        _check_logprobs(x, dtype, [3, 100, 8, 1, 77, 5, -5, 77], 9, exclude=77)


def test_logprobs_nan_and_infinity():
    rng = np.random.default_rng(4)
    for vocab in (300, 30000):
        x = values(rng, (3, vocab), "f32").cuda()
        x[0, 11] = np.nan
        x[1, 12] = np.inf
        lp, en, tl, ti = _logprobs(x, "f32", [5, 5, 5], 4)
        host = f64(x)
        assert np.isnan(lp[:2]).all() and np.isnan(en[:2]).all()
        assert np.isnan(tl[:2]).all() and np.isfinite(tl[2]).all()
        assert ti[0].tolist() == [j for j in np.argsort(-host[0]) if j != 11][:4]
        assert ti[1, 0] == 12
        _check_logprobs(x[2:], "f32", [5], 4)
        x[0] = np.nan
        lp, en, tl, ti = _logprobs(x, "f32", [5, 5, 5], 4)
        assert np.isnan(lp[0]) and np.isnan(en[0]) and (ti[0] == -1).all()


def test_logprobs_subsets_of_outputs():
    rng = np.random.default_rng(9)
    x = values(rng, (2, 700), "f32").cuda()
    want = _logprobs(x, "f32", [3, 4], 5)
    en = torch.empty(2, device="cuda")
    dv.davet_token_logprobs(x, dv.DAVET_F32, entropy=en)
    tl = torch.empty(2, 5, device="cuda")
    ti = torch.empty(2, 5, dtype=torch.int32, device="cuda")
    dv.davet_token_logprobs(x, dv.DAVET_F32, top_logp=tl, top_ids=ti)
    torch.cuda.synchronize()
    assert np.array_equal(f64(en), want[1]) and np.array_equal(f64(tl), want[2])
