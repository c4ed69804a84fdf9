"""davet_beam_select and davet_cache_reorder against the float64 oracle: sizes from one
beam and one token on, types, ties, rows that are over or have nothing to offer, holes;
and steps of a beam search over a cache."""

import numpy as np
import pytest
import torch

import paper_2608_01821_amd as dv
from cache_util import CODE, TORCH, f64, page_table, values
from oracle import cache as oc

pytestmark = pytest.mark.gpu


def select(x, dtype, scores, beams, top, alias=False, **kw):
    rows, vocab = x.shape
    groups = rows // beams
    n = dv.davet_beam_workspace_bytes(groups, beams, vocab, top)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")   # (NaNs)
    sc = scores.cuda()
    o = sc.view(groups, beams) if alias else torch.full((groups + 1, top), 7.0,
                                                        device="cuda")
    r, t = (torch.full((groups + 1, top), 7, dtype=torch.int32, device="cuda")
            for _ in range(2))
    dv.davet_beam_select(x, CODE[dtype], sc, beams, o[:groups], r[:groups], t[:groups],
                         workspace=ws, **kw)
    torch.cuda.synchronize()
    assert (r[groups:] == 7).all() and (t[groups:] == 7).all()
    assert alias or (o[groups:] == 7).all()
    return o[:groups].cpu().numpy(), r[:groups].cpu().numpy(), t[:groups].cpu().numpy()


def check(got, ref, vocab, top):
    """A value carries the roundings of its sum of exponentials: an exponential's
    argument those of a difference and a product (the mean size of arguments is at most
    log2 of the count: under 30, so 42 units of 2^-24), its own and the sum's (64, and
    one a term of a lane); and the store.  Candidates farther apart than that have to be
    the oracle's."""
    o, r, t = got
    for g, want in enumerate(ref):
        n = len(want)
        assert (r[g, n:] == -1).all() and (t[g, n:] == -1).all()
        assert np.isneginf(o[g, n:]).all()
        assert len({(a, b) for a, b in zip(r[g, :n], t[g, :n])}) == n
        v = np.array([w[0] for w in want])
        tol = 2.0 ** -24 * (2 * np.abs(v) + 150 + vocab / 512)
        assert np.all(np.abs(o[g, :n] - v) <= tol)
        for j in range(n):
            near = [i for i in range(n)
                    if i != j and want[i][1] != want[j][1]
                    and abs(v[i] - v[j]) <= 2 * tol[j]]
            last = j == n - 1 or abs(v[j] - v[-1]) <= 2 * tol[j]
            if near or (last and n == top and j != n - 1):
                continue
            if j == n - 1 and (r[g, j], t[g, j]) != want[j][1:]:
                continue                    # (the first one left out may be as near)
            assert (r[g, j], t[g, j]) == want[j][1:], (g, j)


CASES = [  # dtype, groups, beams, vocab, top
    ("f32", 1, 1, 1, 1),
    ("f16", 1, 1, 7, 4),                    # fewer candidates than asked for
    ("f32", 2, 3, 50, 64),
    ("bf16", 3, 4, 1000, 8),
    ("f16", 5, 2, 1024, 2),
    ("f32", 1, 4, 1025, 4),
    ("f32", 1, 4, 32003, 8),                # slices, odd rows
    ("bf16", 2, 5, 50257, 10),
    ("f16", 16, 4, 9001, 4),
    ("f32", 1, 64, 5000, 64),
    ("f16", 4, 16, 16400, 16),
    ("bf16", 70, 4, 2001, 8),               # a slice a row
    ("f32", 1, 2, 126464, 64),
]


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("odd", [False, True])
def test_select(case, odd):
    dtype, groups, beams, vocab, top = case
    rng = np.random.default_rng(vocab + beams)
    rows = groups * beams
    x = values(rng, (rows, vocab + 3 * odd), dtype, 3.0)
    scores = torch.from_numpy(-4 * rng.random(rows)).float()
    kw = {}
    if odd:
        done = (rng.random(rows) < 0.3).astype(np.int32) * 5
        x[torch.from_numpy(done != 0)] = float("nan")        # (not read)
        scores[rows // 2] = float("-inf")
        kw = dict(exclude=vocab // 3, done=torch.from_numpy(done).cuda(), pad=vocab + 9)
    dx = x.cuda()[:, :vocab]
    ref = oc.beam_select(f64(x)[:, :vocab], scores.numpy(), beams, top,
                         exclude=kw.get("exclude", -1),
                         done=done if odd else None, pad=kw.get("pad", 0))
    check(select(dx, dtype, scores, beams, top, **kw), ref, vocab, top)
    if top == beams:
        a = select(dx, dtype, scores, beams, top, **kw)
        b = select(dx, dtype, scores, beams, top, alias=True, **kw)
        assert all(np.array_equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("vocab", [100, 3000, 40000])
def test_ties(vocab):
    """Equal beams, equal logits: the lower row, then the lower token."""
    x = torch.zeros(6, vocab)
    x[:, 11], x[:, 60] = 2.0, 2.0
    o, r, t = select(x.cuda(), "f32", torch.zeros(6), 3, 8)
    assert r.tolist() == [[0, 0, 1, 1, 2, 2, 0, 0], [3, 3, 4, 4, 5, 5, 3, 3]]
    assert t.tolist() == [[11, 60] * 3 + [0, 1]] * 2
    assert (o[:, :6] == o[:, :1]).all() and (o[:, 6:] == o[:, 6:7]).all()
    # minus and plus zero are equal; a score so large that the logits vanish beside it
    x = torch.zeros(2, vocab)
    x[:, 5:] = -0.0
    o, r, t = select(x.cuda(), "f32", torch.tensor([-1e30, -1e30]), 2, 8)
    assert r.tolist() == [[0] * 8] and t.tolist() == [list(range(8))]
    x[:, 9] = 1.0
    _, r, t = select(x.cuda(), "f32", torch.tensor([-1e30, -1e30]), 2, 3)
    assert r.tolist() == [[0] * 3] and t.tolist() == [[9, 0, 1]]


@pytest.mark.parametrize("top", [1, 3, 4, 7, 16, 33, 64])
def test_scores_that_the_logits_vanish_beside(top):
    """Every value of a row is the same: its tokens in order of their logits all the
    same, and the lower row first."""
    rng = np.random.default_rng(top)
    x = values(rng, (6, 33000), "f32")
    scores = torch.tensor([-1e30, -1e30, -2.0, -1e30, 1e25, -1e30])
    o, r, t = select(x.cuda(), "f32", scores, 3, top)
    big = [np.argsort(-f64(x)[i], kind="stable")[:top].tolist() for i in range(6)]
    assert r.tolist() == [[2] * top, [4] * top]
    assert t[0].tolist() == big[2]
    assert t[1].tolist() == big[4]
    o, r, t = select(x[[0, 1, 3]].cuda(), "f32", scores[[0, 1, 3]], 3, top)
    assert r.tolist() == [[0] * top] and t[0].tolist() == big[0]
    if top > 1:
        done = torch.tensor([5, 0, 0], dtype=torch.int32).cuda()
        _, r, t = select(x[[0, 1, 3]].cuda(), "f32", scores[[0, 1, 3]], 3, top, done=done,
                         pad=-7)
        assert r.tolist() == [[0] + [1] * (top - 1)]
        assert t[0].tolist() == [-7] + big[1][:top - 1]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [90, 5000])
def test_rows_with_nothing_to_offer(dtype, vocab):
    x = values(np.random.default_rng(1), (8, vocab), dtype)
    x[0, 3], x[1, 3], x[2] = float("nan"), float("inf"), float("-inf")
    scores = torch.tensor([0, 0, 0, float("nan"), float("inf"), float("-inf"), 0, -1.0])
    done = torch.tensor([0, 0, 0, 1, 1, 1, 0, 0], dtype=torch.int32)
    for d in (None, done.cuda()):
        o, r, t = select(x.cuda(), dtype, scores, 8, 64, done=d)
        assert set(r[0].tolist()) == {6, 7}
        o, r, t = select(x[:6].cuda(), dtype, scores[:6], 6, 4,
                         done=d if d is None else d[:6])
        assert (r == -1).all() and (t == -1).all() and np.isneginf(o).all()
    x[6:, :-1] = float("-inf")              # one token each
    ref = oc.beam_select(f64(x), scores.numpy(), 8, 4)
    o, r, t = select(x.cuda(), dtype, scores, 8, 4)
    assert r.tolist() == [[6, 7, -1, -1]] and t.tolist() == [[vocab - 1] * 2 + [-1] * 2]
    check((o, r, t), ref, vocab, 4)


REORDER = [  # dtype, kv, kv_heads, dim, page
    ("f16", [1], 1, 64, 16),
    ("f16", [0, 16, 17], 2, 64, 16),
    ("bf16", [300] * 4, 8, 128, 64),
    ("f32", [255, 256, 257], 3, 128, 256),
    ("f32", [100] * 64, 2, 64, 32),
    ("bf16", [1999] * 5, 1, 128, 128),
]


@pytest.mark.parametrize("case", REORDER, ids=str)
@pytest.mark.parametrize("odd", [False, True])
def test_reorder(case, odd):
    dtype, kv, hk, dim, page = case
    rng = np.random.default_rng(kv[0] + hk)
    n = len(kv)
    total, table = page_table(rng, [max(kv)] * n, page, extra=n + 1)
    free = np.array([p for p in range(total) if p not in table], np.int32)
    k, v = (values(rng, (total, hk, page, dim), dtype) for _ in range(2))
    parent = rng.integers(0, n, n).astype(np.int32)
    kv = [kv[p] for p in parent]
    fresh, width = free[:n].copy(), table.shape[1] + 2
    if odd:
        parent[0] = [-1, n, 2 ** 31 - 1, -2 ** 31][n % 4]
        fresh[-1] = -1
        if n > 2:
            table[parent[1], -1] = total + 3
            own = int(table[parent[2], kv[2] // page]) if kv[2] % page else -1
            if own not in [int(f) for f in fresh] and parent[2] != parent[1]:
                fresh[2] = own                  # the child keeps its parent's page
    dst = np.full((n, width), 77, np.int32)
    dk, dvv, dd = k.cuda(), v.cuda(), torch.from_numpy(dst).cuda()
    cache = dv.KvCache(dk, dvv, torch.from_numpy(table).cuda(), CODE[dtype])
    dv.davet_cache_reorder(cache, kv, torch.from_numpy(parent).cuda(),
                           torch.from_numpy(fresh).cuda(), dd)
    rk, rv, rd = oc.reorder(dict(k=f64(k), v=f64(v), table=table), kv, parent, fresh, dst)
    assert np.array_equal(dd.cpu().numpy(), rd)
    assert np.array_equal(f64(dk), rk) and np.array_equal(f64(dvv), rv)
    assert np.array_equal(cache.page_table.cpu().numpy(), table)


def test_more_rows_than_one_reordering_takes():
    """Twenty requests of four beams: one selection, the cache moved in two calls of
    whole requests, with the first row of each taken off the parents."""
    rng = np.random.default_rng(5)
    groups, beams, kv, page = 20, 4, 37, 16
    rows = groups * beams
    total, table = page_table(rng, [kv] * rows, page, extra=rows)
    free = np.array([p for p in range(total) if p not in table], np.int32)
    k, v = (values(rng, (total, 2, page, 64), "f16") for _ in range(2))
    dk, dvv, dtable = k.cuda(), v.cuda(), torch.from_numpy(table).cuda()
    x, scores = values(rng, (rows, 50), "f32", 3.0), values(rng, (rows,), "f32")
    o, r, _ = select(x.cuda(), "f32", scores, beams, beams)
    parents, fresh = torch.from_numpy(r).cuda().view(-1), torch.from_numpy(free).cuda()
    dst = torch.full((rows, table.shape[1]), 77, dtype=torch.int32, device="cuda")
    for n in range(0, rows, 64):
        m = slice(n, min(n + 64, rows))
        cache = dv.KvCache(dk, dvv, dtable[m], dv.DAVET_F16)
        dv.davet_cache_reorder(cache, [kv] * (m.stop - n), parents[m] - n, fresh[m],
                               dst[m])
    want = np.full(dst.shape, 77, np.int32)
    rk, rv, rd = oc.reorder(dict(k=f64(k), v=f64(v), table=table), [kv] * rows,
                            r.reshape(-1), free, want)
    assert np.array_equal(dst.cpu().numpy(), rd)
    assert np.array_equal(f64(dk), rk) and np.array_equal(f64(dvv), rv)


def test_steps_of_a_search():
    """Two requests, three beams, five tokens over two layers: selection, reordering,
    append, attention.  The cache a beam ends with is that of its own tokens alone."""
    rng = np.random.default_rng(4)
    beams, groups, vocab, heads, dim, page, past = 3, 2, 700, 2, 64, 16, 29
    rows, layers, steps = beams * groups, 2, 5
    width = -(-(past + steps) // page)
    # a prompt's pages are shared by its beams; each has a last one to itself
    total = groups + rows + 2 * rows + rows * steps
    table = np.full((rows, width), -1, np.int32)
    nxt = iter(rng.permutation(total))
    for g in range(groups):
        whole = next(nxt)
        for b in range(beams):
            table[g * beams + b, :2] = whole, next(nxt)
    embed = values(rng, (vocab, layers, 3 * heads * dim), "f16").cuda()
    head = values(rng, (vocab, heads * dim), "f32", 0.3).cuda()
    prompt = values(rng, (groups, past, layers, 3 * heads * dim), "f16").cuda()
    pools = [[torch.zeros(total, heads, page, dim, dtype=torch.float16, device="cuda")
              for _ in range(2)] for _ in range(layers)]
    tables = [torch.from_numpy(table).cuda(), torch.full((rows, width), -1,
                                                         dtype=torch.int32).cuda()]
    q = torch.empty(rows * past, heads * dim, dtype=torch.float16, device="cuda")
    cu = list(range(0, rows * past + 1, past))
    for (k, v), l in zip(pools, range(layers)):
        qkv = prompt[:, :, l].repeat_interleave(beams, 0).reshape(rows * past, -1)
        # (beams write the same values to the page they share: one at a time)
        for b in range(beams):
            mine = [g * beams + b for g in range(groups)]
            c = dv.KvCache(k, v, tables[0][mine].contiguous(), dv.DAVET_F16)
            part = qkv.view(rows, past, -1)[mine].reshape(groups * past, -1)
            dv.davet_cache_append(c, [0, past, 2 * past], [past, past], part, heads, q)
    ws = torch.empty(max(dv.davet_beam_workspace_bytes(groups, beams, vocab, beams),
                         dv.davet_cache_workspace_bytes(heads, dim, rows)),
                     dtype=torch.uint8, device="cuda")
    scores = torch.zeros(rows, device="cuda")
    scores.view(groups, beams)[:, 1:] = float("-inf")     # at first one beam counts
    logits = values(rng, (rows, vocab), "f32", 2.0).cuda()
    o_rows, o_tok = (torch.empty(groups, beams, dtype=torch.int32, device="cuda")
                     for _ in range(2))
    texts, at = [[] for _ in range(rows)], past
    for _ in range(steps):
        dv.davet_beam_select(logits, dv.DAVET_F32, scores, beams,
                             scores.view(groups, beams), o_rows, o_tok, workspace=ws)
        parents, toks = o_rows.view(-1).tolist(), o_tok.view(-1)
        texts = [texts[p] + [t] for p, t in zip(parents, toks.tolist())]
        fresh = torch.tensor([next(nxt) for _ in range(rows)], dtype=torch.int32).cuda()
        old, new = tables
        for k, v in pools:
            dv.davet_cache_reorder(dv.KvCache(k, v, old, dv.DAVET_F16), [at] * rows,
                                   o_rows.view(-1), fresh, new)
        if at % page == 0:                  # the next token opens a page
            new[:, at // page] = fresh
        tables = [new, old]
        at += 1
        logits = torch.zeros(rows, vocab, device="cuda")
        for l, (k, v) in enumerate(pools):
            c = dv.KvCache(k, v, new, dv.DAVET_F16)
            qkv, qq = embed[toks.long(), l].contiguous(), q[:rows]
            out = torch.empty_like(qq)
            one = list(range(rows + 1))
            dv.davet_cache_append(c, one, [at] * rows, qkv, heads, qq)
            dv.davet_cache_attention(c, one, [at] * rows, qq, heads, out, workspace=ws)
            logits += out.float() @ head.t()
    assert len({tuple(x) for x in texts[:beams]}) == beams
    for r, text in enumerate(texts):
        for l, (k, v) in enumerate(pools):
            qkv = torch.cat([prompt[r // beams, :, l], embed[text, l]])
            t = torch.arange(width, dtype=torch.int32, device="cuda")[None]
            ck, cvv = (torch.zeros(width, heads, page, dim, dtype=torch.float16,
                                   device="cuda") for _ in range(2))
            c = dv.KvCache(ck, cvv, t, dv.DAVET_F16)
            dv.davet_cache_append(c, [0, at], [at], qkv, heads, torch.empty(
                at, heads * dim, dtype=torch.float16, device="cuda"))
            for j in range(at):
                p = tables[0][r, j // page]
                assert torch.equal(k[p, :, j % page], ck[j // page, :, j % page]), (r, j)
                assert torch.equal(v[p, :, j % page], cvv[j // page, :, j % page])


def test_captured_and_on_a_stream():
    rng = np.random.default_rng(9)
    x = values(rng, (8, 20000), "bf16", 3.0).cuda()
    scores = torch.zeros(8, device="cuda")
    ws = torch.empty(dv.davet_beam_workspace_bytes(2, 4, 20000, 4), dtype=torch.uint8,
                     device="cuda")
    o = torch.zeros(2, 4, device="cuda")
    r, t = (torch.zeros(2, 4, dtype=torch.int32, device="cuda") for _ in range(2))

    def step(stream=None, w=ws):
        dv.davet_beam_select(x, dv.DAVET_BF16, scores, 4, o, r, t, workspace=w,
                             stream=stream)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    side = torch.cuda.Stream()
    for i in range(3):
        x.copy_(values(rng, (8, 20000), "bf16", 3.0))
        torch.cuda.synchronize()
        step(side, torch.empty_like(ws))
        side.synchronize()
        want = o.clone(), r.clone(), t.clone()
        for a in (o, r, t):
            a.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((o, r, t), want)), i
