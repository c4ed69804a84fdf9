"""davet_cache_page_bounds, davet_cache_page_select and davet_cache_page_attention
against the float64 oracle: types, head layouts, lengths from one token on, page sizes,
blocks, holes, lists of any kind, values that must not leak."""

import numpy as np
import pytest
import torch

import paper_2608_01821_amd as dv
from cache_util import CODE, TORCH, Setup, check_attention, f64, page_table, values
from oracle import cache as oc

pytestmark = pytest.mark.gpu


def fresh_bounds(s, seed=1):
    """Values of their own everywhere, so that what is left alone shows."""
    n, hk, _, d = s.k.shape
    return values(np.random.default_rng(seed), (n, hk, 2, d), s.dtype)


def whole_bounds(s):
    """Of every page of the sequences, by the call, checked."""
    b = fresh_bounds(s)
    cu = [0] + [int(x) for x in np.cumsum(s.kv)]
    db = b.cuda()
    dv.davet_cache_page_bounds(s.device(), cu, s.kv, db)
    want = oc.page_bounds(s.host, cu, s.kv, f64(b))
    assert np.array_equal(f64(db), want)
    return db, want


BOUNDS = [  # dtype, new, kv, kv_heads, dim, page
    ("f16", [1], [1], 1, 64, 16),
    ("f16", [1], [2965], 8, 128, 64),
    ("bf16", [5, 0, 17, 1], [5, 3, 40, 33], 2, 128, 16),
    ("f32", [9, 3], [9, 67], 4, 64, 32),
    ("f32", [300], [300], 1, 128, 256),
    ("f16", [33, 30], [33, 61], 4, 64, 128),
    ("bf16", [700], [1000], 2, 64, 32),
    ("f32", [64, 1], [64, 65], 3, 128, 64),
]


@pytest.mark.parametrize("case", BOUNDS, ids=str)
def test_bounds(case):
    dtype, new, kv, hk, dim, page = case
    s = Setup(sum(kv), dtype, new, kv, hk, hk, dim, page)
    if len(new) > 1:
        s.table[1, 0] = -1 if kv[1] > 3 else 10 ** 6
    b = fresh_bounds(s)
    db = b.cuda()
    dv.davet_cache_page_bounds(s.device(), s.cu, s.kv, db)
    assert np.array_equal(f64(db), oc.page_bounds(s.host, s.cu, s.kv, f64(b)))
    # without values, and again: the same
    cache = dv.KvCache(s.dk, None, s.dtable, CODE[dtype])
    again = db.clone()
    dv.davet_cache_page_bounds(cache, s.cu, s.kv, again)
    assert torch.equal(again, db)


def test_bounds_of_values_that_are_not_finite():
    s = Setup(1, "f16", [40], [40], 2, 2, 64, 16, fill=float("nan"))
    p = s.table[0]
    s.k[p[0], 0, 3, 7], s.k[p[1], 1, 0, 0] = float("nan"), float("inf")
    s.k[p[2], 0, 7, 1] = -float("inf")
    db = fresh_bounds(s).cuda()
    dv.davet_cache_page_bounds(s.device(), s.cu, s.kv, db)
    got = f64(db)
    assert np.isnan(got[p[0], 0, :, 7]).all()
    assert got[p[1], 1, 1, 0] == np.inf and np.isfinite(got[p[1], 1, 0, 0])
    assert got[p[2], 0, 0, 1] == -np.inf
    got[p[0], 0, :, 7] = got[p[1], 1, 1, 0] = got[p[2], 0, 0, 1] = 0
    assert np.isfinite(got[p[:3]]).all()        # nothing from behind the last token


SELECT = [  # dtype, new, kv, heads, kv_heads, dim, page, block, top, first, last
    ("f16", [1], [1], 1, 1, 64, 16, 0, 1, 0, 0),
    ("f16", [1], [700], 8, 2, 128, 16, 1, 8, 1, 2),
    ("bf16", [1, 1, 1], [31, 700, 400], 4, 2, 128, 16, 1, 3, 0, 0),
    ("f32", [1, 2], [1500, 9], 2, 1, 128, 16, 1, 20, 2, 3),
    ("f32", [3], [1100], 4, 4, 64, 16, 0, 5, 5, 0),
    ("f16", [5, 0, 3], [600, 7, 300], 6, 2, 64, 32, 1, 4, 0, 4),
    ("bf16", [33], [1050], 7, 1, 64, 16, 4, 64, 1, 1),
    ("f16", [2], [16 * 70], 4, 1, 128, 16, 1, 69, 1, 1),     # all but one
    ("f16", [2], [16 * 70], 4, 1, 128, 16, 1, 70, 1, 1),     # all
    ("f16", [1], [16 * 1023 + 5], 1, 1, 64, 16, 0, 1000, 0, 0),
    ("bf16", [1], [16 * 5000], 2, 1, 64, 16, 0, 300, 1, 1),  # more than 4096 pages
    ("f32", [1], [16 * 4200], 1, 1, 64, 16, 0, 7, 0, 0),
    ("f16", [40], [60], 32, 1, 64, 16, 1, 2, 1, 1),
    # many tokens and key heads: a wavefront each
    ("f16", [140, 3], [700, 333], 8, 8, 64, 16, 1, 6, 1, 1),
    ("bf16", [33], [1600], 64, 32, 128, 16, 4, 40, 0, 2),
    ("f32", [70], [16 * 64], 16, 16, 64, 16, 1, 63, 0, 0),
    ("f32", [34], [530], 32, 32, 128, 16, 0, 5, 2, 0),
    ("f16", [2], [16 * 512], 1024, 1024, 64, 16, 0, 7, 0, 1),
    ("bf16", [5] * 8, [100, 200, 31, 500, 5, 77, 333, 480], 32, 32, 128, 16, 1, 6, 1, 2),
    ("f32", [7] * 10, [210] * 10, 16, 16, 64, 16, 4, 5, 0, 1),
    ("f32", [7] * 5, [210] * 5, 30, 30, 128, 16, 1, 13, 0, 1),
    # 16 tokens at a time over up to 1024 pages
    ("f16", [20], [16 * 700], 2, 1, 64, 16, 1, 30, 1, 1),
    ("f32", [9, 1], [16 * 600, 50], 4, 2, 128, 16, 0, 3, 0, 0),
    ("bf16", [8, 0, 17], [16 * 1024, 0, 400], 3, 1, 128, 16, 1, 500, 1, 1),
    # and many of those
    ("f16", [70], [16 * 700], 32, 16, 64, 16, 1, 30, 1, 1),
    ("f32", [35, 1], [16 * 520, 50], 32, 32, 64, 16, 0, 3, 0, 0),
    ("bf16", [64, 0, 17], [16 * 1024, 0, 400], 16, 16, 64, 16, 1, 500, 1, 1),
    # every sequence there may be
    ("f16", [1] * 64, [17 * i + 1 for i in range(64)], 4, 2, 64, 16, 1, 9, 1, 1),
    ("f32", [i % 3 for i in range(64)], [10 * i + 2 for i in range(64)], 16, 16, 64, 16,
     1, 4, 0, 2),
    ("bf16", [8, 0] * 32, [7 * i + 8 for i in range(64)], 4, 4, 64, 16, 0, 5, 1, 0),
]


def select(s, db, top, first, last, block):
    rows, hk = s.cu[-1], s.k.shape[1]
    pages = torch.full((rows + 1, hk, top), 7, dtype=torch.int32, device="cuda")
    dv.davet_cache_page_select(s.device(), s.cu, s.kv, s.q.cuda(), s.heads, db, pages,
                               first=first, last=last, block=block)
    assert (pages[rows:] == 7).all()
    return pages[:rows]


@pytest.mark.parametrize("case", SELECT, ids=str)
def test_select(case):
    dtype, new, kv, heads, hk, dim, page, block, top, first, last = case
    s = Setup(sum(kv) + top, dtype, new, kv, heads, hk, dim, page)
    db, b = whole_bounds(s)
    if max(kv) > 500:
        hole = s.table[kv.index(max(kv))]
        hole[3], hole[5] = -1, 2 ** 31 - 1
    got = select(s, db, top, first, last, block).cpu().numpy()
    want = oc.page_select(s.host, s.cu, s.kv, f64(s.q), heads, b, top, first, last,
                          block)
    for r, row in enumerate(want):
        for h, ps in enumerate(row):
            assert got[r, h].tolist() == ps + [-1] * (top - len(ps)), (r, h)


@pytest.mark.parametrize("dtype,dim", [("f16", 128), ("f16", 64), ("f32", 64),
                                       ("f32", 128)])
def test_equal_and_odd_scores(dtype, dim):
    """Ties go to the lower page; a page whose score is NaN comes last, before none."""
    s = Setup(2, dtype, [2], [16 * 90 + 3], 2, 1, dim, 16)
    s.q[:] = 1.0
    s.k[:] = 0.5
    p = s.table[0]
    s.k[p[40]] = 0.75
    s.k[p[7], 0, 2, 5] = float("nan")
    s.k[p[41], 0, 2, 5] = float("inf")
    s.k[p[88], 0] = -1.0
    cu = [0, s.kv[0]]
    db = fresh_bounds(s).cuda()
    dv.davet_cache_page_bounds(s.device(), cu, s.kv, db)
    got = select(s, db, 6, 0, 0, 0)
    assert got[0, 0].tolist() == [0, 1, 2, 3, 40, 41] == got[1, 0].tolist()
    got = select(s, db, 90, 0, 0, 0)            # all but the NaN
    assert got[0, 0].tolist() == [j for j in range(91) if j != 7]
    got = select(s, db, 89, 0, 0, 0)
    assert got[0, 0].tolist() == [j for j in range(91) if j not in (7, 88)]
    got = select(s, db, 8, 8, 0, 0)             # sure ones, whatever their score
    assert got[0, 0].tolist() == list(range(8))
    s.q[0, 3] = float("nan")                    # nothing to rank by: the first ones
    got = select(s, db, 5, 1, 2, 0)
    assert got[0, 0].tolist() == [0, 1, 2, 89, 90]


@pytest.mark.parametrize("dtype,dim", [("f16", 128), ("bf16", 64), ("f32", 64),
                                       ("f32", 128)])
@pytest.mark.parametrize("new,hk", [(2, 2), (5, 256), (16, 64)],
                         ids=["group", "waves", "tiles"])
def test_scores_of_infinite_bounds(dtype, dim, new, hk):
    """The score is the sum of max(q lo, q hi) also where a bound is infinite: a -inf
    among the keys is nothing to a positive element of the query, +inf nothing to a
    negative one; an element of 0 makes it NaN, which comes last."""
    s = Setup(5 + dim, dtype, [new], [16 * 40 + 3], 2 * hk, hk, dim, 16)
    rng, heads = s.rng, s.q.view(new, hk, 2, dim)
    heads[:, ::2, 1] = heads[:, ::2, 0].abs() * heads[:, ::2, 1].sign()
    heads[:, :, 0, 3] = heads[:, :, 1, 3] = 0.0
    same = torch.from_numpy(rng.random((hk, dim)) < 0.7)    # both heads of one sign
    heads[:, :, 1] = torch.where(same, heads[:, :, 1].abs() * heads[:, :, 0].sign(),
                                 heads[:, :, 1])
    inf = float("inf")
    for h in range(hk):
        for j in rng.permutation(41)[:24]:
            page, e = s.table[0, j], int(rng.integers(0, dim))
            kind = rng.random()
            if kind < 0.9:                      # (most under a sign that ignores it)
                up = rng.random() < (0.8 if heads[0, h, 0, e] < 0 else 0.2)
                s.k[page, h, int(rng.integers(0, 3)), e] = inf if up else -inf
            elif kind < 0.95:                   # either bound
                s.k[page, h, 0, e], s.k[page, h, 1, e] = inf, -inf
            else:                               # no other value
                s.k[page, h, :, e] = inf if rng.random() < 0.5 else -inf
    db, b = whole_bounds(s)
    with np.errstate(invalid="ignore"):
        for top, first, last in ((9, 0, 0), (30, 1, 2)):
            got = select(s, db, top, first, last, 0).cpu().numpy()
            want = oc.page_select(s.host, s.cu, s.kv, f64(s.q), 2 * hk, b, top, first,
                                  last)
            for r, row in enumerate(want):
                for h, ps in enumerate(row):
                    assert got[r, h].tolist() == ps, (r, h, top)


def test_close_scores_do_not_depend_on_order():
    """Pages whose scores differ by less than float32 sums of their terms would be off
    by: chosen as in float64."""
    s = Setup(3, "f16", [1], [16 * 200], 4, 1, 128, 16, q_std=3.0)
    base = s.k[s.table[0, 0], 0, 0].clone()
    s.k[:] = base
    for j in range(200):                        # one last bit of one element
        e = int(s.rng.integers(0, 128))
        bits = s.k[s.table[0, j], 0].view(torch.int16)
        bits[:, e] += 1 if s.rng.random() < 0.5 else -1
    db, b = whole_bounds(s)
    got = select(s, db, 64, 0, 0, 0).cpu().numpy()
    want = oc.page_select(s.host, s.cu, s.kv, f64(s.q), 4, b, 64)
    assert got[0, 0].tolist() == want[0][0]


@pytest.mark.parametrize("dtype,dim", [("f16", 128), ("bf16", 64), ("f32", 64),
                                       ("f32", 128)])
def test_the_batch_around_it_does_not_change_a_choice(dtype, dim):
    """The same five rows by a workgroup each, by a wavefront each (seven such sequences)
    and in tiles (a longer chunk beside them).  16-bit values of a coarse grid: every sum
    is exact, the lists are equal.  fp32: every form's pages are the best ones up to the
    roundings of a score (to float32, and of at most 4 dim products and sums in
    float64)."""
    hk, heads, np_, top = 32, 64, 300, 40
    s = Setup(dim, dtype, [5, 40], [16 * np_, 60], heads, hk, dim, 16)
    if dtype != "f32":
        s.q[:], s.k[:] = (s.q * 8).round() / 8, (s.k * 8).round() / 8
    db, b = whole_bounds(s)
    q, table = s.q.cuda(), torch.from_numpy(s.table).cuda()
    got = []
    for rows, kv, tables in (
            ([5], [16 * np_], table[:1]),
            ([5] * 7, [16 * np_] * 7, table[:1].repeat(7, 1)),
            ([5, 40], [16 * np_, 60], table)):
        cu = [0] + [int(x) for x in np.cumsum(rows)]
        cache = dv.KvCache(s.dk, s.dv, tables.contiguous(), CODE[dtype])
        x = q[:5].repeat(7, 1) if len(rows) == 7 else q[:cu[-1]]
        pages = torch.full((cu[-1], hk, top), 7, dtype=torch.int32, device="cuda")
        dv.davet_cache_page_select(cache, cu, kv, x, heads, db, pages)
        got += [p.cpu().numpy() for p in pages[:35 if len(rows) == 7 else 5].split(5)]
    if dtype != "f32":
        for p in got[1:]:
            assert np.array_equal(p, got[0])
        return
    lo, hi = np.moveaxis(b[s.table[0]].astype(np.longdouble), 2, 0)     # [pages, hk, D]
    qs = f64(s.q)[:5].astype(np.longdouble).reshape(5, hk, 2, 1, dim)
    lo, hi = (np.moveaxis(x, 1, 0)[:, None] for x in (lo, hi))          # [hk, 1, pages, D]
    score = np.maximum(qs * lo, qs * hi).sum((2, 4))                    # [5, hk, pages]
    mass = (np.abs(qs) * np.maximum(np.abs(lo), np.abs(hi))).sum((2, 4))
    off = 2.0 ** -24 * np.abs(score) + 4 * dim * 2.0 ** -53 * mass
    for p in got:
        took = np.zeros(score.shape, bool)
        np.put_along_axis(took, p, True, 2)
        assert (took.sum(2) == top).all()
        least = np.where(took, score + off, np.inf).min(2)
        assert (least >= np.where(took, -np.inf, score - off).max(2)).all()


ATTEND = [  # dtype, new, kv, heads, kv_heads, dim, page, block, top
    ("f16", [1], [1], 1, 1, 64, 16, 0, 1),
    ("f16", [1], [700], 8, 2, 128, 16, 1, 8),
    ("f16", [1], [701], 8, 8, 128, 64, 0, 5),
    ("bf16", [1, 1, 1], [31, 700, 400], 4, 2, 128, 16, 1, 3),
    ("f32", [1, 2], [1500, 9], 2, 1, 128, 16, 1, 60),
    ("f32", [3], [300], 4, 4, 64, 32, 0, 5),
    ("f16", [5, 0, 3], [600, 7, 300], 6, 2, 64, 128, 1, 2),
    ("bf16", [33], [250], 7, 1, 64, 16, 4, 7),
    ("f16", [9], [200], 40, 1, 64, 16, 1, 6),               # two row tiles a token
    ("f16", [2], [2000], 4, 1, 128, 16, 1, 64),             # pieces
    ("bf16", [1], [3000], 2, 1, 64, 256, 0, 11),
    ("f32", [40], [90], 2, 2, 64, 16, 1, 3),
    # lists of more than 1024 keys: pieces
    ("f16", [1], [1500], 8, 2, 128, 64, 1, 20),
    ("bf16", [2, 1], [1300, 2100], 4, 4, 64, 16, 0, 100),
    ("f32", [1], [1400], 2, 1, 128, 256, 0, 6),
    ("f32", [3], [1300], 3, 1, 64, 16, 1, 80),
    # lists enough for a wavefront each
    ("f16", [260, 1], [300, 40], 8, 8, 64, 16, 1, 4),
    ("bf16", [33], [400], 128, 64, 128, 32, 0, 5),
    ("f32", [70], [100], 64, 32, 64, 16, 4, 3),
    ("f32", [66], [90], 32, 32, 128, 16, 1, 2),
    ("f16", [130], [140], 320, 16, 64, 16, 0, 3),           # two row tiles each
    # more than one a CU, of few keys
    ("f16", [70, 1], [300, 40], 8, 8, 64, 16, 1, 4),
    ("bf16", [40], [900], 20, 10, 128, 32, 0, 20),
    ("f32", [33], [1000], 16, 16, 64, 16, 4, 40),
    # every sequence there may be
    ("f16", [1] * 64, [17 * i + 1 for i in range(64)], 8, 2, 128, 16, 1, 9),
    ("bf16", [i % 3 for i in range(64)], [10 * i + 2 for i in range(64)], 4, 4, 64, 16, 1,
     7),
]


def lists(s, block, top, kind):
    """[rows][heads] page lists as a program might hold them."""
    rng, rows = s.rng, []
    size = s.k.shape[2]
    for i, kv in enumerate(s.kv):
        n, np_ = s.cu[i + 1] - s.cu[i], -(-kv // size)
        for r in range(n):
            row = []
            for _ in range(s.k.shape[1]):
                if kind == "some":              # ascending, then -1
                    m = int(rng.integers(0, min(top, np_) + 1))
                    ps = sorted(rng.permutation(np_)[:m].tolist())
                    ps += [-1] * (top - m)
                else:                           # anything, anywhere
                    ps = rng.integers(-2, np_ + 3, top).tolist()
                    if r % 2:
                        ps[0] = 2 ** 31 - 1
                row.append(ps)
            rows.append(row)
    return rows


def attend(s, rows, block, cache=None):
    q, hk = s.q.cuda(), s.k.shape[1]
    out = torch.full((len(q) + 1, q.shape[1]), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((len(q) + 1, s.heads), 7.0, device="cuda")
    pages = torch.tensor(rows, dtype=torch.int32).cuda()
    dv.davet_cache_page_attention(cache or s.device(), s.cu, s.kv, q, s.heads, pages,
                                  out[:len(q)], lse=lse[:len(q)], block=block,
                                  workspace=s.workspace())
    torch.cuda.synchronize()
    assert (out[len(q):] == 7).all() and (lse[len(q):] == 7).all()
    return f64(out)[:len(q)].reshape(len(q), s.heads, -1), f64(lse)[:len(q)]


def seen_by(s, rows, block):
    size = s.k.shape[2]

    def seen(i, r, h):
        kv, n = s.kv[i], s.cu[i + 1] - s.cu[i]
        end = kv if block == 0 else kv - n + min(n, (r // block + 1) * block)
        np_ = -(-kv // size)
        return [j for p in rows[s.cu[i] + r][h][:np_] if 0 <= p < np_
                for j in range(p * size, min(end, p * size + size))]
    return seen


@pytest.mark.parametrize("case", ATTEND, ids=str)
@pytest.mark.parametrize("kind", ["some", "any"])
def test_attention(case, kind):
    dtype, new, kv, heads, hk, dim, page, block, top = case
    s = Setup(sum(kv) + heads, dtype, new, kv, heads, hk, dim, page, fill=float("nan"))
    if max(kv) > 300:
        s.table[kv.index(max(kv)), 1] = -1
    rows = lists(s, block, top, kind)
    ref = oc.attention_of(s.host, s.cu, s.kv, f64(s.q), heads, seen_by(s, rows, block))
    check_attention(attend(s, rows, block), ref, dtype, dim, top * page)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_values_that_are_not_seen(dtype):
    """Infinities behind the visible end of a page, and in pages that are not listed,
    reach nobody; a listed and visible one reaches its rows, as an infinity or NaN (a
    probability is the sum of two 16-bit operands, the second of either sign or 0: an
    infinity times both may be NaN).  A row that sees no key is zeros, its lse -inf."""
    s = Setup(5, dtype, [8], [40], 2, 1, 64, 16)
    s.v[s.table[0, 2], 0, 3] = float("inf")     # index 35: visible from row 3 on
    s.v[s.table[0, 0], 0, 5] = float("nan")     # page 0 is listed by row 7 alone
    rows = [[[1, 2, -1]] for _ in range(8)]
    rows[5] = [[-1, 9, -1]]
    rows[7] = [[0, 1, 2]]
    out, lse = attend(s, rows, 1)
    for r in range(8):
        if r < 3:
            assert np.isfinite(out[r]).all()
        elif r == 5:
            assert (out[r] == 0).all() and np.isneginf(lse[r]).all()
        elif r == 7:
            assert np.isnan(out[r]).all()
        else:
            assert not np.isfinite(out[r]).any()
        assert r == 5 or np.isfinite(lse[r]).all()


@pytest.mark.parametrize("dtype,block", [("f16", 1), ("bf16", 0), ("f32", 4)])
def test_append_bounds_select_attend(dtype, block):
    """Token by token through append, bounds, selection and attention as a program
    runs them; where every page is taken the result is that of the whole cache."""
    rng = np.random.default_rng(6)
    heads, hk, dim, page, past, n = 4, 2, 64, 16, 150, 9
    total, table = page_table(rng, [past + n], page)
    k, v = (values(rng, (total, hk, page, dim), dtype).cuda() for _ in range(2))
    cache = dv.KvCache(k, v, torch.from_numpy(table).cuda(), CODE[dtype])
    bounds = torch.zeros(total, hk, 2, dim, dtype=TORCH[dtype], device="cuda")
    dv.davet_cache_page_bounds(cache, [0, past], [past], bounds)
    ws = torch.empty(dv.davet_cache_workspace_bytes(heads, dim, n), dtype=torch.uint8,
                     device="cuda")
    at = past
    for m in (1, 1, 7):                         # two tokens one by one, then seven
        at += m
        cu, kv = [0, m], [at]
        qkv = values(rng, (m, (heads + 2 * hk) * dim), dtype).cuda()
        q = torch.empty(m, heads * dim, dtype=TORCH[dtype], device="cuda")
        out, lse = torch.empty_like(q), torch.empty(m, heads, device="cuda")
        dv.davet_cache_append(cache, cu, kv, qkv, heads, q)
        dv.davet_cache_page_bounds(cache, cu, kv, bounds)
        host = dict(k=f64(k), v=f64(v), table=table)
        want = oc.page_bounds(host, [0, at], [at], f64(bounds))
        assert np.array_equal(f64(bounds), want)
        for top in (4, 30):
            pages = torch.empty(m, hk, top, dtype=torch.int32, device="cuda")
            dv.davet_cache_page_select(cache, cu, kv, q, heads, bounds, pages, first=1,
                                       last=1, block=block)
            sel = oc.page_select(host, cu, kv, f64(q), heads, want, top, 1, 1, block)
            assert [[h[h >= 0].tolist() for h in r] for r in pages.cpu()] == sel
            dv.davet_cache_page_attention(cache, cu, kv, q, heads, pages, out, lse=lse,
                                          block=block, workspace=ws)
            got = f64(out).reshape(m, heads, dim), f64(lse)

            def seen(_, r, h):
                end = at if block == 0 else at - m + min(m, (r // block + 1) * block)
                return [j for p in sel[r][h]
                        for j in range(p * page, min(end, p * page + page))]
            ref = oc.attention_of(host, cu, kv, f64(q), heads, seen)
            check_attention(got, ref, dtype, dim, at)
        whole = oc.attention(host, cu, kv, f64(q), heads, block=block)
        check_attention(got, whole, dtype, dim, at)


def test_far_pages_need_64_bit_offsets():
    """Pages behind the 2^32nd byte of the bounds, all at the pools' end."""
    hk, d, size = 8, 128, 16
    s = Setup(3, "f32", [2, 1], [300, 45], 8, hk, d, size)
    n = (1 << 32) // (hk * 2 * d * 4) + 40
    far = s.table.copy()
    far[far >= 0] += n - s.k.shape[0]
    pool = torch.empty(n, hk, size, d, device="cuda")
    pool[n - s.k.shape[0]:] = s.k.cuda()        # (keys and values alike)
    cache = dv.KvCache(pool, pool, torch.from_numpy(far).cuda(), dv.DAVET_F32)
    bounds = torch.empty(n, hk, 2, d, device="cuda")
    cu = [0, 300, 345]
    dv.davet_cache_page_bounds(cache, cu, s.kv, bounds)
    last = bounds[n - s.k.shape[0]:]
    db, b = whole_bounds(s)
    used = sorted({int(p) for p in s.table.reshape(-1) if p >= 0})
    assert torch.equal(last[used], db[used])
    q, rows = s.q.cuda(), s.cu[-1]
    pages = torch.empty(rows, hk, 4, dtype=torch.int32, device="cuda")
    dv.davet_cache_page_select(cache, s.cu, s.kv, q, 8, bounds, pages, first=1, last=1)
    want = oc.page_select(s.host, s.cu, s.kv, f64(s.q), 8, b, 4, 1, 1, 0)
    assert [[h[h >= 0].tolist() for h in r] for r in pages.cpu()] == want
    got = attend(s, [[h + [-1] * (4 - len(h)) for h in r] for r in want], 0, cache)
    host = dict(s.host, v=s.host["k"])
    ref = oc.attention_of(host, s.cu, s.kv, f64(s.q), 8, seen_by(s, want, 0))
    check_attention(got, ref, "f32", d, 64)


def test_two_streams_and_captured():
    s = Setup(7, "f16", [1, 1], [900, 500], 8, 2, 128, 16)
    cache = s.device()
    db, _ = whole_bounds(s)
    q = s.q.cuda()
    pages = torch.zeros(2, 2, 12, dtype=torch.int32, device="cuda")
    out, lse, ws = torch.zeros_like(q), torch.zeros(2, 8, device="cuda"), s.workspace()

    def step(p, o, e, w, stream=None):
        dv.davet_cache_page_bounds(cache, s.cu, s.kv, db, stream=stream)
        dv.davet_cache_page_select(cache, s.cu, s.kv, q, 8, db, p, first=1, last=1,
                                   stream=stream)
        dv.davet_cache_page_attention(cache, s.cu, s.kv, q, 8, p, o, lse=e, workspace=w,
                                      stream=stream)
    step(pages, out, lse, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(pages, out, lse, ws)
    side = torch.cuda.Stream()
    for i in range(3):
        q.copy_(values(s.rng, q.shape, "f16", 2.0))
        p2, o2, e2, w2 = (torch.zeros_like(x) for x in (pages, out, lse, ws))
        torch.cuda.synchronize()
        step(p2, o2, e2, w2, side)
        side.synchronize()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(pages, p2) and torch.equal(out, o2) and torch.equal(lse, e2), i
