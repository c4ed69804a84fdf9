"""davet_tree_plan and davet_cache_tree_attention against the float64 oracle: shapes of
trees, types, head layouts, lengths, pages, holes, masks that leave a row empty, values
that masked places must not leak, and a whole step of drafting."""

import numpy as np
import pytest
import torch

import paper_2608_01821_amd as dv
from cache_util import CODE, Setup, check_attention, f64, page_table, values
from oracle import cache as oc

pytestmark = pytest.mark.gpu


def bits(rows_seen, n_rows):
    """int32 [rows, TREE_WORDS] with the named bits set."""
    m = np.zeros((n_rows, dv.TREE_WORDS), np.uint32)
    for r, js in enumerate(rows_seen):
        for j in js:
            m[r, j >> 5] |= np.uint32(1 << (j & 31))
    return torch.from_numpy(m.view(np.int32))


def draft(rng, n, kind):
    if kind == "chain":
        return list(range(-1, n - 1))
    if kind == "star":
        return [-1] * n
    if kind == "wild":                      # also entries that are no parents
        return [int(x) for x in rng.integers(-2 ** 31, 2 ** 31, n)]
    return [int(rng.integers(max(-1, i - 6), i)) for i in range(n)]


@pytest.mark.parametrize("kind", ["chain", "star", "bush", "wild"])
@pytest.mark.parametrize("new", [[1], [26, 0, 5], [64, 63, 65], [256, 1, 255], [31] * 64],
                         ids=str)
def test_plan(kind, new):
    rng = np.random.default_rng(len(new) + new[0])
    cu = [0] + [int(x) for x in np.cumsum(new)]
    kv = [n + int(rng.integers(0, 5000)) for n in new]
    parent = [draft(rng, n, kind) for n in new]
    flat = torch.tensor([p for x in parent for p in x], dtype=torch.int32).cuda()
    pos = torch.full((cu[-1] + 2,), 7, dtype=torch.int32, device="cuda")
    mask = torch.full((cu[-1] + 2, dv.TREE_WORDS), 7, dtype=torch.int32, device="cuda")
    dv.davet_tree_plan(cu, kv, flat, pos=pos, mask=mask)
    want = [[a for a in oc.above(p)] for p in parent]
    rows = [a for x in want for a in x]
    assert torch.equal(mask[:-2].cpu(), bits(rows, cu[-1]))
    first = [kv[s] - new[s] for s in range(len(new)) for _ in range(new[s])]
    assert pos[:-2].tolist() == [f + len(a) - 1 for f, a in zip(first, rows)]
    assert (pos[-2:] == 7).all() and (mask[-2:] == 7).all()
    # positions of their own, either output by itself
    own = [int(x) for x in rng.integers(-100, 10 ** 9, len(new))]
    got = torch.zeros_like(pos)
    dv.davet_tree_plan(cu, None, flat, pos=got, first_pos=own)
    f = [own[s] for s in range(len(new)) for _ in range(new[s])]
    assert got[:-2].tolist() == [x + len(a) - 1 for x, a in zip(f, rows)]
    again = torch.zeros_like(mask)
    dv.davet_tree_plan(cu, kv, flat, mask=again)
    assert torch.equal(again[:-2], mask[:-2])


CASES = [  # dtype, new, kv, heads, kv_heads, dim, page
    ("f16", [1], [1], 1, 1, 64, 16),
    ("f32", [13], [173], 4, 4, 64, 16),
    ("f16", [26], [700], 8, 2, 128, 64),              # wide
    ("bf16", [5, 0, 7], [5, 9, 40], 4, 2, 128, 16),   # nothing before the first tree
    ("f16", [32], [96], 1, 1, 128, 16),               # narrow's last, whole tiles
    ("f16", [33], [97], 1, 1, 128, 32),
    ("bf16", [31, 30], [64, 95], 1, 1, 64, 16),       # the tree crosses a tile
    ("f32", [64], [130], 1, 1, 128, 16),
    ("f32", [65, 70], [131, 70], 2, 2, 64, 64),       # wide
    ("f16", [256], [256], 1, 1, 128, 256),            # every bit
    ("bf16", [256, 255], [1000, 255], 2, 1, 128, 64),
    ("f16", [9], [2500], 7, 1, 64, 16),               # pieces, narrow or wide
    ("f16", [4], [2500], 8, 8, 128, 64),
    ("bf16", [129, 3], [700, 333], 6, 2, 64, 128),
    ("f16", [64] * 5, [300, 65, 64, 191, 257], 4, 2, 128, 16),
    ("f32", [200], [501], 2, 1, 128, 32),
    # every sequence there may be
    ("f16", [i % 4 for i in range(64)], [9 * i + 3 for i in range(64)], 4, 2, 64, 16),
    ("bf16", [i % 40 for i in range(64)], [5 * i + 40 for i in range(64)], 2, 1, 128, 32),
]


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("what", ["bush", "any"])
def test_attention(case, what):
    dtype, new, kv, heads, hk, dim, page = case
    s = Setup(sum(kv) + heads, dtype, new, kv, heads, hk, dim, page, fill=float("nan"))
    if what == "bush":
        rows = [a for n in new for a in oc.above(draft(s.rng, n, "bush"))]
    else:                                   # any bits, some rows without one
        rows = [[j for j in range(n) if s.rng.random() < 0.4 * (i % 3)]
                for n in new for i in range(n)]
    check(s, rows)


def check(s, rows, cache=None):
    kv, cu = s.kv, s.cu
    cache = cache or s.device()
    q = s.q.cuda()
    out = torch.full((len(q) + 1, q.shape[1]), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((len(q) + 1, s.heads), 7.0, device="cuda")
    mask = bits(rows, len(rows))
    for i, a in enumerate(rows):            # bits past the chunk: not looked at
        n = next(b - c for b, c in zip(cu[1:], cu) if b > i)
        for j in range(n, 256):
            mask[i, j >> 5] |= -2 ** 31 if j & 31 == 31 else 1 << (j & 31)
    dv.davet_cache_tree_attention(cache, cu, kv, q, s.heads, mask.cuda(), out[:len(q)],
                                  lse=lse[:len(q)], workspace=s.workspace())
    torch.cuda.synchronize()

    def seen(i, r, _):
        past = kv[i] - (cu[i + 1] - cu[i])
        return list(range(past)) + [past + j for j in rows[cu[i] + r]]
    ref = oc.attention_of(s.host, cu, kv, f64(s.q), s.heads, seen)
    assert (out[len(q):] == 7).all() and (lse[len(q):] == 7).all()
    got = f64(out)[:len(q)].reshape(len(q), s.heads, -1), f64(lse)[:len(q)]
    check_attention(got, ref, s.dtype, s.k.shape[3], max(kv))
    return got, ref


@pytest.mark.parametrize("dtype,new", [("f16", 5), ("f16", 50), ("f32", 5),
                                       ("f32", 70), ("bf16", 40)])
def test_values_that_are_not_seen(dtype, new):
    """Infinities and NaN in drafted tokens reach the rows that see them, and no
    others; a row that sees nothing is zeros, its lse -inf."""
    s = Setup(new, dtype, [new], [new + 40], 2, 1, 128, 16)
    bad = new + 40 - 2                      # the last but one drafted token
    page, off = s.table[0, bad // 16], bad % 16
    s.v[page, 0, off] = float("inf")
    s.v[page, 0, off, 1] = float("nan")
    rows = [list(range(i + 1)) for i in range(new)]
    rows[1] = [0, 1, new - 2]
    ref_rows = [[j for j in r if j != new - 2] for r in rows]
    q = s.q.cuda()
    for cut in (False, True):
        out, lse = torch.empty_like(q), torch.empty(new, 2, device="cuda")
        dv.davet_cache_tree_attention(s.device(), s.cu, s.kv, q, 2,
                                      bits(ref_rows if cut else rows, new).cuda(), out,
                                      lse=lse, workspace=s.workspace())
        o = f64(out).reshape(new, 2, 128)
        for i in range(new):
            hit = not cut and new - 2 in rows[i]
            assert np.isfinite(o[i]).all() != hit
            if hit:
                assert np.isnan(o[i, :, 1]).all() and np.isposinf(o[i, :, 2:]).all()
            assert np.isfinite(f64(lse)[i]).all()
    # nothing before the tree, a row without a bit
    s = Setup(new, dtype, [new], [new], 2, 1, 128, 16)
    s.v[s.table[0, 0], 0, 0] = float("inf")
    rows = [[] if i % 2 else [i, new - 1] for i in range(new)]
    rows[0] = []
    q = s.q.cuda()
    out, lse = torch.full_like(q, 7.0), torch.full((new, 2), 7.0, device="cuda")
    dv.davet_cache_tree_attention(s.device(), s.cu, s.kv, q, 2, bits(rows, new).cuda(),
                                  out, lse=lse, workspace=s.workspace())
    for i in range(new):
        assert bool((out[i] == 0).all()) == (not rows[i])
        assert bool(torch.isneginf(lse[i]).all()) == (not rows[i])


@pytest.mark.parametrize("new", [6, 60])
def test_holes(new):
    s = Setup(3, "f16", [new], [new + 70], 4, 2, 64, 16, fill=float("nan"))
    s.table[0, 1] = -1
    s.table[0, (new + 70) // 16 - 1] = 10 ** 6
    check(s, oc.above(draft(s.rng, new, "bush")))


@pytest.mark.parametrize("dtype,new", [("f16", 20), ("bf16", 50), ("f32", 40)])
def test_a_chain_is_the_causal_chunk(dtype, new):
    """Bit for bit: the same tiles in the same order."""
    s = Setup(new, dtype, [new, 3], [new + 333, 3], 4, 2, 128, 64)
    rows = [list(range(i + 1)) for n in (new, 3) for i in range(n)]
    want = s.attend(block=1)
    got, _ = check(s, rows)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


def test_a_step_of_drafting():
    """Plan, append at the tree's positions, attention; then the accepted path moved
    to the front by the gather, as a chain that had been there would be."""
    rng = np.random.default_rng(8)
    heads, hk, dim, page, past, n = 4, 2, 64, 16, 37, 12
    parent = [-1, 0, 0, 1, 1, 2, 3, 3, 5, 6, 7, -1]
    kv = past + n
    total, table = page_table(rng, [kv], page, extra=4)
    free = [p for p in range(total) if p not in table[0]]
    k, v = (values(rng, (total, hk, page, dim), "f16") for _ in range(2))
    dk, dvv = k.cuda(), v.cuda()
    cache = dv.KvCache(dk, dvv, torch.from_numpy(table).cuda(), dv.DAVET_F16)
    qkv = values(rng, (n, (heads + 2 * hk) * dim), "f16").cuda()
    pos = torch.empty(n, dtype=torch.int32, device="cuda")
    mask = torch.empty(n, dv.TREE_WORDS, dtype=torch.int32, device="cuda")
    q = torch.empty(n, heads * dim, dtype=torch.float16, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(n, heads, device="cuda")
    ws = torch.empty(dv.davet_cache_workspace_bytes(heads, dim, n), dtype=torch.uint8,
                     device="cuda")
    dv.davet_tree_plan([0, n], [kv], torch.tensor(parent, dtype=torch.int32).cuda(),
                       pos=pos, mask=mask)
    dv.davet_cache_append(cache, [0, n], [kv], qkv, heads, q, pos=pos)
    dv.davet_cache_tree_attention(cache, [0, n], [kv], q, heads, mask, out, lse=lse,
                                  workspace=ws)
    path = [0, 1, 3, 7, 10]                 # the accepted tokens, one below the other
    assert pos[path].tolist() == list(range(past, past + 5))
    # the same tokens as a chain, in a cache of its own
    ck, cvv = k.cuda(), v.cuda()
    chain = dv.KvCache(ck, cvv, cache.page_table, dv.DAVET_F16)
    q2 = torch.empty(5, heads * dim, dtype=torch.float16, device="cuda")
    out2, lse2 = torch.empty_like(q2), torch.empty(5, heads, device="cuda")
    dv.davet_cache_append(chain, [0, 5], [past + 5], qkv[path].contiguous(), heads, q2)
    dv.davet_cache_attention(chain, [0, 5], [past + 5], q2, heads, out2, lse=lse2,
                             block=1, workspace=ws)
    assert torch.equal(q[path], q2)
    # (other keys of the tiles in between: the sums' order differs)
    assert np.abs(f64(out[path]) - f64(out2)).max() <= 4 * 2.0 ** -11 * 4
    assert (lse[path] - lse2).abs().max() <= 64 * 2.0 ** -24 * 16
    # accepted tokens to the front: pages from the draft's first one on
    at = past // page
    tail = dv.KvCache(dk, dvv, cache.page_table[:, at:].contiguous(), dv.DAVET_F16)
    keep = past % page + len(path)
    kept = torch.tensor([list(range(past % page)) + [past % page + j for j in path]],
                        dtype=torch.int32).cuda()
    fresh = torch.tensor([free[:2]], dtype=torch.int32).cuda()
    dv.davet_cache_gather(tail, kept, [keep], fresh)
    moved = cache.page_table.clone()
    moved[0, at:at + 2] = fresh[0]
    for a, b in ((dk, ck), (dvv, cvv)):
        for j in range(past + 5):
            assert torch.equal(a[moved[0, j // page], :, j % page],
                               b[cache.page_table[0, j // page], :, j % page]), j


def test_captured_with_masks_that_change():
    s = Setup(4, "f16", [30], [500], 8, 2, 128, 64)
    cache, q, ws = s.device(), s.q.cuda(), s.workspace()
    parent = torch.zeros(30, dtype=torch.int32, device="cuda")
    mask = torch.zeros(30, dv.TREE_WORDS, dtype=torch.int32, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros(30, 8, device="cuda")

    def step(o, e, stream=None):
        dv.davet_tree_plan(s.cu, s.kv, parent, mask=mask, stream=stream)
        dv.davet_cache_tree_attention(cache, s.cu, s.kv, q, 8, mask, o, lse=e,
                                      workspace=ws, stream=stream)
    step(out, lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, lse)
    side = torch.cuda.Stream()
    for i in range(3):
        parent.copy_(torch.tensor(draft(s.rng, 30, "bush"), dtype=torch.int32))
        want, e = torch.zeros_like(q), torch.zeros_like(lse)
        torch.cuda.synchronize()
        step(want, e, side)
        side.synchronize()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, e), i
