"""Calls of documented sizes whose grid has 2^32 threads and more, which is more than one
launch takes: every row of them is answered."""

import pytest
import torch

import paper_2608_01821_amd as dv

pytestmark = pytest.mark.gpu
HALF = torch.float16


def rand(shape, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(HALF)


def cache_of(tables, hk, dim, page, seed):
    """A pool of three pages and these table rows."""
    k = rand((3, hk, page, dim), seed)
    v = rand((3, hk, page, dim), seed + 1)
    return dv.KvCache(k, v, tables, dv.DAVET_F16)


def table_of(seqs, pages):
    t = torch.arange(pages, device="cuda") % 3
    return t.to(torch.int32).expand(seqs, pages).contiguous()


def test_selected_pages_a_workgroup_each():
    """2^22 and more choices, one history of more than 1024 pages among them: 1024
    threads each.  Sequences 1 .. 63 are alike."""
    hk, dim, n = 1024, 64, 66
    seqs = 64
    table = table_of(seqs, 1025)
    table[0, 3] = 1                             # (a history of its own)
    cache = cache_of(table, hk, dim, 16, 3)
    bounds = torch.stack([cache.k.amin(2), cache.k.amax(2)], 2)
    cu = [0, 1] + [1 + n * (i + 1) for i in range(seqs - 1)]
    kv = [16400] + [n] * (seqs - 1)
    q = torch.cat([rand((1, hk * dim), 5), rand((n, hk * dim), 6).repeat(seqs - 1, 1)])
    pages = torch.full((cu[-1], hk, 2), 7, dtype=torch.int32, device="cuda")
    assert cu[-1] * hk * 1024 > 1 << 32
    dv.davet_cache_page_select(cache, cu, kv, q, hk, bounds, pages)
    one = dv.KvCache(cache.k, cache.v, table[1:2].contiguous(), dv.DAVET_F16)
    want = torch.empty(n, hk, 2, dtype=torch.int32, device="cuda")
    dv.davet_cache_page_select(one, [0, n], [n], q[1:1 + n], hk, bounds, want)
    assert torch.equal(pages[1:].view(seqs - 1, n, hk, 2),
                       want.expand(seqs - 1, n, hk, 2))
    assert (want[..., 0] < want[..., 1]).all() and (want[..., 0] >= 0).all()


def test_selected_pages_in_tiles():
    """Chunks of 1041 tokens and 1024 key heads: 2^22 tiles of 16 choices, 1024 threads
    each.  The sequences are alike."""
    hk, dim, n, seqs = 1024, 64, 1041, 64
    table = table_of(seqs, 66)
    cache = cache_of(table, hk, dim, 16, 7)
    bounds = torch.stack([cache.k.amin(2), cache.k.amax(2)], 2)
    one = dv.KvCache(cache.k, cache.v, table[:1].contiguous(), dv.DAVET_F16)
    first = rand((n, hk * dim), 8)
    want = torch.empty(n, hk, 1, dtype=torch.int32, device="cuda")
    dv.davet_cache_page_select(one, [0, n], [n], first, hk, bounds, want)
    assert ((want >= 0) & (want < 3)).all()
    cu, kv = [n * i for i in range(seqs + 1)], [n] * seqs
    assert (n + 15) // 16 * seqs * hk * 1024 > 1 << 32
    pages = torch.full((cu[-1], hk, 1), 7, dtype=torch.int32, device="cuda")
    dv.davet_cache_page_select(cache, cu, kv, first.repeat(seqs, 1), hk, bounds, pages)
    for i in range(seqs):
        assert torch.equal(pages[cu[i]:cu[i + 1]], want), i


def test_attention_over_many_lists():
    """Chunks of 1041 tokens and 1024 key heads: 2^24 workgroups of four lists, 256
    threads each.  The sequences are alike."""
    hk, dim, n, seqs = 1024, 64, 1041, 64
    table = table_of(seqs, 66)
    cache = cache_of(table, hk, dim, 16, 7)
    one = dv.KvCache(cache.k, cache.v, table[:1].contiguous(), dv.DAVET_F16)
    first = rand((n, hk * dim), 8)
    pages = (torch.arange(n * hk, device="cuda") * 7 % 66).int().view(n, hk, 1)
    ws = torch.empty(dv.davet_cache_workspace_bytes(hk, dim, n * seqs),
                     dtype=torch.uint8, device="cuda")
    o, e = torch.empty_like(first), torch.empty(n, hk, device="cuda")
    dv.davet_cache_page_attention(one, [0, n], [n], first, hk, pages, o, lse=e,
                                  workspace=ws)
    assert torch.isfinite(o).all() and torch.isfinite(e).all()
    cu, kv = [n * i for i in range(seqs + 1)], [n] * seqs
    assert cu[-1] * hk // 4 * 256 > 1 << 32
    q = first.repeat(seqs, 1)
    out = torch.full_like(q, 7.0)
    lse = torch.full((cu[-1], hk), 7.0, device="cuda")
    dv.davet_cache_page_attention(cache, cu, kv, q, hk, pages.repeat(seqs, 1, 1), out,
                                  lse=lse, workspace=ws)
    for i in range(seqs):
        rows = slice(cu[i], cu[i + 1])
        assert torch.equal(out[rows], o) and torch.equal(lse[rows], e), i


def test_bounds_of_many_pages():
    """2^24 and more pages and key heads, 256 threads each; most of the pages are
    holes."""
    hk, dim, seqs, count = 1024, 64, 64, 257
    table = torch.full((seqs, count), -1, dtype=torch.int32, device="cuda")
    where = [(0, 0), (31, 5), (seqs - 1, count - 1)]
    for i, (s, p) in enumerate(where):
        table[s, p] = i
    k = rand((4, hk, 16, dim), 9)
    cache = dv.KvCache(k, None, table, dv.DAVET_F16)
    bounds = torch.full((4, hk, 2, dim), 7.0, dtype=HALF, device="cuda")
    kv = [16 * count] * seqs
    assert seqs * count * hk * 256 > 1 << 32
    dv.davet_cache_page_bounds(cache, [16 * count * i for i in range(seqs + 1)], kv, bounds)
    assert torch.equal(bounds[:3], torch.stack([k.amin(2), k.amax(2)], 2)[:3])
    assert (bounds[3:] == 7).all()


def test_beams_of_as_many_requests_as_there_may_be():
    """2^22 requests of one beam: a workgroup of 1024 threads each."""
    n, vocab, top = 1 << 22, 3, 2
    x = rand((n, vocab), 1)
    scores = torch.arange(n, device="cuda").float() / -64
    s = torch.full((n, top), 7.0, device="cuda")
    r, t = (torch.full((n, top), 7, dtype=torch.int32, device="cuda") for _ in range(2))
    ws = torch.empty(dv.davet_beam_workspace_bytes(n, 1, vocab, top), dtype=torch.uint8,
                     device="cuda")
    dv.davet_beam_select(x, dv.DAVET_F16, scores, 1, s, r, t, workspace=ws)
    want, at = x.double().sort(dim=1, descending=True, stable=True)
    assert torch.equal(t, at[:, :top].int())
    assert torch.equal(r, torch.arange(n, device="cuda").int()[:, None].expand(n, top))
    want = scores.double()[:, None] + want[:, :top] - x.double().logsumexp(1)[:, None]
    # the float32 sum of three exponentials (3 roundings of a number up to 3, and those
    # of the exponentials, 2 each), then the value's own
    assert ((s - want).abs() <= 12 * 2.0 ** -24 + 2.0 ** -24 * want.abs()).all()


def test_gather_of_many_entries():
    """2^24 and more blocks of 128 entries and a key head, 256 threads each; most
    destinations are holes."""
    hk, dim, page, seqs, keep = 1024, 64, 16, 64, 128 * 257
    pages = keep // page
    k, v = rand((5, hk, page, dim), 11), rand((5, hk, page, dim), 12)
    table = torch.zeros((seqs, 1), dtype=torch.int32, device="cuda")
    kept = (torch.arange(keep, device="cuda") * 5 % page).int().expand(seqs, keep)
    dst = torch.full((seqs, pages), -1, dtype=torch.int32, device="cuda")
    where = [(0, 0), (31, 5), (seqs - 1, pages - 1)]
    for i, (s, p) in enumerate(where):
        dst[s, p] = i + 1
    want_k, want_v, order = k.clone(), v.clone(), torch.arange(page) * 5 % page
    for i in range(len(where)):
        want_k[i + 1], want_v[i + 1] = k[0][:, order], v[0][:, order]
    assert seqs * keep // 128 * hk * 256 > 1 << 32
    cache = dv.KvCache(k, v, table, dv.DAVET_F16)
    dv.davet_cache_gather(cache, kept.contiguous(), [keep] * seqs, dst)
    assert torch.equal(k, want_k) and torch.equal(v, want_v)


def test_weights_of_many_keys():
    """2^24 and more blocks of 128 keys, 256 threads each: two histories of 2^30 tokens
    that share three pages."""
    page, n = 256, 1 << 30
    table = table_of(3, n // page)
    g = torch.Generator(device="cuda")
    g.manual_seed(13)
    k = torch.randn((3, 1, page, 64), generator=g, device="cuda")
    q = torch.randn((1, 64), generator=g, device="cuda").repeat(3, 1)
    cache = dv.KvCache(k, None, table, dv.DAVET_F32)
    w = torch.full((3, n), 7.0, device="cuda")
    lse = torch.full((3, 1), 2.0, device="cuda")
    ws = torch.empty(dv.davet_cache_workspace_bytes(1, 64, 3), dtype=torch.uint8,
                     device="cuda")
    kv = [n, n, 1]
    assert sum(-(-x // 128) for x in kv) * 256 > 1 << 32
    dv.davet_cache_weights(cache, [0, 1, 2, 3], kv, q, 1, lse, w, workspace=ws)
    one = w[0, :3 * page]
    want = torch.exp(k.view(-1, 64).double() @ q[0].double() / 8 - 2)
    # a score is off by at most 67 roundings of the sum of its terms' magnitudes
    off = 67 * 2.0 ** -24 * (k.view(-1, 64).double().abs() @ q[0].double().abs() / 8 + 4)
    assert ((one - want).abs() <= want * (2 * off + 16 * 2.0 ** -24)).all()
    whole = n // (3 * page) * 3 * page
    for s in range(2):
        assert (w[s, :whole].view(-1, 3 * page) == one).all()
        assert torch.equal(w[s, whole:], one[:n - whole])
    assert w[2, 0] == one[0] and (w[2, 1:] == 7).all()
