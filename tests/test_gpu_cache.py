"""davet_cache_append, davet_cache_attention and davet_cache_weights against
the float64 oracle: types, head layouts, lengths from one token on, pages,
masks, holes, and values that masked places must not leak."""

import numpy as np
import pytest
import torch

import paper_2608_01821_amd as dv
from cache_util import (CODE, TORCH, Setup, check_attention, f64, half_step,
                        page_table, values)
from oracle import cache as oc

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------- append --

APPEND = [  # dtype, new, kv, heads, kv_heads, dim, page, norm
    ("f16", [1], [1], 1, 1, 64, 16, False),
    ("f16", [1], [2965], 32, 8, 128, 64, True),
    ("bf16", [5, 0, 17, 1], [5, 3, 40, 33], 6, 2, 128, 16, True),
    ("f32", [9, 3], [9, 67], 4, 4, 64, 32, True),
    ("f32", [7], [300], 7, 1, 128, 256, False),
    ("f16", [33, 30], [33, 61], 28, 4, 64, 128, True),
    ("bf16", [2100], [2110], 2, 1, 64, 32, True),
    ("f16", [3050, 3200, 0, 1], [3050, 3207, 0, 1], 1, 1, 64, 64, True),  # three rows
    ("bf16", [401], [410], 32, 16, 128, 64, True),    # a workgroup, or two, of 512
]


@pytest.mark.parametrize("case", APPEND, ids=str)
@pytest.mark.parametrize("in_place", [False, True])
def test_append(case, in_place):
    dtype, new, kv, heads, hk, dim, page, norm = case
    rng = np.random.default_rng(len(new) + dim + heads)
    cu = [0] + [int(x) for x in np.cumsum(new)]
    total, table = page_table(rng, kv, page)
    k, v = (values(rng, (total, hk, page, dim), dtype) for _ in range(2))
    width = (heads + 2 * hk) * dim
    qkv = values(rng, (cu[-1] + 2, width + 16), dtype)
    gq, gk = (torch.from_numpy(1 + 0.2 * rng.standard_normal(dim)).float()
              for _ in range(2))
    pos = rng.integers(-5, 2 ** 31 - 1, cu[-1]).astype(np.int32) \
        if len(new) == 2 else None
    dk, dvv, dq = k.cuda(), v.cuda(), qkv.cuda()
    cache = dv.KvCache(dk, dvv, torch.from_numpy(table).cuda(), CODE[dtype])
    if in_place:
        q_out = dq
    else:
        q_out = torch.full((cu[-1] + 2, heads * dim + 8), 7.0,
                           dtype=TORCH[dtype], device="cuda")
    before = q_out.clone()
    dv.davet_cache_append(cache, cu, kv, dq, heads, q_out,
                          pos=None if pos is None else torch.from_numpy(pos).cuda(),
                          norm=norm, q_gain=gq.cuda(),
                          k_gain=gk.cuda() if heads % 2 else None, eps=1e-5,
                          theta=1e4)
    torch.cuda.synchronize()
    rq, rk, rv = oc.append(
        dict(k=f64(k), v=f64(v), table=table), cu, kv, f64(qkv)[:cu[-1], :width],
        heads, pos=pos, norm=norm, q_gain=gq.numpy(),
        k_gain=gk.numpy() if heads % 2 else None, eps=float(np.float32(1e-5)),
        theta=1e4)
    # a turned element is a c - b s of normed a, b (at most ~|x| sqrt(2)): the
    # norm takes 20 roundings in fp32, the sine and cosine (of an argument off
    # by 2^-24 turns: 2 pi 2^-24) and the two products 12 more; then the store
    u = half_step(dtype)
    for got, ref in ((f64(q_out)[:cu[-1], :heads * dim].reshape(rq.shape), rq),
                     (f64(dk), rk)):
        pair = np.sqrt(ref ** 2 + np.roll(ref, dim // 2, -1) ** 2)
        tol = u * np.abs(ref) + 32 * 2.0 ** -24 * pair * (dtype == "f32") + \
            (1 + u) * 32 * 2.0 ** -24 * pair + 2.0 ** -25 * (dtype == "f16")
        assert np.all(np.abs(got - ref) <= tol)
    assert np.array_equal(f64(dvv), rv)                # values bit for bit
    # rows behind the chunk, and columns beside it, are as they were
    assert torch.equal(q_out[cu[-1]:], before[cu[-1]:])
    assert torch.equal(q_out[:, heads * dim:], before[:, heads * dim:])


def test_append_into_holes_and_shared_reads():
    """A hole takes nothing and the queries still come out."""
    rng = np.random.default_rng(5)
    cu, kv, page = [0, 20], [40], 16
    table = np.array([[3, -1, 1]], np.int32)
    k, v = (values(rng, (4, 2, page, 64), "f16") for _ in range(2))
    qkv = values(rng, (20, 6 * 64), "f16")
    dk, dvv = k.cuda(), v.cuda()
    for bad in (-1, 4, 2 ** 31 - 1):
        table[0, 1] = bad
        cache = dv.KvCache(dk, dvv, torch.from_numpy(table).cuda(), dv.DAVET_F16)
        q = torch.empty(20, 128, dtype=torch.float16, device="cuda")
        dv.davet_cache_append(cache, cu, kv, qkv.cuda(), 2, q)
        torch.cuda.synchronize()
        rq, rk, rv = oc.append(dict(k=f64(k), v=f64(v), table=table), cu, kv,
                               f64(qkv), 2)
        assert np.array_equal(f64(dvv), rv)
        assert np.abs(f64(dk) - rk).max() < 4e-3
        assert np.abs(f64(q).reshape(rq.shape) - rq).max() < 4e-3


# ---------------------------------------------------------------- attention --

ATTEND = [  # dtype, new, kv, heads, kv_heads, dim, page, block
    ("f16", [1], [1], 1, 1, 64, 16, 0),
    ("f16", [1], [1], 8, 1, 128, 16, 1),
    ("f32", [1], [17], 4, 4, 64, 16, 0),
    ("bf16", [1, 1, 1], [31, 32, 33], 4, 2, 128, 32, 0),
    ("f16", [1], [700], 32, 8, 128, 64, 0),
    ("f16", [1, 1], [2100, 40], 8, 8, 64, 256, 0),      # pieces, 8 XCDs
    ("bf16", [1], [2500], 7, 1, 128, 16, 0),            # pieces
    ("f32", [1, 2], [1500, 9], 2, 1, 128, 16, 1),
    ("f16", [5, 0, 3], [60, 7, 3], 6, 2, 128, 16, 1),
    ("f32", [32], [192], 4, 4, 64, 16, 0),
    ("bf16", [32, 32], [100, 77], 2, 2, 128, 16, 4),
    ("f16", [9], [9], 28, 4, 64, 32, 3),                # 63 rows a key head
    ("f16", [32], [90], 1, 1, 128, 16, 1),              # narrow's last
    ("f16", [33], [90], 1, 1, 128, 16, 1),              # wide from here
    ("f32", [64], [90], 1, 1, 128, 16, 1),
    ("f32", [65], [90], 1, 1, 128, 16, 1),              # wide from here
    ("bf16", [40], [64], 1, 1, 128, 64, 0),             # one tile, whole
    ("f16", [40], [65], 2, 2, 64, 64, 0),               # two, the last of one key
    ("bf16", [40], [193], 2, 1, 128, 128, 1),           # four
    ("f16", [40, 36], [320, 130], 2, 2, 128, 256, 4),   # five and three
    ("f16", [65], [65], 1, 1, 128, 16, 1),
    ("f16", [33], [200], 4, 2, 128, 64, 0),
    ("bf16", [130, 4], [300, 40], 2, 1, 128, 16, 1),
    ("bf16", [70], [600], 3, 1, 64, 32, 32),
    ("f32", [80, 1], [130, 5], 3, 3, 128, 16, 1),
    ("f32", [129], [129], 2, 2, 64, 64, 0),
    ("f16", [200], [1400], 8, 8, 64, 128, 7),           # wide with pieces
    ("f16", [300, 257, 0, 1], [300, 700, 5, 64], 2, 2, 128, 64, 0),
    # pieces of many rows, several a wavefront: heads in whole and broken groups
    ("f16", [280, 21], [1300, 700], 28, 4, 64, 64, 0),
    ("bf16", [1180], [1300], 7, 1, 64, 32, 5),
    ("f16", [2740], [2760], 3, 1, 128, 64, 0),
    ("f32", [520], [900], 16, 2, 64, 16, 1),
]


@pytest.mark.parametrize("case", ATTEND, ids=str)
def test_attention(case):
    dtype, new, kv, heads, hk, dim, page, block = case
    # NaN wherever no token is: the tails of pages, and unused pages
    t = Setup(7, dtype, new, kv, heads, hk, dim, page, fill=float("nan"))
    ref = oc.attention(t.host, t.cu, t.kv, f64(t.q), heads, block=block)
    check_attention(t.attend(block=block), ref, dtype, dim, max(kv))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("new,kv,block", [([3], [90], 0), ([1], [1300], 1),
                                          ([100], [230], 1), ([66], [66], 0)])
def test_holes_and_empty_rows(dtype, new, kv, block):
    """Bad page ids hold no keys, whatever their value; a sequence without any
    page gives zeros and lse -inf."""
    t = Setup(3, dtype, new + new, kv + kv, 4, 2, 64, 16, fill=float("nan"))
    n = -(-kv[0] // 16)
    bad = np.array([t.k.shape[0], -1, 2 ** 31 - 1, -7], np.int32)
    t.table[0, ::2] = np.resize(bad, len(t.table[0, ::2]))
    t.table[1, :n] = -1
    ref = oc.attention(t.host, t.cu, t.kv, f64(t.q), 4, block=block)
    assert np.isneginf(ref["lse"][new[0]:]).all()
    got = t.attend(block=block)
    check_attention(got, ref, dtype, 64, kv[0])
    assert np.all(got[0][new[0]:] == 0)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("page", [32, 64, 256])
@pytest.mark.parametrize("new", [3, 40, 90])
def test_holes_of_whole_tiles(dtype, page, new):
    """Pages as large as a tile of keys, and larger: every second one a hole."""
    kv = 3 * page + 150
    t = Setup(17, dtype, [new, 1], [kv, page + 1], 2, 2, 128, page,
              fill=float("nan"))
    t.table[0, ::2] = -1
    t.table[1, 0] = t.k.shape[0]
    ref = oc.attention(t.host, t.cu, t.kv, f64(t.q), 2, block=1)
    check_attention(t.attend(block=1), ref, dtype, 128, kv)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("new,heads,hk", [(6, 2, 1), (70, 2, 2)])
def test_invisible_keys_do_not_leak(dtype, bad, new, heads, hk):
    """A value (and key) of NaN or infinity late in a causal chunk reaches the
    rows that see it and no other."""
    kv, cut = new + 21, new - 3                   # rows before `cut` do not see it
    t = Setup(11, dtype, [new], [kv], heads, hk, 128, 16)
    page, off = oc.slot(t.host, 0, kv - new + cut)
    clean = oc.attention(t.host, t.cu, t.kv, f64(t.q), heads, block=1)
    t.v[page, :, off, 5] = bad
    out, lse = t.attend(block=1)
    first = {k: x[:cut] for k, x in clean.items()}
    check_attention((out[:cut], lse[:cut]), first, dtype, 128, kv)
    # rows that see it: that dim only is not finite, the others are as before
    assert not np.isfinite(out[cut:, :, 5]).any()
    rest = np.arange(128) != 5
    tail = {k: x[cut:] if x.ndim == 2 else x[cut:][..., rest]
            for k, x in clean.items()}
    check_attention((out[cut:][..., rest], lse[cut:]), tail, dtype, 128, kv)
    if bad != bad:
        t.k[page, :, off, 9] = bad
        out, lse = t.attend(block=1)
        check_attention((out[:cut], lse[:cut]), first, dtype, 128, kv)
        assert np.isnan(out[cut:]).all() and np.isnan(lse[cut:]).all()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_extreme_scores(dtype):
    """Scores hundreds apart, ascending and descending along the keys (the
    running maximum moves at every tile, or never), and a scale of the
    caller's; queries of zero see uniform weights."""
    for sign in (1, -1):
        t = Setup(2, dtype, [40], [500], 2, 1, 64, 16)
        j = np.arange(500)
        for i in j:
            p, o = oc.slot(t.host, 0, i)
            t.k[p, 0, o] = sign * (i - 250) / 8.0
        t.q = torch.sign(t.q)
        t.q[:5] = 0
        t.q[5:10] = 1
        ref = oc.attention(t.host, t.cu, t.kv, f64(t.q), 2, scale=0.25)
        check_attention(t.attend(scale=0.25), ref, dtype, 64, 500)
        u = t.attend(scale=0.25)
        assert np.allclose(u[1][:5], np.log(500), atol=1e-5)


def test_attention_strided_rows_stay_inside():
    """Row strides of q and out; rows and columns beside the chunk stay."""
    for new, heads in ((2, 4), (40, 4)):
        t = Setup(9, "f16", [new], [70], heads, 2, 64, 16)
        ref = oc.attention(t.host, t.cu, t.kv, f64(t.q), heads)
        q = torch.zeros(new + 3, heads * 64 + 24, dtype=torch.float16, device="cuda")
        q[:new, 8:8 + heads * 64] = t.q.cuda()
        out = torch.full((new + 3, heads * 64 + 40), 7.0, dtype=torch.float16,
                         device="cuda")
        lse = torch.full((new + 1, heads), 7.0, device="cuda")
        dv.davet_cache_attention(t.device(), t.cu, t.kv, q[:, 8:], heads,
                                 out[:, 16:], lse=lse, workspace=t.workspace())
        torch.cuda.synchronize()
        got = f64(out[:new, 16:16 + heads * 64]).reshape(new, heads, 64)
        check_attention((got, f64(lse[:new])), ref, "f16", 64, 70)
        out[:new, 16:16 + heads * 64] = 7.0
        assert bool((out == 7).all()) and bool((lse[new:] == 7).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("scale", [1e-30, 1e-3, 1e4, 1e30])
def test_scales_to_the_limits(dtype, scale):
    """Uniform weights at one end, the largest score alone at the other (keys
    that are one dim each: scores are exact and apart)."""
    t = Setup(13, dtype, [3], [40], 2, 1, 64, 16)
    for j in range(40):
        p, o = oc.slot(t.host, 0, j)
        t.k[p, 0, o] = 0
        t.k[p, 0, o, j] = 1
    ref = oc.attention(t.host, t.cu, t.kv, f64(t.q), 2, scale=scale, block=1)
    out, lse = t.attend(scale=scale, block=1)
    u = half_step(dtype)
    tol = u * np.abs(ref["out"]) + ref["mass"] * (u + 1e-5)
    assert np.all(np.abs(out - ref["out"]) <= tol)
    assert np.all(np.abs(lse - ref["lse"]) <= 1e-5 + 4e-7 * np.abs(ref["lse"]))


def test_one_row_of_any_tensor():
    """A single row has no stride to align: a slice of odd width is taken."""
    t = Setup(14, "f16", [1], [20], 2, 1, 64, 16)
    q = torch.zeros(1, 128 + 5, dtype=torch.float16, device="cuda")
    q[:, :128] = t.q.cuda()
    out = torch.zeros(1, 128 + 3, dtype=torch.float16, device="cuda")
    dv.davet_cache_attention(t.device(), t.cu, t.kv, q, 2, out,
                             workspace=t.workspace())
    torch.cuda.synchronize()
    assert np.array_equal(f64(out[:, :128]).reshape(1, 2, 64), t.attend()[0])
    assert bool((out[:, 128:] == 0).all())


def test_far_pages_need_64_bit_offsets():
    """A pool of more than 2^31 elements, pages at its end."""
    t = Setup(4, "f16", [3], [100], 2, 2, 128, 16)
    n = (1 << 31) // (2 * 16 * 128) + 40
    big = torch.zeros(n, 2, 16, 128, dtype=torch.float16, device="cuda")
    far = t.table.copy()
    far[far >= 0] += n - t.k.shape[0]
    k, v = big, torch.zeros_like(big)
    k[-t.k.shape[0]:], v[-t.k.shape[0]:] = t.k.cuda(), t.v.cuda()
    cache = dv.KvCache(k, v, torch.from_numpy(far).cuda(), dv.DAVET_F16)
    ref = oc.attention(t.host, t.cu, t.kv, f64(t.q), 2)
    check_attention(t.attend(cache), ref, "f16", 128, 100)


# ------------------------------------------------------------------ weights --

@pytest.mark.parametrize("case", [
    ("f16", [1], [1], 1, 1, 64, 16, 0),
    ("bf16", [1, 1], [31, 300], 8, 2, 128, 16, 0),
    ("f32", [32], [192], 4, 4, 64, 16, 0),
    ("f16", [5, 0, 3], [60, 150, 3], 6, 2, 128, 16, 1),
    ("f16", [130], [260], 2, 2, 128, 64, 1),
    ("bf16", [70], [400], 7, 1, 64, 32, 5),
    ("f32", [40], [129], 2, 1, 128, 16, 1),
    ("f16", [300], [130 + 300], 1, 1, 64, 16, 0),      # rows in several ranges
], ids=str)
@pytest.mark.parametrize("accumulate", [False, True])
def test_weights(case, accumulate):
    dtype, new, kv, heads, hk, dim, page, block = case
    t = Setup(21, dtype, new, kv, heads, hk, dim, page, fill=float("nan"))
    if len(kv) == 3:
        t.table[1, 2] = -1                          # a hole
    ref = oc.attention(t.host, t.cu, t.kv, f64(t.q), heads, block=block)
    lse = torch.from_numpy(ref["lse"]).float()
    if len(kv) == 2:
        lse[0, 3] = -np.inf                         # a row that saw nothing
    want = oc.weights(t.host, t.cu, t.kv, f64(t.q), heads, f64(lse), block=block)
    w = torch.full((len(kv) + 1, max(kv) + 5), 7.0, device="cuda")
    prev = None
    if accumulate:
        w[:len(kv), :max(kv)] = torch.from_numpy(
            t.rng.random((len(kv), max(kv)))).float().cuda()
        prev, want = w, want + f64(w[:len(kv), :max(kv)])
    keep = w.clone()
    dv.davet_cache_weights(t.device(), t.cu, t.kv, t.q.cuda(), heads, lse.cuda(),
                           w, prev=prev, block=block, workspace=t.workspace())
    torch.cuda.synchronize()
    # each term: a score off by dim 2^-24 of its magnitudes, the argument's
    # roundings, the exponential; then fp32 sums of rows x heads terms
    terms = max(new) * heads
    rel = (dim + 8) * 2.0 ** -24 * (ref["dot"].max() + np.abs(
        np.where(np.isneginf(ref["lse"]), 0, ref["lse"])).max() + 1) + \
        (terms + 8) * 2.0 ** -24
    for s, n in enumerate(kv):
        got = f64(w[s, :n])
        assert np.all(np.abs(got - want[s, :n]) <= rel * want[s, :n] + 1e-30)
        assert torch.equal(w[s, n:], keep[s, n:])
    assert torch.equal(w[-1], keep[-1])


@pytest.mark.parametrize("dtype,heads,hk,dim,page,block", [
    ("f16", 32, 8, 128, 64, 0), ("bf16", 32, 32, 64, 16, 1), ("f16", 32, 4, 64, 256, 48)])
def test_weights_of_long_chunks(dtype, heads, hk, dim, page, block):
    """Enough rows and keys that a wavefront takes two tiles of keys; a hole, and a
    short sequence beside."""
    new, kv = [700, 20], [5003, 290]
    t = Setup(31, dtype, new, kv, heads, hk, dim, page, fill=float("nan"))
    t.table[0, 1] = -1
    scale, want, most = dim ** -0.5, np.zeros((2, max(kv))), 0.0
    lse = np.zeros((sum(new), heads))
    q = t.q.cuda().double().reshape(-1, heads, dim)
    for s, (n, m) in enumerate(zip(new, kv)):
        ids = torch.from_numpy(t.table[s, :-(-m // page)].astype(np.int64))
        k = t.k[ids.clamp(min=0)].cuda().double().permute(1, 0, 2, 3)
        k = k.reshape(hk, -1, dim)[:, :m]
        i, j = torch.arange(n)[:, None], torch.arange(m)[None]
        end = m if block == 0 else m - n + ((i // block + 1) * block).clamp(max=n)
        seen = ((j < end) & (ids >= 0).repeat_interleave(page)[:m]).cuda()
        rows = slice(t.cu[s], t.cu[s + 1])
        for h in range(heads):
            kh, qh = k[h * hk // heads].nan_to_num(), q[rows, h]
            x = (scale * (qh @ kh.T.contiguous())).masked_fill(~seen, -np.inf)
            z = x.logsumexp(1).float().double()
            want[s, :m] += (x - z[:, None]).exp().sum(0).cpu().numpy()
            lse[rows, h] = z.cpu().numpy()
            most = max(most, float(scale * (qh.abs() @ kh.abs().T.contiguous()).max()))
    w = torch.full((2, max(kv) + 1), 7.0, device="cuda")
    dv.davet_cache_weights(t.device(), t.cu, t.kv, t.q.cuda(), heads,
                           torch.from_numpy(lse).float().cuda(), w, block=block,
                           workspace=t.workspace())
    torch.cuda.synchronize()
    rel = (dim + 8) * 2.0 ** -24 * (most + np.abs(lse).max() + 1) + \
        (max(new) * heads + 8) * 2.0 ** -24         # as in test_weights
    for s, m in enumerate(kv):
        got = f64(w[s, :m])
        assert np.all(np.abs(got - want[s, :m]) <= rel * want[s, :m] + 1e-30)
        assert torch.all(w[s, m:] == 7.0)
    assert np.all(f64(w[0, page:2 * page]) == 0)


def test_weights_sum_to_the_rows():
    """Every row and head gives 1 in all."""
    t = Setup(5, "f16", [50], [300], 4, 2, 128, 32)
    cache = t.device()
    _, lse = t.attend(cache)
    w = torch.zeros(1, 300, device="cuda")
    dv.davet_cache_weights(cache, t.cu, t.kv, t.q.cuda(), 4,
                           torch.from_numpy(lse).float().cuda(), w,
                           workspace=t.workspace())
    assert abs(float(w.double().sum()) / 200 - 1) < 1e-5


def test_no_new_tokens_copies_the_weights():
    t = Setup(6, "f16", [0, 0], [30, 5], 2, 1, 64, 16)
    prev = torch.rand(2, 30, device="cuda")
    w = torch.zeros(2, 30, device="cuda")
    dv.davet_cache_weights(t.device(), [0, 0, 0], [30, 5],
                           torch.zeros(1, 128, dtype=torch.float16, device="cuda"),
                           2, torch.zeros(1, 2, device="cuda"), w, prev=prev,
                           workspace=t.workspace())
    torch.cuda.synchronize()
    assert torch.equal(w[0], prev[0]) and torch.equal(w[1, :5], prev[1, :5])
    assert bool((w[1, 5:] == 0).all())
