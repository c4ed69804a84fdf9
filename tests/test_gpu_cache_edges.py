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

@pytest.mark.filterwarnings("ignore:invalid value")      # (the oracle's 0 inf)
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

@pytest.mark.filterwarnings("ignore:invalid value")      # (the oracle's 0 inf)
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


# --------------------------------------------------- work over many workgroups --

def launches(call):
    """Kernels that a call launches."""
    dv.prof_enable(64)
    dv.prof_reset()
    call()
    n = sum(c for c, _ in dv.prof_read().values())
    dv.prof_enable(0)
    return n


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), -float("inf")])
@pytest.mark.parametrize("new,kv,heads,hk", [
    (9, 1400, 2, 2),            # few rows, joined a wavefront a row
    (90, 1400, 2, 1),           # tiles of many
    (1100, 1900, 8, 8)])        # joined many rows a wavefront
def test_values_that_are_not_finite_in_pieces(dtype, bad, new, kv, heads, hk):
    """Keys cut into pieces, a value of NaN or infinity late in a causal chunk and
    one that every row sees: the first reaches the rows that see it and no other,
    each its own dim only."""
    t = Setup(29, dtype, [new], [kv], heads, hk, 64, 16)
    cut = new - 3
    ref = exact_attention(t, 1)
    put(t, "v", 0, [kv - new + cut], 5, bad)
    put(t, "v", 0, [7], 6, bad)
    out = []
    assert launches(lambda: out.append(t.attend(block=1))) == 2
    out, lse = out[0]
    assert not np.isfinite(out[cut:, :, 5]).any()
    assert not np.isfinite(out[:, :, 6]).any()
    late = [d for d in range(64) if d != 6]
    both = [d for d in range(64) if d not in (5, 6)]
    for rows, dims in ((slice(0, cut), late), (slice(cut, new), both)):
        part = {k: x[rows] if x.ndim == 2 else x[rows][..., dims]
                for k, x in ref.items()}
        check_attention((out[rows][..., dims], lse[rows]), part, dtype, 64, kv)


@pytest.mark.parametrize("dtype,new,kv,heads,hk,dim,page,block,n", [
    # key heads a workgroup, chunks of them: 2 in 4
    ("f16", [3], [17000], 16, 8, 128, 64, 0, 2),
    ("f32", [40], [17000], 8, 8, 64, 32, 1, 2),
    ("bf16", [5, 70], [20000, 20500], 8, 8, 64, 16, 1, 2),      # 3 in 3
    ("f16", [6], [17000], 32, 32, 64, 128, 4, 2),               # 5 in 7
    ("f16", [64], [40000], 32, 8, 64, 64, 1, 2),                # two tiles a wave
    ("bf16", [1] * 4, [20000, 19000, 20011, 17], 8, 8, 128, 256, 0, 2),
    ("f16", [1, 2, 1, 40], [20000, 19000, 20011, 20300], 8, 8, 64, 64, 1, 1),
    ("f32", [2, 1, 1, 9], [20000, 19000, 20011, 20300], 2, 2, 128, 64, 0, 1),
])
def test_weights_of_many_keys(dtype, new, kv, heads, hk, dim, page, block, n):
    """Workgroups that walk over several key heads, with partial sums (two
    launches) and without (one); a hole, pages' ends without a token."""
    t = Setup(33, dtype, new, kv, heads, hk, dim, page)
    t.table[0, 1] = -1
    want, lse, rel = exact_weights(t, block)
    w = torch.full((len(kv), max(kv) + 1), 7.0, device="cuda")
    args = (t.device(), t.cu, t.kv, t.q.cuda(), heads, torch.from_numpy(
        lse).float().cuda(), w)
    ws = t.workspace()
    assert launches(lambda: dv.davet_cache_weights(
        *args, block=block, workspace=ws)) == n
    torch.cuda.synchronize()
    for s, m in enumerate(kv):
        got = f64(w[s, :m])
        assert np.all(np.abs(got - want[s, :m]) <= rel * want[s, :m] + 1e-30)
        assert torch.all(w[s, m:] == 7.0)
    assert np.all(f64(w[0, page:2 * page]) == 0)


def heads_of(t, block):
    """For each sequence and head of a Setup: its number, rows, head, keys and
    values [n, dim] on the GPU in float64, scores with -inf where not visible."""
    _, hk, page, dim = t.k.shape
    q = t.q.cuda().double().reshape(-1, t.heads, dim)
    for s, m in enumerate(t.kv):
        n = t.cu[s + 1] - t.cu[s]
        ids = torch.from_numpy(t.table[s, :-(-m // page)].astype(np.int64))
        k, v = (x[ids.clamp(min=0)].cuda().double().permute(1, 0, 2, 3).reshape(
            hk, -1, dim)[:, :m] for x in (t.k, t.v))
        i, j = torch.arange(n)[:, None], torch.arange(m)[None]
        end = m if block == 0 else m - n + ((i // block + 1) * block).clamp(max=n)
        seen = ((j < end) & (ids >= 0).repeat_interleave(page)[:m]).cuda()
        rows = slice(t.cu[s], t.cu[s + 1])
        for h in range(t.heads):
            g = h * hk // t.heads
            x = dim ** -0.5 * (q[rows, h] @ k[g].T.contiguous())
            yield s, rows, h, q[rows, h], k[g], v[g], x.masked_fill(~seen, -np.inf)


def exact_attention(t, block):
    """As the oracle's, which goes one row at a time."""
    dim, shape = t.k.shape[3], (t.cu[-1], t.heads)
    r = dict(out=np.zeros(shape + (dim,)), mass=np.zeros(shape + (dim,)),
             lse=np.zeros(shape), dot=np.zeros(shape))
    for _, rows, h, q, k, v, x in heads_of(t, block):
        z = x.logsumexp(1)
        p = (x - z[:, None]).exp()
        r["out"][rows, h], r["mass"][rows, h] = f64(p @ v), f64(p @ v.abs())
        r["lse"][rows, h] = f64(z)
        r["dot"][rows, h] = dim ** -0.5 * f64(
            (q.abs() @ k.abs().T.contiguous()).amax(1))
    return r


def exact_weights(t, block):
    """(weights, lse, relative tolerance)."""
    dim = t.k.shape[3]
    want, lse, most = np.zeros((len(t.kv), max(t.kv))), np.zeros((t.cu[-1], t.heads)), 0
    for s, rows, h, q, k, _, x in heads_of(t, block):
        z = x.logsumexp(1).float().double()
        want[s, :t.kv[s]] += f64((x - z[:, None]).exp().sum(0))
        lse[rows, h] = f64(z)
        most = max(most, float(dim ** -0.5 * q.abs().amax() * k.abs().sum(1).amax()))
    # each term: a score off by dim 2^-24 of its magnitudes, the argument's
    # roundings, the exponential; then fp32 sums of rows x heads terms
    rel = (dim + 8) * 2.0 ** -24 * (most + np.abs(lse).max() + 1) + \
        (t.cu[-1] * t.heads + 8) * 2.0 ** -24
    return want, lse, rel


@pytest.mark.parametrize("kv,n", [([17000], 2), ([20000, 19000, 20011, 20300], 1)])
def test_weights_add_up_in_place(kv, n):
    """prev is weights itself, with partial sums and without: three layers."""
    t = Setup(37, "f16", [2] * len(kv), kv, 8, 8, 64, 64)
    want, lse, rel = exact_weights(t, 1)
    w = torch.zeros(len(kv), max(kv), device="cuda")
    args = (t.device(), t.cu, t.kv, t.q.cuda(), 8, torch.from_numpy(
        lse).float().cuda(), w)
    ws = t.workspace()
    for turn in range(1, 4):
        assert launches(lambda: dv.davet_cache_weights(
            *args, prev=w, block=1, workspace=ws)) == n
        torch.cuda.synchronize()
        for s, m in enumerate(kv):
            err = np.abs(f64(w[s, :m]) - turn * want[s, :m])
            assert np.all(err <= turn * (rel + 2.0 ** -24) * want[s, :m] + 1e-30)


# ----------------------------------------------------------- columns of a buffer --

@pytest.mark.parametrize("new", [1, 5, 70])
def test_columns_side_by_side_of_one_buffer(new):
    """Queries and outputs, projected rows and queries, weights and what stays of
    them: the results of buffers of their own, and no other column touched."""
    t = Setup(39, "f16", [new, 2], [150, 40], 4, 2, 64, 16)
    rows, w = new + 2, 4 * 64
    want = t.attend(block=1)
    for first, second in ((0, 1), (1, 0)):      # either may be the left one
        buf = torch.full((rows, 2 * w + 8), 7.0, dtype=torch.float16, device="cuda")
        q, out = (buf[:, i * w:i * w + w] for i in (first, second))
        q.copy_(t.q.cuda())
        dv.davet_cache_attention(t.device(), t.cu, t.kv, q, 4, out, block=1,
                                 workspace=t.workspace())
        torch.cuda.synchronize()
        assert np.array_equal(f64(out).reshape(rows, 4, 64), want[0])
        assert torch.equal(q, t.q.cuda()) and bool((buf[:, 2 * w:] == 7).all())
    qkv = torch.from_numpy(t.rng.standard_normal((rows, 2 * w))).half().cuda()
    own = torch.empty(rows, w, dtype=torch.float16, device="cuda")
    dv.davet_cache_append(t.device(), t.cu, t.kv, qkv, 4, own)
    k = t.dk
    buf = torch.zeros(rows, 3 * w, dtype=torch.float16, device="cuda")
    buf[:, w:] = qkv
    dv.davet_cache_append(t.device(), t.cu, t.kv, buf[:, w:], 4, buf)
    torch.cuda.synchronize()
    assert torch.equal(buf[:, :w], own) and torch.equal(buf[:, w:], qkv)
    assert torch.equal(t.dk, k)
    x = torch.from_numpy(t.rng.random((2, 150 + 60))).float().cuda()
    kept = torch.zeros(2, 60, dtype=torch.int32, device="cuda")
    before = x.clone()
    dv.davet_evict_select(t.kv, [60, 30], x, kept, weights_out=x[:, 150:])
    torch.cuda.synchronize()
    assert torch.equal(x[:, :150], before[:, :150])
    for s, keep in enumerate((60, 30)):
        idx = oc.select(t.kv[s], keep, f64(before[s]))
        assert kept[s, :keep].tolist() == idx
        assert torch.equal(x[s, 150:150 + keep], before[s, idx])
        assert torch.equal(x[s, 150 + keep:], before[s, 150 + keep:])


# -------------------------------------------------------------- large scores --

def one_hot(dtype):
    """Keys of one dim each: the scores are the queries' elements, exactly."""
    t = Setup(35, dtype, [3], [40], 2, 1, 64, 16)
    for j in range(40):
        p, o = oc.slot(t.host, 0, j)
        t.k[p, 0, o] = 0
        t.k[p, 0, o, j] = 1
    return t


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("scale", [1e-30, 1e-3, 30.0, 1e3, 1e4, 1e5])
def test_weights_of_large_scores(dtype, scale):
    """What the header says of scores of any size: a term is off by 2^-22 of the
    sizes of its score and lse together.  (The argument is x c - lse c', c and c' =
    log2(e) rounded to fp32, so are the second product and the result: 2 |x c| + 3
    |lse c'| times 2^-24; then the exponential's 2^-23 and the sums of six.)"""
    t = one_hot(dtype)
    scale = float(np.float32(scale))
    ref = oc.attention(t.host, t.cu, t.kv, f64(t.q), 2, scale=scale, block=1)
    lse = f64(torch.from_numpy(ref["lse"]).float())
    want = oc.weights(t.host, t.cu, t.kv, f64(t.q), 2, lse, scale=scale, block=1)
    got = received(t, lse, 1, scale)
    top = scale * np.abs(f64(t.q)).max()
    rel = np.expm1(2.0 ** -22 * (top + np.abs(lse).max() + 4))
    assert np.all(np.abs(got - want) <= rel * want + 6 * 1e-37)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("block", [0, 1])
@pytest.mark.parametrize("scale", [1e7, 1e9, 1e18, 1e30])
def test_no_term_of_huge_scores_is_above_one(dtype, block, scale):
    """Their lse says less than its own rounding: a term may be anything in [0, 1],
    and a key far below every row's largest score still receives nothing."""
    t = one_hot(dtype)
    lse = oc.attention(t.host, t.cu, t.kv, f64(t.q), 2, scale=scale, block=block)["lse"]
    got = received(t, lse, block, scale)
    assert np.all((got >= 0) & (got <= 6))
    q = f64(t.q).reshape(6, 64)[:, :40]
    low = (q < q.max(1, keepdims=True) - 0.1).all(0)        # 2^-22 of q is far less
    assert low.sum() > 20 and np.all(got[0, low] == 0)
