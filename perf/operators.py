"""Performance cases of the cached denoising operators on one MI355X.

Each case is one call (or the two calls a program makes together) of

  append   davet_cache_append: a chunk's projected rows into the cache, queries
           and keys normed per head and rotated, in one pass
  attend   davet_cache_attention: a chunk of queries over the paged cache
  weigh    davet_cache_weights: the attention weight each cached key received
  evict    davet_evict_select + davet_cache_gather: the entries that stay, and
           their move to new pages
  score    davet_token_logprobs: log probabilities of given tokens, entropy and
           the top alternatives of rows of logits

`own` false: the same operators written with elementary torch operations.
"""

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
THETA, EPS = 10000.0, 1e-6


# ------------------------------------------------------------------- cases --

def _cache(kind, name, **kw):
    # 32 heads x 128 as in the 8B-shaped workloads; kv_heads < heads: grouped
    # queries; `past` cached tokens before the chunk of `new` ones (the largest
    # of a ragged batch), `page` tokens a page; block 0: every key is visible
    # (the bidirectional denoiser), B: block by block (1: causal)
    c = dict(kind=kind, dtype="f16", seqs=1, mix=0, heads=32, kv_heads=32,
             dim=128, page=64, past=0, new=1, even=True, block=0)
    c.update(kw, name=name)
    return c


def listed():
    return [
        # one committed token of one request: the smallest call of a
        # left-to-right decode, latency only
        _cache("append", "append-token", kv_heads=8, past=2964, norm=True),
        # the view and prompt of four crops and a 128-token response enter the
        # cache: once per request and layer
        _cache("append", "append-prompt", dtype="bf16", kv_heads=8, new=3092,
               norm=True),
        # the tiny fp32 model: its response block over its one-crop view
        _cache("attend", "attend-tiny-f32", dtype="f32", heads=4, kv_heads=4,
               dim=64, page=16, past=160, new=32),
        # a batch of eight requests, one new token each, over long histories:
        # the stream of the cache
        _cache("attend", "attend-tokens-long", seqs=8, mix=3, kv_heads=8,
               past=32700, new=1),
        # sixteen ragged requests refine a 32-token block over view and prompt
        # of one to five crops: the step of a semi-autoregressive denoiser
        _cache("attend", "attend-block-ragged16", dtype="bf16", seqs=16, mix=5,
               page=16, past=3741, new=32),
        # four requests' views, prompts and responses in full, the largest call
        _cache("attend", "attend-prompt", seqs=4, mix=7, past=0, new=3092,
               even=False),
        # what a whole response gave to each token of view and prompt
        _cache("weigh", "weigh-response", past=2964, new=128),
        # what one new token of each of eight long histories gave
        _cache("weigh", "weigh-tokens-long", dtype="bf16", seqs=8, mix=3,
               kv_heads=8, past=32700, new=1),
        # half of one request's visual evidence leaves the cache
        _cache("evict", "evict-view", past=2964, keep=0.5),
        # eight long histories cut to half, ragged
        _cache("evict", "evict-long", dtype="bf16", seqs=8, mix=3, kv_heads=8,
               past=32700, keep=0.5),
        # the last two masked positions of a response, logits of the 8B head
        dict(name="score-2", kind="score", dtype="f32", rows=2, vocab=126464,
             top=5),
        # two whole responses scored from 16-bit logits
        dict(name="score-256", kind="score", dtype="bf16", rows=256,
             vocab=126464, top=20),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["append", "attend", "attend", "attend", "weigh",
                       "evict", "score"])
    if kind == "score":
        c = dict(kind=kind, dtype=rng.choice(["f32", "f32", "bf16", "f16"]),
                 rows=log_int(1, 256), vocab=log_int(300, 160000),
                 top=rng.choice([0, 1, 5, 20, 64]))
        return c
    dim = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 32])
    c = dict(kind=kind, dtype=rng.choice(["f32", "bf16", "f16", "f16"]),
             seqs=rng.choice([1, 1, 2, 5, 8, 16, 64]),
             mix=rng.randint(1, 999), kv_heads=kv_heads,
             heads=kv_heads * rng.choice([1, 1, 2, 4, 7] if kv_heads < 32
                                         else [1]),
             dim=dim, page=rng.choice([16, 32, 64, 128, 256]), past=0, new=1,
             even=rng.random() < 0.5, block=0)
    if kind == "append":
        c.update(new=log_int(1, 4000), past=rng.choice([0, log_int(1, 9000)]),
                 norm=rng.random() < 0.6)
    elif kind == "evict":
        c.update(past=log_int(40, 70000), keep=rng.uniform(0.1, 0.95))
    else:
        form = rng.choice(["token", "block", "prompt"])
        c.update(new=dict(token=1, block=log_int(2, 256),
                          prompt=log_int(200, 3600))[form],
                 past=log_int(1, 9000 if form == "prompt" else 70000),
                 block=rng.choice([0, 0, 1, 4, 32]))
        if c["dtype"] == "f32":
            c.update(past=min(c["past"], 9000), new=min(c["new"], 500))
    # no dearer than the largest listed cases of the kind
    most_bytes = 2e8 if kind == "append" else 9e8
    while True:
        w = work(c)
        limit = 1e11 if c["dtype"] == "f32" or kind == "weigh" else 3e11
        if w["bytes"] <= most_bytes and w["flops"] <= limit:
            return c
        if c["seqs"] > 1:
            c["seqs"] = (c["seqs"] + 1) // 2
        elif c["new"] > 16:
            c["new"] = c["new"] * 2 // 3
        else:
            c["past"] = c["past"] * 2 // 3


# ------------------------------------------------------------------ shapes --

def _lens(c):
    """(new tokens, cached tokens before them) of each sequence."""
    if c["seqs"] == 1:
        return [(c["new"], c["past"])]
    rng, out = random.Random(c["mix"]), []
    for _ in range(c["seqs"]):
        past = rng.randint(c["past"] // 4, c["past"])
        new = c["new"] if c["even"] else rng.randint(-(-c["new"] // 2), c["new"])
        out.append((new, past))
    return out


def _visible(new, past, block):
    """Keys visible to each of the chunk's queries."""
    if block == 0:
        return [past + new] * new
    return [past + min(new, (i // block + 1) * block) for i in range(new)]


def _keep(c):
    """Entries that stay, and how many of the first and last are sure to."""
    n = [p for _, p in _lens(c)]
    keep = [max(1, int(round(x * c["keep"]))) for x in n]
    low = min(keep)
    return n, keep, min(4, low // 4), min(32, low // 4)


def work(c):
    if c["kind"] == "score":
        es = 4 if c["dtype"] == "f32" else 2
        return {"bytes": c["rows"] * (c["vocab"] * es + 12 + 8 * c["top"]),
                "flops": 4.0 * c["rows"] * c["vocab"]}
    es = 4 if c["dtype"] == "f32" else 2
    row = c["dim"] * es
    lens = _lens(c)
    rows = sum(n for n, _ in lens)
    if c["kind"] == "append":
        b = 2 * rows * (c["heads"] + 2 * c["kv_heads"]) * row
        return {"bytes": b, "flops": 4.0 * b / es}
    if c["kind"] == "evict":
        n, keep, _, _ = _keep(c)
        return {"bytes": 4 * sum(n) + 8 * sum(keep) +
                4 * sum(keep) * c["kv_heads"] * row, "flops": 0}
    kv = sum(n + p for n, p in lens)
    pairs = sum(sum(_visible(n, p, c["block"])) for n, p in lens)
    if c["kind"] == "weigh":
        return {"bytes": rows * c["heads"] * (row + 4) + kv * c["kv_heads"] * row
                + 8 * kv, "flops": 2.0 * pairs * c["heads"] * c["dim"]}
    return {"bytes": rows * c["heads"] * (2 * row + 4) +
            2 * kv * c["kv_heads"] * row,
            "flops": 4.0 * pairs * c["heads"] * c["dim"]}


# ------------------------------------------------------------------ inputs --

def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + stream)
    return g


def _randn(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _pages(g, lens, page, pool_extra=3):
    """A pool's page count and a shuffled page table for these lengths."""
    counts = [-(-n // page) for n in lens]
    total = sum(counts) + pool_extra
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(1, max(counts))), -1,
                       dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(counts):
        table[s, :n] = order[at:at + n]
        at += n
    return total, table, order[at:]


def _inputs(c, seed):
    """Everything on the GPU that a call reads or writes, as plain torch."""
    g = _gen(seed, 1)
    dt = DTYPES[c["dtype"]]
    if c["kind"] == "score":
        # a few plausible tokens stand out of a broad floor; the mask token is
        # never an answer; most given tokens are among the likely ones
        x = torch.randn((c["rows"], c["vocab"]), generator=g, device="cuda") * 2
        hot = torch.randint(0, c["vocab"], (c["rows"], 24), generator=g,
                            device="cuda")
        x.scatter_add_(1, hot, 3 * torch.randn((c["rows"], 24), generator=g,
                                               device="cuda") + 8)
        tgt = torch.where(torch.rand(c["rows"], generator=g, device="cuda") < 0.7,
                          hot[:, 0], torch.randint(0, c["vocab"], (c["rows"],),
                                                   generator=g, device="cuda"))
        f = dict(device="cuda", dtype=torch.float32)
        return dict(logits=x.to(dt), targets=tgt.to(torch.int32),
                    logp=torch.empty(c["rows"], **f),
                    entropy=torch.empty(c["rows"], **f),
                    top_logp=torch.empty((c["rows"], c["top"]), **f),
                    top_ids=torch.empty((c["rows"], c["top"]),
                                        device="cuda", dtype=torch.int32))
    H, Hk, D, P = c["heads"], c["kv_heads"], c["dim"], c["page"]
    if c["kind"] == "evict":
        n, keep, first, last = _keep(c)
        total, table, free = _pages(g, n, P, sum(-(-k // P) for k in keep))
        dst = torch.full((len(n), max(-(-k // P) for k in keep)), -1,
                         dtype=torch.int32, device="cuda")
        at = 0
        for s, k in enumerate(keep):
            m = -(-k // P)
            dst[s, :m] = free[at:at + m]
            at += m
        # weights as attention leaves them: many small, a heavy tail
        w = torch.exp(2.5 * torch.randn((len(n), max(n)), generator=g,
                                        device="cuda") - 6)
        return dict(k=_randn(g, (total, Hk, P, D), 1, dt),
                    v=_randn(g, (total, Hk, P, D), 1, dt), table=table,
                    dst=dst, n=n, keep=keep, first=first, last=last, weights=w,
                    kept=torch.full((len(n), max(keep)), -1, dtype=torch.int32,
                                    device="cuda"),
                    weights_out=torch.zeros((len(n), max(keep)), device="cuda"))
    lens = _lens(c)
    cu = [0]
    for n, _ in lens:
        cu.append(cu[-1] + n)
    kv = [n + p for n, p in lens]
    total, table, _ = _pages(g, kv, P)
    s = dict(cu=cu, kv=kv, table=table, block=c["block"], heads=H,
             scale=1.0 / math.sqrt(D))
    if c["kind"] == "append":
        s.update(k=torch.zeros((total, Hk, P, D), dtype=dt, device="cuda"),
                 v=torch.zeros((total, Hk, P, D), dtype=dt, device="cuda"),
                 qkv=_randn(g, (cu[-1], (H + 2 * Hk) * D), 1, dt),
                 q=torch.empty((cu[-1], H * D), dtype=dt, device="cuda"),
                 q_gain=1 + 0.2 * _randn(g, (D,), 1, torch.float32),
                 k_gain=1 + 0.2 * _randn(g, (D,), 1, torch.float32),
                 norm=c["norm"])
        return s
    s.update(k=_randn(g, (total, Hk, P, D), 1, dt),
             q=_randn(g, (cu[-1], H * D), 2, dt))
    if c["kind"] == "attend":
        s.update(v=_randn(g, (total, Hk, P, D), 1, dt),
                 out=torch.empty((cu[-1], H * D), dtype=dt, device="cuda"),
                 lse=torch.empty((cu[-1], H), device="cuda"))
    else:
        s.update(prev=torch.rand((len(kv), max(kv)), generator=g, device="cuda"),
                 weights=torch.zeros((len(kv), max(kv)), device="cuda"))
        s["lse"] = torch.cat([torch.logsumexp(x, 2).t() for x in
                              _scores(s, torch.float32)]).contiguous()
    return s


def prepare(c, seed):
    with torch.no_grad():
        s = _inputs(c, seed)
    s["c"] = c
    if own:
        import paper_2608_01821_amd as dv
        s["dv"] = dv
        s["dt"] = dict(f32=dv.DAVET_F32, bf16=dv.DAVET_BF16,
                       f16=dv.DAVET_F16)[c["dtype"]]
        nb = 0
        if c["kind"] == "score":
            nb = dv.davet_logprobs_workspace_bytes(c["rows"], c["vocab"], c["top"])
        else:
            s["cache"] = dv.KvCache(s["k"], s.get("v"), s["table"], s["dt"])
            if c["kind"] in ("attend", "weigh"):
                nb = dv.davet_cache_workspace_bytes(c["heads"], c["dim"],
                                                    s["cu"][-1])
        s["ws"] = torch.empty(max(nb, 256), dtype=torch.uint8, device="cuda")
    return s


# -------------------------------------------------------------------- runs --

def run(s):
    with torch.no_grad():
        return globals()[("_own_" if own else "_plain_") + s["c"]["kind"]](s)


def _own_append(s):
    s["dv"].davet_cache_append(s["cache"], s["cu"], s["kv"], s["qkv"],
                               s["heads"], s["q"], norm=s["norm"],
                               q_gain=s["q_gain"], k_gain=s["k_gain"], eps=EPS,
                               theta=THETA)
    return dict(q=s["q"], k=s["k"], v=s["v"])


def _own_attend(s):
    s["dv"].davet_cache_attention(s["cache"], s["cu"], s["kv"], s["q"],
                                  s["heads"], s["out"], lse=s["lse"],
                                  block=s["block"], workspace=s["ws"])
    return dict(out=s["out"], lse=s["lse"])


def _own_weigh(s):
    s["dv"].davet_cache_weights(s["cache"], s["cu"], s["kv"], s["q"],
                                s["heads"], s["lse"], s["weights"],
                                prev=s["prev"], block=s["block"],
                                workspace=s["ws"])
    return s["weights"]


def _own_evict(s):
    s["dv"].davet_evict_select(s["n"], s["keep"], s["weights"], s["kept"],
                               first=s["first"], last=s["last"],
                               weights_out=s["weights_out"])
    s["dv"].davet_cache_gather(s["cache"], s["kept"], s["keep"], s["dst"])
    return dict(kept=s["kept"], weights=s["weights_out"], k=s["k"], v=s["v"])


def _own_score(s):
    s["dv"].davet_token_logprobs(s["logits"], s["dt"], s["targets"], s["logp"],
                                 s["entropy"], s["top_logp"], s["top_ids"],
                                 exclude=s["c"]["vocab"] - 1, workspace=s["ws"])
    return dict(logp=s["logp"], entropy=s["entropy"], top_logp=s["top_logp"],
                top_ids=s["top_ids"])


def _slots(s, i, lo, hi):
    """(page, offset) of cache indices lo .. hi of sequence i."""
    j = torch.arange(lo, hi, device="cuda")
    P = s["k"].shape[2]
    return s["table"][i].long()[j // P], j % P


def _turn(x, pos, norm, gain, dtype):
    """Per-head norm and rotation of x [rows, heads, D], in `dtype`."""
    D = x.shape[2]
    x = x.to(dtype)
    if norm:
        x = x * torch.rsqrt((x * x).mean(2, keepdim=True) + EPS) * gain.to(dtype)
    inv = THETA ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)
    ang = pos.double()[:, None] * inv
    c, n = ang.cos().to(dtype)[:, None], ang.sin().to(dtype)[:, None]
    a, b = x[..., :D // 2], x[..., D // 2:]
    return torch.cat([a * c - b * n, b * c + a * n], 2)


def _plain_append(s, dtype=torch.float32):
    H, (_, Hk, _, D) = s["heads"], s["k"].shape
    for i in range(len(s["kv"])):
        r0, r1, kv = s["cu"][i], s["cu"][i + 1], s["kv"][i]
        x = s["qkv"][r0:r1].view(r1 - r0, H + 2 * Hk, D)
        pos = torch.arange(kv - (r1 - r0), kv, device="cuda")
        q = _turn(x[:, :H], pos, s["norm"], s["q_gain"], dtype)
        k = _turn(x[:, H:H + Hk], pos, s["norm"], s["k_gain"], dtype)
        page, off = _slots(s, i, kv - (r1 - r0), kv)
        s["q"][r0:r1] = q.reshape(r1 - r0, H * D).to(s["q"].dtype)
        s["k"][page, :, off] = k.to(s["k"].dtype)
        s["v"][page, :, off] = x[:, H + Hk:].to(s["v"].dtype)
    return dict(q=s["q"], k=s["k"], v=s["v"])


def _seq(s, name, i, dtype):
    """[kv_heads, keys, D] of sequence i."""
    P = s["k"].shape[2]
    n = s["kv"][i]
    x = s[name][s["table"][i, :-(-n // P)].long()].to(dtype)
    return x.permute(1, 0, 2, 3).reshape(x.shape[1], -1, x.shape[3])[:, :n]


def _scores(s, dtype):
    """Scaled scores [heads, queries, keys] of each sequence, -inf where a key
    is not visible."""
    H, (_, Hk, _, D) = s["heads"], s["k"].shape
    for i in range(len(s["kv"])):
        n = s["cu"][i + 1] - s["cu"][i]
        q = s["q"][s["cu"][i]:s["cu"][i + 1]].to(dtype).view(n, Hk, H // Hk, D)
        q = q.permute(1, 2, 0, 3).reshape(Hk, H // Hk * n, D)
        k = _seq(s, "k", i, dtype)
        x = torch.matmul(q, k.transpose(1, 2).contiguous())
        x = x.view(H, n, -1) * s["scale"]
        if s["block"]:
            end = torch.tensor(_visible(n, s["kv"][i] - n, s["block"]),
                               device="cuda")
            x = x.masked_fill(torch.arange(s["kv"][i], device="cuda") >=
                              end[:, None], -math.inf)
        yield x


def _plain_attend(s, dtype=torch.float32):
    H, (_, Hk, _, D) = s["heads"], s["k"].shape
    for i, x in enumerate(_scores(s, dtype)):
        r0, r1 = s["cu"][i], s["cu"][i + 1]
        m = x.amax(2, keepdim=True)
        p = torch.exp(x - m)
        den = p.sum(2, keepdim=True)
        o = torch.matmul(p.view(Hk, -1, p.shape[2]), _seq(s, "v", i, dtype))
        o = o.view(H, r1 - r0, D) / den
        s["out"][r0:r1] = o.permute(1, 0, 2).reshape(r1 - r0, H * D).to(
            s["out"].dtype)
        s["lse"][r0:r1] = (m + den.log())[..., 0].t().to(s["lse"].dtype)
    return dict(out=s["out"], lse=s["lse"])


def _plain_weigh(s, dtype=torch.float32):
    for i, x in enumerate(_scores(s, dtype)):
        lse = s["lse"][s["cu"][i]:s["cu"][i + 1]].t().to(dtype)
        w = torch.exp(x - lse[..., None]).sum((0, 1))
        s["weights"][i, :s["kv"][i]] = (
            s["prev"][i, :s["kv"][i]].to(dtype) + w).to(s["weights"].dtype)
    return s["weights"]


def _plain_evict(s):
    for i, (n, keep) in enumerate(zip(s["n"], s["keep"])):
        w = s["weights"][i, :n].clone()
        w[:s["first"]] = math.inf
        w[n - s["last"]:] = math.inf
        idx = torch.sort(w, descending=True, stable=True)[1][:keep].sort()[0]
        s["kept"][i, :keep] = idx.to(torch.int32)
        s["weights_out"][i, :keep] = s["weights"][i, idx]
        P = s["k"].shape[2]
        j = torch.arange(keep, device="cuda")
        src, dst = s["table"][i].long()[idx // P], s["dst"][i].long()[j // P]
        for x in (s["k"], s["v"]):
            x[dst, :, j % P] = x[src, :, idx % P]
    return dict(kept=s["kept"], weights=s["weights_out"], k=s["k"], v=s["v"])


def _plain_score(s, dtype=torch.float32):
    x = s["logits"].to(dtype)
    ids = torch.arange(x.shape[1], device="cuda")
    x = x.masked_fill(ids == s["c"]["vocab"] - 1, -math.inf)
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    S = e.sum(1, keepdim=True)
    logp = x - m - S.log()
    z = torch.where(e > 0, e * (x - m), torch.zeros_like(x)).sum(1)
    s["logp"][:] = logp.gather(1, s["targets"].long()[:, None])[:, 0]
    s["entropy"][:] = S[:, 0].log() - z / S[:, 0]
    v, i = torch.sort(x, dim=1, descending=True, stable=True)
    s["top_ids"][:] = i[:, :s["c"]["top"]].to(torch.int32)
    s["top_logp"][:] = v[:, :s["c"]["top"]] - m - S.log()
    return dict(logp=s["logp"], entropy=s["entropy"], top_logp=s["top_logp"],
                top_ids=s["top_ids"])


# ------------------------------------------------------------------- exact --

def exact(c, seed):
    """What run() returns, from the definitions in 64 bits, one sequence (and
    one head) at a time."""
    with torch.no_grad():
        s = _inputs(c, seed)
        return globals()["_exact_" + c["kind"]](c, s)


def _rows(s, name, i, head):
    """Keys or values [n, D] of sequence i and key/value head `head`."""
    P, n = s[name].shape[2], s["kv"][i]
    return torch.cat([s[name][int(p), head] for p in
                      s["table"][i, :-(-n // P)].tolist()])[:n].double()


def _exact_append(c, s):
    H, Hk, D, P = c["heads"], c["kv_heads"], c["dim"], c["page"]
    half = D // 2
    q = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    k = torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda")
    v = torch.zeros(s["v"].shape, dtype=torch.float64, device="cuda")
    d = torch.arange(half, device="cuda", dtype=torch.float64)
    freq = torch.exp(-math.log(THETA) * 2 * d / D)
    for i, kv in enumerate(s["kv"]):
        n = s["cu"][i + 1] - s["cu"][i]
        x = s["qkv"][s["cu"][i]:s["cu"][i + 1]].double().view(n, H + 2 * Hk, D)
        at = torch.arange(kv - n, kv, device="cuda")
        turn = torch.polar(torch.ones((n, half), dtype=torch.float64,
                                      device="cuda"), at[:, None] * freq)
        page, off = s["table"][i].long()[at // P], at % P
        for h in range(H + Hk):
            y = x[:, h]
            if c["norm"]:
                y = y / (y.pow(2).sum(1, keepdim=True) / D + EPS).sqrt()
                y = y * (s["q_gain"] if h < H else s["k_gain"]).double()
            z = torch.complex(y[:, :half].contiguous(),
                              y[:, half:].contiguous()) * turn
            y = torch.cat([z.real, z.imag], 1)
            if h < H:
                q[s["cu"][i]:s["cu"][i + 1], h * D:(h + 1) * D] = y
            else:
                k[page, h - H, off] = y
        for h in range(Hk):
            v[page, h, off] = x[:, H + Hk + h]
    return dict(q=q, k=k, v=v)


def _exact_pairs(c, s):
    """For each sequence and head: its number, query rows, scores in 64 bits."""
    g, D = c["heads"] // c["kv_heads"], c["dim"]
    for i, kv in enumerate(s["kv"]):
        r0, r1 = s["cu"][i], s["cu"][i + 1]
        for h in range(c["heads"]):
            if h % g == 0:
                key = _rows(s, "k", i, h // g).t().contiguous()
            x = s["q"][r0:r1, h * D:(h + 1) * D].double() @ key / math.sqrt(D)
            if c["block"]:
                r = torch.arange(r1 - r0, device="cuda")
                end = kv - (r1 - r0) + (r // c["block"] + 1) * c["block"]
                x[torch.arange(kv, device="cuda")[None] >= end[:, None]] = -math.inf
            yield i, h, r0, r1, x


def _exact_attend(c, s):
    g, D = c["heads"] // c["kv_heads"], c["dim"]
    out = torch.empty(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda")
    for i, h, r0, r1, x in _exact_pairs(c, s):
        lse[r0:r1, h] = torch.logsumexp(x, 1)
        p = torch.exp(x - lse[r0:r1, h, None])
        out[r0:r1, h * D:(h + 1) * D] = p @ _rows(s, "v", i, h // g)
    return dict(out=out, lse=lse)


def _exact_weigh(c, s):
    w = torch.zeros(s["weights"].shape, dtype=torch.float64, device="cuda")
    for i, h, r0, r1, x in _exact_pairs(c, s):
        w[i, :s["kv"][i]] += torch.exp(
            x - s["lse"][r0:r1, h, None].double()).sum(0)
    for i, n in enumerate(s["kv"]):
        w[i, :n] += s["prev"][i, :n].double()
    return w


def _exact_evict(c, s):
    # choices and copies of given values: nothing is computed
    return None


def _exact_score(c, s):
    logp, ent, top = [], [], []
    for r in range(c["rows"]):
        x = s["logits"][r].double()
        x[c["vocab"] - 1] = -math.inf
        lp = x - torch.logsumexp(x, 0)
        p = lp.exp()
        logp.append(lp[s["targets"][r].long()])
        ent.append(-(p[p > 0] * lp[p > 0]).sum())
        top.append(lp.topk(c["top"])[0])
    return dict(logp=torch.stack(logp), entropy=torch.stack(ent),
                top_logp=torch.stack(top), top_ids=None)
