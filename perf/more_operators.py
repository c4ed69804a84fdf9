"""Performance cases of rotary positions, draft trees, page selection and beams
on one MI355X.

Each case is the calls a program makes together:

  rotary  davet_rotary: queries and keys turned by their positions (halves or
          pairs, part of the head, scaled frequencies; or turned back)
  tree    davet_tree_plan + davet_cache_tree_attention: a tree of drafted
          tokens over the paged cache
  page    davet_cache_page_bounds + davet_cache_page_select +
          davet_cache_page_attention: new tokens attend the pages of a long
          cache that a cheap score selects for each
  beam    davet_beam_select + davet_cache_reorder: the best continuations of
          every beam, and the cache's pages moved along

`own` false: the same operators written with elementary torch operations.
"""

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
THETA = 10000.0
TREE = 256           # most drafted tokens of a sequence: bits of a mask row


# ------------------------------------------------------------------- cases --

def _rotary(name, **kw):
    # `heads` of `width` elements, the first `dim` of each turned; `far`: the
    # largest position; `beside`: columns of the row that are not turned (the
    # values of a projected row)
    c = dict(kind="rotary", dtype="f16", rows=1, heads=40, width=128, dim=128,
             pairs=False, scaling="plain", far=4096, beside=1024, back=False)
    c.update(kw, name=name)
    return c


def _cache(kind, name, **kw):
    # 32 heads x 128 as in the 8B-shaped workloads, 8 key heads; `past` cached
    # tokens before the `new` ones (the largest of a ragged batch), `page`
    # tokens a page
    c = dict(kind=kind, dtype="f16", seqs=1, mix=0, heads=32, kv_heads=8,
             dim=128, page=64, past=0, new=1, even=True)
    if kind == "page":
        c.update(top=32, first=1, last=2, block=1)
    c.update(kw, name=name)
    return c


def _beam(name, **kw):
    c = dict(kind="beam", dtype="f32", groups=1, beams=4, vocab=126464, past=2964,
             page=64, kv_heads=8, dim=128, cache="f16")
    c.update(kw, name=name)
    return c


def listed():
    return [
        # one token of one request far into a long context: latency only
        _rotary("rotary-token", scaling="ramp", far=131072),
        # view, prompt and response of four crops enter the cache, half of each
        # head turned in neighbouring pairs
        _rotary("rotary-prompt", dtype="bf16", rows=3092, dim=64, pairs=True,
                scaling="linear", far=16384),
        # gradients of sixteen responses turned back, heads of 80 with 32 turned
        _rotary("rotary-back-f32", dtype="f32", rows=4099, heads=32, width=80,
                dim=32, scaling="base", beside=0, back=True),
        # the tiny fp32 model checks thirteen drafted tokens
        _cache("tree", "tree-tiny-f32", dtype="f32", heads=4, kv_heads=4, dim=64,
               page=16, past=160, new=13),
        # eight long histories, a tree of 26 drafted tokens each
        _cache("tree", "tree-tokens-long", seqs=8, mix=3, past=32700, new=26),
        # sixteen ragged requests over view and prompt of one to five crops,
        # trees of 32 to 64 tokens
        _cache("tree", "tree-ragged16", dtype="bf16", seqs=16, mix=5, kv_heads=32,
               page=16, past=3741, new=64, even=False),
        # one token of one request, a third of whose history is read
        _cache("page", "page-token", page=16, past=2964, top=64),
        # eight histories of up to 65,400 tokens, 4096 of them read for each
        # new token
        _cache("page", "page-tokens-long", seqs=8, mix=3, past=65400, top=64),
        # sixteen ragged requests refine a 32-token block, every token with
        # its own choice of pages
        _cache("page", "page-block-ragged16", dtype="bf16", seqs=16, mix=5,
               page=16, past=3741, new=32, top=32, block=0),
        # four beams of one request: the smallest call
        _beam("beam-4"),
        # sixteen requests with four beams each, 16-bit logits
        _beam("beam-64", dtype="bf16", groups=16, past=2999),
        # four requests with sixteen beams
        _beam("beam-wide", dtype="bf16", groups=4, beams=16, past=977, page=16),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rotary", "tree", "tree", "page", "page", "beam"])
    if kind == "rotary":
        width = rng.choice([64, 80, 96, 128, 128, 256])
        dim = rng.choice([width, width, width // 2, width // 4,
                          rng.randrange(2, width + 1, 2)])
        c = dict(kind=kind, dtype=rng.choice(["f32", "bf16", "f16"]),
                 rows=log_int(1, 8000), heads=rng.randint(1, 64), width=width,
                 dim=max(2, dim), pairs=rng.random() < 0.5,
                 scaling=rng.choice(["plain", "linear", "base", "ramp"]),
                 far=log_int(100, 1000000), beside=rng.choice([0, 0, 1024, 24]),
                 back=rng.random() < 0.3)
        while work(c)["bytes"] > 1.5e8:
            c["rows"] = c["rows"] * 2 // 3
        return c
    if kind == "beam":
        c = dict(kind=kind, dtype=rng.choice(["f32", "bf16", "f16"]),
                 groups=rng.choice([1, 1, 2, 5, 8, 16]),
                 beams=rng.choice([1, 2, 3, 4, 5, 8, 16]),
                 vocab=log_int(300, 160000), past=log_int(1, 4000),
                 page=rng.choice([16, 32, 64, 128, 256]),
                 kv_heads=rng.choice([1, 2, 4, 8]), dim=rng.choice([64, 128]),
                 cache=rng.choice(["f32", "bf16", "f16"]))
        while c["groups"] * c["beams"] > 64:
            c["groups"] = (c["groups"] + 1) // 2
        return c
    kv_heads = rng.choice([1, 2, 4, 8, 8, 32])
    c = dict(kind=kind, dtype=rng.choice(["f32", "bf16", "f16", "f16"]),
             seqs=rng.choice([1, 1, 2, 5, 8, 16, 64]),
             mix=rng.randint(1, 999), kv_heads=kv_heads,
             heads=kv_heads * (rng.choice([1, 1, 2, 4, 7]) if kv_heads < 32 else 1),
             dim=rng.choice([64, 128, 128]), page=rng.choice([16, 32, 64, 128, 256]),
             even=rng.random() < 0.5, past=log_int(1, 70000))
    if kind == "tree":
        c.update(new=log_int(1, TREE))
    else:
        c.update(new=rng.choice([1, 1, log_int(2, 64)]), top=log_int(2, 160),
                 block=rng.choice([0, 1, 1, 4]))
        c.update(first=min(c["top"] // 2, rng.choice([0, 1, 2])),
                 last=min(c["top"] // 2, rng.choice([0, 1, 3])))
    if c["dtype"] == "f32":
        c.update(past=min(c["past"], 9000))
    # no dearer than the largest listed cases of the kind
    while True:
        w = work(c)
        rows = c["seqs"] * c["new"] * c["kv_heads"]
        read = rows * c["top"] * c["page"] * c["dim"] if kind == "page" else 0
        if w["bytes"] <= 9e8 and read <= 6e8 and \
                w["flops"] <= (2e10 if c["dtype"] == "f32" else 7e10):
            return c
        if c["seqs"] > 1:
            c["seqs"] = (c["seqs"] + 1) // 2
        elif c["new"] > 16:
            c["new"] = c["new"] * 2 // 3
        elif kind == "page" and c["top"] > 16:
            c["top"] = c["top"] * 2 // 3
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
    """Keys visible to each of the chunk's tokens."""
    if block == 0:
        return [past + new] * new
    return [past + min(new, (i // block + 1) * block) for i in range(new)]


def work(c):
    es = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "rotary":
        n = c["rows"] * c["heads"]
        return {"bytes": 2 * n * c["width"] * es + 4 * c["rows"],
                "flops": 3.0 * n * c["dim"]}
    if c["kind"] == "beam":
        rows = c["groups"] * c["beams"]
        ce = 4 if c["cache"] == "f32" else 2
        part = (c["past"] % c["page"]) * 2 * c["kv_heads"] * c["dim"] * ce
        return {"bytes": rows * (c["vocab"] * es + 16 + 2 * part +
                                 8 * -(-c["past"] // c["page"])),
                "flops": 4.0 * rows * c["vocab"]}
    row, lens = c["dim"] * es, _lens(c)
    rows = sum(n for n, _ in lens)
    io = rows * c["heads"] * (2 * row + 4)
    if c["kind"] == "tree":
        kv = sum(n + p for n, p in lens)
        pairs = sum(n * (n + p) for n, p in lens)
        return {"bytes": io + 2 * kv * c["kv_heads"] * row + rows * (8 + TREE // 8),
                "flops": 4.0 * pairs * c["heads"] * c["dim"]}
    # bounds: the keys of the pages that the new tokens enter, once; select: the
    # bounds of all pages, once a sequence; attention: the pages chosen, each at
    # most once a sequence
    P, b, f = c["page"], io, 0.0
    for n, past in lens:
        own_pages = (past + n - 1) // P - past // P + 1
        np_ = [-(-v // P) for v in _visible(n, past, c["block"])]
        took = [min(c["top"], x) for x in np_]
        b += c["kv_heads"] * row * (own_pages * (P + 2) + 2 * np_[-1] +
                                    2 * P * min(np_[-1], sum(took)))
        b += 4 * n * c["kv_heads"] * c["top"]
        f += 4.0 * sum(took) * P * c["heads"] * c["dim"]
        f += 4.0 * sum(np_) * c["kv_heads"] * c["dim"]
    return {"bytes": b, "flops": f}


# ------------------------------------------------------------------ inputs --

def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + stream)
    return g


def _randn(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _pages(g, lens, page, pool_extra=3):
    """A pool's page count, a shuffled page table for these lengths, and the
    pages left."""
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


def _scaling(c):
    """The scaled frequencies' settings as a model's configuration has them."""
    if c["scaling"] == "ramp":
        return dict(factor=8.0, trained=8192.0, fast=32.0, slow=1.0,
                    gain=0.1 * math.log(8.0) + 1.0)
    return dict(factor=dict(plain=1.0, linear=4.0, base=4.0)[c["scaling"]],
                trained=0.0, fast=0.0, slow=0.0, gain=1.0)


def _inputs(c, seed):
    """Everything on the GPU that a call reads or writes, as plain torch."""
    g, dt = _gen(seed, 1), DTYPES[c["dtype"]]
    if c["kind"] == "rotary":
        cols = c["heads"] * c["width"]
        far = torch.randint(0, max(1, c["far"] - c["rows"]), (1,), generator=g,
                            device="cuda")
        return dict(x=_randn(g, (c["rows"], cols + c["beside"]), 1, dt),
                    out=torch.empty((c["rows"], cols), dtype=dt, device="cuda"),
                    pos=(far + torch.arange(c["rows"], device="cuda")).to(torch.int32))
    if c["kind"] == "beam":
        return _beam_inputs(c, g, dt)
    H, Hk, D, P = c["heads"], c["kv_heads"], c["dim"], c["page"]
    lens = _lens(c)
    cu = [0]
    for n, _ in lens:
        cu.append(cu[-1] + n)
    kv = [n + p for n, p in lens]
    total, table, _ = _pages(g, kv, P)
    s = dict(cu=cu, kv=kv, table=table, heads=H, scale=1.0 / math.sqrt(D),
             k=_randn(g, (total, Hk, P, D), 1, dt),
             v=_randn(g, (total, Hk, P, D), 1, dt),
             q=_randn(g, (cu[-1], H * D), 2, dt),
             out=torch.empty((cu[-1], H * D), dtype=dt, device="cuda"),
             lse=torch.empty((cu[-1], H), device="cuda"))
    if c["kind"] == "tree":
        # a draft: every token continues one of the few before it
        r = torch.rand(cu[-1], generator=g, device="cuda").tolist()
        parent = []
        for n, _ in lens:
            for i in range(n):
                lo = max(-1, i - 7)
                parent.append(lo + int(r[len(parent)] * (i - lo)))
        s.update(parent=torch.tensor(parent, dtype=torch.int32, device="cuda"),
                 pos=torch.empty(cu[-1], dtype=torch.int32, device="cuda"),
                 mask=torch.empty((cu[-1], TREE // 32), dtype=torch.int32,
                                  device="cuda"))
    else:
        # some stretches of a history matter more: keys drift from page to page
        s["k"] = (s["k"].float() + 0.7 * torch.randn(
            (total, Hk, 1, D), generator=g, device="cuda")).to(dt)
        s.update(block=c["block"], first=c["first"], last=c["last"], top=c["top"],
                 bounds=torch.stack([s["k"].amin(2), s["k"].amax(2)], 2),
                 pages=torch.empty((cu[-1], Hk, c["top"]), dtype=torch.int32,
                                   device="cuda"))
    return s


def _beam_inputs(c, g, dt):
    rows, P = c["groups"] * c["beams"], c["page"]
    # a few plausible tokens stand out of a broad floor; the mask token is never
    # an answer
    x = torch.randn((rows, c["vocab"]), generator=g, device="cuda") * 2
    hot = torch.randint(0, c["vocab"], (rows, 24), generator=g, device="cuda")
    x.scatter_add_(1, hot, 3 * torch.randn((rows, 24), generator=g,
                                           device="cuda") + 8)
    # a beam has its last two pages to itself and shares the others with those
    # of its request
    n, cd = -(-c["past"] // P), DTYPES[c["cache"]]
    shared = max(0, n - 2)
    total = c["groups"] * shared + rows * (n - shared + 1)
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.empty((rows, n), dtype=torch.int32, device="cuda")
    table[:, :shared] = order[:c["groups"] * shared].view(
        c["groups"], shared).repeat_interleave(c["beams"], 0)
    rest = order[c["groups"] * shared:].view(rows, -1)
    table[:, shared:] = rest[:, :-1]
    shape = (total, c["kv_heads"], P, c["dim"])
    f = dict(device="cuda")
    return dict(logits=x.to(dt), k=_randn(g, shape, 1, cd), v=_randn(g, shape, 1, cd),
                table=table, fresh=rest[:, -1].contiguous(),
                dst=torch.full((rows, n + 1), -1, dtype=torch.int32, **f),
                kv=[c["past"]] * rows,
                scores=-5 - 2 * torch.rand(rows, generator=g, **f),
                out_scores=torch.empty((c["groups"], c["beams"]), **f),
                out_rows=torch.empty((c["groups"], c["beams"]),
                                     dtype=torch.int32, **f),
                out_tokens=torch.empty((c["groups"], c["beams"]),
                                       dtype=torch.int32, **f))


def prepare(c, seed):
    with torch.no_grad():
        s = _inputs(c, seed)
    s["c"] = c
    if own:
        import paper_2608_01821_amd as dv
        codes = dict(f32=dv.DAVET_F32, bf16=dv.DAVET_BF16, f16=dv.DAVET_F16)
        s["dv"], s["dt"], nb = dv, codes[c["dtype"]], 0
        if c["kind"] == "rotary":
            p = _scaling(c)
            kinds = dict(plain=dv.DAVET_ROTARY_PLAIN, linear=dv.DAVET_ROTARY_LINEAR,
                         base=dv.DAVET_ROTARY_BASE, ramp=dv.DAVET_ROTARY_RAMP)
            s["gain"] = p.pop("gain")
            s["turns"] = torch.tensor(
                dv.davet_rotary_turns(c["dim"], THETA, kinds[c["scaling"]], **p),
                dtype=torch.float64, device="cuda")
            s["layout"] = dv.DAVET_ROTARY_PAIRS if c["pairs"] else \
                dv.DAVET_ROTARY_HALVES
            return s
        if c["kind"] == "beam":
            nb = dv.davet_beam_workspace_bytes(c["groups"], c["beams"], c["vocab"],
                                               c["beams"])
            s["cache"] = dv.KvCache(s["k"], s["v"], s["table"], codes[c["cache"]])
        else:
            s["cache"] = dv.KvCache(s["k"], s["v"], s["table"], s["dt"])
            nb = dv.davet_cache_workspace_bytes(c["heads"], c["dim"], s["cu"][-1])
        s["ws"] = torch.empty(max(nb, 256), dtype=torch.uint8, device="cuda")
    return s


# -------------------------------------------------------------------- runs --

def run(s):
    with torch.no_grad():
        return globals()[("_own_" if own else "_plain_") + s["c"]["kind"]](s)


def _own_rotary(s):
    c = s["c"]
    s["dv"].davet_rotary(s["x"], c["heads"], c["width"], s["turns"], s["out"],
                         s["dt"], pos=s["pos"], layout=s["layout"],
                         gain=s["gain"], inverse=c["back"])
    return s["out"]


def _own_tree(s):
    s["dv"].davet_tree_plan(s["cu"], s["kv"], s["parent"], pos=s["pos"],
                            mask=s["mask"])
    s["dv"].davet_cache_tree_attention(s["cache"], s["cu"], s["kv"], s["q"],
                                       s["heads"], s["mask"], s["out"],
                                       lse=s["lse"], workspace=s["ws"])
    return dict(pos=s["pos"], mask=s["mask"], out=s["out"], lse=s["lse"])


def _own_page(s):
    s["dv"].davet_cache_page_bounds(s["cache"], s["cu"], s["kv"], s["bounds"])
    s["dv"].davet_cache_page_select(s["cache"], s["cu"], s["kv"], s["q"],
                                    s["heads"], s["bounds"], s["pages"],
                                    first=s["first"], last=s["last"],
                                    block=s["block"])
    s["dv"].davet_cache_page_attention(s["cache"], s["cu"], s["kv"], s["q"],
                                       s["heads"], s["pages"], s["out"],
                                       lse=s["lse"], block=s["block"],
                                       workspace=s["ws"])
    return dict(bounds=s["bounds"], pages=s["pages"], out=s["out"], lse=s["lse"])


def _own_beam(s):
    s["dv"].davet_beam_select(s["logits"], s["dt"], s["scores"], s["c"]["beams"],
                              s["out_scores"], s["out_rows"], s["out_tokens"],
                              exclude=s["c"]["vocab"] - 1, workspace=s["ws"])
    s["dv"].davet_cache_reorder(s["cache"], s["kv"], s["out_rows"].view(-1),
                                s["fresh"], s["dst"])
    return dict(scores=s["out_scores"], rows=s["out_rows"], tokens=s["out_tokens"],
                table=s["dst"], k=s["k"], v=s["v"])


def _plain_rotary(s):
    c, p = s["c"], _scaling(s["c"])
    dim, half = c["dim"], c["dim"] // 2
    i = torch.arange(half, device="cuda", dtype=torch.float64)
    base = THETA
    if c["scaling"] == "base" and dim > 2:
        base = THETA * p["factor"] ** (dim / (dim - 2))
    f = base ** (-2 * i / dim)
    if c["scaling"] == "linear":
        f = f / p["factor"]
    if c["scaling"] == "ramp":
        keep = (p["trained"] * f / (2 * math.pi) - p["slow"]) / (p["fast"] - p["slow"])
        keep = keep.clamp(0, 1)
        f = f * keep + f / p["factor"] * (1 - keep)
    ang = s["pos"].double()[:, None] * f            # 64 bits: far positions
    co = (ang.cos() * p["gain"]).float()[:, None]
    si = (ang.sin() * (-p["gain"] if c["back"] else p["gain"])).float()[:, None]
    x = s["x"][:, :c["heads"] * c["width"]].float().view(c["rows"], c["heads"], -1)
    y = x.clone()
    lo, hi = (slice(0, dim, 2), slice(1, dim, 2)) if c["pairs"] else \
        (slice(0, half), slice(half, dim))
    a, b = x[..., lo], x[..., hi]
    y[..., lo], y[..., hi] = a * co - b * si, b * co + a * si
    s["out"][:] = y.view(c["rows"], -1).to(s["out"].dtype)
    return s["out"]


def _softmax_rows(x, v):
    """(outputs, log of the sum) of scores x [.., keys] over v [.., keys, D]."""
    m = x.amax(-1, keepdim=True)
    m = torch.where(m > -math.inf, m, torch.zeros_like(m))
    p = torch.exp(x - m)
    den = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(den > 0, den, torch.ones_like(den))
    return o, (m + den.log())[..., 0]


def _plain_tree(s):
    H, (_, Hk, P, D) = s["heads"], s["k"].shape
    s["mask"].zero_()
    for i, kv in enumerate(s["kv"]):
        r0, r1 = s["cu"][i], s["cu"][i + 1]
        n = r1 - r0
        parent = s["parent"][r0:r1].long()
        # who is above whom: parents, then twice as far up at a time
        up = torch.eye(n, device="cuda")
        at = torch.arange(n, device="cuda")[parent >= 0]
        up[at, parent[parent >= 0]] = 1
        for _ in range((n - 1).bit_length()):
            up = (torch.matmul(up, up) > 0).float()
        seen = up > 0
        depth = seen.sum(1) - 1
        s["pos"][r0:r1] = (kv - n + depth).to(torch.int32)
        bit = torch.arange(n, device="cuda")
        for w in range(-(-n // 32)):
            b = seen[:, 32 * w:32 * w + 32].long() << (bit[32 * w:32 * w + 32] % 32)
            s["mask"][r0:r1, w] = b.sum(1).to(torch.int32)
        page = s["table"][i, :-(-kv // P)].long()
        k, v = (s[t][page].float().permute(1, 0, 2, 3).reshape(Hk, -1, D)[:, :kv]
                for t in ("k", "v"))
        q = s["q"][r0:r1].float().view(n, Hk, H // Hk, D).permute(1, 2, 0, 3)
        x = torch.matmul(q.reshape(Hk, -1, D), k.transpose(1, 2).contiguous())
        x = (x * s["scale"]).view(Hk, H // Hk, n, kv)
        x[..., kv - n:] = x[..., kv - n:].masked_fill(~seen, -math.inf)
        o, lse = _softmax_rows(x.view(Hk, -1, kv), v)
        s["out"][r0:r1] = o.view(H, n, D).permute(1, 0, 2).reshape(n, -1).to(
            s["out"].dtype)
        s["lse"][r0:r1] = lse.view(H, n).t()
    return dict(pos=s["pos"], mask=s["mask"], out=s["out"], lse=s["lse"])


def _plain_page(s):
    c, H, (_, Hk, P, D) = s["c"], s["heads"], s["k"].shape
    g, top = H // Hk, s["top"]
    for i, kv in enumerate(s["kv"]):
        r0, r1 = s["cu"][i], s["cu"][i + 1]
        n = r1 - r0
        for p in range((kv - n) // P, (kv - 1) // P + 1):
            at = s["table"][i, p].long()
            k = s["k"][at, :, :min(P, kv - p * P)]
            s["bounds"][at, :, 0], s["bounds"][at, :, 1] = k.amin(1), k.amax(1)
        np_ = -(-kv // P)
        page = s["table"][i, :np_].long()
        b = s["bounds"][page].double()                       # [pages, Hk, 2, D]
        ends = torch.tensor(_visible(n, kv - n, s["block"]), device="cuda")
        idx = torch.arange(np_, device="cuda")
        for a0 in range(0, n, 16):                           # rows at a time
            a1 = min(n, a0 + 16)
            q = s["q"][r0 + a0:r0 + a1].view(a1 - a0, Hk, g, D)
            qd = q.double()
            # in 64 bits, for the borders of the choice
            score = (torch.matmul(qd.clamp(min=0).sum(2).permute(1, 0, 2),
                                  b[:, :, 1].permute(1, 2, 0).contiguous()) +
                     torch.matmul(qd.clamp(max=0).sum(2).permute(1, 0, 2),
                                  b[:, :, 0].permute(1, 2, 0).contiguous()))
            score = score.float().permute(1, 0, 2)           # [rows, Hk, pages]
            end = ends[a0:a1, None]
            mine = -(-end // P)                              # its pages
            sure = (idx < s["first"]) | (idx >= mine - s["last"])
            score = score.masked_fill(sure[:, None], math.inf)
            score = score.masked_fill((idx >= mine)[:, None], -math.inf)
            took = torch.sort(score, dim=2, descending=True, stable=True)[1]
            took = took[..., :top]
            m = took.shape[2]
            none = torch.arange(m, device="cuda") >= mine.clamp(max=top)
            took = took.masked_fill(none[:, None], np_).sort(2)[0]
            s["pages"][r0 + a0:r0 + a1] = -1
            s["pages"][r0 + a0:r0 + a1, :, :m] = torch.where(
                took < np_, took, torch.full_like(took, -1)).to(torch.int32)
            at = page[took.clamp(max=np_ - 1)]               # [rows, Hk, m]
            h = torch.arange(Hk, device="cuda")[:, None]
            k, v = (s[t][at, h].float().view(a1 - a0, Hk, m * P, D)
                    for t in ("k", "v"))
            key = (took[..., None] * P + torch.arange(P, device="cuda")).flatten(2)
            x = torch.matmul(q.float(), k.transpose(2, 3).contiguous()) * s["scale"]
            x = x.masked_fill((key >= end[:, None])[:, :, None], -math.inf)
            o, lse = _softmax_rows(x, v)
            s["out"][r0 + a0:r0 + a1] = o.reshape(a1 - a0, -1).to(s["out"].dtype)
            s["lse"][r0 + a0:r0 + a1] = lse.reshape(a1 - a0, -1)
    return dict(bounds=s["bounds"], pages=s["pages"], out=s["out"], lse=s["lse"])


def _plain_beam(s):
    c, P = s["c"], s["c"]["page"]
    n = c["beams"]
    # in 64 bits: two beams' candidates may lie close together
    x = s["logits"].double()
    x[:, c["vocab"] - 1] = -math.inf
    m = x.amax(1, keepdim=True)
    x = s["scores"].double()[:, None] + (x - m) - torch.exp(x - m).sum(
        1, keepdim=True).log()
    v, at = torch.sort(x.view(c["groups"], -1), dim=1, descending=True, stable=True)
    v, at = v[:, :n], at[:, :n]
    base = torch.arange(c["groups"], device="cuda")[:, None] * n
    s["out_scores"][:] = v.float()
    s["out_rows"][:] = (base + at // c["vocab"]).to(torch.int32)
    s["out_tokens"][:] = (at % c["vocab"]).to(torch.int32)
    parent = s["out_rows"].view(-1).long()
    whole, rest = c["past"] // P, c["past"] % P
    s["dst"][:, :whole] = s["table"][parent, :whole]
    if rest:
        old, new = s["table"][parent, whole].long(), s["fresh"].long()
        s["dst"][:, whole] = s["fresh"]
        for t in (s["k"], s["v"]):
            t[new, :, :rest] = t[old, :, :rest]
    return dict(scores=s["out_scores"], rows=s["out_rows"], tokens=s["out_tokens"],
                table=s["dst"], k=s["k"], v=s["v"])


# ------------------------------------------------------------------- exact --

def exact(c, seed):
    """What run() returns, from the definitions in 64 bits, one sequence and
    head at a time; None for choices and copies."""
    with torch.no_grad():
        return globals()["_exact_" + c["kind"]](c, _inputs(c, seed))


def _exact_rotary(c, s):
    p, half = _scaling(c), c["dim"] // 2
    freq = []
    for i in range(half):
        f = THETA ** (-2.0 * i / c["dim"])
        if c["scaling"] == "linear":
            f /= p["factor"]
        elif c["scaling"] == "base" and c["dim"] > 2:
            f *= p["factor"] ** (-2.0 * i / (c["dim"] - 2))
        elif c["scaling"] == "ramp":
            r = (p["trained"] * f / (2 * math.pi) - p["slow"]) / (p["fast"] - p["slow"])
            f = f / p["factor"] + min(1.0, max(0.0, r)) * (f - f / p["factor"])
        freq.append(f)
    t = s["pos"].double()[:, None] * torch.tensor(freq, dtype=torch.float64,
                                                  device="cuda")
    turn = torch.polar(torch.full_like(t, p["gain"]), -t if c["back"] else t)
    out = s["x"][:, :c["heads"] * c["width"]].double()
    for h in range(c["heads"]):
        x = out[:, h * c["width"]:h * c["width"] + c["dim"]]     # a view
        if c["pairs"]:
            z = torch.view_as_complex(x.reshape(-1, half, 2).contiguous()) * turn
            x[:] = torch.view_as_real(z).reshape(-1, c["dim"])
        else:
            z = torch.complex(x[:, :half].contiguous(), x[:, half:].contiguous())
            z = z * turn
            x[:, :half], x[:, half:] = z.real, z.imag
    return out


def _exact_heads(c, s, seen):
    """(out, lse) in 64 bits; seen(sequence, key head): what its rows see of
    its keys, [rows, keys]."""
    g, D, P = c["heads"] // c["kv_heads"], c["dim"], c["page"]
    out = torch.empty(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda")
    for i, kv in enumerate(s["kv"]):
        r0, r1 = s["cu"][i], s["cu"][i + 1]
        pages = s["table"][i, :-(-kv // P)].long()
        for h in range(c["heads"]):
            if h % g == 0:
                key = s["k"][pages, h // g].reshape(-1, D)[:kv].double()
                val = s["v"][pages, h // g].reshape(-1, D)[:kv].double()
                see = seen(i, h // g)
            x = s["q"][r0:r1, h * D:(h + 1) * D].double() @ key.t().contiguous()
            x = x / math.sqrt(D)
            x[~see] = -math.inf
            lse[r0:r1, h] = torch.logsumexp(x, 1)
            out[r0:r1, h * D:(h + 1) * D] = torch.softmax(x, 1) @ val
    return out, lse


def _exact_tree(c, s):
    parent = s["parent"].tolist()

    def seen(i, _):
        r0, n, kv = s["cu"][i], s["cu"][i + 1] - s["cu"][i], s["kv"][i]
        see = torch.ones((n, kv), dtype=torch.bool)
        see[:, kv - n:] = False
        for r in range(n):
            if parent[r0 + r] >= 0:
                see[r] = see[parent[r0 + r]]
            see[r, kv - n + r] = True
        return see.cuda()

    out, lse = _exact_heads(c, s, seen)
    return dict(pos=None, mask=None, out=out, lse=lse)


def _exact_page(c, s):
    if s["cu"][-1] * c["kv_heads"] > 20000:
        return None                     # (a choice at a time: too many)
    g, D, P = c["heads"] // c["kv_heads"], c["dim"], c["page"]

    def seen(i, h):
        r0, n, kv = s["cu"][i], s["cu"][i + 1] - s["cu"][i], s["kv"][i]
        np_ = -(-kv // P)
        lo = torch.empty((np_, D), dtype=torch.float64, device="cuda")
        hi = torch.empty_like(lo)
        k = s["k"][s["table"][i, :np_].long(), h].double()
        lo[:], hi[:] = k.amin(1), k.amax(1)
        rest = kv - (np_ - 1) * P
        lo[-1], hi[-1] = k[-1, :rest].amin(0), k[-1, :rest].amax(0)
        see = torch.zeros((n, kv), dtype=torch.bool, device="cuda")
        end = _visible(n, kv - n, c["block"])
        for r in range(n):
            q = s["q"][r0 + r].double().view(-1, D)[h * g:(h + 1) * g]
            m = -(-end[r] // P)
            score = torch.maximum(q[:, None] * lo[:m], q[:, None] * hi[:m]).sum((0, 2))
            score = score.float()
            score[:c["first"]] = math.inf
            score[max(0, m - c["last"]):] = math.inf
            took = torch.argsort(-score, stable=True)[:c["top"]]
            on = torch.zeros(np_, dtype=torch.bool, device="cuda")
            on[took] = True
            see[r] = on.repeat_interleave(P)[:kv]
            see[r, end[r]:] = False
        return see

    out, lse = _exact_heads(c, s, seen)
    return dict(bounds=None, pages=None, out=out, lse=lse)


def _exact_beam(c, s):
    best = []
    for b in range(c["groups"]):
        v = []
        for r in range(b * c["beams"], (b + 1) * c["beams"]):
            x = s["logits"][r].double()
            x[c["vocab"] - 1] = -math.inf
            v.append(s["scores"][r].double() + torch.log_softmax(x, 0))
        best.append(torch.cat(v).topk(c["beams"])[0])
    return dict(scores=torch.stack(best), rows=None, tokens=None, table=None,
                k=None, v=None)
