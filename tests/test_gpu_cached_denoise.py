"""The cached operators together, as a serving loop uses them: view and prompt
enter the cache, the response block is refined against it step by step, visual
evidence leaves by the weight it received, positions commit by log probability;
every quantity against the float64 oracle.  Then the ways of calling: captured
and replayed, on other streams, twice, several calls at once."""

import numpy as np
import pytest
import torch

import paper_2608_01821_amd as dv
from cache_util import (CODE, TORCH, Setup, check_attention, f64, half_step,
                        page_table, values)
from oracle import cache as oc

pytestmark = pytest.mark.gpu


class Loop:
    """One layer's cache of two requests on both sides, the host's fed what the
    device holds."""

    def __init__(self, dtype, heads, hk, dim, page):
        self.rng = np.random.default_rng(17)
        self.dtype, self.heads, self.hk, self.dim, self.page = dtype, heads, hk, dim, page
        total = 64
        self.k = torch.full((total, hk, page, dim), float("nan"),
                            dtype=TORCH[dtype], device="cuda")
        self.v = self.k.clone()
        self.free = [int(p) for p in self.rng.permutation(total)]
        self.table = torch.full((2, 24), -1, dtype=torch.int32, device="cuda")
        self.q_gain = torch.from_numpy(1 + .2 * self.rng.standard_normal(dim)).float().cuda()
        self.k_gain = torch.from_numpy(1 + .2 * self.rng.standard_normal(dim)).float().cuda()
        self.ws = torch.empty(dv.davet_cache_workspace_bytes(heads, dim, 400),
                              dtype=torch.uint8, device="cuda")
        self.cache = dv.KvCache(self.k, self.v, self.table, CODE[dtype])

    def host(self):
        return dict(k=f64(self.k), v=f64(self.v), table=self.table.cpu().numpy())

    def room(self, kv):
        """Pages for kv[s] entries of each request."""
        t = self.table.cpu()
        for s, n in enumerate(kv):
            for i in range(-(-n // self.page)):
                if t[s, i] < 0:
                    t[s, i] = self.free.pop()
        self.table.copy_(t)

    def chunk(self, new, kv, pos, block=0):
        """Enters a chunk and attends: (query tensor, out, lse), checked."""
        cu = [0, new[0], new[0] + new[1]]
        width = (self.heads + 2 * self.hk) * self.dim
        qkv = values(self.rng, (cu[-1], width), self.dtype).cuda()
        self.room(kv)
        before = self.host()
        q = torch.empty(cu[-1], self.heads * self.dim, dtype=TORCH[self.dtype],
                        device="cuda")
        out = torch.empty_like(q)
        lse = torch.empty(cu[-1], self.heads, device="cuda")
        p = torch.from_numpy(np.asarray(pos, np.int32)).cuda()
        dv.davet_cache_append(self.cache, cu, kv, qkv, self.heads, q, pos=p,
                              norm=True, q_gain=self.q_gain, k_gain=self.k_gain)
        dv.davet_cache_attention(self.cache, cu, kv, q, self.heads, out, lse=lse,
                                 block=block, workspace=self.ws)
        torch.cuda.synchronize()
        rq, rk, rv = oc.append(before, cu, kv, f64(qkv), self.heads, pos=pos,
                               norm=True, q_gain=f64(self.q_gain),
                               k_gain=f64(self.k_gain))
        u = half_step(self.dtype)
        # norms make every element at most sqrt(D) gains; one rounding, and the
        # fp32 steps before it (see the append tests)
        for got, ref in ((f64(q).reshape(rq.shape), rq), (f64(self.k), rk)):
            top = np.nanmax(np.abs(ref))
            assert np.nanmax(np.abs(got - ref)) <= u * top + 64 * 2.0 ** -24 * top
            assert np.array_equal(np.isnan(got), np.isnan(ref))
        assert np.array_equal(f64(self.v), rv, equal_nan=True)
        # attention against the oracle on what the device's cache now holds
        ref = oc.attention(self.host(), cu, kv, f64(q), self.heads, block=block)
        check_attention((f64(out).reshape(rq.shape), f64(lse)), ref, self.dtype,
                        self.dim, max(kv))
        return cu, q, lse, ref


@pytest.mark.parametrize("dtype,heads,hk,dim,page", [
    ("f16", 4, 2, 128, 16), ("bf16", 4, 4, 64, 32), ("f32", 2, 1, 64, 16)])
def test_cached_denoising_with_eviction(dtype, heads, hk, dim, page):
    lp = Loop(dtype, heads, hk, dim, page)
    visual, prompt, resp = [80, 49], [7, 12], 9
    pre = [a + b for a, b in zip(visual, prompt)]
    weights = torch.zeros(2, max(pre) + resp, device="cuda")
    # 1. view and prompt enter, bidirectional among themselves
    pos = [p for n in pre for p in range(n)]
    lp.chunk(pre, pre, pos)
    # 2. two refinements of the response block over them: the same cache slots
    #    are written again, the weights that the cache received add up
    kv = [n + resp for n in pre]
    want = np.zeros((2, max(kv)))
    rpos = [p for n in pre for p in range(n, n + resp)]
    for _ in range(2):
        cu, q, lse, ref = lp.chunk([resp, resp], kv, rpos)
        dv.davet_cache_weights(lp.cache, cu, kv, q, heads, lse, weights,
                               prev=weights, workspace=lp.ws)
        torch.cuda.synchronize()
        want += oc.weights(lp.host(), cu, kv, f64(q), heads, f64(lse))
    for s in range(2):
        # as in the weights tests: scores off by dim 2^-24 of their magnitudes
        rel = (dim + 40 + resp * heads) * 2.0 ** -24 * (ref["dot"].max() + 8)
        assert np.all(np.abs(f64(weights)[s, :kv[s]] - want[s, :kv[s]])
                      <= rel * want[s, :kv[s]])
    # 3. half of the view and prompt leaves; the prompt stays for sure
    keep = [n // 2 for n in pre]
    kept = torch.full((2, max(keep)), -1, dtype=torch.int32, device="cuda")
    left = torch.zeros(2, max(pre) + resp, device="cuda")
    dv.davet_evict_select(pre, keep, weights, kept, first=1, last=min(prompt),
                          weights_out=left)
    dst = torch.full((2, 24), -1, dtype=torch.int32)
    for s in range(2):
        for i in range(-(-keep[s] // page)):
            dst[s, i] = lp.free.pop()
    before = lp.host()
    dst = dst.cuda()
    dv.davet_cache_gather(lp.cache, kept, keep, dst)
    torch.cuda.synchronize()
    after = dict(lp.host(), table=dst.cpu().numpy())
    for s in range(2):
        idx = oc.select(pre[s], keep[s], f64(weights)[s], 1, min(prompt))
        assert kept[s, :keep[s]].tolist() == idx
        for h in range(hk):
            for name in ("k", "v"):
                assert np.array_equal(oc.gathered(after, name, s, h, range(keep[s])),
                                      oc.gathered(before, name, s, h, idx))
    lp.table.copy_(dst)
    # 4. the next block, token groups of 4 in turn, over what is left: its
    #    rotary positions go on where they were
    kv = [k + resp for k in keep]
    lp.chunk([resp, resp], kv, rpos, block=4)


def test_logprobs_drive_commitment():
    """Logits of a denoising step's open rows: the top alternative and its
    probability are the argmax and confidence that davet_unmask ranks by."""
    rng = np.random.default_rng(3)
    n, L, vocab = 2, 24, 1000
    logits = values(rng, (n * L, vocab), "f32", 3.0).cuda()
    top_lp = torch.empty(n * L, 1, device="cuda")
    top_id = torch.empty(n * L, 1, dtype=torch.int32, device="cuda")
    nb = dv.davet_logprobs_workspace_bytes(n * L, vocab, 1)
    ws = torch.empty(max(nb, 256), dtype=torch.uint8, device="cuda")
    dv.davet_token_logprobs(logits, dv.DAVET_F32, top_logp=top_lp, top_ids=top_id,
                            exclude=vocab - 1, workspace=ws)
    ids = torch.full((n * L,), vocab - 1, dtype=torch.int32, device="cuda")
    masked = torch.ones(n * L, dtype=torch.uint8, device="cuda")
    sel = torch.empty(n * 5, dtype=torch.int32, device="cuda")
    dv.davet_unmask(n, L, 5, top_lp.exp().reshape(-1), top_id.reshape(-1), ids,
                    masked, sel)
    torch.cuda.synchronize()
    host = f64(logits)
    for s in range(n):
        rows = [oc.logprobs(host[s * L + i], 0, vocab - 1, 1)[2][0] for i in range(L)]
        order = sorted(range(L), key=lambda i: -rows[i][1])[:5]
        assert sel[s * 5:s * 5 + 5].tolist() == order
        for i in order:
            assert int(ids[s * L + i]) == rows[i][0]


def test_step_logits_give_its_confidences():
    """davet_denoise_step's logits through davet_token_logprobs: its argmaxes
    and confidences."""
    import synth
    cfg = synth.get_any_config(11)
    s = synth.gen_sample(cfg)

    def dev(a):
        return torch.from_numpy(np.ascontiguousarray(a, np.float32).astype(
            np.float16)).cuda()
    W = dv.Weights(dev(synth.gen_embed(cfg)), dev(synth.gen_head(cfg)), [
        {k: dev(x) for k, x in synth.gen_layer_weights(cfg, i).items()}
        for i in range(cfg.n_layers)])
    v, prompt, L = s["visual"][0], s["prompts"][0], cfg.resp_len
    m = dv.ModelCfg(cfg.n_layers, cfg.d, cfg.n_heads, cfg.head_dim, cfg.ffn,
                    cfg.vocab, cfg.mask_id, cfg.rms_eps, cfg.rope_theta,
                    dv.DAVET_F16)
    ws = torch.empty(dv.davet_workspace_bytes(m, len(v) + len(prompt) + L, 1, L),
                     dtype=torch.uint8, device="cuda")
    ids = torch.full((L,), cfg.mask_id, dtype=torch.int32, device="cuda")
    msk = torch.ones(L, dtype=torch.uint8, device="cuda")
    conf, am = torch.empty(L, device="cuda"), torch.empty(L, dtype=torch.int32,
                                                          device="cuda")
    logits = torch.empty(L, cfg.vocab, device="cuda")
    dv.davet_denoise_step(m, W, [dev(v)], [len(v)], torch.from_numpy(prompt).cuda(),
                          [0, len(prompt)], ids, msk, L, conf, am, logits, ws)
    lp, ent = torch.empty(L, device="cuda"), torch.empty(L, device="cuda")
    tl = torch.empty(L, 3, device="cuda")
    ti = torch.empty(L, 3, dtype=torch.int32, device="cuda")
    dv.davet_token_logprobs(logits, dv.DAVET_F32, targets=am, logp=lp, entropy=ent,
                            top_logp=tl, top_ids=ti, exclude=cfg.mask_id)
    torch.cuda.synchronize()
    assert torch.equal(ti[:, 0], am) and torch.equal(tl[:, 0], lp)
    # both sum exp in fp32: 1e-5 covers the vocabulary's 1000 terms twice
    assert np.abs(f64(lp.exp()) - f64(conf)).max() < 1e-5
    assert bool((ent >= 0).all()) and bool((tl[:, 0] >= tl[:, 1]).all())


# ------------------------------------------------------------ ways of calling --

def _everything(t, cache, ws, q, out, lse, w, kept, kw):
    dv.davet_cache_attention(cache, t.cu, t.kv, q, t.heads, out, lse=lse,
                             workspace=ws, **kw)
    dv.davet_cache_weights(cache, t.cu, t.kv, q, t.heads, lse, w, workspace=ws, **kw)
    s = {k: v for k, v in kw.items() if k == "stream"}
    dv.davet_evict_select(t.kv, [n // 2 for n in t.kv], w, kept, **s)


@pytest.mark.parametrize("new,kv,heads,hk", [([1, 1], [1700, 900], 8, 2),
                                             ([70, 80], [300, 500], 4, 2)])
def test_captured_replayed_and_repeated(new, kv, heads, hk):
    """Bit for bit the eager call's results, on every replay, with eager work in
    between and new inputs in the same buffers; two graphs have a workspace
    each."""
    t = Setup(31, "f16", new, kv, heads, hk, 128, 32)
    cache = t.device()
    q = t.q.cuda()

    def buffers():
        return (t.workspace(), torch.empty_like(q),
                torch.empty(len(q), heads, device="cuda"),
                torch.zeros(2, max(kv), device="cuda"),
                torch.full((2, max(kv)), -1, dtype=torch.int32, device="cuda"))

    eager = buffers()
    _everything(t, cache, eager[0], q, *eager[1:], {})
    torch.cuda.synchronize()
    again = buffers()
    _everything(t, cache, again[0], q, *again[1:], {})
    torch.cuda.synchronize()
    for a, b in zip(eager[1:], again[1:]):
        assert torch.equal(a, b)
    graphs = []
    for _ in range(2):
        b = buffers()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _everything(t, cache, b[0], q, *b[1:], {})
        graphs.append((g, b))
    for turn in range(3):
        q.copy_(t.q.cuda() * (1 + turn))
        ref = buffers()
        _everything(t, cache, ref[0], q, *ref[1:], {})
        torch.cuda.synchronize()
        for g, b in graphs:
            for x in b[1:]:
                x.zero_()
            b[4].fill_(-1)
            g.replay()
        torch.cuda.synchronize()
        for _, b in graphs:
            for x, y in zip(b[1:], ref[1:]):
                assert torch.equal(x, y)


def test_other_streams_and_two_calls_at_once():
    """Two requests on two streams, each with its workspace, while the default
    stream works."""
    ts = [Setup(40 + i, "bf16", [1], [2500], 8, 8, 128, 64) for i in range(2)]
    refs, runs = [], []
    for t in ts:
        c = t.device()
        b = (t.workspace(), torch.empty_like(t.q.cuda()),
             torch.empty(1, 8, device="cuda"), torch.zeros(1, 2500, device="cuda"),
             torch.zeros(1, 1250, dtype=torch.int32, device="cuda"))
        q = t.q.cuda()
        _everything(t, c, b[0], q, *b[1:], {})
        torch.cuda.synchronize()
        refs.append([x.clone() for x in b[1:]])
        for x in b[1:]:
            x.zero_()
        runs.append((t, c, b, q))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    junk = torch.zeros(1 << 20, device="cuda")
    for turn in range(4):
        for st, (t, c, b, q) in zip(streams, runs):
            # by handle, by object, and by the current stream
            if turn == 0:
                _everything(t, c, b[0], q, *b[1:], dict(stream=st.cuda_stream))
            elif turn == 1:
                _everything(t, c, b[0], q, *b[1:], dict(stream=st))
            else:
                with torch.cuda.stream(st):
                    _everything(t, c, b[0], q, *b[1:], {})
        junk.add_(1)
    torch.cuda.synchronize()
    for (t, c, b, q), ref in zip(runs, refs):
        for x, y in zip(b[1:], ref):
            assert torch.equal(x, y)


def test_pages_shared_by_two_requests():
    """A common prefix held once: both read its pages, each has its own after."""
    t = Setup(50, "f16", [3, 3], [70, 70], 2, 1, 64, 16)
    t.table[1, :3] = t.table[0, :3]
    ref = oc.attention(t.host, t.cu, t.kv, f64(t.q), 2)
    check_attention(t.attend(), ref, "f16", 64, 70)


def test_largest_batch():
    """64 requests of every length from none, and heads to the limit."""
    rng = np.random.default_rng(1)
    kv = [int(x) for x in rng.integers(0, 200, 64)]
    kv[:3] = [0, 1, 16]
    new = [min(n, int(rng.integers(0, 4))) for n in kv]
    t = Setup(60, "f16", new, kv, 6, 3, 64, 16, fill=float("nan"))
    ref = oc.attention(t.host, t.cu, t.kv, f64(t.q), 6, block=1)
    check_attention(t.attend(block=1), ref, "f16", 64, 200)
    t = Setup(61, "bf16", [2], [40], 1024, 512, 64, 16)
    ref = oc.attention(t.host, t.cu, t.kv, f64(t.q), 1024)
    check_attention(t.attend(), ref, "bf16", 64, 40)


def test_cpu_tensors_are_refused():
    t = Setup(70, "f16", [2], [20], 2, 1, 64, 16)
    c = t.device()
    q = t.q.cuda()
    with pytest.raises(ValueError):
        dv.davet_cache_attention(c, t.cu, t.kv, t.q, 2, torch.empty_like(q),
                                 workspace=t.workspace())
    with pytest.raises(ValueError):
        dv.davet_cache_attention(c, t.cu, t.kv, q, 2, torch.empty_like(q),
                                 workspace=t.workspace().cpu())
    with pytest.raises(dv.DavetError) as e:
        dv.davet_cache_attention(c, t.cu, t.kv, q, 2, torch.empty_like(q))
    assert e.value.status == -4
