"""Paged caches for the tests: seeded values on the host, their exact 16-bit
(or fp32) copies on the device, shuffled pages."""

import numpy as np
import torch

import paper_2608_01821_amd as dv

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CODE = {"f32": dv.DAVET_F32, "f16": dv.DAVET_F16, "bf16": dv.DAVET_BF16}


def half_step(dtype):
    """Largest relative error of one rounding."""
    return torch.finfo(TORCH[dtype]).eps / 2


def values(rng, shape, dtype, std=1.0):
    """A host tensor of `dtype`."""
    return torch.from_numpy(rng.standard_normal(shape) * std).to(TORCH[dtype])


def f64(t):
    return t.detach().cpu().double().numpy()


def page_table(rng, kv_len, page, extra=2, max_pages=None):
    """(n_pages, table): each sequence's pages at random places of the pool,
    unused entries -1."""
    counts = [-(-n // page) for n in kv_len]
    total = sum(counts) + extra
    order = rng.permutation(total).astype(np.int32)
    width = max_pages or max(1, max(counts))
    table = np.full((len(kv_len), width), -1, np.int32)
    at = 0
    for s, c in enumerate(counts):
        table[s, :c] = order[at:at + c]
        at += c
    return total, table


class Setup:
    """A cache with keys and values everywhere (also outside the sequences)."""

    def __init__(self, seed, dtype, new, kv, heads, kv_heads, dim, page,
                 q_std=2.0, fill=None):
        rng = np.random.default_rng(seed)
        self.rng, self.dtype, self.heads = rng, dtype, heads
        self.cu = [0] + [int(x) for x in np.cumsum(new)]
        self.kv = list(kv)
        total, self.table = page_table(rng, kv, page)
        shape = (total, kv_heads, page, dim)
        self.k, self.v = values(rng, shape, dtype), values(rng, shape, dtype)
        if fill is not None:            # outside the sequences
            used = np.zeros((total, page), bool)
            for s, n in enumerate(kv):
                for j in range(n):
                    used[self.table[s, j // page], j % page] = True
            out = torch.from_numpy(~used)[:, None, :, None].expand(shape)
            self.k[out], self.v[out] = fill, fill
        self.q = values(rng, (self.cu[-1], heads * dim), dtype, q_std)

    @property
    def host(self):
        return dict(k=f64(self.k), v=f64(self.v), table=self.table)

    def device(self):
        self.dk, self.dv = self.k.cuda(), self.v.cuda()
        self.dtable = torch.from_numpy(self.table).cuda()
        return dv.KvCache(self.dk, self.dv, self.dtable, CODE[self.dtype])

    def workspace(self):
        n = dv.davet_cache_workspace_bytes(self.heads, self.k.shape[3],
                                           max(1, self.cu[-1]))
        return torch.empty(n, dtype=torch.uint8, device="cuda")

    def attend(self, cache=None, block=0, scale=0.0):
        """(out [rows, heads, D], lse [rows, heads]) as float64 arrays."""
        cache = cache or self.device()
        q = self.q.cuda()
        out = torch.full_like(q, 7.0)
        lse = torch.full((len(q), self.heads), 7.0, device="cuda")
        dv.davet_cache_attention(cache, self.cu, self.kv, q, self.heads, out,
                                 lse=lse, scale=scale, block=block,
                                 workspace=self.workspace())
        torch.cuda.synchronize()
        return f64(out).reshape(len(q), self.heads, -1), f64(lse)


def check_attention(got, ref, dtype, dim, keys):
    """Element by element against the float64 reference.  A score is a sum of
    `dim` products in fp32: off by at most dim 2^-24 times the sum of their
    magnitudes, and by the roundings of the exponent's argument (a multiply-add
    and the constant: 3 2^-24 of the largest score); that moves every weight by
    twice as much, relative.  The output adds one rounding of each weight to the
    element type, the fp32 sums over the keys, and its own store."""
    out, lse = got
    u = half_step(dtype)
    dot = ref["dot"][..., None]
    ds = (dim + 3) * 2.0 ** -24 * dot
    tol = u * np.abs(ref["out"]) + ref["mass"] * (
        (u if dtype != "f32" else 0) + 2 * ds + (keys + 64) * 2.0 ** -24) + 1e-30
    err = np.abs(out - ref["out"])
    assert np.all(err <= tol), (err / tol).max()
    empty = np.isneginf(ref["lse"])
    assert np.array_equal(np.isneginf(lse), empty)
    d = np.abs(lse[~empty] - ref["lse"][~empty])
    tol = (ds[..., 0] + (keys + 64) * 2.0 ** -24 +
           4 * 2.0 ** -24 * (1 + np.abs(ref["dot"]) + np.abs(
               np.where(empty, 0, ref["lse"]))))[~empty]
    assert np.all(d <= tol), (d / tol).max()
