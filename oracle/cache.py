"""The paged cache and the token log probabilities in float64, one sequence,
head and token at a time, with no tiling and no running statistics.

A cache here is a dict: k, v [n_pages, n_kv_heads, page_size, head_dim] and
table [n_seqs, max_pages]; an entry of the table outside [0, n_pages) is a hole.
"""

import numpy as np


def slot(cache, s, j):
    """(page, offset) of cache index j of sequence s, or None in a hole."""
    n_pages, _, size, _ = cache["k"].shape
    page = int(cache["table"][s, j // size])
    return (page, j % size) if 0 <= page < n_pages else None


def turned(x, pos, theta):
    """Elements (i, i + D/2) of x [D] turned by pos * theta^(-2i/D)."""
    half = len(x) // 2
    a = float(pos) * float(theta) ** (-2.0 * np.arange(half) / len(x))
    c, s = np.cos(a), np.sin(a)
    return np.concatenate([x[:half] * c - x[half:] * s,
                           x[half:] * c + x[:half] * s])


def append(cache, cu_q, kv_len, qkv, n_heads, pos=None, norm=False, q_gain=None,
           k_gain=None, eps=1e-6, theta=10000.0):
    """(queries [rows, n_heads, D], new k, new v), the caches as copies."""
    k, v = cache["k"].astype(np.float64), cache["v"].astype(np.float64)
    _, hk, _, D = k.shape
    x = np.asarray(qkv, np.float64).reshape(len(qkv), -1, D)
    q = np.zeros((cu_q[-1], n_heads, D))
    for s, kv in enumerate(kv_len):
        for r in range(cu_q[s], cu_q[s + 1]):
            j = kv - cu_q[s + 1] + r
            p = j if pos is None else pos[r]
            at = slot(cache, s, j)
            for h in range(n_heads + hk):
                y, gain = x[r, h], q_gain if h < n_heads else k_gain
                if norm:
                    y = y / np.sqrt(np.mean(y * y) + eps)
                    y = y if gain is None else y * np.asarray(gain, np.float64)
                y = turned(y, p, theta)
                if h < n_heads:
                    q[r, h] = y
                elif at:
                    k[at[0], h - n_heads, at[1]] = y
            if at:
                v[at[0], :, at[1]] = x[r, n_heads + hk:]
    return q, k, v


def visible(cache, s, i, n, kv, block):
    """Cache indices that query i of a chunk of n sees."""
    end = kv if block == 0 else kv - n + min(n, (i // block + 1) * block)
    return [j for j in range(end) if slot(cache, s, j)]


def gathered(cache, name, s, h, js):
    at = [slot(cache, s, j) for j in js]
    out = np.zeros((len(js), cache["k"].shape[3]))
    for i, (p, o) in enumerate(at):
        out[i] = cache[name][p, h, o]
    return out


def attention(cache, cu_q, kv_len, q, n_heads, scale=0.0, block=0):
    """dict of out, lse and, for error bounds, `mass` = sum p |v| of every
    output element and `dot` = max_j scale sum |q k_j| of every row and head;
    q [rows, n_heads, D]."""
    _, hk, _, D = cache["k"].shape
    q = np.asarray(q, np.float64).reshape(len(q), n_heads, D)
    scale = scale or 1.0 / np.sqrt(D)
    rows = cu_q[-1]
    r = dict(out=np.zeros((rows, n_heads, D)), mass=np.zeros((rows, n_heads, D)),
             lse=np.full((rows, n_heads), -np.inf), dot=np.zeros((rows, n_heads)))
    for s, kv in enumerate(kv_len):
        n = cu_q[s + 1] - cu_q[s]
        for h in range(n_heads):
            g = h // (n_heads // hk)
            every = [j for j in range(kv) if slot(cache, s, j)]
            k = gathered(cache, "k", s, g, every)
            v = gathered(cache, "v", s, g, every)
            for i in range(n):
                m = len(visible(cache, s, i, n, kv, block))
                if m == 0:
                    continue
                row = cu_q[s] + i
                x = scale * (k[:m] @ q[row, h])
                top = x.max()
                if top == -np.inf:              # zeros, lse -inf
                    continue
                e = np.exp(x - top)
                p = e / e.sum()
                r["out"][row, h] = p @ v[:m]
                r["mass"][row, h] = p @ np.abs(v[:m])
                r["lse"][row, h] = top + np.log(e.sum())
                r["dot"][row, h] = scale * (np.abs(k[:m]) @ np.abs(q[row, h])).max()
    return r


def attention_of(cache, cu_q, kv_len, q, n_heads, seen, scale=0.0):
    """attention() where seen(s, i, h) lists the cache indices that row i of
    sequence s sees of key head h (those in holes hold no keys)."""
    _, hk, _, D = cache["k"].shape
    q = np.asarray(q, np.float64).reshape(len(q), n_heads, D)
    scale = scale or 1.0 / np.sqrt(D)
    rows = cu_q[-1]
    r = dict(out=np.zeros((rows, n_heads, D)), mass=np.zeros((rows, n_heads, D)),
             lse=np.full((rows, n_heads), -np.inf), dot=np.zeros((rows, n_heads)))
    for s in range(len(kv_len)):
        for row in range(cu_q[s], cu_q[s + 1]):
            for g in range(hk):
                js = [j for j in seen(s, row - cu_q[s], g) if slot(cache, s, j)]
                if not js:
                    continue
                k = gathered(cache, "k", s, g, js)
                v = gathered(cache, "v", s, g, js)
                for h in range(g * (n_heads // hk), (g + 1) * (n_heads // hk)):
                    x = scale * (k @ q[row, h])
                    top = x.max()
                    if top == -np.inf:
                        continue
                    e = np.exp(x - top)
                    p = e / e.sum()
                    r["out"][row, h] = p @ v
                    r["mass"][row, h] = p @ np.abs(v)
                    r["lse"][row, h] = top + np.log(e.sum())
                    r["dot"][row, h] = scale * (np.abs(k) @ np.abs(q[row, h])).max()
    return r


def above(parent):
    """For each drafted token of one tree, those above it and itself, ascending."""
    out = []
    for i, p in enumerate(parent):
        out.append((out[p] if 0 <= p < i else []) + [i])
    return out


def page_bounds(cache, cu_q, kv_len, bounds):
    """bounds [n_pages, n_kv_heads, 2, D] with those of the chunk's pages brought up
    to date: the elementwise smallest and largest of the keys below kv_len."""
    b = np.array(bounds, np.float64)
    _, hk, size, _ = cache["k"].shape
    for s, kv in enumerate(kv_len):
        n = cu_q[s + 1] - cu_q[s]
        for page in sorted({j // size for j in range(kv - n, kv)}):
            js = [j for j in range(page * size, min(kv, page * size + size))]
            if slot(cache, s, js[0]):
                for h in range(hk):
                    k = gathered(cache, "k", s, h, js)
                    b[cache["table"][s, page], h] = k.min(0), k.max(0)
    return b


def page_select(cache, cu_q, kv_len, q, n_heads, bounds, top, first=0, last=0,
                block=0):
    """[rows][n_kv_heads] lists of the pages that each new token reads."""
    n_pages, hk, size, D = cache["k"].shape
    q = np.asarray(q, np.float64).reshape(len(q), hk, n_heads // hk, D)
    out = []
    for s, kv in enumerate(kv_len):
        n = cu_q[s + 1] - cu_q[s]
        for i in range(n):
            end = kv if block == 0 else kv - n + min(n, (i // block + 1) * block)
            count = -(-end // size)
            there = [p for p in range(count) if 0 <= cache["table"][s, p] < n_pages]
            row = []
            for h in range(hk):
                score = {}
                for p in there:
                    lo, hi = bounds[cache["table"][s, p], h].astype(np.float64)
                    x = np.float32(np.maximum(q[cu_q[s] + i, h] * lo,
                                              q[cu_q[s] + i, h] * hi).sum())
                    score[p] = np.float32(-np.inf) if np.isnan(x) else x
                if count <= top:
                    row.append(there)
                    continue
                sure = [p for p in there if p < first or p >= count - last]
                rest = sorted((p for p in there if p not in sure),
                              key=lambda p: (-score[p], p))
                row.append(sorted(sure + rest[:top - len(sure)]))
            out.append(row)
    return out


def weights(cache, cu_q, kv_len, q, n_heads, lse, scale=0.0, block=0):
    """[n_seqs, max kv]: what each cached key received."""
    _, hk, _, D = cache["k"].shape
    q = np.asarray(q, np.float64).reshape(len(q), n_heads, D)
    scale = scale or 1.0 / np.sqrt(D)
    w = np.zeros((len(kv_len), max(kv_len)))
    for s, kv in enumerate(kv_len):
        n = cu_q[s + 1] - cu_q[s]
        for h in range(n_heads):
            for i in range(n):
                js = visible(cache, s, i, n, kv, block)
                row = cu_q[s] + i
                if not js or lse[row, h] == -np.inf:
                    continue
                k = gathered(cache, "k", s, h // (n_heads // hk), js)
                w[s, js] += np.exp(scale * (k @ q[row, h]) - float(lse[row, h]))
    return w


def select(n, keep, w, first=0, last=0):
    """Indices that stay, ascending: the first and last ones, then by (weight
    descending, index ascending), NaN with -inf."""
    w = [-np.inf if np.isnan(x) else float(x) for x in w[:n]]
    sure = [j for j in range(n) if j < first or j >= n - last] if keep else []
    rest = sorted((j for j in range(n) if j not in set(sure)),
                  key=lambda j: (-w[j], j))
    return sorted(sure + rest[:keep - len(sure)])


def logprobs(x, target, exclude=-1, top=0):
    """(logp of the target, entropy, [(id, logp)] of the top) of one row."""
    x = np.array(x, np.float64)
    if 0 <= exclude < len(x):
        x[exclude] = -np.inf
    order = sorted((j for j in range(len(x)) if x[j] > -np.inf),
                   key=lambda j: (-x[j], j))
    if not order and not np.isnan(x).any():
        return -np.inf, 0.0, []
    with np.errstate(invalid="ignore"):
        m = x[order[0]] if order else np.nan
        z = m + np.log(np.sum(np.exp(x - m)))
        lp = x - z
        p = np.exp(lp)
        ent = -np.sum(np.where(p == 0, 0.0, p * np.where(p == 0, 0.0, lp)))
    out = -np.inf
    if 0 <= target < len(x) and target != exclude:
        out = lp[target]
    return out, ent, [(j, lp[j]) for j in order[:top]]


def beam_select(x, scores, beams, top, exclude=-1, done=None, pad=0):
    """For each request the `top` best (value, row, token); x [rows, vocab]."""
    out = []
    for g in range(len(x) // beams):
        cands = []
        for r in range(g * beams, (g + 1) * beams):
            score = float(scores[r])
            if done is not None and done[r]:
                if np.isfinite(score):
                    cands.append((-score, r, 0.0, pad))
                continue
            row = np.array(x[r], np.float64)
            if 0 <= exclude < len(row):
                row[exclude] = -np.inf
            with np.errstate(invalid="ignore"):
                m = row[row > -np.inf].max() if (row > -np.inf).any() else np.nan
                lse = m + np.log(np.sum(np.exp(row - m)))
            if not np.isfinite(score - lse):
                continue
            best = sorted((j for j in range(len(row)) if row[j] > -np.inf),
                          key=lambda j: (-row[j], j))[:top]
            cands += [(-(score + row[j] - lse), r, -row[j], j) for j in best]
        out.append([(-v, r, j) for v, r, _, j in sorted(cands)[:top]])
    return out


def reorder(cache, kv_len, parent, fresh, dst):
    """(k, v, dst) after the cache moved along, as copies."""
    n_pages, _, size, _ = cache["k"].shape
    k, v, dst = cache["k"].copy(), cache["v"].copy(), np.array(dst)
    for s, kv in enumerate(kv_len):
        known = 0 <= parent[s] < len(kv_len)
        whole, rest = kv // size, kv % size
        dst[s, :whole] = cache["table"][parent[s], :whole] if known else -1
        if rest:
            a = int(cache["table"][parent[s], whole]) if known else -1
            b = int(fresh[s])
            move = 0 <= a < n_pages and 0 <= b < n_pages
            dst[s, whole] = b if move else -1
            if move:
                k[b, :, :rest] = cache["k"][a, :, :rest]
                v[b, :, :rest] = cache["v"][a, :, :rest]
    return k, v, dst
