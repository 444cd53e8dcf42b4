"""Plain forms in 64 bits, with numpy, of rotary positions, the paged cache and the
shaping of logits; and how far the library's float32 results may lie from them."""
import math

import numpy as np

U = 2.0 ** -24                                   # half a step of float32
HALF = {"f32": 0.0, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}     # half a step of the type, relative
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}   # half its smallest step
TORCH = {"f32": "float32", "f16": "float16", "bf16": "bfloat16"}


def torch_type(name):
    import torch
    return getattr(torch, TORCH[name])


def rounding(y, to):
    return HALF[to] * np.abs(y) + TINY[to]


def rotate(x, pos, freq, interleaved=False, scale=1.0, inverse=False):
    """x [N, H, d] float64 turned; and the bound on a float32 result: each of cosine, sine
    (rounded from 64 bits), product and sum is off by at most half a step of m (|a| + |b|)."""
    n = len(freq)
    t = np.asarray(pos, dtype=np.float64)[:, None] * freq
    c, s = scale * np.cos(t)[:, None], scale * np.sin(t)[:, None] * (-1.0 if inverse else 1.0)
    i = np.arange(n)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, n + i)
    y, tol = x.copy(), np.zeros_like(x)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    m = 4 * U * abs(scale) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    tol[..., a] = tol[..., b] = m
    return y, tol


def key_rows(k):
    """[n_pages, H, page/16, d/8, 16, 8] as [n_pages, H, page, d]."""
    n, h, p, c = k.shape[:4]
    return np.ascontiguousarray(k.transpose(0, 1, 2, 4, 3, 5)).reshape(n, h, p * 16, c * 8)


def value_rows(v):
    """[n_pages, H, page/8, d, 8] as [n_pages, H, page, d]."""
    n, h, p, d = v.shape[:4]
    return np.ascontiguousarray(v.transpose(0, 1, 2, 4, 3)).reshape(n, h, p * 8, d)


def attend(q, k, v, table, lens, window=0, sm_scale=None):
    """q [B, Hq, d], k and v [n_pages, H, page, d] float64 -> (out, tol).

    A score's float32 sum of d products is off by d U sum |q k| and its scaling by a step; that
    is a probability's relative error, once in the weight and once in the sum of weights.
    exp2, the reference and the split into terms add 2^-20, and T / 32 + 64 additions one U each.
    Probabilities below 2^-12 of the largest are kept to 2^-34 of it."""
    B, Hq, d = q.shape
    n_pages, H, page, _ = k.shape
    G = Hq // H
    sm = 1.0 / math.sqrt(d) if not sm_scale else sm_scale
    out, tol = np.zeros((B, Hq, d)), np.zeros((B, Hq, d))
    for b in range(B):
        n = min(max(int(lens[b]), 0), table.shape[1] * page)
        ts = [t for t in range(max(0, n - window) if window > 0 else 0, n) if 0 <= table[b, t // page] < n_pages]
        if not ts:
            continue
        at = [(int(table[b, t // page]), t % page) for t in ts]
        p, o = np.array([x[0] for x in at]), np.array([x[1] for x in at])
        for h in range(H):
            K, V = k[p, h, o], v[p, h, o]
            for g in range(G):
                s = sm * (K @ q[b, h * G + g])
                off = d * U * sm * (np.abs(K) @ np.abs(q[b, h * G + g])) + 4 * U * np.abs(s)
                w = np.exp(s - s.max())
                w /= w.sum()
                out[b, h * G + g] = w @ V
                rel = 2.0 * off.max() + 2.0 ** -20 + (len(ts) / 32 + 64) * U
                tol[b, h * G + g] = rel * (w @ np.abs(V)) + 2.0 ** -34 * np.abs(V).sum(0) + 1e-37
    return out, tol


def path_of(parent, i):
    """Nodes from node i up to node 0, node 0 not among them."""
    out = []
    while i > 0:
        out.append(i)
        i = parent[i] if parent[i] < i else -1
    return out


def shape_logits(l, params=None, history=None, history_len=None, prompt_len=None, bias=None, mask=None, tree=None, token=None,
                 probs=False):
    """Rows l [N, V] float64 -> (out, tol); tree (cu_nodes, parent)."""
    N, V = l.shape
    out, tol = np.zeros((N, V)), np.zeros((N, V))
    for i in range(N):
        b, path = i, []
        if tree is not None:
            cu, parent = tree
            b = max(k for k in range(len(cu) - 1) if cu[k] <= i)
            par = [int(x) for x in parent[cu[b]:cu[b + 1]]]
            path = [int(token[cu[b] + a]) for a in path_of(par, i - cu[b])]
        rep, pres, freq, temp = (float(x) for x in params[b]) if params is not None else (1.0, 0.0, 0.0, 1.0)
        ids, m = [], 0
        if history is not None:
            n = min(max(int(history_len[b]), 0), history.shape[1])
            ids = [int(x) for x in history[b, :n]]
            m = min(max(int(prompt_len[b]), 0), n) if prompt_len is not None else 0
        ok = lambda xs: [x for x in xs if 0 <= x < V]
        said = ok(ids[m:] + path)
        z = l[i].copy()
        seen = np.zeros(V, bool)
        seen[ok(ids)] = True
        seen[said] = True
        z[seen] = np.where(z[seen] > 0, z[seen] / rep, z[seen] * rep)
        with np.errstate(invalid="ignore"):
            big = np.abs(z)
            c = np.bincount(said, minlength=V).astype(np.float64) if said else np.zeros(V)
            z = np.where(c > 0, z - freq * c - pres, z)
            big = big + np.abs(freq) * c + np.abs(pres) * (c > 0)
            if bias is not None:
                start, bid, val = bias
                for e in range(max(int(start[b]), 0), min(int(start[b + 1]), len(bid))):
                    if 0 <= bid[e] < V:
                        z[bid[e]] += float(val[e])
                        big[bid[e]] += 2 * abs(float(val[e]))
            if mask is not None:
                t = np.arange(V)
                z = np.where((mask[i].view(np.uint32)[t // 32] >> (t % 32).astype(np.uint32)) & 1, z, -np.inf)
        off = 6 * U * np.where(np.isfinite(big), big, 0.0)
        if not probs:
            out[i], tol[i] = z, off
            continue
        live = ~np.isnan(z)
        top = z[live].max() if live.any() else -np.inf
        if not temp > 0:
            if top > -np.inf:
                out[i, int(np.argmax(np.where(live, z, -np.inf)))] = 1.0
            continue
        if np.isnan(z).any() or top == np.inf:
            out[i] = np.nan
            continue
        if top == -np.inf:
            continue
        x = (z - top) / temp
        p = np.exp(x)
        S = p.sum()
        out[i] = p / S
        # the exponent's error, relative in p: both entries' and the largest's, scaling, exp2;
        # the sum's is the mean of its entries', and V / 4096 + 32 additions
        fin = np.isfinite(x)
        e = 2 * off / temp + off[z == top].max() / temp + 4 * U * np.where(fin, np.abs(x), 0.0) + 2.0 ** -22
        tol[i] = out[i] * (e + float((p * e).sum() / S) + (V / 4096 + 48) * U) + 2.0 ** -120
    return out, tol


def check(got, want, tol, label):
    """Equal where want is not finite, within tol elsewhere."""
    got, want = np.asarray(got, dtype=np.float64), np.asarray(want)
    fin = np.isfinite(want)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    assert same[~fin].all(), f"{label}: numbers that are not finite differ at {np.argwhere(~fin & ~same)[:4].tolist()}"
    bad = fin & ~(np.abs(got - want) <= tol)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{label}: {bad.sum()} of {bad.size} off, first at {i}: {got[i]!r} for {want[i]!r}, allowed {np.broadcast_to(tol, got.shape)[i]:.3e}")
