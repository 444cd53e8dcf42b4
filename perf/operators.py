"""The operators of a speculative decoding step over the factorized cache, as measured cases.

A program that serves from the cache drafts a small tree of tokens per
sequence, scores all of them in one pass, keeps the ones that stand and lays the
cache out for what comes next:

* ``decode``  attention of a tree of drafted tokens over one layer of the
              factorized cache, each node seeing the cache and its ancestors
* ``verify``  which drafted tokens stand against the target's probabilities,
              from given random numbers, and the token that follows them
* ``repack``  a new packed cache from tokens of an old one: sequences forked,
              compacted, freed or grown

``run`` with ``own`` false computes them with elementary torch operations; with
``own`` true it calls the library.  The cache arrays are in the layouts of
include/dwkv.h.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

D = 128
DEV = "cuda"

_DECODE = {"kind": "decode", "batch": 1, "tokens": 65536, "ragged": False, "nodes": 16, "shape": "tree", "kv_heads": 8,
           "group": 4, "rank": 48, "levels": "0,4,8,16", "probs": "0.75,0.12,0.08,0.05", "q": "bf16", "coef": "f16"}
_VERIFY = {"kind": "verify", "batch": 1, "nodes": 16, "shape": "tree", "children": 4, "vocab": 131072, "draft": True,
           "p": "f32"}
_REPACK = {"kind": "repack", "use": "grow", "batch": 1, "tokens": 65536, "layers": 4, "window": 4, "kv_heads": 8,
           "rank": 48, "levels": "0,4,8,16", "probs": "0.75,0.12,0.08,0.05", "coef": "f16"}
_L70B = {"levels": "0,4,8,16,32", "probs": "0.70,0.12,0.10,0.06,0.02"}
_L3 = {"levels": "0,8,16", "probs": "0.80,0.15,0.05"}


def listed():
    def case(base, name, **kw):
        return {**base, "name": name, **kw}
    return [
        # the smallest call: a short context of a small model and a chain of 5 nodes, bound by latency
        case(_DECODE, "decode-1k-chain5", tokens=1000, nodes=5, shape="chain", kv_heads=2, rank=32, q="f16", **_L3),
        # an 8B-class decoder's layer at 64K with a small tree
        case(_DECODE, "decode-64k-tree8", nodes=8),
        # the same with the largest tree, whose products outweigh the cache's bytes
        case(_DECODE, "decode-64k-tree64", nodes=64),
        # a ragged serving batch (8K..16K tokens, up to 12 nodes), 8-bit blockwise coefficients
        case(_DECODE, "decode-batch16-int8", batch=16, tokens=16384, ragged=True, nodes=12, rank=32, coef="int8", **_L3),
        # the largest: a 70B-class decoder's layer, 2 x 128K, groups of 8, trees of 32
        case(_DECODE, "decode-70b-tree32", batch=2, tokens=131072, nodes=32, group=8, rank=64, **_L70B),
        # one chain of 4 drafts, sampled
        case(_VERIFY, "verify-chain5", nodes=5, shape="chain", children=1, vocab=32000),
        # one large sampled tree
        case(_VERIFY, "verify-tree64", nodes=64),
        # a batch of trees of the most likely tokens (no draft distribution), 16-bit probabilities
        case(_VERIFY, "verify-batch16-topk", batch=16, nodes=32, draft=False, p="bf16"),
        # a small cache that grows by a few slots
        case(_REPACK, "repack-grow-1k", tokens=1000, layers=2, window=2, kv_heads=2, rank=32, **_L3),
        # a 64K cache that grows
        case(_REPACK, "repack-grow-64k"),
        # a 16K prompt forked into four sequences
        case(_REPACK, "repack-fork-16k", use="fork", batch=4, tokens=16384),
        # a ragged batch: two sequences freed, a few tokens of each other one dropped, slots added
        case(_REPACK, "repack-compact-batch16-int8", use="compact", batch=16, tokens=8192, layers=2, window=2, rank=32,
             coef="int8", **_L3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any operator, sizes over the whole range of the listed cases."""
    kind = rng.choice(["decode", "decode", "verify", "repack"])
    if kind == "verify":
        c = dict(_VERIFY, batch=rng.choice([1, 1, 2, 3, 5, 16]), nodes=_log(rng, 1, 64), vocab=_log(rng, 1000, 131072))
        c["shape"] = rng.choice(["tree", "tree", "chain"])
        c["children"] = 1 if c["shape"] == "chain" else rng.choice([2, 3, 4, 6])
        c["draft"] = rng.random() < 0.6
        c["p"] = rng.choice(["f32", "f32", "bf16", "f16"])
        return c
    c = dict(_DECODE if kind == "decode" else _REPACK)
    c["kv_heads"] = rng.choice([1, 2, 4, 8])
    c["rank"] = rng.choice([16, 32, 32, 48, 48, 64, 96, 128])
    c["batch"] = rng.choice([1, 1, 1, 2, 3, 16])
    c["coef"] = rng.choice(["f16", "f16", "int8"])
    c.update(rng.choice([{}, _L3, _L70B]))
    if kind == "decode":
        c["q"] = rng.choice(["bf16", "f16"])
        c["group"] = rng.choice([1, 2, 4, 4, 8, 16])
        c["nodes"] = _log(rng, 1, 64)
        c["shape"] = rng.choice(["tree", "tree", "chain", "padded"])
        c["tokens"] = _log(rng, 1, 131072)
        c["ragged"] = c["batch"] > 1 and rng.random() < 0.7
        room = 2 * 131072 * 8 * 256 // (c["kv_heads"] * max(32, c["nodes"] * c["group"]))
        c["tokens"] = max(1, min(c["tokens"], min(262144, room) // c["batch"]))
    else:
        c["use"] = rng.choice(["grow", "fork", "compact"])
        c["layers"] = c["window"] = rng.choice([1, 2, 4])
        if c["use"] == "fork":
            c["batch"] = rng.choice([2, 3, 4, 8])
        c["tokens"] = min(_log(rng, 100, 65536), 65536 * 4 * 8 * 48 // (c["batch"] * c["layers"] * c["kv_heads"] * c["rank"]))
    return c


# ---- shapes -----------------------------------------------------------------------------------

def _shape_rng(case):
    return random.Random("%s/%d/%d" % (case["kind"], case["batch"], case.get("tokens", 0) + 7 * case.get("nodes", 0)))


def _lens(case):
    """Cached tokens of each sequence (of a repack: of the source)."""
    if case["kind"] == "repack":
        r = _shape_rng(case)
        if case["use"] == "fork":
            return [case["tokens"]]
        return [case["tokens"]] if case["batch"] == 1 else [r.randint(max(1, case["tokens"] // 2), case["tokens"])
                                                             for _ in range(case["batch"])]
    if not case["ragged"]:
        return [case["tokens"]] * case["batch"]
    r = _shape_rng(case)
    return [r.randint(max(1, case["tokens"] // 2), case["tokens"]) for _ in range(case["batch"])]


def _node_counts(case):
    if not case.get("ragged") and case["kind"] == "decode" or case["batch"] == 1:
        return [case["nodes"]] * case["batch"]
    r = _shape_rng(case)
    return [r.randint(max(1, case["nodes"] // 2), case["nodes"]) for _ in range(case["batch"])]


def _levels(case):
    return [int(x) for x in case["levels"].split(",")]


def _mean_rank(case):
    return sum(float(p) * l for p, l in zip(case["probs"].split(","), _levels(case)))


def _parents(case, seed):
    """Parent of each node inside its sequence: a chain, or a tree of at most ``children`` children per
    node that prefers early children's subtrees, as drafts ordered by likelihood do; "padded" trees end in
    absent nodes (-2)."""
    r = random.Random(seed * 7919 + 11)
    out = []
    for n in _node_counts(case):
        par, kids = [-1], [0] * n
        for i in range(1, n):
            p = i - 1
            if case["shape"] != "chain":
                p = min(r.randrange(i), r.randrange(i))
                while kids[p] >= case.get("children", 4):
                    p += 1
            kids[p] += 1
            par.append(p)
        if case["shape"] == "padded":
            keep = max(1, n - n // 4)
            par = par[:keep] + [-2] * (n - keep)
        out += par
    return out


def _gen(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * (seed + 1) + 29)
    return g


def _cu(lens):
    return np.concatenate([[0], np.cumsum(np.asarray(lens, dtype=np.int64))]).astype(np.int32)


def _dev(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device=DEV)


# ---- inputs ------------------------------------------------------------------------------------

def _factors(case, lens, layers, g, seed):
    """The arrays of a filled cache (one depth window): orthonormal fp16 bases, N(0, 1) coefficients or their 8-bit
    blockwise form, categorical ranks, entries of distinct channels ordered by |code| then channel."""
    H, rb, L, T, B = case["kv_heads"], case["rank"], layers, sum(lens), len(lens)
    T16, lv = -(-T // 16) * 16, _levels(case)
    c = {"cu": _cu(lens), "levels": tuple(lv), "layers": L, "window": L, "kv_heads": H, "rank": rb, "coef_format": case["coef"]}
    r = np.random.default_rng(seed + 99)
    bas = np.linalg.qr(r.standard_normal((B * H * 2, D, rb)))[0].transpose(0, 2, 1)
    c["basis"] = torch.from_numpy(np.ascontiguousarray(bas)).to(DEV).half().view(B, 1, H, 2, rb, D)
    cum = torch.tensor(np.cumsum([float(x) for x in case["probs"].split(",")])[:-1], device=DEV, dtype=torch.float32)
    code = torch.bucketize(torch.rand((H, T), generator=g, device=DEV), cum, right=True)
    rho = torch.tensor(lv, device=DEV)[code]
    off = torch.zeros((H, T + 1), dtype=torch.int64, device=DEV)
    off[:, 1:] = rho.cumsum(1)
    top = lv[-1]
    room = min(T * top, int(T * _mean_rank(case) + 8 * top * math.sqrt(T)))
    stride = -(-(room + 512) // 256) * 256
    idx = torch.zeros((L, 2, H, stride), dtype=torch.uint8, device=DEV)
    nib = torch.zeros((L, 2, H, stride), dtype=torch.uint8, device=DEV)
    h, t = torch.nonzero(rho, as_tuple=True)                         # the tokens that hold entries
    j = torch.arange(top, device=DEV)
    ri = lambda lo, hi, *s: torch.randint(lo, hi, (L, 2) + s, generator=g, device=DEV, dtype=torch.int32)  # noqa: E731
    ch = (ri(0, D, h.numel(), 1) + j * (2 * ri(0, D // 2, h.numel(), 1) + 1)) % D
    q = ri(-7, 8, h.numel(), top)
    valid = j < rho[h, t][:, None]
    key = ((7 - q.abs()) * 256 + ch) * 2 + (q < 0)
    key = torch.where(valid, key, 1 << 20).to(torch.int32).sort(dim=-1).values
    q = torch.where(key % 2 == 1, key // 512 - 7, 7 - key // 512)
    at = (h[:, None] * stride + off[h, t][:, None] + j)[valid]
    idx.view(L, 2, -1)[:, :, at] = ((key // 2) % 256)[:, :, valid].to(torch.uint8)
    nib.view(L, 2, -1)[:, :, at] = (q & 15)[:, :, valid].to(torch.uint8)
    c["res_idx"], c["res_val"] = idx, nib[..., 0::2] | (nib[..., 1::2] << 4)
    c["rank_code"], c["res_off"], c["res_stride"] = code.to(torch.uint8).view(1, H, T), off.to(torch.int32).view(1, H, T + 1), stride
    c["res_scale"] = (0.01 + 0.09 * torch.rand((L, 2, H, T), generator=g, device=DEV)).half()
    rows = lambda: torch.randn((L, H, T16, rb), generator=g, device=DEV)  # noqa: E731
    pad = torch.arange(T16, device=DEV)[:, None] < T                    # padding tokens are zero
    if case["coef"] == "int8":
        k, v = ((rows() * 8).round_().clamp_(-127, 127) * pad for _ in range(2))
        c["coef_k"] = k.to(torch.int8).view(L, H, T16 // 16, 16, rb // 16, 16).transpose(3, 4).contiguous()
        c["coef_v"] = v.to(torch.int8).view(L, H, T16 // 16, 16, rb).transpose(3, 4).contiguous()
        for z in "kv":
            c["coef_scale_" + z] = (0.11 + 0.03 * torch.rand((L, H, rb // 16, T), generator=g, device=DEV)).half()
    else:
        k, v = (rows() * pad for _ in range(2))
        c["coef_k"] = k.half().view(L, H, T16 // 16, 16, rb // 8, 8).transpose(3, 4).contiguous()
        c["coef_v"] = v.half().view(L, H, T16 // 8, 8, rb).transpose(3, 4).contiguous()
    return c


def _empty_like(c, lens, stride):
    """Room for a cache of the same kind with other sequences."""
    T, L, H, rb, i8 = sum(lens), c["layers"], c["kv_heads"], c["rank"], c["coef_format"] == "int8"
    T16, z = -(-T // 16) * 16, lambda *s, dtype=torch.uint8: torch.zeros(s, dtype=dtype, device=DEV)
    e = {k: c[k] for k in ("levels", "layers", "window", "kv_heads", "rank", "coef_format")}
    e.update(cu=_cu(lens), res_stride=stride, basis=z(len(lens), 1, H, 2, rb, D, dtype=torch.float16), rank_code=z(1, H, T),
             res_off=z(1, H, T + 1, dtype=torch.int32), res_idx=z(L, 2, H, stride), res_val=z(L, 2, H, stride // 2),
             res_scale=z(L, 2, H, T, dtype=torch.float16))
    if i8:
        e.update(coef_k=z(L, H, T16 // 16, rb // 16, 16, 16, dtype=torch.int8), coef_v=z(L, H, T16 // 16, rb, 16, dtype=torch.int8),
                 coef_scale_k=z(L, H, rb // 16, T, dtype=torch.float16), coef_scale_v=z(L, H, rb // 16, T, dtype=torch.float16))
    else:
        e.update(coef_k=z(L, H, T16 // 16, rb // 8, 16, 8, dtype=torch.float16), coef_v=z(L, H, T16 // 8, rb, 8, dtype=torch.float16))
    return e


def _moves(case, lens, seed):
    """A repack's destination: lengths, source token of each slot (negative: fresh slot -1 - j), source sequences."""
    r, cu = random.Random(seed * 31 + 5), _cu(lens)
    out_lens, token, seq, fresh = [], [], [], 0
    if case["use"] == "fork":
        order = [0] * case["batch"]
    elif case["use"] == "compact":
        gone = {i for i in range(len(lens)) if i % 8 == 3}
        order = [i for i in range(len(lens)) if i not in gone]
    else:
        order = list(range(len(lens)))
    for i in order:
        src = np.arange(cu[i], cu[i + 1])
        if case["use"] == "compact":                                   # the rejected ones of the last few tokens
            tail = min(len(src), 24)
            drop = set(random.Random(len(out_lens)).sample(range(tail), tail // 3))
            src = np.asarray([t for k, t in enumerate(src) if k < len(src) - tail or k - (len(src) - tail) not in drop], dtype=np.int64)
        add = 8 if case["use"] != "fork" else 1
        token.append(np.concatenate([src, -1 - np.arange(fresh, fresh + add)]))
        fresh += add
        out_lens.append(len(src) + add)
        seq.append(i)
    if case["use"] != "fork" and r.random() < 0.5:                        # the batch in another order
        k = len(seq) // 2
        out_lens, token, seq = out_lens[k:] + out_lens[:k], token[k:] + token[:k], seq[k:] + seq[:k]
    return out_lens, np.concatenate(token).astype(np.int32), seq, fresh


_DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def prepare(case, seed):
    g = _gen(case, seed)
    s = {"kind": case["kind"]}
    if case["kind"] == "decode":
        s["cache"] = _factors(case, _lens(case), 1, g, seed)
        s["cu_nodes"] = _cu(_node_counts(case))
        N, H, G = int(s["cu_nodes"][-1]), case["kv_heads"], case["group"]
        s["parent"] = _dev(_parents(case, seed))
        sharp = 0.5 + 3.5 * torch.rand((H * G, 1), generator=g, device=DEV)   # heads from spread out to peaked
        s["q"] = (torch.randn((N, H * G, D), generator=g, device=DEV) * sharp).to(_DTYPE[case["q"]])
        s["k"], s["v"] = (torch.randn((N, H, D), generator=g, device=DEV).half() for _ in range(2))
        s["out"] = torch.empty((N, H * G, D), dtype=torch.float32, device=DEV)
    elif case["kind"] == "verify":
        s["cu_nodes"] = _cu(_node_counts(case))
        N, V, dt = int(s["cu_nodes"][-1]), case["vocab"], _DTYPE[case["p"]]
        par, cu = _parents(case, seed), s["cu_nodes"]
        s["parent"], s["children"], s["vocab"] = _dev(par), case["children"], V
        row = _dev([max(p, 0) + int(cu[b]) for b in range(case["batch"]) for p in par[cu[b]:cu[b + 1]]], torch.int64)
        # target and draft distributions that agree on most of their mass, as a good draft's do
        a = torch.randn((N, V), generator=g, device=DEV).mul_(3.0)
        q = torch.softmax(a, 1)
        s["target"] = torch.softmax(a.add_(torch.randn((N, V), generator=g, device=DEV), alpha=0.7), 1).to(dt)
        s["draft"] = q.to(dt) if case["draft"] else None
        if case["draft"]:                                                # children drawn from the parent's row
            race = torch.empty((N, V), device=DEV).exponential_(generator=g).clamp_(min=1e-30)
            token = (q[row] / race).argmax(1)
        else:                                                            # the k-th child is the k-th most likely token
            order = q.topk(min(V, 8), 1).indices
            kid = _dev([sum(p2 == p for p2 in par[cu[b]:cu[b] + i]) for b in range(case["batch"])
                        for i, p in enumerate(par[cu[b]:cu[b + 1]])], torch.int64).clamp(max=order.shape[1] - 1)
            token = order[row, kid]
        s["token"] = token.to(torch.int32)
        s["u"] = torch.rand((N,), generator=g, device=DEV)
        s["u_next"] = torch.rand((case["batch"],), generator=g, device=DEV)
    else:
        lens = _lens(case)
        s["cache"] = _factors(case, lens, case["layers"], g, seed)
        out_lens, token, seq, fresh = _moves(case, lens, seed)
        top = _levels(case)[-1]
        copies = case["batch"] if case["use"] == "fork" else 1
        room = copies * (s["cache"]["res_stride"] - 512) + fresh * top
        s["token"], s["seq"] = _dev(token), _dev(seq)
        s["new_code"] = torch.randint(0, len(_levels(case)), (1, case["kv_heads"], fresh), generator=g, device=DEV, dtype=torch.uint8)
        s["to"] = _empty_like(s["cache"], out_lens, -(-(room + 512) // 256) * 256)
    return s


# ---- the library's calls -------------------------------------------------------------------------

def _handle(c, group):
    from paper_2607_06523_amd import DeviceCache
    return DeviceCache.from_device(
        basis=c["basis"], coef_k=c["coef_k"], coef_v=c["coef_v"], rank_code=c["rank_code"], res_off=c["res_off"],
        res_idx=c["res_idx"], res_val=c["res_val"], res_scale=c["res_scale"], coef_scale_k=c.get("coef_scale_k"),
        coef_scale_v=c.get("coef_scale_v"), cu_seqlens=c["cu"], window=c["window"], n_q_heads=c["kv_heads"] * group,
        levels=c["levels"], coef_format=c["coef_format"])


def _run_own(s):
    import paper_2607_06523_amd as fw
    if s["kind"] == "decode":
        if "dc" not in s:                                                # the program's handles
            s["dc"] = _handle(s["cache"], s["q"].shape[1] // s["k"].shape[1])
            s["tree"] = fw.DraftTree(s["cu_nodes"], s["parent"])
            s["ws"] = s["dc"].tree_workspace(s["tree"])
        return s["dc"].tree_decode(0, s["tree"], s["q"], s["k"], s["v"], out=s["out"], workspace=s["ws"])
    if s["kind"] == "verify":
        if "tree" not in s:
            s["tree"] = fw.DraftTree(s["cu_nodes"], s["parent"])
            s["ws"] = fw.tree_verify_workspace(s["tree"], s["vocab"], s["children"])
        path, count, nxt = fw.tree_verify(s["tree"], s["token"], s["target"], s["u"], s["u_next"], draft=s["draft"],
                                          max_children=s["children"], workspace=s["ws"])
        return {"path": path, "count": count, "next": nxt}
    if "dc" not in s:
        s["dc"], s["dst"] = _handle(s["cache"], 1), _handle(s["to"], 1)
        s["ws"] = s["dst"].repack_workspace()
    s["dst"].repack_from(s["dc"], s["token"], s["seq"], new_code=s["new_code"], workspace=s["ws"])
    return _arrays(s["to"])


_MOVED = ("basis", "coef_k", "coef_v", "coef_scale_k", "coef_scale_v", "rank_code", "res_off", "res_idx", "res_val", "res_scale")


def _arrays(c):
    """A cache's arrays; its codes are moved as they are, so they are returned as the whole numbers they are held in."""
    return {k: c[k] for k in _MOVED if k in c}


# ---- the plain forms -----------------------------------------------------------------------------

def _key_rows(c):
    """[L, H, T, rb] coefficient rows of the key tiles, in the stored type."""
    k = c["coef_k"].transpose(3, 4).flatten(4, 5).flatten(2, 3)
    return k[:, :, :int(c["cu"][-1])]


def _value_rows(c):
    v = c["coef_v"].transpose(3, 4).flatten(2, 3)
    return v[:, :, :int(c["cu"][-1])]


def _code_values(packed):
    both = torch.stack([packed & 15, packed >> 4], -1).flatten(-2)
    return ((both ^ 8).to(torch.int16) - 8)


def _ancestors(parent, n):
    """[B, n, n] whether node i sees node j (itself and its ancestors up to the context)."""
    B = parent.shape[0]
    eye = torch.eye(n, dtype=torch.bool, device=DEV).expand(B, n, n)
    up = parent.clamp(min=0)
    live = parent >= -1
    see, at, more = eye & live[:, :, None], up, parent >= 0
    for _ in range(n):                                                    # one generation at a time
        if n == 1:
            break
        see = see | (torch.nn.functional.one_hot(at, n).bool() & more[:, :, None])
        more = more & (parent.gather(1, at) >= 0)
        at = up.gather(1, at)
    return see


def _rebuilt(c):
    """K_hat, V_hat [2, H, T, D] of layer 0 in float32 (Eq. 1), each sequence under its own bases."""
    H, T = c["kv_heads"], int(c["cu"][-1])
    lens = torch.from_numpy(np.diff(c["cu"]).astype(np.int64)).to(DEV)
    B, Tm = lens.numel(), int(np.diff(c["cu"]).max())
    seq = torch.repeat_interleave(torch.arange(B, device=DEV), lens, output_size=T)
    pos = torch.arange(T, device=DEV) - torch.from_numpy(c["cu"].astype(np.int64)).to(DEV)[seq]
    off = c["res_off"][0].long()
    rho = off[:, 1:] - off[:, :-1]
    E = off[:, -1]
    ent = torch.arange(c["res_stride"], device=DEV)
    valid = ent < E[:, None]
    tok = torch.searchsorted(off[:, 1:].contiguous(), ent.expand(H, -1).contiguous(), right=True).clamp(max=T - 1)
    out = []
    for z, rows in enumerate((_key_rows(c)[0], _value_rows(c)[0])):
        rows = rows.float()
        if c["coef_format"] == "int8":
            sc = c["coef_scale_k" if z == 0 else "coef_scale_v"][0].float()
            rows = rows * sc.transpose(1, 2).repeat_interleave(16, 2)
        a = torch.zeros((B, H, Tm, rows.shape[-1]), device=DEV)
        a[seq, :, pos] = rows.transpose(0, 1)
        x = torch.matmul(a, c["basis"][:, 0, :, z].float())               # [B, H, Tm, D]
        r = torch.zeros((H, T, D), device=DEV)
        val = _code_values(c["res_val"][0, z]).float() * c["res_scale"][0, z].float().gather(1, tok)
        hh = torch.arange(H, device=DEV)[:, None].expand_as(tok)
        r[hh[valid], tok[valid], c["res_idx"][0, z].long()[valid]] = val[valid]
        x[seq, :, pos] += r.transpose(0, 1)
        out.append(x)
    return out[0], out[1], lens, rho


def _plain_decode(s):
    c, q, H = s["cache"], s["q"].float(), s["cache"]["kv_heads"]
    G = q.shape[1] // H
    K, V, lens, _ = _rebuilt(c)
    counts = torch.from_numpy(np.diff(s["cu_nodes"]).astype(np.int64)).to(DEV)
    B, n, N = counts.numel(), int(np.diff(s["cu_nodes"]).max()), q.shape[0]
    seq = torch.repeat_interleave(torch.arange(B, device=DEV), counts, output_size=N)
    pos = torch.arange(N, device=DEV) - torch.from_numpy(s["cu_nodes"].astype(np.int64)).to(DEV)[seq]

    def padded(x, fill=0.0):
        y = torch.full((B, n) + tuple(x.shape[1:]), fill, device=DEV, dtype=x.dtype)
        y[seq, pos] = x
        return y
    Q = padded(q).view(B, n, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, n * G, D) * (D ** -0.5)
    kn, vn = (padded(x.float()).transpose(1, 2).contiguous() for x in (s["k"], s["v"]))     # [B, H, n, D]
    parent = padded(s["parent"].long(), -2)
    see = _ancestors(parent, n)
    live = parent >= -1
    cached = (torch.arange(K.shape[2], device=DEV) < lens[:, None])[:, None, :] & live[:, :, None]   # [B, n, Tm]
    mask = torch.cat([cached, see], 2).repeat_interleave(G, 1)[:, None]                              # [B, 1, n G, Tm + n]
    S = torch.cat([torch.matmul(Q, K.transpose(2, 3).contiguous()), torch.matmul(Q, kn.transpose(2, 3).contiguous())], 3)
    S = S.masked_fill_(~mask, -math.inf)
    P = (S - S.amax(3, keepdim=True).clamp(min=-1e30)).exp_()
    P = P / P.sum(3, keepdim=True).clamp(min=1e-37)
    O = torch.matmul(P[..., :K.shape[2]].contiguous(), V) + torch.matmul(P[..., K.shape[2]:].contiguous(), vn)
    return O.view(B, H, n, G, D).permute(0, 2, 1, 3, 4).reshape(B, n, H * G, D)[seq, pos]


def _usable(x):
    """Probabilities in 64 bits; what is not a positive finite number counts as zero."""
    x = x.double()
    return torch.where((x > 0) & torch.isfinite(x), x, 0.0)


def _plain_verify(s):
    """Acceptance of every node as its parent's k-th child, then the walk; 64 bits next to the borders."""
    cu = torch.from_numpy(s["cu_nodes"].astype(np.int64)).to(DEV)
    N, B, V = s["parent"].numel(), cu.numel() - 1, s["vocab"]
    ar = torch.arange(N, device=DEV)
    first = cu[:-1].repeat_interleave(cu[1:] - cu[:-1], output_size=N)
    par = torch.where((s["parent"] >= 0) & (ar > first), s["parent"].long() + first, -1)
    same = (par[:, None] == par[None, :]) & (par[:, None] >= 0)
    kid = (same & (ar[None, :] < ar[:, None])).sum(1)
    p, x = _usable(s["target"]), s["token"].long()
    q = _usable(s["draft"]) if s["draft"] is not None else None
    c = torch.zeros((N,), dtype=torch.float64, device=DEV)                # of a parent's row
    Z = torch.ones((N,), dtype=torch.float64, device=DEV)
    chosen = torch.full((N,), -1, dtype=torch.int64, device=DEV)           # accepted child of a row
    tried = torch.zeros((N,), dtype=torch.int64, device=DEV)
    w = p.clone() if q is None else None
    u = s["u"].double()
    for k in range(s["children"]):                                         # the k-th children of all rows
        node = torch.nonzero((par >= 0) & (kid == k) & (chosen[par.clamp(min=0)] < 0)).flatten()
        row = par[node]
        if q is None:
            r = w[row, x[node]]
            ok = u[node] * Z[row] < r
            w[row, x[node]] = 0.0
            Z[row] -= r
        else:
            qx = q[row, x[node]]
            r = (p[row, x[node]] - c[row] * qx).clamp(min=0.0)
            ok = u[node] * qx * Z[row] < r
            c[row] += Z[row]
            Z[row] = (p[row] - c[row][:, None] * q[row]).clamp(min=0.0).sum(1)
        chosen[row] = torch.where(ok, node, -1)
        tried[row] += 1
    path, at, count = torch.full((N,), -1, dtype=torch.int32, device=DEV), cu[:-1].clone(), torch.zeros((B,), dtype=torch.int64, device=DEV)
    live = cu[1:] > cu[:-1]
    last = at.clone()
    for _ in range(int(np.diff(s["cu_nodes"]).max())):                      # one generation at a time
        path[(cu[:-1] + count)[live]] = (at - cu[:-1])[live].to(torch.int32)
        count += live
        last = torch.where(live, at, last)
        nxt = chosen[at.clamp(min=0, max=N - 1)]
        live = live & (nxt >= 0)
        at = torch.where(live, nxt, at)
    r = w[last] if q is None else (p[last] - c[last][:, None] * q[last]).clamp(min=0.0)
    cum = r.cumsum(1)
    total = cum[:, -1:]
    hit = (cum > s["u_next"].double()[:, None] * total) & (r > 0)
    token = torch.where(total[:, 0] > 0, hit.to(torch.uint8).argmax(1), p[last].argmax(1))
    return {"path": path, "count": count.to(torch.int32), "next": token.to(torch.int32)}


def _plain_repack(s):
    c, e, tok, H, L = s["cache"], s["to"], s["token"].long(), s["cache"]["kv_heads"], s["cache"]["layers"]
    T, rb, i8 = tok.numel(), c["rank"], c["coef_format"] == "int8"
    T16, old = -(-T // 16) * 16, tok >= 0
    src = tok.clamp(min=0)
    out = {"basis": c["basis"][s["seq"].long()]}

    def rows(x):                                                           # [L, H, T, rb] -> padded, moved
        y = torch.zeros((L, H, T16, rb), dtype=x.dtype, device=DEV)
        y[:, :, :T] = x[:, :, src] * old[:, None]
        return y
    k, v = rows(_key_rows(c)), rows(_value_rows(c))
    if i8:
        out["coef_k"] = k.view(L, H, T16 // 16, 16, rb // 16, 16).transpose(3, 4).contiguous()
        out["coef_v"] = v.view(L, H, T16 // 16, 16, rb).transpose(3, 4).contiguous()
        for z in ("coef_scale_k", "coef_scale_v"):
            out[z] = c[z][..., src] * old
    else:
        out["coef_k"] = k.view(L, H, T16 // 16, 16, rb // 8, 8).transpose(3, 4).contiguous()
        out["coef_v"] = v.view(L, H, T16 // 8, 8, rb).transpose(3, 4).contiguous()
    code = torch.where(old, c["rank_code"][0][:, src], s["new_code"][0][:, (-1 - tok).clamp(min=0)])
    rho = torch.tensor(c["levels"], device=DEV)[code.long()]
    off = torch.zeros((H, T + 1), dtype=torch.int64, device=DEV)
    off[:, 1:] = rho.cumsum(1)
    out["rank_code"], out["res_off"] = code[None], off.to(torch.int32)[None]
    out["res_scale"] = c["res_scale"][..., src] * old
    ent = torch.arange(e["res_stride"], device=DEV).expand(H, -1).contiguous()
    t = torch.searchsorted(off[:, 1:].contiguous(), ent, right=True).clamp(max=T - 1)   # slot of each entry
    j = ent - off[:, :-1].gather(1, t)
    at = (c["res_off"][0].long().gather(1, src[t]) + j).clamp(min=0, max=c["res_stride"] - 1)
    live, fresh = ent < off[:, -1:], ~old[t]
    at, live, fresh, j = at[None, None], live[None, None], fresh[None, None], j[None, None]
    shape = (L, 2) + tuple(ent.shape)
    idx = c["res_idx"].gather(3, at.expand(shape))
    val = (_code_values(c["res_val"]).gather(3, at.expand(shape)) & 15).to(torch.uint8)
    idx = torch.where(fresh, j.to(torch.uint8), idx)
    out["res_idx"] = torch.where(live, idx, 0).to(torch.uint8)
    val = torch.where(live & ~fresh, val, 0).to(torch.uint8)
    out["res_val"] = val[..., 0::2] | (val[..., 1::2] << 4)
    return {k: out[k] for k in _MOVED if k in out}


def run(state):
    if own:
        return _run_own(state)
    return {"decode": _plain_decode, "verify": _plain_verify, "repack": _plain_repack}[state["kind"]](state)


# ---- what a pass cannot do without ----------------------------------------------------------------

def _token_bytes(case, entries=True):
    """Bytes of one token of one KV head of one layer, keys and values (offsets and rank codes apart)."""
    rb = case["rank"]
    coef = 2 * rb * 2 if case["coef"] == "f16" else 2 * (rb + 2 * (rb // 16))
    return coef + 4 + (2 * 1.5 * _mean_rank(case) if entries else 0)


def work(case):
    if case["kind"] == "decode":
        H, G, rb, rho = case["kv_heads"], case["group"], case["rank"], _mean_rank(case)
        lens, nodes = _lens(case), _node_counts(case)
        N, T = sum(nodes), sum(lens)
        byts = T * H * (_token_bytes(case) + 4) + len(lens) * H * 2 * rb * D * 2 + N * H * D * (G * (2 + 4) + 2 * 2)
        flops = sum(4.0 * t * n * G * H * (rb + rho) + 4.0 * n * G * H * D * (rb + n / 2) for t, n in zip(lens, nodes))
        return {"bytes": byts, "flops": flops}
    if case["kind"] == "verify":
        elt = 4 if case["p"] == "f32" else 2
        rows = case["batch"] * (2 if case["draft"] else 1)                 # the rows the next tokens are drawn from
        return {"bytes": rows * case["vocab"] * elt + sum(_node_counts(case)) * (4 * 4 + 2 * elt), "flops": 3.0 * rows * case["vocab"]}
    lens, L, H = _lens(case), case["layers"], case["kv_heads"]
    out, token, seq, _ = _moves(case, lens, 1)
    src = len(set(int(t) for t in token if t >= 0))
    per = H * (L * _token_bytes(case) + 5)
    return {"bytes": (src + sum(out)) * per + 4 * sum(out) + 2 * len(seq) * H * 2 * case["rank"] * D * 2, "flops": 0.0}


# ---- from the definitions, in 64 bits --------------------------------------------------------------

def exact(case, seed):
    if case["kind"] == "repack":
        return None                                                       # nothing is computed
    s = prepare(case, seed)
    return _exact_decode(case, s) if case["kind"] == "decode" else _exact_verify(case, s)


def _exact_decode(case, s):
    """Every sequence and KV head on its own: rebuilt keys and values, each node's own set of keys."""
    c, H, G, f8 = s["cache"], case["kv_heads"], case["group"], torch.float64
    cu, cn, par = c["cu"], s["cu_nodes"], s["parent"].tolist()
    kt, vt, rb = c["coef_k"][0], c["coef_v"][0], case["rank"]
    out = torch.zeros(s["out"].shape, dtype=f8, device=DEV)
    off = c["res_off"][0].long()
    for b in range(case["batch"]):
        t0, t1, n0, n1 = int(cu[b]), int(cu[b + 1]), int(cn[b]), int(cn[b + 1])
        t = torch.arange(t0, t1, device=DEV)[:, None]
        i = torch.arange(rb, device=DEV)
        for h in range(H):
            hat = []
            for z in (0, 1):
                if case["coef"] == "int8":
                    x = kt[h][t // 16, i // 16, t % 16, i % 16] if z == 0 else vt[h][t // 16, i, t % 16]
                    x = x.to(f8) * (c["coef_scale_k"] if z == 0 else c["coef_scale_v"])[0, h][i // 16, t].to(f8)
                else:
                    x = (kt[h][t // 16, i // 8, t % 16, i % 8] if z == 0 else vt[h][t // 8, i, t % 8]).to(f8)
                x = x @ c["basis"][b, 0, h, z].to(f8)
                e = torch.arange(int(off[h, t0]), int(off[h, t1]), device=DEV)
                owner = torch.bucketize(e, off[h, t0 + 1:t1 + 1], right=True)
                byte = c["res_val"][0, z, h][e // 2].to(torch.int64)
                code = torch.where(e % 2 == 0, byte % 16, byte // 16)
                code = torch.where(code > 7, code - 16, code).to(f8)
                x.index_put_((owner, c["res_idx"][0, z, h][e].long()), code * c["res_scale"][0, z, h, t0:t1].to(f8)[owner], accumulate=True)
                hat.append(x)
            K = torch.cat([hat[0], s["k"][n0:n1, h].to(f8)])
            V = torch.cat([hat[1], s["v"][n0:n1, h].to(f8)])
            sc = s["q"][n0:n1, h * G:(h + 1) * G].to(f8) @ K.T / math.sqrt(D)       # [n, G, T + n]
            for k in range(n1 - n0):
                seen, a = [], k
                while a >= 0:
                    seen.append(a)
                    a = par[n0 + a]
                if a < -1:
                    continue
                keep = torch.zeros((K.shape[0],), dtype=torch.bool, device=DEV)
                keep[:t1 - t0] = True
                keep[[t1 - t0 + a for a in seen]] = True
                out[n0 + k, h * G:(h + 1) * G] = torch.softmax(sc[k][:, keep], 1) @ V[keep]
    return out


def _exact_verify(case, s):
    """Sequence by sequence: test the children of the node reached, in order, against what is left of the
    target after each rejection."""
    cn, par, tok, u = s["cu_nodes"], s["parent"].tolist(), s["token"].tolist(), s["u"].double().tolist()
    path, count, nxt = [], [], []
    for b in range(case["batch"]):
        n0, n = int(cn[b]), int(cn[b + 1] - cn[b])
        at, stood = 0, [0]
        while True:
            p = s["target"][n0 + at].double().cpu().numpy()
            q = s["draft"][n0 + at].double().cpu().numpy() if s["draft"] is not None else None
            left, mass, found = p.copy(), 1.0, -1                            # what is left, unnormalised, and its sum
            for k in [i for i in range(1, n) if par[n0 + i] == at][:case["children"]]:
                x = tok[n0 + k]
                if q is None:
                    ok = u[n0 + k] * mass < left[x]
                    mass, left[x] = mass - left[x], left[x] if ok else 0.0
                else:
                    ok = u[n0 + k] * q[x] * mass < left[x]
                    if not ok:
                        left = np.maximum(left - mass * q, 0.0)
                        mass = float(np.sum(left))
                if ok:
                    found = k
                    break
            if found < 0:
                break
            at = found
            stood.append(at)
        run_sum = np.cumsum(left)
        nxt.append(int(np.argmax(run_sum > float(s["u_next"][b].double()) * run_sum[-1])) if run_sum[-1] > 0 else int(np.argmax(p)))
        path += stood + [-1] * (n - len(stood))
        count.append(len(stood))
    return {"path": _dev(path), "count": _dev(count), "next": _dev(nxt)}
