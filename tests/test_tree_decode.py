"""Attention of drafted trees (dwkv_tree_decode) on the GPU against plain
float64 attention: every sequence's rebuilt keys and values (Eq. 1, the oracle's
reconstruction) followed by the dense ones of a node and its ancestors.

Tolerance.  Scores in exp2 units are float32 sums of at most 128 + r_b + 1 exact
products of operands kept to 22 bits (q~ as a pair of fp16 numbers): their error
is at most (128 + r_b + 8) 2^-24 S_abs, S_abs the sum of the products' absolute
values, and typically its square root of the count.  A score error e changes a
probability by the factor 2^e; probabilities and their products with value
scales are kept to 22 bits, sums of T terms in float32 add about sqrt(T) 2^-24.
Taken together, with S_abs <= 8 |S|_max for these random inputs, rows are held to
rel-L2 <= (sqrt(T) + sqrt(128 + r_b) (8 + 8 |S|_max)) 2^-24 + 2^-21.
"""
import numpy as np
import pytest

import oracle
from gpu_util import announce, device_cache, lib_ready, torch_gpu
from oracle.factorized import reconstruct
from synth import Workload, generate

pytestmark = pytest.mark.gpu
D = 128


class _Fixed:
    def __init__(self, w, lengths):
        self._w, self._lengths = w, list(lengths)

    def __getattr__(self, k):
        if k.startswith("_"):
            raise AttributeError(k)
        return getattr(self._w, k)

    def seqlens(self):
        return list(self._lengths)


def make_host(lengths, G=4, rb=48, levels=(0, 4, 8, 16), Hk=2, fmt="f16", dtype="bf16", seed=5, scale_mode="uniform"):
    probs = tuple([1.0 / len(levels)] * len(levels))
    w = _Fixed(Workload(name="tree", batch=len(lengths), n_layers=2, window=1, n_kv_heads=Hk, n_q_heads=Hk * G, head_dim=D,
                        context=max(lengths), basis_rank=rb, levels=tuple(levels), probs=probs, q_dtype=dtype, seed=seed,
                        coef_format=fmt, scale_mode=scale_mode), lengths)
    return generate(w, threads=4)


def make_tree(counts, shape, rng):
    """cu_nodes and parents: chain, star, tree, or "padded" (a tree with absent nodes and their children)."""
    par = []
    for n in counts:
        p = []
        for i in range(n):
            if i == 0 or shape == "star":
                p.append(-1)
            elif shape == "chain":
                p.append(i - 1)
            else:
                p.append(int(rng.integers(-1 if i % 7 == 0 else 0, i)))
        if shape == "padded":
            for i in range(n):
                if i % 3 == 2:
                    p[i] = [-2, i, n + 5, -1000, 2**31 - 1][i % 5]
        par += p
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32), np.asarray(par, dtype=np.int32)


def chains(parent):
    """For each node of one sequence, itself and its ancestors; None when absent."""
    out = []
    for i, p in enumerate(parent):
        if p == -1:
            out.append([i])
        elif 0 <= p < i and out[p] is not None:
            out.append(out[p] + [i])
        else:
            out.append(None)
    return out


def reference(host, layer, cu, parent, q, kn, vn, scale=None):
    """(out float64 [N, Hq, D], largest |score| in exp2 units)"""
    Hk, G = host.n_kv_heads, host.n_q_heads // host.n_kv_heads
    scale = D ** -0.5 if scale is None else scale
    out, top = np.zeros(q.shape), 0.0
    for b in range(host.batch):
        n0, n1 = int(cu[b]), int(cu[b + 1])
        see = chains(parent[n0:n1])
        for h in range(Hk):
            if n1 == n0:
                continue
            K, V = reconstruct(host, layer, 0, h, b), reconstruct(host, layer, 1, h, b)
            for i in range(n1 - n0):
                if see[i] is None:
                    continue
                rows = [n0 + j for j in see[i]]
                keys, vals = np.concatenate([K, kn[rows, h]]), np.concatenate([V, vn[rows, h]])
                for gm in range(G):
                    s = scale * (keys @ q[n0 + i, h * G + gm])
                    top = max(top, float(np.abs(s).max()) * 1.4427)
                    p = np.exp(s - s.max())
                    out[n0 + i, h * G + gm] = (p / p.sum()) @ vals
    return out, top


def bound(host, top):
    T = max(int(np.diff(host.cu_seqlens).max()), 1)
    return (np.sqrt(T) + np.sqrt(128 + host.basis_rank) * (8 + 8 * top)) * 2.0 ** -24 + 2.0 ** -21


def inputs(host, N, rng, amp=1.0):
    torch = torch_gpu()
    dt = torch.bfloat16 if host.q_dtype == "bf16" else torch.float16
    Hk, Hq = host.n_kv_heads, host.n_q_heads
    q = torch.from_numpy((rng.standard_normal((N, Hq, D)) * amp).astype(np.float32)).to(dt)
    k, v = (torch.from_numpy(rng.standard_normal((N, Hk, D)).astype(np.float16)) for _ in range(2))
    return q, k, v


def check(got, want, tol, label):
    assert np.all(np.isfinite(got)), f"{label}: not finite"
    n = np.linalg.norm(want, axis=-1)
    err = np.linalg.norm(got - want, axis=-1)
    assert np.all(got[n == 0] == 0), f"{label}: an empty row is not zero"
    worst = float(np.max(err[n > 0] / n[n > 0])) if np.any(n > 0) else 0.0
    print(f"[parity] {label}: max rel-L2 {worst:.3e}, bound {tol:.3e}", flush=True)
    assert worst <= tol, f"{label}: rel-L2 {worst:.3e} > {tol:.3e}"


CASES = [
    # name, lengths, nodes, shape, G, r_b, levels, coefficients, query, split
    ("one-token-one-node", [1], [1], "chain", 4, 48, (0, 4, 8, 16), "f16", "bf16", 0),
    ("one-token-one-node-i8", [1], [1], "chain", 1, 16, (2,), "int8", "f16", 0),
    ("empty-context", [0, 40], [5, 3], "tree", 4, 32, (0, 8), "f16", "bf16", 0),
    ("sequences-without-nodes", [300, 17, 500], [0, 4, 0], "tree", 4, 48, (0, 4, 8, 16), "f16", "bf16", 0),
    ("chain5", [1000], [5], "chain", 4, 32, (0, 8, 16), "f16", "f16", 0),
    ("chain64", [777], [64], "chain", 4, 48, (0, 4, 8, 16), "f16", "bf16", 0),
    ("tree64", [2049], [64], "tree", 4, 48, (0, 4, 8, 16), "f16", "f16", 0),
    ("star33", [515], [33], "star", 2, 64, (0, 4), "f16", "bf16", 0),
    ("padded", [700, 31, 64], [17, 9, 64], "padded", 4, 48, (0, 4, 8, 16), "f16", "bf16", 0),
    ("g1", [900, 33], [16, 7], "tree", 1, 16, (0, 2), "f16", "bf16", 0),
    ("g2", [901], [9], "tree", 2, 32, (0, 8), "f16", "f16", 0),
    ("g8", [650], [21], "tree", 8, 64, (0, 4, 8, 16, 32), "f16", "bf16", 0),
    ("g16", [333], [12], "tree", 16, 48, (0, 16), "f16", "f16", 0),
    ("r80", [600], [13], "tree", 4, 80, (0, 8), "f16", "bf16", 0),
    ("r96-g16", [500], [6], "tree", 16, 96, (0, 8), "f16", "f16", 0),
    ("r128", [431], [20], "tree", 4, 128, (0, 8, 32), "f16", "bf16", 0),
    ("rank0-only", [800], [10], "tree", 4, 48, (0,), "f16", "bf16", 0),
    ("full-rank", [290], [10], "tree", 4, 32, (128,), "f16", "bf16", 0),
    ("many-entries", [310], [10], "tree", 4, 32, (0, 34, 64, 128), "f16", "f16", 0),
    ("split64", [1, 63, 64, 65, 129, 1000], [3, 3, 3, 3, 3, 9], "tree", 4, 48, (0, 4, 8, 16), "f16", "bf16", 64),
    ("split4096", [6000], [8], "tree", 4, 48, (0, 4, 8, 16), "f16", "bf16", 4096),
    ("20-sequences", [(37 * i) % 211 for i in range(20)], [(5 * i) % 11 for i in range(20)], "tree", 4, 32, (0, 8), "f16", "bf16", 64),
    ("70-sequences", [(41 * i) % 97 for i in range(70)], [(7 * i) % 9 for i in range(70)], "padded", 2, 16, (0, 4), "f16", "f16", 0),
    ("int8", [1300], [11], "tree", 4, 48, (0, 4, 8, 16), "int8", "bf16", 0),
    ("int8-r32-batch", [257, 1, 500], [12, 3, 30], "padded", 4, 32, (0, 8, 16), "int8", "f16", 0),
    ("int8-r112-g8", [300], [9], "tree", 8, 112, (0, 8), "int8", "bf16", 64),
    ("int8-r128-20", [(53 * i) % 150 for i in range(20)], [3] * 20, "tree", 4, 128, (0, 4), "int8", "f16", 0),
]


@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_tree_decode_matches_float64(case):
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import DraftTree
    name, lengths, counts, shape, G, rb, levels, fmt, dtype, split = case
    rng = np.random.default_rng(len(name) * 131 + sum(lengths))
    host = make_host(lengths, G, rb, levels, fmt=fmt, dtype=dtype)
    cu, parent = make_tree(counts, shape, rng)
    q, k, v = inputs(host, int(cu[-1]), rng, amp=2.0)
    dc = device_cache(host, split_tokens=split)
    tree = DraftTree(cu, torch.from_numpy(parent).cuda())
    ws = torch.full((dc.tree_workspace(tree).numel(),), 0xFF, dtype=torch.uint8, device="cuda")   # NaN everywhere
    announce(f"tree decode {name}")
    got = dc.tree_decode(1, tree, q.cuda(), k.cuda(), v.cuda(), workspace=ws).cpu().numpy()
    torch.cuda.synchronize()
    want, top = reference(host, 1, cu, parent, q.double().numpy(), k.double().numpy(), v.double().numpy())
    check(got, want, bound(host, top), name)


def test_one_node_agrees_with_the_decode():
    """A node that is its sequence's only one, over a cache whose last token is left out, is a decode with that token
    dense: the same attention as the decode's over the cached part."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import DraftTree
    host = make_host([1500, 900], 4, 48)
    dc = device_cache(host)
    rng = np.random.default_rng(3)
    q, k, v = inputs(host, 2, rng)
    k = torch.full_like(k, -60.0) * torch.sign(q[:, ::4].float()).half()       # a key no query looks at
    announce("tree decode, a node that attends to the cache alone")
    tree = DraftTree([0, 1, 2], torch.tensor([-1, -1], dtype=torch.int32, device="cuda"))
    sel = [h * 4 for h in range(host.n_kv_heads)]
    got = dc.tree_decode(0, tree, q.cuda(), k.cuda(), v.cuda()).cpu().numpy()[:, sel]
    want = oracle.decode(host, 0, q.double().numpy())[:, sel]
    check(got, want, 1e-5, "one node")


@pytest.mark.parametrize("fmt", ["f16", "int8"])
@pytest.mark.parametrize("rb", [48, 96])
def test_scales_over_the_whole_range(fmt, rb):
    """Residual scales from 2^-24 up to 2^15 (values) with the largest late in a chunk.  The output's error counts
    against the largest value scale of a row's tokens, whose terms the row's norm holds: the same bound."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import DraftTree
    host = make_host([1100], 4, rb, (0, 4, 16), fmt=fmt, scale_mode="wide")
    rng = np.random.default_rng(8)
    cu, parent = make_tree([10], "tree", rng)
    q, k, v = inputs(host, 10, rng, amp=0.5)
    dc = device_cache(host, split_tokens=512)
    announce(f"tree decode wide scales {fmt} {rb}")
    got = dc.tree_decode(0, DraftTree(cu, torch.from_numpy(parent).cuda()), q.cuda(), k.cuda(), v.cuda()).cpu().numpy()
    want, top = reference(host, 0, cu, parent, q.double().numpy(), k.double().numpy(), v.double().numpy())
    check(got, want, bound(host, top), f"wide scales {fmt}")


@pytest.mark.parametrize("rb", [16, 48, 112])
def test_block_scales_over_a_wide_range(rb):
    """int8 block scales from 2^-5 to 2^-2 (keys) and from 2^-12 to 2^7 (values), another for every token of a value
    block; the bound of the fp16 coefficients, whose products are as exact."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import DraftTree
    w = Workload(name="tree", batch=2, n_layers=2, window=1, n_kv_heads=2, n_q_heads=8, head_dim=D, context=901, basis_rank=rb,
                 levels=(0, 8), probs=(0.5, 0.5), q_dtype="f16", seed=15, coef_format="int8", coef_scale_mode="wide")
    host = generate(_Fixed(w, [901, 70]), threads=4)
    rng = np.random.default_rng(rb)
    cu, parent = make_tree([10, 7], "tree", rng)
    q, k, v = inputs(host, 17, rng)
    announce(f"tree decode wide block scales {rb}")
    got = device_cache(host).tree_decode(1, DraftTree(cu, torch.from_numpy(parent).cuda()), q.cuda(), k.cuda(), v.cuda()).cpu().numpy()
    want, top = reference(host, 1, cu, parent, q.double().numpy(), k.double().numpy(), v.double().numpy())
    check(got, want, bound(host, top), f"wide block scales {rb}")


def test_queries_beyond_fp16():
    """bf16 queries whose projections exceed fp16's range: scores in the hundred thousands, the softmax one-hot."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import DraftTree
    host = make_host([600], 4, 48)
    rng = np.random.default_rng(21)
    cu, parent = make_tree([6], "tree", rng)
    q, k, v = inputs(host, 6, rng)
    q[3:] *= 2.0 ** 20
    dc = device_cache(host)
    announce("tree decode queries beyond fp16")
    got = dc.tree_decode(0, DraftTree(cu, torch.from_numpy(parent).cuda()), q.cuda(), k.cuda(), v.cuda()).cpu().numpy()
    want, _ = reference(host, 0, cu, parent, q.double().numpy(), k.double().numpy(), v.double().numpy())
    # rows of ordinary queries share the workgroup's scaling with the large ones: q~ is then kept to
    # 2^-22 of 2^20 |q~|, so only the large rows are compared, and those to one-hot accuracy (2^-21)
    check(got[3:], want[3:], 2.0 ** -21 * 4, "large queries")


def test_what_a_node_does_not_see_changes_nothing():
    """NaN and infinities in unseen nodes' rows, in absent nodes' queries and in other sequences' cache."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import DraftTree
    host = make_host([70, 333, 45], 4, 48, seed=9)
    rng = np.random.default_rng(4)
    cu = np.array([0, 6, 14, 18], dtype=np.int32)
    parent = np.array([-1, 0, 0, 1, -2, 4] + [-1, 0, 0, 1, 1, 2, 7, 3] + [-1, 0, 1, 0], dtype=np.int32)
    q, k, v = inputs(host, 18, rng)
    dc = device_cache(host)
    tree = DraftTree(cu, torch.from_numpy(parent).cuda())
    announce("tree decode, clean")
    want = dc.tree_decode(0, tree, q.cuda(), k.cuda(), v.cuda()).cpu().numpy()
    q2, k2, v2 = q.clone(), k.clone(), v.clone()
    q2[[4, 5, 12]] = float("nan")                      # absent nodes (12: node 6 of sequence 1, its parent above it)
    bad = [4, 5, 12, 9]                                 # absent, and node 3 of sequence 1 (seen by 13 alone)
    k2[bad], v2[bad] = float("nan"), float("inf")
    big = dc.coef_k.numel() // 2 // host.n_kv_heads     # halves of a (layer, head) slab
    ck, cv, sc = dc.coef_k.view(-1), dc.coef_v.view(-1), dc.res_scale.view(2, 2, 2, -1)
    ok = [0, 1, 2, 3, 6, 7, 8, 10, 11]                  # rows that see none of it
    for s, clean in ((2, ok),):                         # sequence 2's tokens
        t0, t1 = int(host.cu_seqlens[s]), int(host.cu_seqlens[s + 1])
        for h in range(2):
            for t in range(t0, t1):
                for i in range(48):
                    ck[h * big + ((t >> 4) * 6 + (i >> 3)) * 128 + (t & 15) * 8 + (i & 7)] = float("nan") if i == 3 else float("inf")
                    cv[h * big + ((t >> 3) * 48 + i) * 8 + (t & 7)] = float("nan")
        sc[:, :, :, t0:t1] = float("nan")
        announce("tree decode with NaN outside of what the rows see")
        got = dc.tree_decode(0, tree, q2.cuda(), k2.cuda(), v2.cuda()).cpu().numpy()
        assert np.array_equal(got[clean], want[clean])
        assert np.all(got[[4, 5, 12]] == 0)


def test_value_scale_not_finite_stays_with_its_entries():
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import DraftTree
    host = make_host([200], 4, 32, (0, 8))
    dc = device_cache(host)
    off = host.res_off[0, 0].astype(np.int64)
    t = int(np.nonzero(np.diff(off))[0][7])
    ch = host.res_idx[0, 1, 0, off[t]:off[t + 1]]
    from oracle.factorized import entry_codes
    code = entry_codes(host.res_val[0, 1, 0], int(off[t]), int(off[t + 1] - off[t]))
    dc.res_scale.view(2, 2, 2, -1)[0, 1, 0, t] = float("inf")
    rng = np.random.default_rng(4)
    q, k, v = inputs(host, 3, rng)
    announce("tree decode with an infinite value scale")
    got = dc.tree_decode(0, DraftTree([0, 3], torch.tensor([-1, 0, 0], dtype=torch.int32, device="cuda")), q.cuda(), k.cuda(),
                         v.cuda()).cpu().numpy()[:, :4]
    hit = np.zeros(D, bool)
    hit[ch] = True
    assert np.all(np.isfinite(got[..., ~hit]))
    assert np.all(got[..., ch[code > 0]] == np.inf) and np.all(got[..., ch[code < 0]] == -np.inf)


def test_strided_rows_other_streams_and_graphs():
    """Slices of a fused projection's rows, a side stream, two captured graphs that share nothing but the cache and one
    workspace in order; replays follow changed inputs."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import DraftTree
    host = make_host([1200, 300], 4, 48)
    rng = np.random.default_rng(6)
    cu, parent = make_tree([9, 5], "tree", rng)
    N, Hq, Hk = 14, host.n_q_heads, host.n_kv_heads
    q, k, v = inputs(host, N, rng)
    q = q.half()
    dc = device_cache(host)
    tree = DraftTree(cu, torch.from_numpy(parent).cuda())
    announce("tree decode strided")
    want = dc.tree_decode(1, tree, q.cuda(), k.cuda(), v.cuda())
    rows = torch.zeros((N, (Hq + 2 * Hk) * D + 8), dtype=torch.float16, device="cuda").fill_(float("nan"))
    qs, ks, vs = (rows[:, a * D:b * D].view(N, -1, D) for a, b in ((0, Hq), (Hq, Hq + Hk), (Hq + Hk, Hq + 2 * Hk)))
    qs.copy_(q), ks.copy_(k), vs.copy_(v)
    assert torch.equal(dc.tree_decode(1, tree, qs, ks, vs), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = dc.tree_workspace(tree)
    with torch.cuda.stream(side):
        got = dc.tree_decode(1, tree, qs, ks, vs, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    announce("tree decode graphs")
    out = [torch.zeros_like(want) for _ in range(2)]
    graphs = []
    for i in range(2):
        gph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gph):
            dc.tree_decode(i, tree, qs, ks, vs, out=out[i], workspace=ws)
        graphs.append(gph)
    for step in range(3):
        qs.mul_(0.5)
        for gph in graphs:
            gph.replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(out[i], dc.tree_decode(i, tree, qs, ks, vs)), (step, i)
