"""The calls as a program makes them: prompts and steps over the paged cache into the
probabilities that a drafted tree is verified against, and turned keys into the
factorized cache."""
import copy

import numpy as np
import pytest

from gpu_util import announce, lib_ready, torch_gpu
from serving_ref import attend, check, rotate, rounding, shape_logits

pytestmark = pytest.mark.gpu


def test_prompts_steps_and_verification():
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import DraftTree, LogitsRules, PagedCache, RopeTable, adjust_logits, rope_freqs, tree_verify
    announce("serving step")
    B, H, G, d, page, V = 3, 2, 4, 64, 16, 3000
    prompts, steps = [37, 1, 64], 5
    rng = np.random.default_rng(0)
    g = torch.Generator().manual_seed(0)
    draw = lambda n: torch.randn((n, H * G + 2 * H, d), generator=g).bfloat16().cuda()
    table = torch.from_numpy(rng.permutation(24).astype(np.int32).reshape(3, 8)).cuda()
    lens = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    cache = PagedCache.empty(table, lens, n_pages=24, page_size=page, n_kv_heads=H, n_q_heads=H * G, head_dim=d, dtype=torch.bfloat16)
    freq = rope_freqs(32, base=500000.0, scaling="linear", factor=2.0)
    t = RopeTable(freq, interleaved=True)
    split = lambda x: (x[:, :H * G], x[:, H * G:H * G + H], x[:, H * G + H:])
    rows = draw(sum(prompts))
    q, k, v = split(rows)
    cu = np.concatenate([[0], np.cumsum(prompts)])
    cache.append(0, k, v, cu_new=torch.from_numpy(cu.astype(np.int32)).cuda(), q=q, rope=t)
    keys = [[x] for x in np.split(k.double().cpu().numpy(), cu[1:-1])]
    vals = [[x] for x in np.split(v.double().cpu().numpy(), cu[1:-1])]
    for _ in range(steps):
        lens += 1
        rows = draw(B)
        q, k, v = split(rows)
        qt = cache.append(0, k, v, q=q, rope=t)
        out = cache.decode(0, qt)
        n = lens.cpu().numpy()
        for b in range(B):
            keys[b].append(k[b:b + 1].double().cpu().numpy())
            vals[b].append(v[b:b + 1].double().cpu().numpy())
            K, V_ = np.concatenate(keys[b]), np.concatenate(vals[b])
            K, tol_k = rotate(K, np.arange(n[b]), freq.numpy(), True)
            # the stored keys and the turned query are rounded to bfloat16: what the scores may differ by
            Q, tol_q = rotate(q[b:b + 1].double().cpu().numpy(), [n[b] - 1], freq.numpy(), True)
            pages = lambda x: x.transpose(1, 0, 2)[None]
            want, tol = attend(Q, pages(K), pages(V_), np.zeros((1, 1), np.int32), [n[b]])
            ek, eq = rounding(np.abs(K) + tol_k, "bf16") + tol_k, rounding(np.abs(Q) + tol_q, "bf16") + tol_q
            for hq in range(H * G):
                h = hq // G
                ds = (np.abs(K[:, h]) @ eq[0, hq] + ek[:, h] @ (np.abs(Q[0, hq]) + eq[0, hq])) / np.sqrt(d)
                # probabilities change by a factor between exp(-2 ds) and exp(2 ds), of weights that sum to one
                tol[0, hq] += np.expm1(2 * ds.max()) * 2 * np.abs(V_[:, h]).max(0)
            check(out[b:b + 1].cpu().numpy(), want, tol, f"step, sequence {b}")
    # a drafted tree per sequence, its logits, and what stands
    nodes = [4, 1, 6]
    cn = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
    parent = np.array([-1, 0, 0, 1, -1, -1, 0, 1, 1, 2, 0], dtype=np.int32)
    N = int(cn[-1])
    token = rng.integers(0, V, N).astype(np.int32)
    logits = rng.normal(0, 2, (N, V)).astype(np.float32)
    hist = rng.integers(0, V, (B, 60)).astype(np.int32)
    hist_len = np.array([30, 60, 12], dtype=np.int32)
    params = np.array([[1.2, 0.3, 0.2, 0.8], [1.0, 0.0, 0.0, 0.0], [1.1, 0.0, 0.1, 1.0]], dtype=np.float32)
    up = lambda x: torch.from_numpy(x).cuda()
    tree = DraftTree(cn, up(parent))
    rules = LogitsRules(params=up(params), history=up(hist), history_len=up(hist_len))
    target = adjust_logits(up(logits), rules, tree=tree, token=up(token))
    want, tol = shape_logits(logits.astype(np.float64), params, hist, hist_len, tree=(cn, parent), token=token, probs=True)
    check(target.cpu().numpy(), want, tol, "target")
    path, kept, nxt = tree_verify(tree, up(token), target, up(np.full(N, 0.999, np.float32)), up(np.full(B, 0.5, np.float32)), max_children=4)
    assert (kept.cpu().numpy() >= 1).all()
    assert int(nxt[1]) == int(np.argmax(want[4]))            # the greedy sequence's only node


def test_turned_keys_into_the_factorized_cache():
    """The fused rows' queries and keys turned in place, then compressed and decoded, as the keys turned in numpy are."""
    torch = torch_gpu()
    lib_ready()
    import oracle
    import oracle.compress
    from gpu_util import compare, device_cache
    from paper_2607_06523_amd import RopeTable, rope, rope_freqs
    from synth import TINY, generate
    announce("turned keys compressed")
    host = generate(TINY, threads=4)
    dc = device_cache(host)
    T, H, d = dc.total_tokens, dc.n_kv_heads, dc.head_dim
    G, t0 = dc.n_q_heads // H, T - 40
    rows = torch.randn((40, (G + 2) * H, d), device="cuda").half()
    pos = torch.arange(t0, T, dtype=torch.int32, device="cuda")
    freq = rope_freqs(d, base=500000.0)
    turned, tol = rotate(rows[:, :(G + 1) * H].double().cpu().numpy(), pos.cpu().numpy(), freq.numpy())
    qk = rows[:, :(G + 1) * H]
    rope(qk, pos, RopeTable(freq), out=qk)
    check(qk.double().cpu().numpy(), turned, tol + rounding(np.abs(turned) + tol, "f16"), "turned")
    k, v = rows[:, G * H:(G + 1) * H].contiguous(), rows[:, (G + 1) * H:].contiguous()
    q = rows[-1:, :G * H].contiguous()
    dc.compress(0, k, v, t0, T)
    out = dc.decode(0, q).cpu().numpy()
    want = copy.deepcopy(host)
    oracle.compress.compress(want, 0, k.cpu().numpy(), v.cpu().numpy(), t0, T)
    ref = oracle.decode(want, 0, q=q.double().cpu().numpy())
    compare(out, ref, [(0, h) for h in range(H)], G, "turned keys")
