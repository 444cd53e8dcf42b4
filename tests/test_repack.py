"""Repacking of a cache (dwkv_repack): copies, forks, compaction, freeing and
growth, every byte against plain indexing on the host, and a whole speculative
step: drafted trees scored and verified, the cache grown, the kept tokens
compressed into it, and decoded."""
import numpy as np
import pytest

import oracle
import oracle.compress as OC
from gpu_util import announce, compare, device_cache, lib_ready, torch_gpu
from synth.layout import block_values, unblock_values
from test_tree_decode import _Fixed, make_host
from synth import Workload, generate

pytestmark = pytest.mark.gpu


def host_of(dc):
    """A device cache's arrays in the host layout."""
    keys, values = dc.coef_host()
    i8 = dc.coef_format == "int8"
    out = {"coef_k": keys.view(np.int8 if i8 else np.uint16), "coef_v": values.view(np.int8 if i8 else np.uint16),
           "rank_code": dc.rank_code.cpu().numpy(), "res_off": dc.res_off.cpu().numpy().view(np.uint32),
           "res_idx": dc.res_idx.cpu().numpy(), "res_val": dc.res_val.cpu().numpy(),
           "res_scale": dc.res_scale.cpu().numpy().view(np.uint16), "basis": dc.basis.cpu().numpy().view(np.uint16)}
    if i8:
        out["coef_scale_k"], out["coef_scale_v"] = (x.cpu().numpy().view(np.uint16) for x in (dc.coef_scale_k, dc.coef_scale_v))
    return out


def expected(src, to, levels, src_token, src_seq, new_code, window):
    """Plain indexing; `to`: the destination's arrays before the call."""
    out = {k: v.copy() for k, v in to.items()}
    T, T0 = len(src_token), src["rank_code"].shape[-1]
    L, H = src["coef_k"].shape[:2]
    n_new = 0 if new_code is None else new_code.shape[-1]
    old = (src_token >= 0) & (src_token < T0)
    s = np.where(old, src_token, 0)
    out["coef_k"] = np.where(old[None, None, :, None], src["coef_k"][:, :, s], 0).astype(src["coef_k"].dtype)
    rows = unblock_values(src["coef_v"], T0)[:, :, s]
    out["coef_v"] = block_values(np.where(old[None, None, :, None], rows, 0).astype(rows.dtype))
    out["res_scale"] = np.where(old, src["res_scale"][..., s], 0).astype(np.uint16)
    for k in ("coef_scale_k", "coef_scale_v"):
        if k in src:
            out[k] = np.where(old, src[k][..., s], 0).astype(np.uint16)
    code = np.where(old, src["rank_code"][..., s], 0)
    slot = -1 - src_token.astype(np.int64)
    fresh = (src_token < 0) & (slot < n_new)
    if n_new:
        code = np.where(fresh, new_code[..., np.clip(slot, 0, n_new - 1)], code)
    code = np.where(code < len(levels), code, 0)
    out["rank_code"] = code.astype(np.uint8)
    rho = np.asarray(levels)[code]
    off = np.zeros((*rho.shape[:-1], T + 1), np.int64)
    off[..., 1:] = np.cumsum(rho, -1)
    out["res_off"] = off.astype(np.uint32)
    nib = lambda v: np.stack([v & 15, v >> 4], -1).reshape(*v.shape[:-1], -1)
    idx, val, sidx, sval = out["res_idx"], nib(out["res_val"]), src["res_idx"], nib(src["res_val"])
    for l in range(L):
        for h in range(H):
            m = l // window
            o, o0 = off[m, h], src["res_off"][m, h].astype(np.int64)
            for t in range(T):
                a, b = int(o[t]), int(o[t + 1])
                if old[t]:
                    c = int(o0[s[t]])
                    idx[l, :, h, a:b], val[l, :, h, a:b] = sidx[l, :, h, c:c + b - a], sval[l, :, h, c:c + b - a]
                else:
                    idx[l, :, h, a:b], val[l, :, h, a:b] = np.arange(b - a), 0
    out["res_val"] = (val[..., 0::2] | (val[..., 1::2] << 4)).astype(np.uint8)
    for b, q in enumerate(src_seq):
        if 0 <= q < src["basis"].shape[0]:
            out["basis"][b] = src["basis"][q]
    return out


def moves(kind, cu, rng):
    """(lengths, src_token, src_seq, slots)"""
    seqs = [np.arange(cu[i], cu[i + 1]) for i in range(len(cu) - 1)]
    fresh = lambda a, n: -1 - np.arange(a, a + n)
    if kind == "copy":
        parts, seq, n = seqs, list(range(len(seqs))), 0
    elif kind == "grow":
        parts, n = [], 0
        for s in seqs:
            parts.append(np.concatenate([s, fresh(n, 3)]))
            n += 3
        seq = list(range(len(seqs)))
    elif kind == "fork":
        parts, seq, n = [seqs[-1], seqs[0], seqs[-1], np.concatenate([seqs[-1][:5], fresh(0, 1)])], [len(seqs) - 1, 0, len(seqs) - 1, len(seqs) - 1], 1
    elif kind == "compact":
        parts = [s[rng.random(len(s)) < 0.8] for s in seqs[1:]][::-1]
        seq, n = list(range(1, len(seqs)))[::-1], 0
    elif kind == "shuffle":                                 # any order inside a sequence, tokens repeated
        parts, seq, n = [rng.choice(s, size=len(s) + 9) if len(s) else s for s in seqs], list(range(len(seqs))), 0
    elif kind == "new":                                     # fresh sequences only, one without a base
        parts, seq, n = [fresh(0, 33), fresh(33, 2)], [0, -1], 35
    else:                                                   # nothing at all
        parts, seq, n = [seqs[0][:0], seqs[0][:0]], [0, -1], 0
    return [len(p) for p in parts], np.concatenate(parts).astype(np.int32), np.asarray(seq, np.int32), n


KINDS = ["copy", "grow", "fork", "compact", "shuffle", "new", "nothing"]


@pytest.mark.parametrize("fmt,rb,levels,lengths", [
    ("f16", 48, (0, 4, 8, 16), [130, 0, 1, 77]),
    ("f16", 16, (0,), [64, 65]),
    ("f16", 128, (2, 128), [37, 20]),
    ("int8", 32, (0, 8, 16), [200, 15, 16]),
    ("int8", 112, (0, 30), [49, 33]),
    ("f16", 32, (0, 2, 4, 6, 8, 10, 12, 34), [1100, 950]),
], ids=["r48", "rank0", "r128", "int8-r32", "int8-r112", "two-blocks"])
@pytest.mark.parametrize("kind", KINDS)
def test_moves_every_byte(kind, fmt, rb, levels, lengths):
    torch = torch_gpu()
    lib_ready()
    rng = np.random.default_rng(rb + len(kind))
    host = make_host(lengths, 4, rb, levels, fmt=fmt)
    dc = device_cache(host)
    lens, token, seq, n = moves(kind, host.cu_seqlens, rng)
    codes = rng.integers(0, len(levels), (2, 2, n)).astype(np.uint8) if n else None
    to = dc.empty_like(lens)
    for x in (to.basis, to.coef_k, to.coef_v, to.res_scale, to.rank_code, to.res_idx, to.res_val, to.res_off):
        x.view(torch.uint8).fill_(0xA5)                     # what must be written and what must be left alone
    before, src = host_of(to), host_of(dc)
    announce(f"repack {kind} {fmt} r_b {rb}")
    ws = to.repack_workspace()
    ws.fill_(0xFF)
    to.repack_from(dc, torch.from_numpy(token).cuda(), torch.from_numpy(seq).cuda(),
                   new_code=None if codes is None else torch.from_numpy(codes).cuda(), workspace=ws)
    torch.cuda.synchronize()
    want, got = expected(src, before, levels, token, seq, codes, host.window), host_of(to)
    for k in want:
        if not np.array_equal(got[k], want[k]):
            raise AssertionError(f"{kind}: {k} differs at {np.argwhere(got[k] != want[k])[:4].tolist()}")
    if sum(lens) > 0:                                       # an empty cache has no arrays to look at
        assert to.validate() == (True, -1)
    after = host_of(dc)
    for k in src:
        assert np.array_equal(after[k], src[k]), f"the source's {k} changed"


def test_sources_out_of_range_are_fresh_slots():
    torch = torch_gpu()
    lib_ready()
    host = make_host([50], 4, 32, (0, 8, 16))
    dc = device_cache(host)
    token = np.array([3, 50, 2**31 - 1, -1, -2, -3, -2**31, 49], np.int32)
    codes = np.full((2, 2, 2), 1, np.uint8)
    codes[..., 1] = 200                                     # no such level
    to = dc.empty_like([8])
    before, src = host_of(to), host_of(dc)
    announce("repack, sources out of range")
    to.repack_from(dc, torch.from_numpy(token).cuda(), torch.tensor([0], dtype=torch.int32, device="cuda"),
                   new_code=torch.from_numpy(codes).cuda())
    got, want = host_of(to), expected(src, before, (0, 8, 16), token, [0], codes, host.window)
    for k in want:
        assert np.array_equal(got[k], want[k]), k
    assert to.validate() == (True, -1)


def test_a_slab_without_room_is_reported():
    torch = torch_gpu()
    lib_ready()
    host = make_host([300], 4, 32, (8,))
    dc = device_cache(host)
    to = dc.empty_like([300], res_stride=2048)              # 2400 entries do not fit
    guard = to.res_idx.clone()
    announce("repack without room")
    to.repack_from(dc, torch.arange(300, dtype=torch.int32, device="cuda"), torch.tensor([0], dtype=torch.int32, device="cuda"))
    assert not to.validate()[0]
    assert torch.equal(to.res_idx[..., 2048 - 512:], guard[..., 2048 - 512:])
    assert torch.equal(to.res_off, dc.res_off)


def test_a_fork_decodes_as_its_source():
    torch = torch_gpu()
    lib_ready()
    host = make_host([1000, 400], 4, 48)
    dc = device_cache(host)
    lens, order = [400, 1000, 400], [1, 0, 1]
    token = np.concatenate([np.arange(host.cu_seqlens[i], host.cu_seqlens[i + 1]) for i in order]).astype(np.int32)
    to = dc.empty_like(lens, res_stride=dc.res_stride * 2)
    announce("repack fork and decode")
    to.repack_from(dc, torch.from_numpy(token).cuda(), torch.tensor(order, dtype=torch.int32, device="cuda"))
    q = dc.q[1][order].contiguous()
    got = to.decode(1, q=q).cpu().numpy()
    want = oracle.decode(host, 1)[order]
    compare(got, want, [(b, h) for b in range(3) for h in range(2)], 4, "fork")


@pytest.mark.parametrize("fmt,all_stand", [("f16", False), ("int8", False), ("f16", True), ("int8", True)])
def test_a_speculative_step(fmt, all_stand):
    """Drafts scored over the cache, verified, the cache grown by what stands, its keys and values compressed, and the
    next decode: each part against the oracle on what the parts before it gave."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import DraftTree, tree_verify
    from test_tree_decode import bound, check, inputs, make_tree, reference
    from test_tree_verify import reference as verify_reference
    rng = np.random.default_rng(31)
    levels, V = (0, 4, 8), 400
    host = make_host([210, 64, 333], 4, 32, levels, fmt=fmt)
    dc = device_cache(host)
    cu, parent = make_tree([9, 5, 1], "tree", rng)
    for b in range(3):
        first = parent[cu[b]:cu[b + 1]]
        first[1:] = np.maximum(first[1:], 0)                # one root each
    N = int(cu[-1])
    q, k, v = inputs(host, N, rng)
    tree = DraftTree(cu, torch.from_numpy(parent).cuda())
    kg, vg = k.cuda(), v.cuda()
    announce(f"speculative step {fmt}")
    for layer in range(2):
        got = dc.tree_decode(layer, tree, q.cuda(), kg, vg).cpu().numpy()
        want, top = reference(host, layer, cu, parent, q.double().numpy(), k.double().numpy(), v.double().numpy())
        check(got, want, bound(host, top), f"step layer {layer}")
    p = rng.dirichlet(np.ones(V) * 0.05, size=N).astype(np.float32)
    token = rng.integers(0, V, N).astype(np.int32)
    for i in range(N):                                      # most drafts are likely ones
        b = int(np.searchsorted(cu, i, side="right")) - 1
        if i > cu[b] and rng.random() < 0.7:
            token[i] = int(np.argmax(p[cu[b] + parent[i]]))
    u, un = rng.random(N).astype(np.float32) * 0.5, rng.random(3).astype(np.float32) * 0.99
    if all_stand:                                           # every draft with a chance stands
        u[:] = 0.0
    path, kept, nxt = tree_verify(tree, torch.from_numpy(token).cuda(), torch.from_numpy(p).cuda(), torch.from_numpy(u).cuda(),
                                  torch.from_numpy(un).cuda(), max_children=4)
    path, kept, nxt = path.cpu().numpy(), kept.cpu().numpy(), nxt.cpu().numpy()
    wv = verify_reference(cu, parent, token, p.astype(np.float64), None, u, un, 4)
    assert np.array_equal(path, wv[0]) and np.array_equal(kept, wv[1]) and np.array_equal(nxt, wv[2])
    assert np.all(kept >= 1) and (not all_stand or kept.sum() > 3)
    # grow by the kept tokens, at routed levels
    lens = [int(n) for n in np.diff(host.cu_seqlens) + kept]
    token_map, nodes, done = [], [], 0
    for b in range(3):
        token_map += list(range(host.cu_seqlens[b], host.cu_seqlens[b + 1])) + [-1 - done - j for j in range(kept[b])]
        nodes += [int(cu[b] + path[cu[b] + j]) for j in range(kept[b])]
        done += int(kept[b])
    codes = rng.integers(0, len(levels), (2, 2, done)).astype(np.uint8)
    new = dc.empty_like(lens)
    new.repack_from(dc, torch.tensor(token_map, dtype=torch.int32, device="cuda"), torch.arange(3, dtype=torch.int32, device="cuda"),
                    new_code=torch.from_numpy(codes).cuda())
    at = 0
    for b in range(3):
        t1, n = int(new.cu_host[b + 1]), int(kept[b])
        rows = torch.tensor(nodes[at:at + n], device="cuda")
        at += n
        for layer in range(2):
            new.compress(layer, kg[rows].contiguous(), vg[rows].contiguous(), t1 - n, t1)
    assert new.validate() == (True, -1)
    # the oracle's cache: the same moves, then its own compression
    w = _Fixed(Workload(name="step", batch=3, n_layers=2, window=1, n_kv_heads=2, n_q_heads=8, head_dim=128, context=max(lens),
                        basis_rank=32, levels=levels, probs=(1.0, 0.0, 0.0), q_dtype="bf16", seed=5, coef_format=fmt), lens)
    exp = generate(w, threads=2)
    moved = expected(host_of(dc), {k2: np.zeros_like(x) for k2, x in host_of(new).items()}, levels, np.asarray(token_map), [0, 1, 2], codes, 1)
    for name, x in moved.items():
        setattr(exp, name, x.view(np.float16) if x.dtype == np.uint16 else x)
    exp.res_stride = new.res_stride
    at = 0
    for b in range(3):
        t1, n = int(new.cu_host[b + 1]), int(kept[b])
        for layer in range(2):
            OC.compress(exp, layer, k.numpy()[nodes[at:at + n]], v.numpy()[nodes[at:at + n]], t1 - n, t1, None)
        at += n
    got = host_of(new)
    for name in moved:
        want = np.ascontiguousarray(getattr(exp, name))
        assert np.array_equal(got[name].view(np.uint8).ravel(), want.view(np.uint8).ravel()), name
    q1 = torch.from_numpy(rng.standard_normal((3, 8, 128)).astype(np.float32) / 11.3).to(torch.bfloat16)
    out = new.decode(1, q=q1.cuda()).cpu().numpy()
    compare(out, oracle.decode(exp, 1, q1.double().numpy()), [(b, h) for b in range(3) for h in range(2)], 4, "the next decode")
