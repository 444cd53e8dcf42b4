"""The speculative step's calls where little is left to spare: at once, captured, a cache
without a token, and one whose arrays pass 2^32 bytes and 2^31 elements, against
plain computation on the GPU in float64 (attention) and plain indexing
(repacking)."""
import types

import numpy as np
import pytest

from gpu_util import announce, device_cache, lib_ready, torch_gpu
from test_tree_decode import D, bound, chains, check, make_host, make_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["f16", "int8"])
def test_a_cache_without_a_token(fmt):
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import DraftTree
    dc = device_cache(make_host([40], 4, 32, (0, 8), fmt=fmt)).empty_like([0, 0])
    rng = np.random.default_rng(7)
    cu, parent = make_tree([9, 40], "tree", rng)
    q = torch.from_numpy(rng.standard_normal((49, 8, D)).astype(np.float16))
    k, v = (torch.from_numpy(rng.standard_normal((49, 2, D)).astype(np.float16)) for _ in range(2))
    announce(f"tree decode over no cached token {fmt}")
    got = dc.tree_decode(1, DraftTree(cu, torch.from_numpy(parent).cuda()), q.cuda(), k.cuda(), v.cuda()).cpu().numpy()
    want, top = np.zeros((49, 8, D)), 0.0
    kn, vn, qn = k.double().numpy(), v.double().numpy(), q.double().numpy()
    for b in range(2):
        for i, see in enumerate(chains(parent[cu[b]:cu[b + 1]])):
            rows = [cu[b] + j for j in see]
            for hq in range(8):
                s = D ** -0.5 * (kn[rows, hq // 4] @ qn[cu[b] + i, hq])
                top = max(top, float(np.abs(s).max()) * 1.4427)
                p = np.exp(s - s.max())
                want[cu[b] + i, hq] = (p / p.sum()) @ vn[rows, hq // 4]
    check(got, want, bound(types.SimpleNamespace(cu_seqlens=np.array([0, 40]), basis_rank=32), top), "no cached token")


def test_arrays_past_32_bits():
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import DeviceCache, DraftTree
    L, H, rb, T = 6, 8, 48, 2**20 + 13                       # 2.4e9 coefficients of 2 bytes each for keys and values
    T16, stride = -(-T // 16) * 16, 2 * T // 256 * 256 + 768
    gen = torch.Generator(device="cuda")
    gen.manual_seed(11)
    f16 = lambda *s: torch.empty(s, dtype=torch.float16, device="cuda").normal_(generator=gen)
    u8 = lambda top, *s: torch.randint(0, top, s, dtype=torch.uint8, device="cuda", generator=gen)
    announce("a cache past 2^32 bytes")
    ck, cv = f16(L, H, T16 // 16, rb // 8, 16, 8), f16(L, H, T16 // 8, rb, 8)
    ck[:, :, -1, :, T % 16:] = 0
    cv[:, :, T // 8, :, T % 8:] = 0
    cv[:, :, T // 8 + 1:] = 0
    idx = u8(64, L, 2, H, stride)
    idx[..., 1::2] += 64                                     # two channels of a token are never the same
    code = torch.ones((1, H, T), dtype=torch.uint8, device="cuda")
    off = (2 * torch.arange(T + 1, dtype=torch.int32, device="cuda")).expand(1, H, T + 1).contiguous()
    val = torch.tensor([0x11, 0x72, 0xF3, 0x97], dtype=torch.uint8, device="cuda")[u8(4, L, 2, H, stride // 2).long()]
    src = DeviceCache.from_device(basis=f16(1, 1, H, 2, rb, D).mul_(0.1), coef_k=ck, coef_v=cv, rank_code=code, res_off=off,
                                  res_idx=idx, res_val=val, res_scale=f16(L, 2, H, T).mul_(0.1), cu_seqlens=[0, T], window=L,
                                  n_q_heads=2 * H, levels=(0, 2))
    q = f16(3, 2 * H, D)
    kn, vn = f16(3, H, D), f16(3, H, D)
    parent = torch.tensor([-1, 0, 0], dtype=torch.int32, device="cuda")
    got = src.tree_decode(L - 1, DraftTree([0, 3], parent), q, kn, vn).cpu().numpy()
    h, l = H - 1, L - 1
    dense = []
    for z, coef in ((0, ck[l, h].permute(0, 2, 1, 3).reshape(T16, rb)), (1, cv[l, h].permute(0, 2, 1).reshape(T16, rb))):
        x = coef[:T].double() @ src.basis[0, 0, h, z].double()
        e = idx[l, z, h, :2 * T].long().view(T, 2)
        n = torch.stack([val[l, z, h, :T] & 15, val[l, z, h, :T] >> 4], -1).to(torch.int8)
        n = torch.where(n > 7, n - 16, n).double() * src.res_scale[l, z, h, :, None].double()
        dense.append(x.scatter_add_(1, e, n))
    want, top = np.zeros((3, 2, D)), 0.0
    for i, see in enumerate(([0], [0, 1], [0, 2])):
        K, V = (torch.cat([x, y[see, h].double()]) for x, y in zip(dense, (kn, vn)))
        for g in range(2):
            s = D ** -0.5 * (K @ q[i, 2 * h + g].double())
            top = max(top, float(s.abs().max()) * 1.4427)
            want[i, g] = (torch.softmax(s, 0) @ V).cpu().numpy()
    check(got[:, 2 * h:2 * h + 2], want, bound(types.SimpleNamespace(cu_seqlens=src.cu_host, basis_rank=rb), top), "long cache")
    del dense
    announce("repacking past 2^32 bytes")
    dst = src.empty_like([T], res_stride=stride)
    dst.repack_from(src, torch.arange(1, T + 1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"))
    flat_k = lambda c, l, h: c.coef_k[l, h].permute(0, 2, 1, 3).reshape(T16, rb)
    flat_v = lambda c, l, h: c.coef_v[l, h].permute(0, 2, 1).reshape(T16, rb)
    for l, h in ((0, 0), (3, 2), (L - 1, H - 1)):            # the last token is a fresh slot at level 0
        for flat in (flat_k, flat_v):
            assert torch.equal(flat(dst, l, h)[:T - 1], flat(src, l, h)[1:T]) and not flat(dst, l, h)[T - 1:].any()
        assert torch.equal(dst.res_scale[l, :, h, :T - 1], src.res_scale[l, :, h, 1:])
        assert torch.equal(dst.res_idx[l, :, h, :2 * T - 2], src.res_idx[l, :, h, 2:2 * T])
        assert torch.equal(dst.res_val[l, :, h, :T - 1], src.res_val[l, :, h, 1:T])
    assert torch.equal(dst.res_off[0, H - 1, :T], off[0, 0, :T]) and int(dst.res_off[0, H - 1, T]) == 2 * T - 2


def test_calls_at_once_and_a_captured_repack():
    """Calls on two streams with workspaces of their own, nothing between them, and a captured repack whose source
    tokens change between its replays: all as the calls one after another."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import DraftTree, tree_verify, tree_verify_workspace
    host = make_host([2100, 900], 4, 48)
    dc = device_cache(host)
    rng = np.random.default_rng(21)
    cu, parent = make_tree([30, 11], "tree", rng)
    tree = DraftTree(cu, torch.from_numpy(parent).cuda())
    x = [[torch.from_numpy(rng.standard_normal((41, h, D)).astype(np.float16)).cuda() for h in (8, 2, 2)] for _ in range(2)]
    p = torch.softmax(torch.from_numpy(rng.standard_normal((2, 41, 5003)).astype(np.float32)).cuda(), -1)
    tok = torch.from_numpy(rng.integers(0, 5003, 41).astype(np.int32)).cuda()
    u = torch.from_numpy(rng.random(43).astype(np.float32)).cuda()
    perm = [torch.from_numpy(rng.permutation(3000).astype(np.int32)).cuda() for _ in range(4)]
    seq = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    dst = [dc.empty_like([2100, 900]) for _ in range(2)]
    arrays = lambda c: [c.coef_k, c.coef_v, c.rank_code, c.res_off, c.res_idx, c.res_val, c.res_scale, c.basis]

    def calls(i, ws):
        out = dc.tree_decode(i, tree, *x[i], workspace=ws[0])
        kept = tree_verify(tree, tok, p[i], u[:41], u[41:], draft=p[1 - i], max_children=3, workspace=ws[1])
        dst[i].repack_from(dc, perm[i], seq, workspace=ws[2])
        return [out, *kept]

    ws = [(dc.tree_workspace(tree), tree_verify_workspace(tree, 5003, 3), dst[i].repack_workspace()) for i in range(2)]
    announce("one call after another")
    want = []
    for i in range(2):
        want.append([t.clone() for t in calls(i, ws[i]) + arrays(dst[i])])
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    announce("calls at once")
    for _ in range(3):
        got = []
        for i, s in enumerate(streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(calls(i, ws[i]))
        torch.cuda.synchronize()
        for i in range(2):
            for a, b in zip(got[i] + arrays(dst[i]), want[i]):
                assert torch.equal(a, b)
    announce("a captured repack")
    src_token = perm[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dst[0].repack_from(dc, src_token, seq, workspace=ws[0][2])
    for i in (2, 3, 1):
        src_token.copy_(perm[i])
        graph.replay()
        dst[1].repack_from(dc, perm[i], seq, workspace=ws[1][2])
        torch.cuda.synchronize()
        e = int(dst[0].res_off[..., -1].min())
        for a, b in zip(arrays(dst[0]), arrays(dst[1])):
            cut = {id(dst[0].res_idx): e, id(dst[0].res_val): e // 2}.get(id(a))      # entries past the last keep older ones
            assert torch.equal(a[..., :cut], b[..., :cut])


@pytest.mark.parametrize("dt", ["float32", "float16", "bfloat16"])
def test_verify_without_nodes_and_rows_off_16_bytes(dt):
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import DraftTree, tree_verify
    dtype = getattr(torch, dt)
    announce(f"verify without nodes {dt}")
    u = torch.rand(60, generator=torch.Generator().manual_seed(3)).cuda()
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    p0 = torch.zeros((0, 77), dtype=dtype, device="cuda")
    path, kept, after = tree_verify(DraftTree([0, 0, 0], none), none, p0, u[:0], u[:2], draft=p0, max_children=2)
    assert path.numel() == 0 and kept.tolist() == [0, 0] and after.tolist() == [-1, -1]
    announce(f"verify of rows off 16 bytes {dt}")
    rng = np.random.default_rng(9)
    N, V = 40, 4099
    cu, parent = make_tree([33, 7], "tree", rng)
    tree = DraftTree(cu, torch.from_numpy(parent).cuda())
    tok = torch.from_numpy(rng.integers(0, V, N).astype(np.int32)).cuda()
    p, q = (torch.softmax(torch.from_numpy(rng.standard_normal((N, V)).astype(np.float32) * 3), -1).to(dtype).cuda() for _ in range(2))
    want = tree_verify(tree, tok, p, u[:N], u[N:N + 2], draft=q, max_children=3)
    for a, b in ((1, 0), (0, 3), (5, 2)):
        off = []
        for x, o in ((p, a), (q, b)):
            buf = torch.full((N * V + 8,), float("nan"), dtype=dtype, device="cuda")
            buf[o:o + N * V] = x.flatten()
            off.append(buf[o:o + N * V].view(N, V))
        got = tree_verify(tree, tok, off[0], u[:N], u[N:N + 2], draft=off[1], max_children=3)
        for x, y in zip(got, want):
            assert torch.equal(x, y)
