"""Calls of the speculative step as programs make them: layouts that are contiguous
in fact, and calls that share a workspace between a graph's replays."""
import numpy as np
import pytest

from gpu_util import announce, device_cache, lib_ready, torch_gpu
from test_tree_decode import D, bound, check, make_host, make_tree, reference
from test_tree_verify import make as make_drafts
from test_tree_verify import reference as verify_reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("G", [1, 4])
def test_one_kv_head_from_a_turned_tensor(G):
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import DraftTree
    host = make_host([300, 41], G, 32, (0, 8), Hk=1, dtype="f16")
    rng = np.random.default_rng(2)
    cu, parent = make_tree([7, 3], "tree", rng)
    q, k, v = (torch.from_numpy(rng.standard_normal((h, 10, D)).astype(np.float16)).cuda().transpose(0, 1) for h in (G, 1, 1))
    q = q if G == 1 else q.contiguous()
    assert k.is_contiguous() and k.stride(1) != D
    announce(f"tree decode, one KV head, G {G}")
    got = device_cache(host).tree_decode(1, DraftTree(cu, torch.from_numpy(parent).cuda()), q, k, v).cpu().numpy()
    want, top = reference(host, 1, cu, parent, *(x.cpu().double().numpy() for x in (q, k, v)))
    check(got, want, bound(host, top), f"one KV head, G {G}")


def test_a_graph_and_other_verifications_share_a_workspace():
    """Between the replays of a captured call with a draft its workspace serves a call without one and one of another
    tree, whose parts lie elsewhere in it: each gives the definition's outputs, each time."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import DraftTree, tree_verify, tree_verify_workspace
    rng = np.random.default_rng(41)
    sets = [make_drafts([20, 9], 3001, rng, 3, True), make_drafts([33, 1, 6], 3001, rng, 5, True)]
    trees = [DraftTree(a[0], torch.from_numpy(a[1]).cuda()) for a in sets]
    ws = max((tree_verify_workspace(t, 3001, n) for t, n in zip(trees, (3, 5))), key=lambda w: w.numel())
    ws.fill_(0xFF)
    gpu = [[x.cuda() if hasattr(x, "cuda") else torch.from_numpy(x).cuda() for x in a[2:]] for a in sets]

    def call(i, children, draft):
        token, target, q, u, un = gpu[i]
        return tree_verify(trees[i], token, target, u, un, draft=q if draft else None, max_children=children, workspace=ws)

    def want(i, children, draft):
        cu, parent, token, target, q, _, _ = sets[i]
        u, un = (x.cpu().numpy() for x in gpu[i][3:])
        out = verify_reference(cu, parent, token, target.double().numpy(), q.double().numpy() if draft else None, u, un, children)
        assert out[3] > 1e-12
        return out[:3]
    announce("tree verify, a graph and other calls in one workspace")
    call(0, 3, True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = call(0, 3, True)
    for step in range(4):
        for i in range(2):
            for x in gpu[i][3:]:
                x.copy_(torch.from_numpy(np.minimum(rng.random(x.numel()).astype(np.float32), 0.9999999)))
        graph.replay()
        got = [(captured, (0, 3, True)), (call(0, 2, False), (0, 2, False)), (call(1, 5, True), (1, 5, True))]
        torch.cuda.synchronize()
        for out, args in got:
            for a, b in zip(out, want(*args)):
                assert np.array_equal(a.cpu().numpy(), b), (step, args)


@pytest.mark.parametrize("fmt", ["f16", "int8"])
def test_growth_into_spare_room(fmt):
    """A cache laid out with fresh slots as a sequence of its own behind each live one takes the kept tokens without being
    copied: a handle over the same tensors with the starts moved, then compress.  Its live sequences are those of a cache
    grown by a repack."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import DeviceCache, DraftTree
    host = make_host([200, 90], 4, 32, (0, 4, 8), fmt=fmt)
    dc = device_cache(host)
    rng = np.random.default_rng(6)
    dev = lambda x: torch.from_numpy(np.asarray(x, dtype=np.int32)).cuda()
    codes = torch.from_numpy(rng.integers(0, 3, (2, 2, 32)).astype(np.uint8)).cuda()
    room = dc.empty_like([200, 16, 90, 16])
    slots = -1 - np.arange(32)
    announce(f"a cache with spare room {fmt}")
    room.repack_from(dc, dev(np.concatenate([np.arange(200), slots[:16], np.arange(200, 290), slots[16:]])), dev([0, 0, 1, 1]),
                     new_code=codes)
    kept = (3, 5)
    grown = DeviceCache.from_device(
        basis=room.basis, coef_k=room.coef_k, coef_v=room.coef_v, rank_code=room.rank_code, res_off=room.res_off, res_idx=room.res_idx,
        res_val=room.res_val, res_scale=room.res_scale, coef_scale_k=room.coef_scale_k, coef_scale_v=room.coef_scale_v,
        cu_seqlens=np.cumsum([0, 203, 13, 95, 11]), window=room.window, n_q_heads=room.n_q_heads, levels=room.levels, coef_format=fmt)
    plain = dc.empty_like([203, 95])
    plain.repack_from(dc, dev(np.concatenate([np.arange(200), slots[:3], np.arange(200, 290), slots[16:21]])), dev([0, 1]), new_code=codes)
    x = [[torch.from_numpy(rng.standard_normal((n, 2, D)).astype(np.float16)).cuda() for n in kept] for _ in range(2)]
    for layer in range(2):
        for c, ends in ((grown, (203, 311)), (plain, (203, 298))):
            for b, t1 in enumerate(ends):
                c.compress(layer, x[0][b], x[1][b], t1 - kept[b], t1)
    assert grown.validate() == (True, -1) and plain.validate() == (True, -1)
    cu, parent = make_tree([6, 4], "tree", rng)
    q, k, v = (torch.from_numpy(rng.standard_normal((10, h, D)).astype(np.float16)).cuda() for h in (8, 2, 2))
    parent = torch.from_numpy(parent).cuda()
    for layer in range(2):
        a = grown.tree_decode(layer, DraftTree([0, 6, 6, 10, 10], parent), q, k, v)
        b = plain.tree_decode(layer, DraftTree(cu, parent), q, k, v)
        # the same attention over chunks that start elsewhere: twice what a sum of 298 float32 terms may be off by
        check(a.cpu().numpy(), b.cpu().numpy(), 2 * bound(host, 20.0), f"spare room, layer {layer}")
        qd = q[:4].contiguous()
        c, d = grown.decode(layer, q=qd)[[0, 2]], plain.decode(layer, q=qd[[0, 2]].contiguous())
        check(c.cpu().numpy(), d.cpu().numpy(), 2 * bound(host, 20.0), f"spare room, decode of layer {layer}")
