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
