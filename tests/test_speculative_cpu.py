"""Refusals of the speculative step's calls (dwkv_tree_decode, dwkv_tree_verify,
dwkv_repack) and of their Python forms: every case returns on the host before
anything is enqueued, so none needs a GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2607_06523_amd import DeviceCache, DraftTree, DwkvError, binding, tree_verify, tree_verify_workspace
from test_abi_cpu import FAKE, dims, lib  # noqa: F401

OK, NULL, DIMS, UNSUPPORTED, WORKSPACE, ALIGN = 0, 1, 2, 3, 4, 7


def up256(x):
    return (x + 255) // 256 * 256


def tree_of(cu, **kw):
    host = np.ascontiguousarray(cu, dtype=np.int32)
    t = binding.Tree()
    t.n_nodes = int(host[-1])
    t.cu_nodes_host = host.ctypes.data_as(C.POINTER(C.c_int32))
    t.cu_nodes, t.parent = FAKE, FAKE
    for k, v in kw.items():
        setattr(t, k, v)
    return t, host


def tree_decode(lib, d, t, cache=None, layer=0, q=FAKE, q_type=0, q_stride=0, k=FAKE, v=FAKE, kv_stride=0, out=FAKE, ws=FAKE,
                ws_bytes=1 << 40):
    c = cache or binding.Cache(*([FAKE] * 10))
    return lib.dwkv_tree_decode(C.byref(d), C.byref(c), layer, C.byref(t) if t is not None else None, q, q_type, q_stride, k, v,
                                kv_stride, 0.0, out, ws, ws_bytes, None)


@pytest.mark.parametrize("cu,kw,status", [
    ([0, 5, 9], dict(n_nodes=8), DIMS),             # cu[B] != N
    ([0, 5, 9], dict(n_nodes=-1), DIMS),
    ([1, 5, 9], {}, DIMS),
    ([0, 9, 5], {}, DIMS),                          # descending
    ([0, 65, 70], {}, UNSUPPORTED),                 # 65 nodes in one sequence
    ([0, 5, 9], dict(cu_nodes=None), NULL),
    ([0, 5, 9], dict(parent=None), NULL),
    ([0, 5, 9], dict(cu_nodes_host=C.POINTER(C.c_int32)()), NULL),
    ([0, 5, 9], dict(cu_nodes=FAKE + 2), ALIGN),
    ([0, 5, 9], dict(parent=FAKE + 1), ALIGN),
])
def test_trees_that_do_not_fit(lib, cu, kw, status):  # noqa: F811
    d, keep = dims()
    t, host = tree_of(cu, **kw)
    assert lib.dwkv_tree_workspace_bytes(C.byref(d), C.byref(t)) == 0
    assert tree_decode(lib, d, t) == status
    assert lib.dwkv_tree_verify_workspace_bytes(2, C.byref(t), 100, 2) == 0
    assert lib.dwkv_tree_verify(2, C.byref(t), FAKE, 100, 2, FAKE, FAKE, FAKE, FAKE, 2, FAKE, FAKE, FAKE, FAKE, 1 << 40,
                                None) == status


def test_tree_decode_arguments(lib):  # noqa: F811
    d, keep = dims()
    t, host = tree_of([0, 5, 9])
    need = lib.dwkv_tree_workspace_bytes(C.byref(d), C.byref(t))
    # a chunk or more and one item of drafted nodes per 32 rows: 20 and 16 rows are one block each
    item = 32 * (128 + 32 + 4) * 4
    assert need >= up256(2 * (2 + 2) * item)
    assert tree_decode(lib, d, t, ws_bytes=need - 1) == WORKSPACE
    assert tree_decode(lib, d, None) == NULL
    for name in ("q", "k", "v", "out", "ws"):
        assert tree_decode(lib, d, t, **{name: None}) == NULL
        assert tree_decode(lib, d, t, **{name: FAKE + 8}) == ALIGN
    for layer in (-1, 4):
        assert tree_decode(lib, d, t, layer=layer) == DIMS
    assert tree_decode(lib, d, t, q_type=2) == DIMS                   # probabilities only
    row, kvrow = 8 * 128, 2 * 128
    for s in (row - 8, row + 4, -row, 8):
        assert tree_decode(lib, d, t, q_stride=s) == DIMS
    for s in (kvrow - 8, kvrow + 4, -kvrow, 8):
        assert tree_decode(lib, d, t, kv_stride=s) == DIMS
    bad, keepb = dims(basis_rank=24)
    assert tree_decode(lib, bad, t) == UNSUPPORTED
    assert lib.dwkv_tree_workspace_bytes(C.byref(bad), C.byref(t)) == 0
    for i in range(8):
        if i == 3:                                                    # the levels are in res_off already
            continue
        c = binding.Cache(*([FAKE] * 10))
        setattr(c, c._fields_[i][0], None)
        assert tree_decode(lib, d, t, cache=c) == NULL, c._fields_[i][0]
    d8, keep8 = dims(coef_format=binding.COEF_I8)
    for name in ("coef_k_scale", "coef_v_scale"):
        c = binding.Cache(*([FAKE] * 10))
        setattr(c, name, None)
        assert tree_decode(lib, d8, t, cache=c) == NULL
        setattr(c, name, FAKE + 1)
        assert tree_decode(lib, d8, t, cache=c) == ALIGN


def test_tree_decode_sizes_past_its_addressing(lib):  # noqa: F811
    B = 65536
    d, keep = dims(batch=B, cu_seqlens_host=np.arange(B + 1, dtype=np.int32), total_tokens=B, res_stride=B * 16 + 512)
    t, host = tree_of(np.arange(B + 1))
    assert tree_decode(lib, d, t) == UNSUPPORTED
    T = 2**28 + 16                                                    # r_b / 16 T = 2^29 + 32 block scales
    t, host = tree_of([0, 1])
    kw = dict(batch=1, cu_seqlens_host=[0, T], total_tokens=T, levels=(0, 2), res_stride=2**30)
    d, keep = dims(coef_format=binding.COEF_I8, **kw)
    assert tree_decode(lib, d, t) == UNSUPPORTED
    d, keep = dims(split_tokens=64, **kw)                             # 2^22 chunks of 2 heads, 1 block of rows
    need = lib.dwkv_tree_workspace_bytes(C.byref(d), C.byref(t))
    assert tree_decode(lib, d, t, ws_bytes=need - 1) == WORKSPACE and tree_decode(lib, d, t, ws_bytes=need) == UNSUPPORTED


def test_a_tree_without_nodes_is_no_call(lib):  # noqa: F811
    d, keep = dims()
    t, host = tree_of([0, 0, 0])
    assert lib.dwkv_tree_workspace_bytes(C.byref(d), C.byref(t)) == 256
    assert tree_decode(lib, d, t, ws_bytes=256) == OK
    t.parent = None                                                   # an empty array
    assert tree_decode(lib, d, t, ws_bytes=256) == OK
    empty, keep0 = dims(batch=1, cu_seqlens_host=[0, 0], total_tokens=0, res_stride=512)
    t, host = tree_of([0, 0])
    c = binding.Cache(FAKE, None, None, None, FAKE, FAKE, FAKE, None)  # arrays of tokens are not there
    assert tree_decode(lib, empty, t, cache=c, ws_bytes=256) == OK


def test_tree_verify_arguments(lib):  # noqa: F811
    t, host = tree_of([0, 5, 9])
    V, kids = 1000, 3
    need = lib.dwkv_tree_verify_workspace_bytes(2, C.byref(t), V, kids)
    assert need > 0
    base = dict(token=FAKE, vocab=V, p_type=2, target=FAKE, draft=FAKE, u=FAKE, u_next=FAKE, max_children=kids, path=FAKE,
                n_kept=FAKE, next=FAKE, workspace=FAKE, ws_bytes=need)

    def call(batch=2, tree=t, **kw):
        a = {**base, **kw}
        return lib.dwkv_tree_verify(batch, C.byref(tree) if tree is not None else None, *a.values(), None)
    assert call(tree=None) == NULL
    assert call(batch=0) == DIMS
    for name in ("token", "target", "u", "u_next", "path", "n_kept", "next", "workspace"):
        assert call(**{name: None}) == NULL, name
        assert call(**{name: FAKE + 1}) == ALIGN, name
    assert call(draft=FAKE + 2) == ALIGN
    assert call(workspace=FAKE + 8) == ALIGN
    for p_type in (0, 1):                                             # 2-byte rows
        assert call(p_type=p_type, target=FAKE + 2, ws_bytes=need - 1) == WORKSPACE
        assert call(p_type=p_type, target=FAKE + 1) == ALIGN
    assert call(ws_bytes=need - 1) == WORKSPACE
    for kw in (dict(vocab=0), dict(vocab=-5), dict(max_children=0), dict(max_children=65), dict(p_type=3), dict(p_type=-1)):
        assert call(**kw) == DIMS, kw
    assert call(vocab=2**31 - 1) == UNSUPPORTED
    assert lib.dwkv_tree_verify_workspace_bytes(2, C.byref(t), 0, kids) == 0
    big, hostb = tree_of(np.arange(0, 65537 * 16, 16).clip(max=65536))
    assert call(batch=65536, tree=big) == UNSUPPORTED
    many, hostm = tree_of(np.arange(1025) * 64)                       # 65536 nodes
    assert call(batch=1024, tree=many) == UNSUPPORTED


def repack(lib, dst, src, to=None, frm=None, src_token=FAKE, src_seq=FAKE, new_code=None, n_new=0, ws=FAKE, ws_bytes=1 << 40):
    to = to or binding.Cache(*([FAKE] * 10))
    frm = frm or binding.Cache(*([2 * FAKE] * 10))
    return lib.dwkv_repack(C.byref(dst), C.byref(to), C.byref(src), C.byref(frm), src_token, src_seq, new_code, n_new, ws, ws_bytes,
                           None)


@pytest.mark.parametrize("kw", [dict(n_layers=8), dict(window=4), dict(n_kv_heads=4), dict(n_q_heads=4), dict(basis_rank=48),
                                dict(levels=(0, 8)), dict(levels=(0, 8, 32)), dict(coef_format=1)])
def test_repack_of_another_kind_of_cache(lib, kw):  # noqa: F811
    dst, keep = dims()
    src, keep2 = dims(**kw)
    assert repack(lib, dst, src) == DIMS


def test_repack_arguments(lib):  # noqa: F811
    dst, keep = dims(batch=1, cu_seqlens_host=[0, 2000], total_tokens=2000)
    src, keep2 = dims()
    need = lib.dwkv_repack_workspace_bytes(C.byref(dst))
    assert need == up256(2 * 2 * 2 * 4)                               # 2 blocks of 1024 tokens, 2 windows, 2 heads
    assert repack(lib, dst, src, ws_bytes=need - 1) == WORKSPACE
    assert repack(lib, dst, src, n_new=-1) == DIMS
    for name in ("src_token", "src_seq", "ws"):
        assert repack(lib, dst, src, **{name: None}) == NULL
        assert repack(lib, dst, src, **{name: FAKE + 2}) == ALIGN
    bad, keepb = dims(n_q_heads=7)
    assert lib.dwkv_repack_workspace_bytes(C.byref(bad)) == 0
    assert repack(lib, bad, src) == DIMS and repack(lib, dst, bad) == DIMS
    fields = [f[0] for f in binding.Cache._fields_]
    for side, at in (("to", FAKE), ("frm", 2 * FAKE)):
        for name in fields[:8]:
            c = binding.Cache(*([at] * 10))
            setattr(c, name, None)
            assert repack(lib, dst, src, **{side: c}) == NULL, name
        for name in ("basis", "coef_k", "coef_v", "res_off", "res_idx", "res_scale"):
            c = binding.Cache(*([at] * 10))
            setattr(c, name, at + 1)
            assert repack(lib, dst, src, **{side: c}) == ALIGN, name
    dst8, k8 = dims(coef_format=binding.COEF_I8)
    for side, at in (("to", FAKE), ("frm", 2 * FAKE)):
        for name in ("coef_k_scale", "coef_v_scale"):
            c = binding.Cache(*([at] * 10))
            setattr(c, name, None)
            assert repack(lib, dst8, dst8, **{side: c}) == NULL
            setattr(c, name, at + 1)
            assert repack(lib, dst8, dst8, **{side: c}) == ALIGN
    for i in range(10):                                               # in place, any array of it
        c = binding.Cache(*([2 * FAKE] * 10))
        setattr(c, fields[i], FAKE)
        assert repack(lib, dst8, dst8, frm=c) == DIMS, fields[i]


# -- Python forms ---------------------------------------------------------------------

def test_draft_trees():
    p = torch.tensor([-1, 0, 1], dtype=torch.int32)
    for bad in (p.long(), p[None], torch.zeros(6, dtype=torch.int32)[::2]):
        with pytest.raises(TypeError):
            DraftTree([0, 3], bad)
    for cu in ([0, 2], [3], [[0, 3]]):
        with pytest.raises(ValueError):
            DraftTree(cu, p)
    with pytest.raises(DwkvError):
        tree_verify_workspace(DraftTree([0, 3], p), 0, 1)
    with pytest.raises(DwkvError):
        tree_verify_workspace(DraftTree([0, 4, 3], p), 10, 1)


def test_python_tree_verify():
    t = DraftTree([0, 3], torch.tensor([-1, 0, 1], dtype=torch.int32))
    tok, p, u, un = torch.zeros(3, dtype=torch.int32), torch.full((3, 10), 0.1), torch.zeros(3), torch.zeros(1)
    for kw in (dict(target=p.double()), dict(target=p[0]), dict(target=p[:2]), dict(target=p.t().contiguous().t()), dict(draft=p.half()),
               dict(draft=p[:, :5]), dict(token=tok.long()), dict(token=tok[:2]), dict(u=u.double()), dict(u=u[:1]),
               dict(u_next=u)):
        a = {**dict(token=tok, target=p, u=u, u_next=un), **kw}
        with pytest.raises(TypeError):
            tree_verify(t, a["token"], a["target"], a["u"], a["u_next"], draft=a.get("draft"), max_children=2)
    with pytest.raises(ValueError):                                   # nothing of it on a GPU
        tree_verify(t, tok, p, u, un, max_children=2)


def a_cache(lengths=(5,)):
    B, T = len(lengths), sum(lengths)
    T16 = -(-T // 16) * 16
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    f16 = lambda *s: torch.zeros(s, dtype=torch.float16)
    return dict(basis=f16(B, 1, 2, 2, 16, 128), coef_k=f16(2, 2, T16, 16), coef_v=f16(2, 2, T16, 16), rank_code=u8(1, 2, T),
                res_off=torch.zeros((1, 2, T + 1), dtype=torch.int32), res_idx=u8(2, 2, 2, 1024), res_val=u8(2, 2, 2, 512),
                res_scale=f16(2, 2, 2, T), cu_seqlens=np.cumsum([0, *lengths]), window=2, n_q_heads=8, levels=(0, 2))


def test_python_tree_decode():
    dc = DeviceCache.from_device(**a_cache())
    t = DraftTree([0, 3], torch.tensor([-1, 0, 1], dtype=torch.int32))
    q, k = torch.zeros(3, 8, 128, dtype=torch.float16), torch.zeros(3, 2, 128, dtype=torch.float16)
    for err, args in [(TypeError, (q.float(), k, k)), (TypeError, (q, k.bfloat16(), k)), (TypeError, (q, k, k.float())),
                      (ValueError, (q[:2], k, k)), (ValueError, (q[:, :4], k, k)), (ValueError, (q, k[:, :1], k)),
                      (ValueError, (q, k, k[:2])),
                      (ValueError, (q.transpose(1, 2).contiguous().transpose(1, 2), k, k)),
                      (ValueError, (q, k, torch.zeros(3, 4, 128, dtype=torch.float16)[:, :2])),
                      (ValueError, (q, k, k))]:                       # the last: nothing of it on a GPU
        with pytest.raises(err):
            dc.tree_decode(0, t, *args)
    one = k[:1].expand(3, 2, 128)
    for args in [(q[:1].expand(3, 8, 128), k, k), (q, one, one)]:     # a row stride of 0 is no gapless row
        with pytest.raises(ValueError, match="overlap"):
            dc.tree_decode(0, t, *args)
    with pytest.raises(ValueError):
        dc.tree_decode(0, DraftTree([0, 1, 3], t.parent), q, k, k)
    with pytest.raises(DwkvError):
        dc.tree_workspace(DraftTree([0, 65], torch.zeros(65, dtype=torch.int32)))


def test_python_caches_and_repack():
    with pytest.raises(ValueError):
        DeviceCache.from_device(**{**a_cache(), "coef_k": torch.zeros(2, 2, 5, 16, dtype=torch.float16)})
    with pytest.raises(ValueError):
        DeviceCache.from_device(**{**a_cache(), "coef_format": "int8"})
    with pytest.raises(ValueError):
        DeviceCache.from_device(**{**a_cache(), "res_off": torch.zeros((1, 2, 6), dtype=torch.int64)})
    src = DeviceCache.from_device(**a_cache((5, 3)))
    dst = src.empty_like([4])
    assert dst.cu_host.tolist() == [0, 4] and dst.res_stride == 768 and dst.basis.shape == (1, 1, 2, 2, 16, 128)
    tok, seq = torch.zeros(4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for args in [(tok.long(), seq), (tok[:3], seq), (torch.zeros(8, dtype=torch.int32)[::2], seq), (tok, seq.long()),
                 (tok, torch.zeros(2, dtype=torch.int32)), (tok, seq, torch.zeros(1, 2, 3)),
                 (tok, seq, torch.zeros(2, 2, 3, dtype=torch.uint8))]:
        with pytest.raises(TypeError):
            dst.repack_from(src, *args)
    with pytest.raises(ValueError):                                   # nothing of it on a GPU
        dst.repack_from(src, tok, seq)
