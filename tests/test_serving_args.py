"""Refusals and host code of rotary positions, the paged cache and the shaping of
logits: none of these cases needs a GPU (every call returns before the first launch)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

FAKE = 1 << 20


@pytest.fixture(scope="module")
def lib():
    import os
    from paper_2607_06523_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return binding.load()


# ---- frequencies -----------------------------------------------------------------------------

def freqs(lib, n, base=10000.0, scaling=0, factor=1.0, context=0.0, low=1.0, high=4.0):
    out = (C.c_double * max(n, 1))()
    return lib.dwkv_rope_freqs(n, base, scaling, factor, context, low, high, out), np.array(out[:max(n, 0)])


@pytest.mark.parametrize("n", [1, 2, 5, 64])
def test_frequencies(lib, n):
    i = np.arange(n)
    plain = 10000.0 ** (-i / n)
    for scaling, args, want in [(0, {}, plain), (1, dict(factor=4.0), plain / 4.0)]:
        st, f = freqs(lib, n, scaling=scaling, **args)
        assert st == 0
        np.testing.assert_allclose(f, want, rtol=1e-14)
    st, f = freqs(lib, n, scaling=2, factor=8.0)
    assert st == 0 and f[0] == 1.0
    if n > 1:                                              # the lowest divided by the factor
        np.testing.assert_allclose(f[-1], plain[-1] / 8.0, rtol=1e-13)
    st, f = freqs(lib, n, scaling=3, factor=8.0, context=4096.0, low=1.0, high=32.0)
    turns = 4096.0 * plain / (2 * math.pi)
    s = np.clip((turns - 1.0) / 31.0, 0.0, 1.0)
    assert st == 0
    np.testing.assert_allclose(f, s * plain + (1 - s) * plain / 8.0, rtol=1e-13)
    assert (f[turns > 32.01] == freqs(lib, n)[1][turns > 32.01]).all()       # those stay as they are


def test_frequencies_refused(lib):
    out = (C.c_double * 4)()
    call = lambda n=4, base=1e4, sc=0, factor=1.0, ctx=0.0, lo=1.0, hi=4.0, o=out: lib.dwkv_rope_freqs(n, base, sc, factor, ctx, lo, hi, o)
    assert call() == 0
    assert call(o=None) == 1
    for kw in (dict(n=0), dict(base=0.0), dict(base=math.inf), dict(base=math.nan), dict(sc=4), dict(sc=-1), dict(sc=1, factor=0.0),
               dict(sc=2, factor=math.nan), dict(sc=3, factor=2.0), dict(sc=3, factor=2.0, ctx=100.0, lo=4.0, hi=4.0),
               dict(sc=3, factor=2.0, ctx=100.0, lo=math.nan)):
        assert call(**kw) == 2, kw


def test_frequencies_in_python(lib):
    from paper_2607_06523_amd import RopeTable, rope_freqs
    f = rope_freqs(128, base=500000.0, scaling="ramp", factor=8.0, context=8192)
    assert f.dtype == torch.float64 and f.shape == (64,) and f[0] == 1.0
    for bad in (dict(rot_dim=7), dict(rot_dim=0), dict(rot_dim=8, scaling="cubic")):
        with pytest.raises(ValueError):
            rope_freqs(**bad)
    for bad in (torch.ones(4), torch.ones((2, 2), dtype=torch.float64), torch.ones(0, dtype=torch.float64)):
        with pytest.raises(TypeError):
            RopeTable(bad)


# ---- rope ------------------------------------------------------------------------------------------

def rope_status(lib, rows=4, heads=2, d=64, table="yes", x=FAKE, xt=0, xs=0, pos=FAKE, out=2 * FAKE, ot=0, os=0, freq=FAKE, pairs=32):
    from paper_2607_06523_amd import binding
    t = binding.RopeTable(freq, pairs, 0, 1.0) if table else None
    return lib.dwkv_rope(rows, heads, d, C.byref(t) if t else None, 0, x, xt, xs, pos, out, ot, os, None)


def test_rope_refused(lib):
    assert rope_status(lib, rows=0) == 0                    # nothing to do
    for kw, want in [(dict(table=None), 1), (dict(freq=None), 1), (dict(x=None), 1), (dict(pos=None), 1), (dict(out=None), 1),
                     (dict(rows=-1), 2), (dict(heads=0), 2), (dict(d=0), 2), (dict(xt=3), 2), (dict(ot=-1), 2), (dict(pairs=0), 2),
                     (dict(pairs=33), 2), (dict(xs=64), 2), (dict(xs=132), 2), (dict(os=120), 2),
                     (dict(out=FAKE, ot=2), 2), (dict(out=FAKE, xs=136), 2),
                     (dict(d=60, pairs=4), 3), (dict(d=520), 3), (dict(rows=(1 << 24) + 1), 3), (dict(heads=65536), 3),
                     (dict(x=FAKE + 8), 7), (dict(out=FAKE + 2), 7), (dict(pos=FAKE + 2), 7), (dict(freq=FAKE + 4), 7)]:
        assert rope_status(lib, **kw) == want, kw


def test_rope_in_python_refused(lib):
    from paper_2607_06523_amd import rope

    class Table:                                            # a table on no GPU
        index, ref = -1, None
    x, pos = torch.zeros(4, 2, 64).half(), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):                         # the CPU is no GPU
        rope(x, pos, Table())
    with pytest.raises(TypeError):
        rope(x.double(), pos, Table())
    with pytest.raises(TypeError):
        rope(x, pos.long(), Table())
    with pytest.raises(TypeError):
        rope(x, pos[:3], Table())
    with pytest.raises(TypeError):
        rope(x, pos, Table(), out=x[:, :1])
    with pytest.raises(ValueError):
        rope(x[0], pos, Table())
    with pytest.raises(ValueError):                         # gaps between the heads of a row
        rope(torch.zeros(4, 4, 64).half()[:, ::2], pos, Table())
    with pytest.raises(ValueError):                         # rows on top of each other
        rope(x[:1].expand(4, 2, 64), pos, Table())


@pytest.fixture
def doubling(monkeypatch):
    """The call as a host function that doubles its rows, and halves them where it turns back, so that it and autograd
    around it run without a GPU: (a table for it, the calls' `inverse`)."""
    import paper_2607_06523_amd as fw
    monkeypatch.setattr(fw, "_all_on", lambda index, *tensors: True)
    rt, calls = fw._runtime(), []
    monkeypatch.setattr(rt, "device", lambda: -1)
    monkeypatch.setattr(rt, "stream", lambda index: 0)

    class Lib:
        @staticmethod
        def dwkv_rope(N, H, d, table, inverse, x, x_type, xs, pos, out, out_type, os, stream):
            calls.append(inverse)
            rows = lambda p, r, s, t: np.ctypeslib.as_array(C.cast(p + r * (s or H * d) * (4 if t == 2 else 2), C.POINTER(
                C.c_float if t == 2 else C.c_uint16)), (H * d,)).view(np.float32 if t == 2 else np.float16)
            for r in range(N):
                rows(out, r, os, out_type)[:] = rows(x, r, xs, x_type) * (0.5 if inverse else 2.0)
            return 0

    class Table:
        index, ref, lib, freq = -1, None, Lib, torch.ones(4, dtype=torch.float64)
    return Table(), calls


def test_rope_gradient_flows(doubling):
    from paper_2607_06523_amd import rope
    table, calls = doubling
    pos = torch.arange(4, dtype=torch.int32)
    leaf = torch.randn(4, 3, 8, requires_grad=True)
    y = rope(leaf, pos, table)
    assert torch.equal(y, 2 * leaf)
    y.sum().backward()                                       # a gradient without strides of its own
    assert calls == [0, 1] and torch.equal(leaf.grad, torch.full_like(leaf, 0.5))
    # the inverse's gradient, and a gradient's gradient
    g, = torch.autograd.grad(rope(leaf, pos, table, inverse=True).pow(2).sum(), leaf, create_graph=True)
    assert torch.equal(g, leaf.detach() * 2)                 # d (x / 2)^2: 2 (x / 2), turned by 2
    h, = torch.autograd.grad(g.sum(), leaf)                  # ones through the doubling that made g, the square, the halving
    assert torch.equal(h, torch.full_like(leaf, 0.5 * 2 * 2))
    # another type out, and back into the input's
    half = torch.empty(4, 3, 8, dtype=torch.float16)
    y = rope(leaf, pos, table, out=half)
    assert y is half and y.requires_grad and torch.equal(y, (2 * leaf).half())
    g, = torch.autograd.grad(y.float().sum(), leaf)
    assert g.dtype == torch.float32 and torch.equal(g, torch.full_like(leaf, 0.5))
    # nothing to do with gradients
    with torch.no_grad():
        assert not rope(leaf, pos, table).requires_grad
    assert not rope(leaf.detach(), pos, table).requires_grad


def test_rope_gradient_in_place(doubling):
    """Slices of a fused projection turned in place, through one name for them and through two."""
    from paper_2607_06523_amd import rope
    table, _ = doubling
    pos = torch.arange(4, dtype=torch.int32)
    for two in (False, True):
        w = torch.randn(4, 6, 8, requires_grad=True)
        rows = w * 1.0
        qk = rows[:, 1:4]
        assert rope(qk, pos, table, out=rows[:, 1:4] if two else qk) is not None
        want = torch.ones(4, 6, 8)
        want[:, 1:4] = 2.0
        assert torch.equal(rows, w * want)
        weights = torch.randn(4, 6, 8)
        g, = torch.autograd.grad((rows * weights).sum(), w)
        back = torch.ones(4, 6, 8)
        back[:, 1:4] = 0.5
        assert torch.equal(g, weights * back)
    # the result into a slice of something else that has a gradient
    a, w = torch.randn(4, 6, 8, requires_grad=True), torch.randn(4, 2, 8, requires_grad=True)
    rows = a * 1.0
    rope(w, pos, table, out=rows[:, 2:4])
    weights = torch.randn(4, 6, 8)
    ga, gw = torch.autograd.grad((rows * weights).sum(), (a, w))
    assert torch.equal(gw, 0.5 * weights[:, 2:4])
    weights[:, 2:4] = 0
    assert torch.equal(ga, weights)
    before = a.detach().clone()
    for out in (a, a[:, :3]):                                # leaves stay as they are
        with pytest.raises(ValueError):
            rope(out, pos, table, out=out)
    assert torch.equal(a, before)
    # positions that change before the gradient is taken
    y = rope(w, pos, table)
    pos += 1
    with pytest.raises(RuntimeError):
        y.sum().backward()


# ---- pages -----------------------------------------------------------------------------------------

def pages(**kw):
    from paper_2607_06523_amd import binding
    base = dict(type=0, batch=2, n_layers=2, n_kv_heads=2, head_dim=64, page_size=16, n_pages=8, max_pages=4, k=FAKE, v=FAKE,
                page_table=FAKE, seq_len=FAKE)
    base.update(kw)
    return binding.Pages(*[base[n] for n, _ in binding.Pages._fields_])


BAD_PAGES = [(dict(batch=0), 2), (dict(n_layers=0), 2), (dict(n_kv_heads=0), 2), (dict(n_pages=0), 2), (dict(max_pages=0), 2),
             (dict(type=2), 3), (dict(head_dim=48), 3), (dict(head_dim=288), 3), (dict(page_size=8), 3), (dict(page_size=48), 3),
             (dict(batch=4097), 3), (dict(max_pages=1 << 27), 3), (dict(k=None), 1), (dict(v=None), 1), (dict(page_table=None), 1),
             (dict(seq_len=None), 1), (dict(k=FAKE + 8), 7), (dict(v=FAKE + 2), 7), (dict(page_table=FAKE + 1), 7), (dict(seq_len=FAKE + 2), 7)]


def append_status(lib, p=None, layer=0, n=2, cu=None, k=FAKE, v=FAKE, xt=0, ks=0, q=FAKE, qs=0, nq=4, table=None, pos=None, q_out=FAKE):
    p = pages() if p is None else p
    return lib.dwkv_page_append(C.byref(p), layer, n, cu, k, v, xt, ks, q, qs, nq, C.byref(table) if table else None, pos, q_out, None)


def decode_status(lib, p=None, layer=0, q=FAKE, qs=0, nq=4, window=0, out=FAKE, ws=FAKE, ws_bytes=1 << 40):
    p = pages() if p is None else p
    return lib.dwkv_page_decode(C.byref(p), layer, q, qs, nq, 0.0, window, out, ws, ws_bytes, None)


def test_pages_refused(lib):
    for kw, want in BAD_PAGES:
        p = pages(**kw)
        assert append_status(lib, p, n=p.batch) == want, kw
        assert decode_status(lib, p) == want, kw
        assert lib.dwkv_page_workspace_bytes(C.byref(p), 4) == 0, kw
    assert lib.dwkv_page_append(None, 0, 2, None, FAKE, FAKE, 0, 0, None, 0, 0, None, None, None, None) == 1
    assert lib.dwkv_page_decode(None, 0, FAKE, 0, 4, 0.0, 0, FAKE, FAKE, 1 << 30, None) == 1


def test_append_refused(lib):
    from paper_2607_06523_amd import binding
    T = lambda freq=FAKE, pairs=32: binding.RopeTable(freq, pairs, 0, 1.0)
    assert append_status(lib, n=0, cu=FAKE) == 0
    for kw, want in [(dict(layer=2), 2), (dict(layer=-1), 2), (dict(n=-1, cu=FAKE), 2), (dict(n=3), 2), (dict(xt=3), 2),
                     (dict(ks=64), 2), (dict(ks=130), 2), (dict(nq=0), 2), (dict(qs=128), 2), (dict(qs=260), 2),
                     (dict(table=T(pairs=0)), 2), (dict(table=T(pairs=33)), 2), (dict(table=T(freq=None)), 1), (dict(table=T(freq=FAKE + 4)), 7),
                     (dict(k=None), 1), (dict(v=None), 1), (dict(q_out=None), 1), (dict(n=(1 << 24) + 1, cu=FAKE), 3),
                     (dict(k=FAKE + 8), 7), (dict(v=FAKE + 8), 7), (dict(q=FAKE + 8), 7), (dict(q_out=FAKE + 8), 7),
                     (dict(cu=FAKE + 2), 7), (dict(pos=FAKE + 2), 7),
                     (dict(xt=1), 2), (dict(xt=2), 2), (dict(qs=264), 2)]:           # q_out over q: of another type, with gaps
        assert append_status(lib, **kw) == want, kw


def test_page_decode_refused(lib):
    need = lib.dwkv_page_workspace_bytes(C.byref(pages()), 4)
    assert need > 0
    for kw, want in [(dict(layer=2), 2), (dict(layer=-1), 2), (dict(nq=0), 2), (dict(nq=3), 2), (dict(window=-1), 2), (dict(qs=128), 2),
                     (dict(qs=258), 2), (dict(q=None), 1), (dict(out=None), 1), (dict(ws=None), 1), (dict(ws_bytes=need - 1), 4),
                     (dict(q=FAKE + 2), 7), (dict(out=FAKE + 4), 7), (dict(ws=FAKE + 8), 7)]:
        assert decode_status(lib, **kw) == want, kw
    p = pages(batch=4096)
    assert decode_status(lib, p, nq=2048) == 3 and decode_status(lib, p, nq=1026) == 3 and decode_status(lib, p, nq=65536) == 3
    # a list of tiles past 2^31
    p = pages(batch=4096, max_pages=1 << 23, n_kv_heads=2)
    assert decode_status(lib, p) == 3 and lib.dwkv_page_workspace_bytes(C.byref(p), 4) == 0


def test_paged_cache_in_python_refused(lib):
    from paper_2607_06523_amd import PagedCache
    z = lambda *s: torch.zeros(s, dtype=torch.float16)
    k, v = z(1, 4, 2, 1, 8, 16, 8), z(1, 4, 2, 2, 64, 8)
    table, lens = torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for err, args in [(TypeError, (k.float(), v.float(), table, lens)), (TypeError, (k, v.bfloat16(), table, lens)),
                      (ValueError, (k[..., :4], v, table, lens)), (ValueError, (k, v[:, :3], table, lens)),
                      (ValueError, (k[0], v, table, lens)), (ValueError, (k.transpose(1, 2), v, table, lens)),
                      (TypeError, (k, v, table.long(), lens)), (TypeError, (k, v, table[0], lens)), (TypeError, (k, v, table, lens[:1])),
                      (ValueError, (k, v, table, lens))]:       # on no GPU
        with pytest.raises(err):
            PagedCache(*args, n_q_heads=4)
    with pytest.raises(ValueError):
        PagedCache.empty(table, lens, n_pages=4, page_size=24, n_kv_heads=2, n_q_heads=4)


def test_decodes_that_overlap_share_no_workspace(lib, monkeypatch):
    """A call without a workspace, made while another one's two launches are under way (here between its
    arguments and its return), works in memory of its own."""
    import paper_2607_06523_amd as fw
    monkeypatch.setattr(fw, "_all_on", lambda index, *tensors: True)
    z = lambda *s: torch.zeros(s, dtype=torch.float16)
    cache = fw.PagedCache(z(1, 4, 2, 1, 8, 16, 8), z(1, 4, 2, 2, 64, 8), torch.zeros((2, 3), dtype=torch.int32),
                          torch.zeros(2, dtype=torch.int32), n_q_heads=4)
    q, seen = z(2, 4, 64), []

    class Lib:                                              # records the calls and enqueues nothing
        @staticmethod
        def dwkv_page_decode(*args):
            seen.append((args[8], args[9]))
            if len(seen) < 3:
                cache.decode(0, q)
            return 0
    cache.lib = Lib
    rt = fw._runtime()
    monkeypatch.setattr(rt, "device", lambda: cache.index)
    monkeypatch.setattr(rt, "stream", lambda index: 0)
    cache.decode(0, q)
    seen.sort()
    assert len(seen) == 3 and all(a + n <= b for (a, n), (b, _) in zip(seen, seen[1:])), seen
    given = cache.workspace()
    cache.decode(0, q, workspace=given)
    assert seen[-1] == (given.data_ptr(), given.nbytes)


def test_windows_past_32_bits_are_none(lib, monkeypatch):
    """They are not cut off to their low bits."""
    import paper_2607_06523_amd as fw
    monkeypatch.setattr(fw, "_all_on", lambda index, *tensors: True)
    z = lambda *s: torch.zeros(s, dtype=torch.float16)
    cache = fw.PagedCache(z(1, 4, 2, 1, 8, 16, 8), z(1, 4, 2, 2, 64, 8), torch.zeros((2, 3), dtype=torch.int32),
                          torch.zeros(2, dtype=torch.int32), n_q_heads=4)
    seen = []

    class Lib:
        @staticmethod
        def dwkv_page_decode(*args):
            seen.append(C.c_int32(args[6]).value)           # as the call gets it
            return 0
    cache.lib = Lib
    monkeypatch.setattr(fw._runtime(), "device", lambda: cache.index)
    monkeypatch.setattr(fw._runtime(), "stream", lambda index: 0)
    for window in (0, 7, 2 ** 31 - 1, 2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 63 - 1):
        cache.decode(0, z(2, 4, 64), window=window)
    assert seen == [0, 7] + [2 ** 31 - 1] * 5
    cache.decode(0, z(2, 4, 64), window=-2 ** 32 + 9)        # and stay below 0, which the call refuses
    assert seen[-1] < 0


# ---- logits ----------------------------------------------------------------------------------------

def logits_status(lib, batch=2, tree=None, token=None, vocab=100, l=FAKE, lt=2, ls=0, rules="yes", probs=1, out=2 * FAKE, ot=2, ws=FAKE,
                  ws_bytes=1 << 30, **kw):
    from paper_2607_06523_amd import binding
    r = binding.LogitsRules(**kw) if rules else None
    return lib.dwkv_logits(batch, C.byref(tree) if tree else None, token, vocab, l, lt, ls, C.byref(r) if r else None, probs, out, ot, ws,
                           ws_bytes, None)


def test_logits_refused(lib):
    from paper_2607_06523_amd import binding
    cu = (C.c_int32 * 3)(0, 3, 5)

    def tree(n=5, host=cu, parent=FAKE):
        return binding.Tree(n, host, FAKE, parent)
    need = lib.dwkv_logits_workspace_bytes(2, 100)
    assert need > 0 and lib.dwkv_logits_workspace_bytes(65536, 10) == 0 and lib.dwkv_logits_workspace_bytes(1, 0) == 0
    empty = (C.c_int32 * 3)(0, 0, 0)
    assert logits_status(lib, tree=binding.Tree(0, empty, FAKE, None)) == 0
    for kw, want in [(dict(rules=None), 1), (dict(l=None), 1), (dict(out=None), 1), (dict(ws=None), 1), (dict(tree=tree()), 1),
                     (dict(history=FAKE, history_stride=4), 1), (dict(bias=FAKE, n_bias=1), 1),
                     (dict(batch=0), 2), (dict(vocab=0), 2), (dict(lt=3), 2), (dict(ot=-1), 2), (dict(ls=99), 2),
                     (dict(tree=tree(n=4), token=FAKE), 2), (dict(mask=FAKE, mask_stride=3), 2), (dict(history=FAKE, history_stride=-1), 2),
                     (dict(out=FAKE, ot=0), 2), (dict(out=FAKE, ls=128), 2),
                     (dict(batch=65536), 3), (dict(vocab=(1 << 30) + 1), 3), (dict(ws_bytes=need - 1), 4),
                     (dict(l=FAKE + 2), 7), (dict(lt=0, l=FAKE + 1), 7), (dict(out=FAKE + 2), 7), (dict(params=FAKE + 2), 7),
                     (dict(history=FAKE + 1, history_stride=4, history_len=FAKE), 7), (dict(mask=FAKE + 2, mask_stride=4), 7),
                     (dict(ws=FAKE + 8), 7), (dict(tree=tree(), token=FAKE + 2), 7)]:
        assert logits_status(lib, **kw) == want, kw


def test_logits_in_python_refused(lib):
    from paper_2607_06523_amd import LogitsRules, adjust_logits
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    for err, kw in [(TypeError, dict(params=torch.zeros(2, 3))), (TypeError, dict(params=torch.zeros(2, 4).half())),
                    (TypeError, dict(history=torch.zeros(2, 4), history_len=i32(2))), (ValueError, dict(history=i32(2, 4))),
                    (ValueError, dict(history_len=i32(2))), (ValueError, dict(prompt_len=i32(2))),
                    (TypeError, dict(history=i32(2, 4), history_len=i32(2).long())),
                    (ValueError, dict(params=torch.zeros(3, 4), history=i32(2, 4), history_len=i32(2))),
                    (TypeError, dict(bias=(i32(3), i32(4), torch.zeros(5)))), (TypeError, dict(bias=(i32(3), i32(4).long(), torch.zeros(4)))),
                    (TypeError, dict(mask=torch.zeros(2, 4))), (TypeError, dict(mask=i32(2, 8)[:, ::2])),
                    (ValueError, dict(mask=i32(1, 4).expand(2, 4))), (ValueError, dict(params=torch.zeros(2, 4)))]:   # the CPU is no GPU
        with pytest.raises(err):
            LogitsRules(**kw)
    none = LogitsRules()
    l = torch.zeros(2, 100)
    for err, kw in [(TypeError, dict(logits=l.double())), (TypeError, dict(logits=l.t())), (ValueError, dict(logits=l[:1].expand(2, 100))),
                    (ValueError, dict(logits=l, token=i32(2))), (TypeError, dict(logits=l, out=l.double())), (TypeError, dict(logits=l, out=l[:1])),
                    (ValueError, dict(logits=l))]:
        with pytest.raises(err):
            adjust_logits(rules=none, **kw)
