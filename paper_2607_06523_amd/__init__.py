"""MI355X-native decode attention over the DepthWeave-KV cross-depth factorized cache.

The hot path lives in ``libdwkv.so`` (hand-written HIP for gfx950, C ABI in
``include/dwkv.h``).  This package only marshals arguments: torch tensors
provide device memory and the current HIP stream.

    cache = DeviceCache(host_cache)        # upload the compressed layout
    out = cache.decode(layer)              # fp32 [B, Hq, d]
    out, err, out_ref = cache.decode(layer, probe=ProbeRef(heads, k_ref, v_ref))
    codes, offsets = cache.route(phi, u, theta)
    cache.route_range(phi, u, theta, t0, t1)      # routing of new tokens, in place
    cache.compress(layer, x_k, x_v, t0, t1)       # their Eq. 1 factors, in place

Several drafted tokens per sequence:

    tree = DraftTree(cu_nodes, parent)            # nodes of every sequence, packed
    out = cache.tree_decode(layer, tree, q, k, v) # fp32 [N, Hq, d]
    path, n_kept, nxt = tree_verify(tree, token, target, u, u_next, draft=draft)
    new = cache.empty_like(seqlens, res_stride)   # then the tokens that stay, with room for the kept ones
    new.repack_from(cache, src_token, src_seq, new_code=codes)
"""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass

import numpy as np

from . import binding, layout
from .binding import DwkvError, F16, BF16, F32

__all__ = ["DeviceCache", "ProbeRef", "DraftTree", "DwkvError", "load", "F16", "BF16", "F32", "hbm_read",
           "hbm_read_blocks", "probe_schedule", "tree_verify", "tree_verify_workspace"]


def load():
    return binding.load()


def _ptr(t):
    return C.c_void_p(t.data_ptr()) if t is not None else C.c_void_p(0)


def _stream(torch, device):
    return C.c_void_p(torch.cuda.current_stream(device).cuda_stream)


class _on:
    """``with _on(torch, index)``: the device current, left alone when it is already."""

    def __init__(self, torch, index):
        self.torch, self.index, self.was = torch, index, torch.cuda.current_device()

    def __enter__(self):
        if self.was != self.index:
            self.torch.cuda.set_device(self.index)

    def __exit__(self, *exc):
        if self.was != self.index:
            self.torch.cuda.set_device(self.was)


def _all_on(index, *tensors):
    """Whether every tensor (None aside) is on GPU ``index`` (-1, the CPU, is none)."""
    for x in tensors:
        if x is not None and x.get_device() != index:
            return False
    return index >= 0


def _nbytes(workspace):
    """Bytes from a workspace's start on."""
    if not workspace.is_contiguous():
        raise TypeError("workspace must be contiguous")
    return workspace.nbytes


def probe_schedule(step: int, period: int, n_heads: int, n_kv_heads: int, n_pos: int = 1):
    """dwkv_probe_schedule: (probed KV heads, positions) at decode step
    `step`, ([], 0) on a step that does not probe."""
    lib = load()
    heads = (C.c_int32 * max(1, n_heads))()
    npos = C.c_int32(0)
    n = lib.dwkv_probe_schedule(int(step), int(period), int(n_heads), int(n_kv_heads), int(n_pos), heads,
                                C.byref(npos))
    if n < 0:
        raise DwkvError(2, "dwkv_probe_schedule")
    return list(heads[:n]), int(npos.value)


def hbm_read_blocks() -> int:
    """Words of the sink that ``hbm_read`` writes."""
    return int(binding.load().dwkv_hbm_read_blocks())


def hbm_read(buf, sink):
    """Enqueue one read of the device tensor ``buf`` (its bytes, a multiple of
    16) on the current stream; ``sink`` is a device int32 tensor of at least
    ``hbm_read_blocks()`` elements whose xor becomes the xor of buf's 32-bit
    words.  The HBM read-stream ceiling of the device is its bytes over its
    time."""
    import torch
    lib = binding.load()
    nbytes = buf.numel() * buf.element_size()
    binding.check(lib.dwkv_hbm_read(_ptr(buf), nbytes, _ptr(sink), sink.numel(), _stream(torch, buf.device)),
                  "dwkv_hbm_read")


@dataclass
class ProbeRef:
    """Dense higher-fidelity reference cache for Eq. 3 (fp16 [n][T][d] device
    tensors).  q_prev, optional, holds the queries of earlier decode positions
    ([P-1][B][Hq][d], the decode query's dtype, slice j-1 from j steps back):
    the probe then evaluates P positions, the norms over positions and d."""
    kv_heads: list
    k_ref: object
    v_ref: object
    eps: float = 1e-6
    q_prev: object = None

    @property
    def n_pos(self) -> int:
        return 1 if self.q_prev is None else 1 + int(self.q_prev.shape[0])


class DraftTree:
    """Drafted nodes of a batch: cu_nodes [B+1] (host) packed starts, parent int32
    [N] (device) each node's parent inside its sequence, lower than its own
    index, -1 for the cached context; any other value marks an absent node."""

    def __init__(self, cu_nodes, parent):
        import torch
        if parent.dtype != torch.int32 or parent.dim() != 1 or not parent.is_contiguous():
            raise TypeError("parent must be a contiguous int32 vector")
        self.cu_host = np.array(cu_nodes, dtype=np.int32, order="C")    # a copy: the caller's array may change, the device's does not
        if self.cu_host.ndim != 1 or len(self.cu_host) < 2 or int(self.cu_host[-1]) != parent.numel():
            raise ValueError("cu_nodes must be [B+1] and end at the number of nodes")
        self.parent = parent
        self.cu = torch.from_numpy(self.cu_host).to(parent.device)
        self.batch, self.n_nodes = len(self.cu_host) - 1, parent.numel()
        t = binding.Tree()
        t.n_nodes = self.n_nodes
        t.cu_nodes_host = self.cu_host.ctypes.data_as(C.POINTER(C.c_int32))
        t.cu_nodes, t.parent = self.cu.data_ptr(), parent.data_ptr()
        self.cstruct, self.ref, self.index = t, C.byref(t), parent.get_device()


def tree_verify_workspace(tree: DraftTree, vocab: int, max_children: int):
    """A workspace for ``tree_verify`` of such trees."""
    import torch
    n = int(load().dwkv_tree_verify_workspace_bytes(tree.batch, C.byref(tree.cstruct), int(vocab), int(max_children)))
    if n == 0:
        raise DwkvError(2, "dwkv_tree_verify_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=tree.parent.device)


def tree_verify(tree: DraftTree, token, target, u, u_next, draft=None, max_children: int = 1, workspace=None):
    """dwkv_tree_verify: which drafted tokens stand against the target's
    probabilities.  token int32 [N], target [N, vocab] (float32, float16 or
    bfloat16), draft None or like target (row i: what node i's children were
    drawn from), u fp32 [N] and u_next fp32 [B] in [0, 1).  Returns (path int32
    [N], n_kept int32 [B], next int32 [B])."""
    import torch
    kinds = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
    N, B = tree.n_nodes, tree.batch
    if target.dtype not in kinds or target.dim() != 2 or target.shape[0] != N or not target.is_contiguous():
        raise TypeError("target must be a contiguous [N, vocab] tensor of float32, float16 or bfloat16")
    if draft is not None and (draft.dtype != target.dtype or draft.shape != target.shape or not draft.is_contiguous()):
        raise TypeError("draft must be like target")
    if token.dtype != torch.int32 or token.numel() != N or not token.is_contiguous():
        raise TypeError("token must be contiguous int32 [N]")
    for x, n in ((u, N), (u_next, B)):
        if x.dtype != torch.float32 or x.numel() != n or not x.is_contiguous():
            raise TypeError("u and u_next must be contiguous float32 [N] and [B]")
    dev = tree.parent.device
    if not _all_on(tree.index, token, target, draft, u, u_next, workspace):
        raise ValueError("every tensor must be on the tree's device")
    V = target.shape[1]
    ws = workspace if workspace is not None else tree_verify_workspace(tree, V, max_children)
    path, n_kept, nxt = torch.empty(N + 2 * B, dtype=torch.int32, device=dev).split((N, B, B))
    with _on(torch, tree.index):
        st = load().dwkv_tree_verify(B, tree.ref, token.data_ptr(), V, kinds[target.dtype], target.data_ptr(),
                                     draft.data_ptr() if draft is not None else None, u.data_ptr(), u_next.data_ptr(),
                                     int(max_children), path.data_ptr(), n_kept.data_ptr(), nxt.data_ptr(), ws.data_ptr(),
                                     _nbytes(ws), torch.cuda.current_stream(tree.index).cuda_stream)
    binding.check(st, "dwkv_tree_verify")
    return path, n_kept, nxt


class DeviceCache:
    """One factorized cache resident on the GPU in the C-ABI layout.

    ``host`` is any object carrying the layout arrays (basis, coef, rank_code,
    res_off, res_idx, res_val, res_scale, q_bits, cu_seqlens, levels, ...), for
    example a synthetic cache from ``synth.generate``."""

    def __init__(self, host, device: str = "cuda", split_tokens: int = 0):
        import torch
        self.torch = torch
        self.lib = binding.load()
        self.device = torch.device(device)
        dev = self.device
        up = lambda a, dt: torch.from_numpy(np.ascontiguousarray(a)).view(dt).to(dev)
        self.basis = up(host.basis.view(np.uint16), torch.float16)
        self.coef_format = getattr(host, "coef_format", "f16")
        if self.coef_format == "int8":        # codes and their fp16 block scales
            self.coef_k = up(layout.keys_to_abi(host.coef_k.view(np.uint8), group=16), torch.uint8)
            self.coef_v = up(host.coef_v.view(np.uint8), torch.uint8)
            self.coef_scale_k = up(host.coef_scale_k.view(np.uint16), torch.float16)
            self.coef_scale_v = up(host.coef_scale_v.view(np.uint16), torch.float16)
        else:                                 # fp16: the ABI's tiled layouts
            self.coef_k = up(layout.keys_to_abi(host.coef_k.view(np.uint16)), torch.float16)
            self.coef_v = up(layout.values_to_abi(host.coef_v.view(np.uint16)), torch.float16)
            self.coef_scale_k = self.coef_scale_v = None
        self.rank_code = up(host.rank_code, torch.uint8)
        self.res_off = up(host.res_off.view(np.int32), torch.int32)
        self.res_idx = up(host.res_idx, torch.uint8)
        self.res_val = up(host.res_val, torch.uint8)
        self.res_scale = up(host.res_scale.view(np.uint16), torch.float16)
        self.q_dtype = host.q_dtype
        qdt = torch.float16 if host.q_dtype == "f16" else torch.bfloat16
        self.q = up(host.q_bits.view(np.int16), torch.int16).view(qdt)
        self.cu_host = np.array(host.cu_seqlens, dtype=np.int32, order="C")   # a copy, as the device's
        self.cu = torch.from_numpy(self.cu_host).to(dev)
        self.batch = len(self.cu_host) - 1
        self.n_layers = host.n_layers
        self.window = host.window
        self.n_kv_heads = host.n_kv_heads
        self.n_q_heads = host.n_q_heads
        self.head_dim = host.head_dim
        self.basis_rank = host.basis_rank
        self.levels = tuple(host.levels)
        self.total_tokens = int(self.cu_host[-1])
        self.res_stride = int(host.res_stride)
        self.set_split(split_tokens)

    @classmethod
    def from_device(cls, *, basis, coef_k, coef_v, rank_code, res_off, res_idx, res_val, res_scale, cu_seqlens, window: int,
                    n_q_heads: int, levels, coef_scale_k=None, coef_scale_v=None, coef_format: str = "f16",
                    q_dtype: str = "bf16", split_tokens: int = 0):
        """A cache over device tensors that are in the C ABI's layouts already
        (include/dwkv.h, dwkv_cache); they are used in place.  coef_format is "f16"
        or "int8".  Tensors have the layouts' types or are integers of their
        bits (res_off: int32); cu_seqlens [B+1] is a host array.  Such a cache holds
        no queries."""
        import torch
        if coef_format not in ("f16", "int8"):
            raise ValueError(f'coef_format must be "f16" or "int8", not {coef_format!r}')
        self = cls.__new__(cls)
        self.torch, self.lib, self.device = torch, binding.load(), basis.device
        self.coef_format, self.q_dtype, self.q = coef_format, q_dtype, None
        self.cu_host = np.array(cu_seqlens, dtype=np.int32, order="C")  # a copy, as the device's
        self.cu = torch.from_numpy(self.cu_host).to(self.device)
        self.batch, self.total_tokens = len(self.cu_host) - 1, int(self.cu_host[-1])
        self.window, self.levels, self.n_q_heads = int(window), tuple(int(x) for x in levels), int(n_q_heads)
        self.n_layers, self.n_kv_heads, self.head_dim = int(coef_k.shape[0]), int(coef_k.shape[1]), int(basis.shape[-1])
        self.basis_rank, self.res_stride = int(basis.shape[-2]), int(res_idx.shape[-1])
        L, H, T, rb, M = self.n_layers, self.n_kv_heads, self.total_tokens, self.basis_rank, self.n_layers // self.window
        T16, i8 = -(-T // 16) * 16, coef_format == "int8"
        byte, half = (torch.uint8, torch.int8), (torch.float16, torch.int16, torch.uint16)
        word, coef = (torch.int32, torch.uint32), byte if i8 else half
        want = {"basis": (basis, self.batch * M * H * 2 * rb * self.head_dim, half), "coef_k": (coef_k, L * H * T16 * rb, coef),
                "coef_v": (coef_v, L * H * T16 * rb, coef), "rank_code": (rank_code, M * H * T, byte),
                "res_off": (res_off, M * H * (T + 1), word), "res_idx": (res_idx, L * 2 * H * self.res_stride, byte),
                "res_val": (res_val, L * 2 * H * (self.res_stride // 2), byte), "res_scale": (res_scale, L * 2 * H * T, half)}
        if i8:
            want.update(coef_scale_k=(coef_scale_k, L * H * (rb // 16) * T, half),
                        coef_scale_v=(coef_scale_v, L * H * (rb // 16) * T, half))
        else:
            coef_scale_k = coef_scale_v = None
        for name, (x, n, types) in want.items():
            if x is None or x.numel() != n or x.dtype not in types or not x.is_contiguous() or x.device != self.device:
                raise ValueError(f"{name} must be a contiguous {types[0]} tensor of {n} elements on {self.device}")
        self.basis, self.coef_k, self.coef_v = basis, coef_k, coef_v
        self.coef_scale_k, self.coef_scale_v = coef_scale_k, coef_scale_v
        self.rank_code, self.res_off, self.res_idx, self.res_val, self.res_scale = rank_code, res_off, res_idx, res_val, res_scale
        self.set_split(split_tokens)
        return self

    def empty_like(self, seqlens, res_stride: int | None = None):
        """A zero-filled cache of this one's kind for other sequence lengths;
        res_stride: residual entries per slab (a multiple of 256, 512 of them spare),
        by default room for every token at the highest level."""
        torch = self.torch
        cu = np.concatenate([[0], np.cumsum(np.asarray(list(seqlens), dtype=np.int64))])
        T, B, L, H, rb, d = int(cu[-1]), len(cu) - 1, self.n_layers, self.n_kv_heads, self.basis_rank, self.head_dim
        M, T16 = L // self.window, -(-T // 16) * 16
        if res_stride is None:
            res_stride = -(-(T * self.levels[-1] + 512) // 256) * 256
        z = lambda *s, dtype=torch.uint8: torch.zeros(s, dtype=dtype, device=self.basis.device)
        f16, i8 = torch.float16, self.coef_format == "int8"
        if i8:
            k, v = z(L, H, T16 // 16, rb // 16, 16, 16, dtype=self.coef_k.dtype), z(L, H, T16 // 16, rb, 16, dtype=self.coef_v.dtype)
        else:
            k, v = z(L, H, T16 // 16, rb // 8, 16, 8, dtype=f16), z(L, H, T16 // 8, rb, 8, dtype=f16)
        return DeviceCache.from_device(
            basis=z(B, M, H, 2, rb, d, dtype=f16), coef_k=k, coef_v=v, rank_code=z(M, H, T),
            res_off=z(M, H, T + 1, dtype=torch.int32), res_idx=z(L, 2, H, res_stride), res_val=z(L, 2, H, res_stride // 2),
            res_scale=z(L, 2, H, T, dtype=f16), coef_scale_k=z(L, H, rb // 16, T, dtype=f16) if i8 else None,
            coef_scale_v=z(L, H, rb // 16, T, dtype=f16) if i8 else None, cu_seqlens=cu, window=self.window,
            n_q_heads=self.n_q_heads, levels=self.levels, coef_format=self.coef_format, q_dtype=self.q_dtype)

    # -- descriptors -----------------------------------------------------------------
    def set_split(self, split_tokens: int):
        self.dims, self._cu_keep = binding.make_dims(
            batch=self.batch, n_layers=self.n_layers, window=self.window,
            n_kv_heads=self.n_kv_heads, n_q_heads=self.n_q_heads, head_dim=self.head_dim,
            basis_rank=self.basis_rank, levels=self.levels, cu_seqlens_host=self.cu_host,
            cu_seqlens_dev_ptr=self.cu.data_ptr(), total_tokens=self.total_tokens,
            res_stride=self.res_stride, split_tokens=split_tokens,
            coef_format=binding.COEF_I8 if self.coef_format == "int8" else binding.COEF_F16)
        c = binding.Cache()
        c.basis, c.rank_code = self.basis.data_ptr(), self.rank_code.data_ptr()
        c.coef_k, c.coef_v = self.coef_k.data_ptr(), self.coef_v.data_ptr()
        c.res_off, c.res_idx, c.res_val = self.res_off.data_ptr(), self.res_idx.data_ptr(), self.res_val.data_ptr()
        c.res_scale = self.res_scale.data_ptr()
        if self.coef_scale_k is not None:
            c.coef_k_scale, c.coef_v_scale = self.coef_scale_k.data_ptr(), self.coef_scale_v.data_ptr()
        self.cstruct = c
        self._ws = {}

    @property
    def split_tokens(self) -> int:
        return int(self.lib.dwkv_split_tokens(C.byref(self.dims)))

    @property
    def uses_token_lane(self) -> bool:
        """True when dwkv_decode runs the token-lane split kernel for this cache."""
        return int(self.lib.dwkv_decode_kernel(C.byref(self.dims))) == 1

    @property
    def decode_launches(self) -> int:
        """Kernel launches of one decode call without a probe (the split-K pass and the merge)."""
        return int(self.lib.dwkv_decode_launches(C.byref(self.dims), None))

    def _probe_struct(self, probe: ProbeRef | None, err, out_ref):
        if probe is None:
            return None, None
        heads = np.ascontiguousarray(probe.kv_heads, dtype=np.int32)
        p = binding.Probe()
        p.n_heads = len(heads)
        p.kv_heads_host = heads.ctypes.data_as(C.POINTER(C.c_int32))
        p.k_ref, p.v_ref = probe.k_ref.data_ptr(), probe.v_ref.data_ptr()
        p.eps = probe.eps
        p.err = err.data_ptr()
        p.out_ref = out_ref.data_ptr() if out_ref is not None else None
        p.n_pos = probe.n_pos
        if probe.q_prev is not None:
            qp = probe.q_prev
            if tuple(qp.shape[1:]) != (self.batch, self.n_q_heads, self.head_dim) or not qp.is_contiguous():
                raise ValueError("q_prev must be a contiguous [P-1, B, Hq, d] tensor")
            p.q_prev = qp.data_ptr()
        return p, heads

    def workspace_bytes(self, probe: ProbeRef | None = None) -> int:
        torch = self.torch
        G = self.n_q_heads // self.n_kv_heads
        err = torch.empty(1, device=self.device)
        p, keep = self._probe_struct(probe, err, None)
        n = self.lib.dwkv_workspace_bytes(C.byref(self.dims), C.byref(p) if p is not None else None)
        if n == 0:
            raise DwkvError(2, "dwkv_workspace_bytes")
        return int(n)

    def new_workspace(self, probe: ProbeRef | None = None):
        """A fresh decode workspace (zero-filled; the library needs no initial contents)."""
        return self.torch.zeros(self.workspace_bytes(probe), dtype=self.torch.uint8, device=self.device)

    def workspace(self, probe: ProbeRef | None = None):
        """A decode workspace, allocated once per probe shape and reused."""
        need = self.workspace_bytes(probe)
        key = None if probe is None else (len(probe.kv_heads), probe.n_pos)
        ws = self._ws.get(key)
        if ws is None or ws.numel() < need:
            ws = self.new_workspace(probe)
            self._ws[key] = ws
        return ws

    # -- calls -----------------------------------------------------------------------
    def _query(self, layer: int, q):
        if q is not None:
            return q
        if self.q is None:
            raise ValueError("this cache holds no queries: q must be given")
        return self.q[layer]

    def decode(self, layer: int, q=None, sm_scale: float | None = None, probe: ProbeRef | None = None,
               out=None, workspace=None, with_ref: bool = True, err=None):
        """Per-layer decode attention; returns out [B,Hq,d] fp32, or
        (out, err [B, n*G], out_ref [B, n*G, d]) with a probe (err may be given)."""
        torch = self.torch
        q = self._query(layer, q)
        qt = F16 if q.dtype == torch.float16 else BF16
        if q.dtype not in (torch.float16, torch.bfloat16):
            raise TypeError("q must be float16 or bfloat16")
        B, Hq, d = self.batch, self.n_q_heads, self.head_dim
        if out is None:
            out = torch.empty((B, Hq, d), dtype=torch.float32, device=self.device)
        G = Hq // self.n_kv_heads
        out_ref = None
        if probe is not None:
            if probe.q_prev is not None and probe.q_prev.dtype != q.dtype:
                raise TypeError("q_prev must have the decode query's dtype")
            n = len(probe.kv_heads)
            if err is None:
                err = torch.empty((B, n * G), dtype=torch.float32, device=self.device)
            out_ref = torch.empty((B, n * G, d), dtype=torch.float32, device=self.device) if with_ref else None
        p, keep = self._probe_struct(probe, err, out_ref)
        ws = workspace if workspace is not None else self.workspace(probe)
        st = self.lib.dwkv_decode(C.byref(self.dims), C.byref(self.cstruct), int(layer), _ptr(q), qt,
                                  float(sm_scale or 0.0), _ptr(out), C.byref(p) if p is not None else None,
                                  _ptr(ws), ws.numel(), _stream(torch, self.device))
        binding.check(st, "dwkv_decode")
        return out if probe is None else (out, err, out_ref)

    def decode_noalloc(self, layer: int, q=None, sm_scale: float | None = None, out=None,
                       probe: ProbeRef | None = None, err=None):
        """dwkv_decode_noalloc: decode with the library's static scratch (no
        workspace); out [B,Hq,d] fp32 (and err [B, n*G] with a probe) must be
        given or are allocated here by torch.  Returns out, or (out, err)."""
        torch = self.torch
        q = self._query(layer, q)
        if q.dtype not in (torch.float16, torch.bfloat16):
            raise TypeError("q must be float16 or bfloat16")
        qt = F16 if q.dtype == torch.float16 else BF16
        if out is None:
            out = torch.empty((self.batch, self.n_q_heads, self.head_dim), dtype=torch.float32, device=self.device)
        if probe is not None and err is None:
            G = self.n_q_heads // self.n_kv_heads
            err = torch.empty((self.batch, len(probe.kv_heads) * G), dtype=torch.float32, device=self.device)
        p, keep = self._probe_struct(probe, err, None)
        st = self.lib.dwkv_decode_noalloc(C.byref(self.dims), C.byref(self.cstruct), int(layer), _ptr(q), qt,
                                          float(sm_scale or 0.0), _ptr(out), C.byref(p) if p is not None else None,
                                          _stream(torch, self.device))
        binding.check(st, "dwkv_decode_noalloc")
        return out if probe is None else (out, err)

    def decode_partials(self, layer: int, q=None, sm_scale: float | None = None, workspace=None,
                        probe: ProbeRef | None = None, err=None):
        """First half of decode: the split-K pass(es); dwkv_decode_merge finishes it
        (with the same probe and err)."""
        torch = self.torch
        q = self._query(layer, q)
        qt = F16 if q.dtype == torch.float16 else BF16
        p, keep = self._probe_struct(probe, err, None)
        ws = workspace if workspace is not None else self.workspace(probe)
        st = self.lib.dwkv_decode_partials(C.byref(self.dims), C.byref(self.cstruct), int(layer), _ptr(q), qt,
                                           float(sm_scale or 0.0), C.byref(p) if p is not None else None,
                                           _ptr(ws), ws.numel(), _stream(torch, self.device))
        binding.check(st, "dwkv_decode_partials")

    def decode_merge(self, layer: int, out=None, workspace=None, probe: ProbeRef | None = None, err=None):
        """Second half of decode: merges the split partials of `layer` into out [B,Hq,d]
        (and, with a probe, writes err [B, n*G])."""
        torch = self.torch
        if out is None:
            out = torch.empty((self.batch, self.n_q_heads, self.head_dim), dtype=torch.float32, device=self.device)
        p, keep = self._probe_struct(probe, err, None)
        ws = workspace if workspace is not None else self.workspace(probe)
        st = self.lib.dwkv_decode_merge(C.byref(self.dims), C.byref(self.cstruct), int(layer), _ptr(out),
                                        C.byref(p) if p is not None else None, _ptr(ws), ws.numel(),
                                        _stream(torch, self.device))
        binding.check(st, "dwkv_decode_merge")
        return out

    def probe_feature(self, layer: int, kv_heads, err, phi, fresh: bool):
        """dwkv_probe_feature: fold one probed layer's Eq. 3 errors err [B, n*G]
        into column 3 of the layer's window of phi [M, Hkv, T, 4] (in place)."""
        heads = np.ascontiguousarray(kv_heads, dtype=np.int32)
        st = self.lib.dwkv_probe_feature(C.byref(self.dims), int(layer), len(heads),
                                         heads.ctypes.data_as(C.POINTER(C.c_int32)), _ptr(err), int(bool(fresh)),
                                         _ptr(phi), _stream(self.torch, self.device))
        binding.check(st, "dwkv_probe_feature")
        return phi

    def route(self, phi, u, theta, rank_code=None, res_off=None):
        """Eq. 2 routing on the GPU; returns (rank_code uint8 [M,Hkv,T], res_off int32-view [M,Hkv,T+1])."""
        torch = self.torch
        M, Hk, T = self.n_layers // self.window, self.n_kv_heads, self.total_tokens
        if rank_code is None:
            rank_code = torch.empty((M, Hk, T), dtype=torch.uint8, device=self.device)
        if res_off is None:
            res_off = torch.empty((M, Hk, T + 1), dtype=torch.int32, device=self.device)
        need = self.lib.dwkv_route_workspace_bytes(C.byref(self.dims))
        ws = torch.empty(max(int(need), 1), dtype=torch.uint8, device=self.device)
        st = self.lib.dwkv_route(C.byref(self.dims), _ptr(phi), _ptr(u), _ptr(theta), _ptr(rank_code),
                                 _ptr(res_off), _ptr(ws), ws.numel(), _stream(torch, self.device))
        binding.check(st, "dwkv_route")
        return rank_code, res_off

    def route_range(self, phi, u, theta, t0: int, t1: int, rank_code=None, res_off=None):
        """Eq. 2 routing of packed tokens [t0, t1), continuing the offset table in
        place (by default the cache's own rank_code / res_off)."""
        torch = self.torch
        rank_code = self.rank_code if rank_code is None else rank_code
        res_off = self.res_off if res_off is None else res_off
        need = self.lib.dwkv_route_workspace_bytes(C.byref(self.dims))
        ws = torch.empty(max(int(need), 1), dtype=torch.uint8, device=self.device)
        st = self.lib.dwkv_route_range(C.byref(self.dims), _ptr(phi), _ptr(u), _ptr(theta), int(t0), int(t1),
                                       _ptr(rank_code), _ptr(res_off), _ptr(ws), ws.numel(),
                                       _stream(torch, self.device))
        binding.check(st, "dwkv_route_range")
        return rank_code, res_off

    def route_budget(self, phi, u, entries, t0: int, t1: int, rank_code=None, res_off=None):
        """Two-level Eq. 2 routing of tokens [t0, t1) under a budget of entries
        (int64 [M, Hkv], device) per (window, head); in place by default."""
        torch = self.torch
        rank_code = self.rank_code if rank_code is None else rank_code
        res_off = self.res_off if res_off is None else res_off
        need = int(self.lib.dwkv_route_budget_workspace_bytes(C.byref(self.dims)))
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
        st = self.lib.dwkv_route_budget(C.byref(self.dims), _ptr(phi), _ptr(u), _ptr(entries), int(t0), int(t1),
                                        _ptr(rank_code), _ptr(res_off), _ptr(ws), ws.numel(),
                                        _stream(torch, self.device))
        binding.check(st, "dwkv_route_budget")
        return rank_code, res_off

    def compress(self, layer: int, x_k, x_v, t0: int, t1: int, gate=None):
        """Append/compress packed tokens [t0, t1) of `layer` in place from dense
        fp16 keys / values x_k, x_v [t1-t0, Hkv, d]; gate: None or fp32 [2, Hkv, t1-t0]."""
        torch = self.torch
        for x in (x_k, x_v):
            if x.dtype != torch.float16 or not x.is_contiguous():
                raise TypeError("x_k / x_v must be contiguous float16")
        if gate is not None and (gate.dtype != torch.float32 or not gate.is_contiguous()):
            raise TypeError("gate must be contiguous float32")
        st = self.lib.dwkv_compress(C.byref(self.dims), C.byref(self.cstruct), int(layer), _ptr(x_k), _ptr(x_v),
                                    _ptr(gate), int(t0), int(t1), _stream(torch, self.device))
        binding.check(st, "dwkv_compress")

    @property
    def decode_append_launches(self) -> int:
        return int(self.lib.dwkv_decode_append_launches(C.byref(self.dims)))

    def decode_append(self, layer: int, x_k, x_v, gate=None, q=None, sm_scale: float | None = None, out=None,
                      workspace=None):
        """dwkv_decode_append: append the new token of every sequence (its
        last) from x_k, x_v [B, Hkv, d] fp16 (gate None or fp32 [2, Hkv, B]),
        then decode the layer; returns out [B, Hq, d] fp32."""
        torch = self.torch
        for x in (x_k, x_v):
            if x.dtype != torch.float16 or not x.is_contiguous():
                raise TypeError("x_k / x_v must be contiguous float16")
        if gate is not None and (gate.dtype != torch.float32 or not gate.is_contiguous()):
            raise TypeError("gate must be contiguous float32")
        q = self._query(layer, q)
        if q.dtype not in (torch.float16, torch.bfloat16):
            raise TypeError("q must be float16 or bfloat16")
        qt = F16 if q.dtype == torch.float16 else BF16
        if out is None:
            out = torch.empty((self.batch, self.n_q_heads, self.head_dim), dtype=torch.float32, device=self.device)
        need = int(self.lib.dwkv_decode_append_workspace_bytes(C.byref(self.dims)))
        if need == 0:
            raise DwkvError(2, "dwkv_decode_append_workspace_bytes")
        if workspace is None:
            ws = self._ws.get("append")
            if ws is None or ws.numel() < need:
                ws = torch.zeros(need, dtype=torch.uint8, device=self.device)
                self._ws["append"] = ws
            workspace = ws
        st = self.lib.dwkv_decode_append(C.byref(self.dims), C.byref(self.cstruct), int(layer), _ptr(q), qt,
                                         float(sm_scale or 0.0), _ptr(out), _ptr(x_k), _ptr(x_v), _ptr(gate),
                                         _ptr(workspace), workspace.numel(), _stream(torch, self.device))
        binding.check(st, "dwkv_decode_append")
        return out

    def decode_features(self, layer: int, phi, q=None, sm_scale: float | None = None, out=None, workspace=None):
        """dwkv_decode plus the router's attention features: phi fp32 [M, Hkv, T, 4]
        (columns 0 mass, 1 spike) is updated in place; returns out [B, Hq, d]."""
        torch = self.torch
        q = self._query(layer, q)
        qt = F16 if q.dtype == torch.float16 else BF16
        if out is None:
            out = torch.empty((self.batch, self.n_q_heads, self.head_dim), dtype=torch.float32, device=self.device)
        if workspace is None:
            n = int(self.lib.dwkv_features_workspace_bytes(C.byref(self.dims)))
            if n == 0:
                raise DwkvError(3, "dwkv_features_workspace_bytes")
            workspace = torch.empty(n, dtype=torch.uint8, device=self.device)
        st = self.lib.dwkv_decode_features(C.byref(self.dims), C.byref(self.cstruct), int(layer), _ptr(q), qt,
                                           float(sm_scale or 0.0), _ptr(out), _ptr(phi), _ptr(workspace),
                                           workspace.numel(), _stream(torch, self.device))
        binding.check(st, "dwkv_decode_features")
        return out

    def sketch_basis(self, window: int, seq: int, x, omega):
        """Randomized-sketch bases of (seq, window) from its prefill x fp16
        [w, 2, n, Hkv, d] and sketch matrix omega fp16 [w*n, r_b]; in place."""
        torch = self.torch
        n = int(x.shape[2])
        need = int(self.lib.dwkv_sketch_workspace_bytes(C.byref(self.dims), n))
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
        st = self.lib.dwkv_sketch_basis(C.byref(self.dims), C.byref(self.cstruct), int(window), int(seq), _ptr(x),
                                        _ptr(omega), n, _ptr(ws), ws.numel(), _stream(torch, self.device))
        binding.check(st, "dwkv_sketch_basis")

    def materialize(self, layer: int, k_out=None, v_out=None):
        """Eq. 1 written out for `layer`: K_hat fp16 [Hkv, T, d] and V_hat fp16
        [Hkv, T16/16, d, 16] (the blocked layout of the dense decode)."""
        torch = self.torch
        Hk, T, d = self.n_kv_heads, self.total_tokens, self.head_dim
        T16 = -(-T // 16) * 16
        if k_out is None:
            k_out = torch.empty((Hk, T, d), dtype=torch.float16, device=self.device)
        if v_out is None:
            v_out = torch.empty((Hk, T16 // 16, d, 16), dtype=torch.float16, device=self.device)
        st = self.lib.dwkv_materialize(C.byref(self.dims), C.byref(self.cstruct), int(layer), _ptr(k_out),
                                       _ptr(v_out), _stream(torch, self.device))
        binding.check(st, "dwkv_materialize")
        return k_out, v_out

    def dense_decode(self, k, v, q, sm_scale: float | None = None, out=None, workspace=None):
        """Decode attention over a dense fp16 cache k [Hkv, T, d], v [Hkv, T16/16, d, 16]."""
        torch = self.torch
        qt = F16 if q.dtype == torch.float16 else BF16
        if out is None:
            out = torch.empty((self.batch, self.n_q_heads, self.head_dim), dtype=torch.float32, device=self.device)
        if workspace is None:
            workspace = torch.empty(int(self.lib.dwkv_dense_workspace_bytes(C.byref(self.dims))),
                                    dtype=torch.uint8, device=self.device)
        st = self.lib.dwkv_dense_decode(C.byref(self.dims), _ptr(k), _ptr(v), _ptr(q), qt, float(sm_scale or 0.0),
                                        _ptr(out), _ptr(workspace), workspace.numel(),
                                        _stream(torch, self.device))
        binding.check(st, "dwkv_dense_decode")
        return out

    def tree_workspace(self, tree: DraftTree):
        """A workspace for ``tree_decode`` of such trees over this cache."""
        n = int(self.lib.dwkv_tree_workspace_bytes(C.byref(self.dims), C.byref(tree.cstruct)))
        if n == 0:
            raise DwkvError(2, "dwkv_tree_workspace_bytes")
        return self.torch.empty(n, dtype=self.torch.uint8, device=self.basis.device)

    def tree_decode(self, layer: int, tree: DraftTree, q, k_new, v_new, sm_scale: float | None = None, out=None,
                    workspace=None):
        """dwkv_tree_decode: attention of the drafted nodes' queries q [N, Hq, d]
        over the cache and their ancestors' keys and values k_new, v_new fp16
        [N, Hkv, d] (q and k_new, v_new may be slices of wider rows); returns out
        fp32 [N, Hq, d]."""
        torch = self.torch
        N, Hq, Hk, d = tree.n_nodes, self.n_q_heads, self.n_kv_heads, self.head_dim
        if tree.batch != self.batch:
            raise ValueError("the tree and the cache have different batches")
        if q.dtype not in (torch.float16, torch.bfloat16):
            raise TypeError("q must be float16 or bfloat16")
        if k_new.dtype != torch.float16 or v_new.dtype != torch.float16:
            raise TypeError("k_new and v_new must be float16")
        if q.shape != (N, Hq, d) or k_new.shape != (N, Hk, d) or v_new.shape != (N, Hk, d):
            raise ValueError("q must be [N, Hq, d], k_new and v_new [N, Hkv, d]")
        qs, ks, vs = q.stride(), k_new.stride(), v_new.stride()
        if N > 0 and not qs[1:] == ks[1:] == vs[1:] == (d, 1) and any(
                x.stride(2) != 1 or x.shape[1] > 1 and x.stride(1) != d for x in (q, k_new, v_new)):   # one head has no stride
            raise ValueError("the rows of q, k_new and v_new must have no gaps inside")
        if N > 1 and ks[0] != vs[0]:
            raise ValueError("k_new and v_new must have the same row stride")
        if N > 1 and (qs[0] < Hq * d or ks[0] < Hk * d):
            raise ValueError("the rows of q, k_new and v_new must not overlap")
        index = self.basis.get_device()
        if tree.index != index or not _all_on(index, q, k_new, v_new, out, workspace):
            raise ValueError("every tensor must be on the cache's device")
        if out is None:
            out = torch.empty((N, Hq, d), dtype=torch.float32, device=self.basis.device)
        elif out.dtype != torch.float32 or out.shape != (N, Hq, d) or not out.is_contiguous():
            raise TypeError("out must be contiguous float32 [N, Hq, d]")
        if N == 0:
            return out
        ws = workspace if workspace is not None else self.tree_workspace(tree)
        with _on(torch, index):
            st = self.lib.dwkv_tree_decode(C.byref(self.dims), C.byref(self.cstruct), int(layer), tree.ref, q.data_ptr(),
                                           F16 if q.dtype == torch.float16 else BF16, qs[0] if N > 1 else 0, k_new.data_ptr(),
                                           v_new.data_ptr(), ks[0] if N > 1 else 0, float(sm_scale or 0.0), out.data_ptr(),
                                           ws.data_ptr(), _nbytes(ws), torch.cuda.current_stream(index).cuda_stream)
        binding.check(st, "dwkv_tree_decode")
        return out

    def repack_workspace(self):
        """A workspace for ``repack_from`` into this cache."""
        n = int(self.lib.dwkv_repack_workspace_bytes(C.byref(self.dims)))
        if n == 0:
            raise DwkvError(2, "dwkv_repack_workspace_bytes")
        return self.torch.empty(n, dtype=self.torch.uint8, device=self.basis.device)

    def repack_from(self, src: "DeviceCache", src_token, src_seq, new_code=None, workspace=None):
        """dwkv_repack: fill this cache with tokens of ``src``: token t is
        src_token[t] (int32 [T], device), or the fresh slot -1 - src_token[t] at
        level new_code[m, h, slot] (uint8 [M, Hkv, n], None: level 0); sequence b
        takes the bases of src_seq[b] (int32 [B], device; negative: unchanged)."""
        torch = self.torch
        M, H = self.n_layers // self.window, self.n_kv_heads
        if src_token.dtype != torch.int32 or src_token.numel() != self.total_tokens or not src_token.is_contiguous():
            raise TypeError("src_token must be contiguous int32 [T]")
        if src_seq.dtype != torch.int32 or src_seq.numel() != self.batch or not src_seq.is_contiguous():
            raise TypeError("src_seq must be contiguous int32 [B]")
        n_new = 0
        if new_code is not None:
            n_new = int(new_code.shape[-1])
            if new_code.dtype != torch.uint8 or tuple(new_code.shape) != (M, H, n_new) or not new_code.is_contiguous():
                raise TypeError("new_code must be contiguous uint8 [M, Hkv, n]")
        index = self.basis.get_device()
        if not _all_on(index, src_token, src_seq, new_code, workspace, src.basis):
            raise ValueError("every tensor must be on the cache's device")
        ws = workspace if workspace is not None else self.repack_workspace()
        with _on(torch, index):
            st = self.lib.dwkv_repack(C.byref(self.dims), C.byref(self.cstruct), C.byref(src.dims), C.byref(src.cstruct),
                                      src_token.data_ptr() or None, src_seq.data_ptr(), None if new_code is None else new_code.data_ptr(),
                                      n_new, ws.data_ptr(), _nbytes(ws), torch.cuda.current_stream(index).cuda_stream)
        binding.check(st, "dwkv_repack")

    def residual_map(self, layer: int, z: int, kv_head: int, t0: int, t1: int):
        torch = self.torch
        dense = torch.empty((max(t1 - t0, 0), self.head_dim), dtype=torch.float32, device=self.device)
        st = self.lib.dwkv_residual_map(C.byref(self.dims), C.byref(self.cstruct), int(layer), int(z),
                                        int(kv_head), int(t0), int(t1), _ptr(dense),
                                        _stream(torch, self.device))
        binding.check(st, "dwkv_residual_map")
        return dense

    def coef_host(self):
        """The device coefficients in the host layout (fp16 as uint16): keys
        [L][Hkv][T][r_b], values [L][Hkv][T16/16][r_b][16] (int8: codes, same shapes)."""
        k = self.coef_k.cpu().numpy()
        v = self.coef_v.cpu().numpy()
        L, Hk, T, rb = self.n_layers, self.n_kv_heads, self.total_tokens, self.basis_rank
        T16 = -(-T // 16) * 16
        if self.coef_format == "int8":
            return layout.keys_from_abi(k.reshape(L, Hk, T16 // 16, rb // 16, 16, 16), T), v
        k, v = k.view(np.uint16), v.view(np.uint16)
        keys = layout.keys_from_abi(k.reshape(L, Hk, T16 // 16, rb // 8, 16, 8), T)
        vals = layout.values_from_abi(v.reshape(L, Hk, T16 // 8, rb, 8))
        return keys, vals

    def validate(self):
        """Returns (ok, bad_index); raises on argument errors."""
        torch = self.torch
        ws = torch.empty(int(self.lib.dwkv_validate_workspace_bytes()), dtype=torch.uint8, device=self.device)
        bad = C.c_int64(-1)
        st = self.lib.dwkv_validate(C.byref(self.dims), C.byref(self.cstruct), C.byref(bad), _ptr(ws),
                                    ws.numel(), _stream(torch, self.device))
        if st == 5:
            return False, int(bad.value)
        binding.check(st, "dwkv_validate")
        return True, -1
