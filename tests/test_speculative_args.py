"""Arguments of the speculative step's Python forms that the host can tell to be
right or wrong by itself: none of these cases needs a GPU."""
import numpy as np
import pytest
import torch

from paper_2607_06523_amd import DeviceCache, DraftTree
from test_speculative_cpu import a_cache


def int8_cache(lengths=(5,)):
    a = a_cache(lengths)
    T = sum(lengths)
    for k in ("coef_k", "coef_v"):
        a[k] = torch.zeros(a[k].shape, dtype=torch.uint8)
    scale = lambda: torch.zeros((2, 2, 1, T), dtype=torch.float16)
    return {**a, "coef_scale_k": scale(), "coef_scale_v": scale(), "coef_format": "int8"}


@pytest.mark.parametrize("name", ["basis", "coef_k", "coef_v", "res_scale", "coef_scale_k", "coef_scale_v"])
def test_caches_of_bfloat16_are_refused(name):
    """As wide as float16, and something else."""
    a = int8_cache() if name.startswith("coef_scale") else a_cache()
    with pytest.raises(ValueError, match=name):
        DeviceCache.from_device(**{**a, name: a[name].to(torch.bfloat16)})


@pytest.mark.parametrize("name,other", [("coef_k", torch.bool), ("rank_code", torch.bool), ("res_idx", torch.float8_e4m3fn),
                                        ("res_off", torch.float32)])
def test_caches_of_other_types_of_the_same_size_are_refused(name, other):
    a = int8_cache()
    with pytest.raises(ValueError, match=name):
        DeviceCache.from_device(**{**a, name: torch.zeros(a[name].shape).to(other)})


@pytest.mark.parametrize("fmt", ["fp16", "i8", "INT8", "", None])
def test_unknown_coefficient_formats_are_refused(fmt):
    with pytest.raises(ValueError, match="coef_format"):
        DeviceCache.from_device(**{**a_cache(), "coef_format": fmt})


def test_caches_of_the_types_or_their_bits_are_taken():
    for a in (a_cache(), int8_cache()):
        bits = {torch.float16: torch.int16, torch.uint8: torch.int8}
        other = {k: x.view(bits.get(x.dtype, x.dtype)) if isinstance(x, torch.Tensor) else x for k, x in a.items()}
        for b in (a, other):
            dc = DeviceCache.from_device(**b)
            assert dc.coef_k.data_ptr() == b["coef_k"].data_ptr()
            new = dc.empty_like([4, 9])
            assert new.coef_format == dc.coef_format and np.array_equal(new.cu_host, [0, 4, 13])


def test_trees_and_caches_keep_their_own_starts():
    """A program refills its arrays for the next step: the handles' host sides stay with their device sides."""
    cu, parent = np.array([0, 3, 7], np.int32), torch.tensor([-1, 0, 1, -1, 0, 0, 2], dtype=torch.int32)
    tree = DraftTree(cu, parent)
    lens = np.array([0, 5, 8], np.int32)
    dc = DeviceCache.from_device(**{**a_cache((5, 3)), "cu_seqlens": lens})
    cu[1], lens[1] = 1, 2
    for x, want in ((tree, [0, 3, 7]), (dc, [0, 5, 8])):
        assert x.cu.tolist() == want and x.cu_host.tolist() == want
    assert tree.cstruct.cu_nodes_host[:3] == [0, 3, 7] and dc.dims.cu_seqlens_host[:3] == [0, 5, 8]
    dc.set_split(64)
    assert dc.dims.cu_seqlens_host[:3] == [0, 5, 8]


def test_host_caches_keep_their_own_starts():
    from synth import TINY, generate
    host = generate(TINY, threads=2)
    want = host.cu_seqlens = np.array(host.cu_seqlens, dtype=np.int32)
    dc = DeviceCache(host, device="cpu")
    want = want.copy()
    host.cu_seqlens[1:] -= 1
    assert np.array_equal(dc.cu_host, want) and dc.cu.tolist() == want.tolist()


def test_caches_without_queries_say_so():
    x = torch.zeros((1, 2, 128), dtype=torch.float16)
    dc = DeviceCache.from_device(**a_cache())
    for cache in (dc, dc.empty_like([7])):
        for call in (lambda: cache.decode(0), lambda: cache.decode_noalloc(0), lambda: cache.decode_partials(0),
                     lambda: cache.decode_append(0, x, x), lambda: cache.decode_features(0, None)):
            with pytest.raises(ValueError, match="holds no queries"):
                call()


def test_one_head_has_no_stride():
    """[1, N, d] turned to [N, 1, d] is contiguous, whatever stride its one head carries."""
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    f16 = lambda *s: torch.zeros(s, dtype=torch.float16)
    dc = DeviceCache.from_device(basis=f16(1, 1, 1, 2, 16, 128), coef_k=f16(2, 1, 16, 16), coef_v=f16(2, 1, 16, 16), rank_code=u8(1, 1, 5),
                                 res_off=torch.zeros((1, 1, 6), dtype=torch.int32), res_idx=u8(2, 2, 1, 1024), res_val=u8(2, 2, 1, 512),
                                 res_scale=f16(2, 2, 1, 5), cu_seqlens=[0, 5], window=2, n_q_heads=1, levels=(0, 2))
    tree = DraftTree([0, 3], torch.tensor([-1, 0, 1], dtype=torch.int32))
    one = f16(1, 3, 128).transpose(0, 1)
    assert one.is_contiguous() and one.stride(1) != 128
    with pytest.raises(ValueError, match="device"):     # past the strides: nothing of it is on a GPU
        dc.tree_decode(0, tree, one, one, one)
    gaps = f16(3, 1, 256)[:, :, ::2]
    for args in ((gaps, one, one), (one, gaps, one), (one, one, gaps)):
        with pytest.raises(ValueError, match="gaps"):
            dc.tree_decode(0, tree, *args)
