"""Arguments of the speculative step's Python forms that the host can tell to be
right or wrong by itself: none of these cases needs a GPU."""
import numpy as np
import pytest
import torch

from paper_2607_06523_amd import DeviceCache
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
