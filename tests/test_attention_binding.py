"""Host: what the binding of the attention and paged calls refuses before anything is launched."""

from types import SimpleNamespace

import numpy as np
import pytest

from paper_2609_32259_amd import heterofold as hf

torch = pytest.importorskip("torch")


def test_a_stream_of_another_device_is_refused():
    """(The launch would have gone to the tensors' device's current stream instead.)"""
    here, there = torch.device("cuda", 0), torch.device("cuda", 1)
    with pytest.raises(ValueError, match="stream"):
        with hf._call_on(here, SimpleNamespace(device=there, cuda_stream=0)):
            pass


@pytest.mark.parametrize("make", [list, np.asarray, torch.tensor], ids=["list", "numpy", "torch"])
def test_lengths_are_whole_numbers(make):
    for lens in ([2.7], [1.0, 2.5], [float("nan")]):
        with pytest.raises((TypeError, ValueError)):
            hf._lens(make(lens), "n")
    with pytest.raises((TypeError, ValueError)):
        hf._lens(make([[1, 2]]), "n")
    array, lens = hf._lens(make([3, 0, 5]), "n", 3)
    assert lens == [3, 0, 5] and list(array) == lens


def test_nested_lengths_are_refused():
    with pytest.raises(TypeError):
        hf._lens([[1, 2]], "n")
    with pytest.raises(ValueError):
        hf._lens(np.zeros((2, 2), np.int32), "n")


def test_dense_cache_refuses_lengths_that_do_not_fit():
    """(64-bit lengths were cut to 32 bits.)"""
    from paper_2609_32259_amd.path import dense_cache
    cache = SimpleNamespace(L=1, H=1, d_h=64, pages=torch.zeros(1), batch=1)
    for lens in (np.array([(1 << 32) + 5]), [1 << 31], np.array([5.5]), [5.5]):
        with pytest.raises((TypeError, ValueError)):
            dense_cache(cache, lens)
