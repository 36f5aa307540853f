"""Host: what the binding of the attention and paged calls refuses before anything is launched."""

from types import SimpleNamespace

import pytest

from paper_2609_32259_amd import heterofold as hf

torch = pytest.importorskip("torch")


def test_a_stream_of_another_device_is_refused():
    """(The launch would have gone to the tensors' device's current stream instead.)"""
    here, there = torch.device("cuda", 0), torch.device("cuda", 1)
    with pytest.raises(ValueError, match="stream"):
        with hf._call_on(here, SimpleNamespace(device=there, cuda_stream=0)):
            pass
