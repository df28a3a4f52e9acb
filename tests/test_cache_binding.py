"""What the binding of the cache and scoring calls refuses before it needs a GPU."""

from types import SimpleNamespace

import pytest


def test_streams_of_another_device_are_refused():
    from paper_2609_21827_amd import binding
    import torch
    h = binding._OnDevice()
    h._index, h.device = 0, torch.device("cuda", 0)
    other = SimpleNamespace(device_index=1, cuda_stream=64)
    for call in (lambda: h._stream(other, ()),
                 lambda: h._made(None, torch.int32, (3,), "out", other)):
        with pytest.raises(binding.RheoError, match="stream must be of") as e:
            call()
        assert e.value.code == binding.RHEO_EINVAL
