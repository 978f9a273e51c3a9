"""What the gate and the experts' operators refuse at the limits of their ranges, without a GPU."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def ep():
    from paper_2603_13606_amd import binding, build
    if not build.is_current():
        build.build()
    binding.load()
    return binding


class OnGpu:
    """Looks like a tensor of a GPU to the check of devices."""
    is_cuda, device = True, torch.device("cuda", 0)


def test_tensors_in_host_memory_among_those_of_a_gpu_are_refused(ep, monkeypatch):
    """A kernel that is handed their address would fault.  Pinned memory and empty tensors pass, and so do calls on the host alone
    (whose descriptors are checked before anything is launched)."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    host, empty = torch.zeros(4, dtype=torch.int32), torch.zeros(0, dtype=torch.int32)
    with pytest.raises(ValueError):
        ep._one_device([OnGpu(), host])
    with pytest.raises(ValueError):
        ep._one_device([host, OnGpu(), OnGpu()])
    pinned = type("Pinned", (), dict(is_cuda=False, device=torch.device("cpu"), numel=lambda self: 4, is_pinned=lambda self: True))()
    assert ep._one_device([OnGpu(), empty, pinned]) == 0
    assert ep._one_device([host, empty]) is None
