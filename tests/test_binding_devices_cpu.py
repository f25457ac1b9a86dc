"""The binding's checks of devices and streams, on the CPU with stand-ins for
device tensors and streams."""
import pytest
import torch

from paper_2607_08526_amd import qlinear as ql


class DeviceTensor:
    is_cuda = True

    def __init__(self, index):
        self.index = index
        self.device = f"cuda:{index}"

    def get_device(self):
        return self.index


@pytest.fixture(params=[True, False], ids=["torch has _cuda_getDevice", "it does not"])
def device0(request, monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(ql, "_device", (lambda: 0) if request.param else None)


def test_tensors_on_the_current_device(device0):
    ql._on_current_device(DeviceTensor(0), None, DeviceTensor(0))
    with pytest.raises(ValueError, match="current device"):
        ql._on_current_device(DeviceTensor(0), DeviceTensor(1))
    with pytest.raises(ValueError, match="device"):
        ql._on_current_device(torch.zeros(1))


def test_stream_of_the_current_device(device0):
    class Stream:
        cuda_stream = 7
        device_index = 0

    assert ql._stream(Stream()) == 7
    Stream.device_index = 1
    with pytest.raises(ValueError, match="stream"):
        ql._stream(Stream())
