"""What the binding refuses, keeps and forgets, on the host alone."""
import pytest
import torch

from paper_2609_40093_b200 import ep


class _OnDevice:
    """Answers the device query as a tensor of CUDA device 1 would."""
    device = torch.device("cuda", 1)

    def get_device(self):
        return 1


def test_tensors_on_another_device_than_the_current_one_are_refused(monkeypatch):
    """The library launches on the current device: a stream and addresses of another one may not reach it."""
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    with pytest.raises(ValueError, match="current"):
        ep._stream_of(_OnDevice(), _OnDevice(), None)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    assert ep._stream_of(_OnDevice(), _OnDevice(), None) == 0
