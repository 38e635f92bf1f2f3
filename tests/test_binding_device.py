"""The binding asks torch's public interface for the current device (what ends a forked child's use of CUDA with a reason, and picks up a device
that was never set)."""
import pytest
import torch

from paper_2502_16880_b200 import lmhead


class _On:
    def __init__(self, device):
        self.device = device

    def get_device(self):
        return self.device


def test_current_device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    assert lmhead._op_device(_On(3), "x") == 3
    for other in (-1, 0, 2):
        with pytest.raises(ValueError, match="x must be on the current CUDA device"):
            lmhead._op_device(_On(other), "x")
