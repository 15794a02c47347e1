"""The round driver's calls for the selected batch, host side (no kernel is launched here)."""
import pytest
import torch

from paper_2505_09142_amd.driver import DeviceRoundDriver


def test_logits_take_no_stream():
    """The histories are packed on the current stream: an adjustment on another one would read them too early."""
    drv = DeviceRoundDriver.__new__(DeviceRoundDriver)
    drv.appended, drv.slot_of = {1: 3}, {1: 0}
    with pytest.raises(TypeError, match="stream"):
        drv.adjust_logits([1], torch.zeros((1, 9)), [1], stream=object())
    with pytest.raises(TypeError):
        drv.adjust_logits([1], torch.zeros((1, 9)), [1], cu_seqlens=torch.zeros(2))
