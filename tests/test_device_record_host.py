"""The device's failure record without a device: the call exists and reports the runtime's failure.  No GPU needed."""
import pytest
import torch


def test_without_a_device():
    from paper_1911_04070_b200 import build, binding
    build.build()
    lib = binding.load_library()
    assert "bpt_check_device" in binding.EXPORTS
    if torch.cuda.is_available():
        pytest.skip("there is a device")
    assert lib.bpt_check_device(None) == 4
