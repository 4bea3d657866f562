"""Tensors that agree with one another but are not on the current device are refused."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_not_the_current_device(dev):
    from paper_2607_08565_amd import kv
    if torch.cuda.device_count() < 2:
        pytest.skip("one device")
    x = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda:1")
    with torch.cuda.device(0), pytest.raises(ValueError, match="current device"):
        kv.qk_rotate(x, x, kv.Rotary(), q_out=x, k_out=x)
    with torch.cuda.device(1):
        kv.qk_rotate(x, x, kv.Rotary(), q_out=x, k_out=x)
