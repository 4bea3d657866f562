"""What the paged cache's binding refuses before it hands on an address, on tensors without memory."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2607_08565_amd import kv
from paper_2607_08565_amd.smetric import SmetricError

pytestmark = pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")
SHAPE = (2, 3, 4, 2, 64, 1)


def test_plan_takes_device_memory_only():
    with pytest.raises(TypeError):
        kv.Plan(*SHAPE, device="cpu")
    for w in (torch.empty(1 << 22, dtype=torch.uint8), "x", torch.empty(1 << 22)):
        with pytest.raises(TypeError):
            kv.Plan(*SHAPE, workspace=w)
    with FakeTensorMode():
        u8 = lambda n, **how: torch.empty(n, dtype=torch.uint8, device="cuda")  # noqa: E731
        for w in (u8(1).expand(1 << 22), u8(1 << 23)[::2], torch.empty(1 << 22, device="cuda"), u8(1 << 22).cpu()):
            with pytest.raises(TypeError):
                kv.Plan(*SHAPE, workspace=w)
        with pytest.raises(SmetricError):
            kv.Plan(*SHAPE, workspace=u8(16))
