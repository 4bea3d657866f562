"""The binding where torch has no 4-bit type: 16- and 8-bit caches are as they are with one."""
import subprocess
import sys

SCRIPT = """
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
with FakeTensorMode():  # (what torch itself imports for its stand-ins asks for the types)
    torch.empty(2, device="cuda:0").data_ptr(), torch.empty((2, 2), device="cuda:0")[:, 0].stride()
for name in ("float4_e2m1fn_x2", "float8_e8m0fnu"):
    delattr(torch, name)
from paper_2607_08565_amd import kv
with FakeTensorMode():
    for dtype in (torch.bfloat16, torch.float16, torch.float8_e4m3fn):
        c = kv.PagedCache.empty(5, 2, 64, dtype=dtype, device="cuda:0")
        assert c.head_dim == 64 and c.c.exps is None
    for dtype in (torch.float32, torch.uint8):
        try:
            kv.PagedCache.empty(5, 2, 64, dtype=dtype, device="cuda:0")
        except TypeError:
            continue
        raise AssertionError(dtype)
    e = torch.empty((5, 2, 16, 2), dtype=torch.uint8, device="cuda:0")
    try:
        kv.PagedCache(c.k, c.v, k_exp=e, v_exp=e)
    except ValueError:
        print("fine")
"""


def test_import_and_caches():
    r = subprocess.run([sys.executable, "-W", "ignore", "-c", SCRIPT], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "fine", r.stderr[-2000:]
