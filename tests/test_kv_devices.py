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


def _args(on):
    """A call's tensors by name, on cuda:0 or, where `on` names them, on cuda:1."""
    dev = lambda name: "cuda:1" if name == on else "cuda:0"  # noqa: E731
    bf = lambda name, *s: torch.empty(s, dtype=torch.bfloat16, device=dev(name))  # noqa: E731
    num = lambda name, t, *s: torch.empty(s, dtype=t, device=dev(name))  # noqa: E731
    return dict(q=bf("q", 3, 4, 64), k=bf("k", 3, 2, 64), v=bf("v", 3, 2, 64), out=bf("out", 3, 4, 64), k_out=bf("k_out", 3, 2, 64),
                table=num("table", torch.int32, 2, 4), q_off=num("q_off", torch.int64, 3), kv_len=num("kv_len", torch.int32, 2),
                positions=num("positions", torch.int32, 3), status=num("status", torch.int32, 1),
                lse=num("lse", torch.float32, 3, 4), cache=kv.PagedCache(*[bf("cache", 5, 2, 16, 64) for _ in "kv"]),
                rotary=kv.Rotary(num("rotary", torch.float32, 8, 64)), plan=kv.Plan(*SHAPE, device=dev("plan")))


def _calls(x):
    p = x["plan"]
    return dict(
        rotate=(("q", "k", "rotary", "positions", "out", "k_out", "status"),
                lambda: kv.qk_rotate(x["q"], x["k"], x["rotary"], x["positions"], x["out"], x["k_out"], x["status"])),
        append=(("cache", "table", "q_off", "kv_len", "k", "v", "q", "out", "rotary", "positions", "status"),
                lambda: kv.append(x["cache"], x["table"], x["q_off"], x["kv_len"], x["k"], x["v"], x["q"], x["out"], x["rotary"],
                                  x["positions"], x["status"])),
        make=(("plan", "q_off", "kv_len", "status"), lambda: p.make(x["q_off"], x["kv_len"], x["status"])),
        attend=(("q", "cache", "table", "plan", "out", "lse", "q_off", "kv_len", "status"),
                lambda: kv.attend(x["q"], x["cache"], x["table"], p, out=x["out"], lse=x["lse"], status=x["status"])))


@pytest.mark.parametrize("call", ["rotate", "append", "make", "attend"])
def test_tensors_of_another_device(call):
    """One tensor, cache, table of angles or plan of another device than the others is refused."""
    if torch.cuda.is_available() and torch.cuda.device_count() < 2:
        pytest.skip("torch makes no stand-in for a second device beside a single real one")
    with FakeTensorMode():
        names = _calls(_args(None))[call][0]
        for name in names:
            x = _args(name)
            x["plan"].q_off, x["plan"].kv_len = x["q_off"], x["kv_len"]
            with pytest.raises(ValueError, match="device"):
                _calls(x)[call][1]()
        z = torch.empty(5, 2, 16, 64, dtype=torch.float8_e4m3fn, device="cuda:0")
        one = lambda d: torch.empty(2, device=d)  # noqa: E731
        for t in ((z, z.to("cuda:1")), (z, z, one("cuda:1"), one("cuda:0")), (z, z, one("cuda:1"), one("cuda:1"))):
            with pytest.raises(ValueError, match="device"):
                kv.PagedCache(*t)
        with pytest.raises(ValueError, match="device"):
            kv.Rotary(torch.empty(8, 64, device="cuda:1"), q_weight=torch.empty(64, device="cuda:0"))
        with pytest.raises(ValueError, match="device"):
            kv.Plan(*SHAPE, device="cuda:0", workspace=torch.empty(1 << 24, dtype=torch.uint8, device="cuda:1"))


def test_host_memory_is_another_type():
    """A host tensor is a TypeError also beside device tensors."""
    with FakeTensorMode():
        t, w = torch.empty(8, 64, device="cuda"), torch.empty(64, device="cuda")
        for args in (dict(table=t.cpu()), dict(table=t, q_weight=w.cpu()), dict(table=t.cpu(), k_weight=w)):
            with pytest.raises(TypeError):
                kv.Rotary(**args)
        z = torch.empty(5, 2, 16, 64, dtype=torch.float8_e4m3fn, device="cuda")
        s = torch.empty(2, device="cuda")
        for args in ((z, z.cpu()), (z, z, s, s.cpu()), (z, z, s.cpu(), s.cpu())):
            with pytest.raises(TypeError):
                kv.PagedCache(*args)
