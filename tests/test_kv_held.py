"""Structures that the library is given by address stay whole as long as the one that points to them."""
import ctypes as C

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2607_08565_amd import kv


@pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")
def test_exponents_of_a_dropped_cache():
    """A 4-bit cache made for one call and dropped: its structure's address shows its exponents' strides still."""
    with FakeTensorMode():
        at = [kv.PagedCache.empty(5 + i, 2, 64, 16, kv._E2M1, device="cuda:0").ref for i in range(20)]
    other = [bytes(C.sizeof(kv._Exps)) for _ in range(1000)] + [bytearray(64) for _ in range(1000)]
    for i, a in enumerate(at):
        c = kv._Cache.from_address(a)
        e = kv._Exps.from_address(c.exps)
        # [page][head][k, v][token][group]
        assert c.n_pages == 5 + i and list(e.k_stride) == list(e.v_stride) == [128, 64, 2]
    assert len(other) == 2000


@pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")
def test_a_cache_holds_its_exponents():
    with FakeTensorMode():
        z = lambda t, *s: torch.empty(s, dtype=t, device="cuda:0")  # noqa: E731
        k, e = z(kv._E2M1, 5, 2, 16, 32), z(kv._E8M0, 5, 2, 16, 2)
        c = kv.PagedCache(k, k, k_exp=e, v_exp=e)
        assert c.c.held == (c.exps,) and c.c.exps == C.addressof(c.exps)
        assert kv.PagedCache.empty(5, 2, 64, device="cuda:0").c.held == ()
