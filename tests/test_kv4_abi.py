"""4-bit pages, reading back and other scores on the host: what is refused (no GPU work is launched), and
the plain forms that the GPU tests compare with."""
import ctypes as C
import math
import struct

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2607_08565_amd import kv, smetric as S
from paper_2607_08565_amd.smetric import SmetricError
from tests import kv4_reference as ref4
from tests.test_kv_abi import FAKE, batch, heads

strides = lambda *x: (C.c_int64 * 3)(*x)  # noqa: E731
F4, E8 = ref4.F4, ref4.E8


class Cache4(kv._Cache):
    """A cache and, kept with it, its exponents; names with exp_ are theirs."""

    def __init__(self, **how):
        super().__init__(FAKE, FAKE, 4, strides(2048, 1024, 64), strides(2048, 1024, 64), 16, 2, 64, 3, None, None)
        self.kept = kv._Exps(FAKE, FAKE, strides(64, 32, 2), strides(64, 32, 2))
        self.exps = C.addressof(self.kept)
        for k, v in how.items():
            setattr(self.kept if k.startswith("exp_") else self, k.replace("exp_", ""), v)


cache4 = Cache4
BAD = (dict(exps=None), dict(exp_k=None), dict(exp_v=None), dict(exp_k=FAKE + 1), dict(exp_v=FAKE + 1),
       dict(exp_k_stride=strides(64, 32, 1)), dict(exp_v_stride=strides(64, 31, 2)), dict(exp_k_stride=strides(-64, 32, 2)),
       dict(exp_v_stride=strides(64, 32, 1 << 24)),
       dict(k_stride=strides(2048, 1024, 48)), dict(v_stride=strides(2048, 1040, 64)), dict(v=FAKE + 8), dict(head_dim=96),
       dict(head_dim=256, exp_k_stride=strides(64, 32, 4)), dict(dtype=4))


def test_append_and_read_refusals():
    f = S._lib.smetric_kv_append

    def append(c, b=batch()):
        return f(0, C.addressof(c), b, None, None, 0, None, None, heads(), heads(), None, None)
    assert append(cache4(), batch(n_tokens=0)) == S.OK
    for how in BAD:
        assert append(cache4(**how)) == S.EINVAL, how
    g = S._lib.smetric_kv_read

    def read(c=cache4(), dtype=0, b=batch(), k=heads(), v=heads()):
        return g(dtype, C.addressof(c), b, k, v, None, None)
    assert read(b=batch(n_tokens=0)) == S.OK and read(k=None, v=None) == S.OK
    for how in BAD:
        assert read(cache4(**how)) == S.EINVAL, how
    for how in (dict(dtype=2), dict(dtype=3), dict(c=cache4(dtype=1)), dict(b=batch(table=0)), dict(b=batch(n_req=0)),
                dict(b=batch(n_tokens=-1)), dict(b=batch(n_tokens=1 << 31)), dict(k=heads(data=FAKE + 8)),
                dict(v=heads(token=4)), dict(k=None, v=heads(data=0))):
        assert read(**how) == S.EINVAL, how


def test_scores_refusals():
    a, b = C.c_uint64(), C.c_uint64()
    S._lib.smetric_attend_plan_bytes(2, 3, 4, 2, 64, 1, C.byref(a), C.byref(b))

    def call(scores, c=cache4(), dtype=0, bt=batch(n_tokens=0), scale=0.125, ws=b.value):
        return S._lib.smetric_attend_scores(dtype, C.addressof(c), bt, 4, heads(), heads(), None, scale, scores, 1, 0,
                                            FAKE, a.value, FAKE, ws, None, None)
    s = lambda cap, slopes=0: struct.pack("fxxxxP", cap, slopes)  # noqa: E731
    for ok in (s(0.0), s(30.0), s(2.0 ** -20), s(2.0 ** 20), s(0.0, FAKE), s(50.0, FAKE + 4)):
        assert call(ok) == S.OK
    for bad in (None, s(-1.0), s(math.inf), s(math.nan), s(2.0 ** -21), s(2.0 ** 21), s(0.0, FAKE + 2)):
        assert call(bad) == S.EINVAL
    full = batch()
    for how in (dict(scale=0.0), dict(scale=math.nan), dict(dtype=3), dict(c=cache4(exps=None)), dict(c=cache4(exp_v=FAKE + 1))):
        assert call(s(30.0), **dict(dict(bt=full), **how)) == S.EINVAL, how
    assert call(s(30.0), bt=full, ws=b.value - 1) == S.EWORKSPACE


@pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")
def test_binding_refusals():
    with FakeTensorMode():
        z = lambda *s, t=torch.uint8, d="cuda:0": torch.empty(s, dtype=t, device=d)  # noqa: E731
        k, e = z(5, 2, 16, 32, t=F4), z(5, 2, 16, 2, t=E8)
        c = kv.PagedCache(k, k, k_exp=e, v_exp=e)
        assert c.head_dim == 64 and list(c.c.k_stride) == [2048, 1024, 64] and list(c.exps.v_stride) == [64, 32, 2]
        assert kv.PagedCache.empty(5, 2, 128, dtype=F4, device="cuda:0").k_exp.shape == (5, 2, 16, 4)
        b = z(5, 2, 16, 64, t=torch.bfloat16)
        for args in (dict(k=k, v=k), dict(k=k, v=k, k_exp=e), dict(k=b, v=b, k_exp=e, v_exp=e), dict(k=k, v=k, k_exp=e, v_exp=e[:4]),
                     dict(k=k, v=k, k_exp=z(5, 2, 16, 4, t=E8), v_exp=e), dict(k=k, v=k, k_exp=z(5, 2, 16, 4, t=E8)[..., ::2], v_exp=e),
                     dict(k=k, v=k, k_exp=e, v_exp=e, k_scale=z(2, t=torch.float32), v_scale=z(2, t=torch.float32))):
            with pytest.raises(ValueError):
                kv.PagedCache(**args)
        for args in (dict(k_exp=e.view(torch.uint8), v_exp=e), dict(k_exp=e, v_exp=e.cpu()), dict(k_exp="x", v_exp=e)):
            with pytest.raises(TypeError):
                kv.PagedCache(k, k, **args)
        if not torch.cuda.is_available():
            with pytest.raises(ValueError, match="device"):
                kv.PagedCache(k, k, k_exp=e, v_exp=z(5, 2, 16, 2, t=E8, d="cuda:1"))
        i32 = lambda *s: z(*s, t=torch.int32)  # noqa: E731
        where = (c, i32(2, 4), z(3, t=torch.int64), i32(2))
        bf = lambda *s, t=torch.bfloat16: z(*s, t=t)  # noqa: E731
        with pytest.raises(ValueError):
            kv.read(*where)
        with pytest.raises(ValueError):
            kv.read(*where, k_out=bf(3, 2, 64), v_out=bf(2, 2, 64))
        with pytest.raises(ValueError):
            kv.read(*where, k_out=bf(3, 2, 32))
        with pytest.raises(ValueError):
            kv.read(c, i32(3, 4), *where[2:], n_tokens=3)
        with pytest.raises(TypeError):
            kv.read(*where, n_tokens=3, dtype=torch.float32)
        with pytest.raises(TypeError):
            kv.read(*where, k_out=bf(3, 2, 64), v_out=bf(3, 2, 64, t=torch.float16))
        plan = kv.Plan(2, 3, 4, 2, 64, 1, device="cuda:0")
        plan.q_off, plan.kv_len = where[2], where[3]
        q, f32 = bf(3, 4, 64), lambda *s: z(*s, t=torch.float32)  # noqa: E731
        with pytest.raises(ValueError):
            kv.attend(q, c, where[1], plan, slopes=f32(2))
        with pytest.raises(TypeError):
            kv.attend(q, c, where[1], plan, slopes=bf(4))
        with pytest.raises(TypeError):
            kv.attend(q, c, where[1], plan, cap="x")
        if not torch.cuda.is_available():
            with pytest.raises(ValueError, match="device"):
                kv.attend(q, c, where[1], plan, slopes=z(4, t=torch.float32, d="cuda:1"))


def test_binding_refuses_caps():
    """Through the binding a bad cap is an error before anything is enqueued (no tokens: nothing would be)."""
    with FakeTensorMode():
        e = lambda t, *s: torch.empty(s, dtype=t, device="cuda:0")  # noqa: E731
        c = kv.PagedCache.empty(5, 2, 64, dtype=F4, device="cuda:0")
        plan = kv.Plan(0, 0, 4, 2, 64, 1, device="cuda:0")
        plan.q_off, plan.kv_len = e(torch.int64, 1), e(torch.int32, 0)
        if torch.cuda.is_available():
            pytest.skip("stand-ins have no memory to hand on")
        for cap in (-1.0, math.inf, math.nan, 1e9):
            with pytest.raises((SmetricError, RuntimeError)):
                kv.attend(e(torch.bfloat16, 0, 4, 64), c, e(torch.int32, 0, 4), plan, cap=cap)


def test_addresses_of_a_call_stay_good():
    """A structure made for one call and dropped is still what its address shows, after much else was made."""
    at = [C.addressof(kv._Cache(FAKE + 16 * i, FAKE, 7, strides(1, 2, 3), strides(4, 5, 6), 16, 2, 64, 0, None, None)) for i in range(20)]
    at.append(C.addressof(kv._Rotary(FAKE, FAKE, FAKE, 9, 64, 0, 1e-6)))
    other = [bytes(112) for _ in range(1000)] + [bytearray(104) for _ in range(1000)]
    for i, a in enumerate(at[:20]):
        c = kv._Cache.from_address(a)
        assert (c.k, c.v, c.n_pages, list(c.v_stride), c.head_dim) == (FAKE + 16 * i, FAKE, 7, [4, 5, 6], 64)
    assert kv._Rotary.from_address(at[20]).n_pos == 9 and len(other) == 2000


def test_plain_form_of_the_codes():
    """The reference against the levels' own table: every midpoint goes to the even code, k is smallest."""
    lv = ref4.LEVELS
    mid = (lv[1:] + lv[:-1]) / 2
    assert ref4.codes(mid).tolist() == [0, 2, 2, 4, 4, 6, 6] and ref4.codes(lv).tolist() == list(range(8))
    assert ref4.codes(-lv).tolist() == [8, 9, 10, 11, 12, 13, 14, 15] and ref4.codes(torch.tensor([6.9, 100.0]).double()).tolist() == [7, 7]
    x = torch.zeros(4, 32).double()
    x[:, 3] = torch.tensor([7.0, 7.000001, 3.5, 0.0])
    assert ref4.exponents(x, torch.bfloat16).tolist() == [0, 1, -1, -125]
    x[:, 3] = torch.tensor([7e30, 65504.0, 2.0 ** -24, 7 * 2.0 ** 13])
    assert ref4.exponents(x, torch.float16).tolist() == [13, 13, -23, 13]
    c, e = ref4.quantise(torch.randn(5, 64).double(), torch.bfloat16)
    assert torch.equal(ref4.unpack(ref4.pack(c)), c) and e.shape == (5, 2)
    # no component is further away than half of the largest step
    g = torch.Generator().manual_seed(1)
    x = torch.randn(2000, 32, generator=g).double() * 2.0 ** torch.randint(-20, 20, (2000, 1), generator=g).double()
    c, e = ref4.quantise(x, torch.bfloat16)
    assert bool(((ref4.values(c, e) - x).abs() <= 2.0 ** (e.double() - 127)).all())
