"""The paged cache's entry points on the host: sizes and refusals (no GPU work is launched)."""
import ctypes as C
import struct

import pytest

from paper_2607_08565_amd import kv, smetric as S

FAKE = 1 << 20  # an aligned address that nothing reads: every call below returns first


def heads(data=FAKE, token=256, head=64):
    return struct.pack("Pqq", data, token, head)


def cache(**how):
    c = kv._Cache(FAKE, FAKE, 4, (C.c_int64 * 3)(2048, 1024, 64), (C.c_int64 * 3)(2048, 1024, 64), 16, 2, 64, 0, None, None)
    for k, v in how.items():
        setattr(c, k, v)
    return c


def rotary(**how):
    r = kv._Rotary(None, None, FAKE, 8, 64, 0, 1e-6)
    for k, v in how.items():
        setattr(r, k, v)
    return r


def batch(table=FAKE, stride=4, pages=4, n_req=2, q_off=FAKE, kv_len=FAKE, n_tokens=3):
    return struct.pack("PqiiPPq", table, stride, pages, n_req, q_off, kv_len, n_tokens)


def test_plan_sizes():
    a, b = C.c_uint64(), C.c_uint64()
    f = lambda *x: S._lib.smetric_attend_plan_bytes(*x, C.byref(a), C.byref(b))  # noqa: E731
    assert f(1, 1, 32, 4, 128, 1) == S.OK and a.value % 256 == 0 and 0 < b.value < 1 << 26
    few = a.value, b.value
    assert f(1, 4096, 32, 4, 128, 4096) == S.OK and a.value > few[0] and b.value > few[1]
    assert f(0, 0, 32, 4, 128, 1) == S.OK
    for bad in ((-1, 1, 32, 4, 128, 1), (1, -1, 32, 4, 128, 1), (0, 1, 32, 4, 128, 1), (1, 1, 30, 4, 128, 1),
                (1, 1, 2, 4, 128, 1), (1, 1, 32, 0, 128, 1), (1, 1, 32, 4, 96, 1), (1, 1, 32, 4, 128, 0),
                (1, 1 << 28, 32, 4, 128, 1), (1, 1, 65540, 4, 128, 1)):
        assert f(*bad) == S.EINVAL, bad
    assert S._lib.smetric_attend_plan_bytes(1, 1, 32, 4, 128, 1, None, C.byref(b)) == S.EINVAL


def test_rotate_refusals():
    def call(dtype=0, dim=64, n=2, r=None, pos=FAKE, n_q=2, q=heads(), q_out=heads(), n_kv=1, k=heads(), k_out=heads()):
        return S._lib.smetric_qk_rotate(dtype, dim, n, C.addressof(r or rotary()), pos, n_q, q, q_out, n_kv, k, k_out,
                                        None, None)
    assert call(n=0) == S.OK and call(n_q=0, n_kv=0) == S.OK
    for how in (dict(dtype=2), dict(dtype=-1), dict(dim=96), dict(n=-1), dict(n_q=-1), dict(n_kv=70000), dict(pos=None),
                dict(q=None), dict(q_out=heads(data=None or 0)), dict(k=heads(data=FAKE + 8)), dict(k_out=heads(token=252)),
                dict(q=heads(head=60)), dict(r=rotary(rot_dim=24)), dict(r=rotary(rot_dim=128)), dict(r=rotary(rot_dim=-16)),
                dict(r=rotary(table=None)), dict(r=rotary(table=FAKE + 4)), dict(r=rotary(n_pos=0)),
                dict(r=rotary(eps=-1.0)), dict(r=rotary(eps=float("nan"))), dict(r=rotary(q_weight=FAKE + 2))):
        assert call(**how) == S.EINVAL, how
    assert S._lib.smetric_qk_rotate(0, 64, 2, None, FAKE, 2, heads(), heads(), 0, None, None, None, None) == S.EINVAL


def test_append_refusals():
    def call(dtype=0, c=None, b=batch(), r=None, n_q=0, q=None, q_out=None, k=heads(), v=heads()):
        return S._lib.smetric_kv_append(dtype, C.addressof(c or cache()), b, None if r is None else C.addressof(r), None,
                                        n_q, q, q_out, k, v, None, None)
    assert call(b=batch(n_tokens=0)) == S.OK and call(b=batch(n_req=0, n_tokens=0, table=0, q_off=0, kv_len=0)) == S.OK
    strides = lambda *x: (C.c_int64 * 3)(*x)  # noqa: E731
    for how in (dict(dtype=1), dict(dtype=2), dict(c=cache(k=None)), dict(c=cache(v=FAKE + 8)), dict(c=cache(n_pages=0)),
                dict(c=cache(n_pages=1 << 31)), dict(c=cache(page_size=0)), dict(c=cache(page_size=65537)),
                dict(c=cache(n_kv_heads=0)), dict(c=cache(head_dim=80)), dict(c=cache(dtype=3)),
                dict(c=cache(k_scale=FAKE)), dict(c=cache(k_stride=strides(2048, 1024, 60))),
                dict(c=cache(v_stride=strides(2048, -1024, 64))), dict(c=cache(v_stride=strides(2048, 1024, 1 << 24))),
                dict(c=cache(dtype=2, k_stride=strides(2048, 1024, 72))), dict(b=batch(stride=3)), dict(b=batch(table=0)),
                dict(b=batch(q_off=0)), dict(b=batch(kv_len=0)), dict(b=batch(n_req=0)), dict(b=batch(n_tokens=-1)),
                dict(b=batch(n_req=-1)), dict(k=None), dict(v=heads(data=FAKE + 2)), dict(n_q=2), dict(n_q=-1),
                dict(r=rotary(rot_dim=128))):
        assert call(**how) == S.EINVAL, how


def test_attend_refusals():
    a, b = C.c_uint64(), C.c_uint64()
    S._lib.smetric_attend_plan_bytes(2, 3, 4, 2, 64, 1, C.byref(a), C.byref(b))

    def call(dtype=0, c=None, bt=batch(), n_q=4, q=heads(), out=heads(), scale=0.125, max_new=1, window=0, plan=FAKE,
             plan_bytes=a.value, ws=FAKE, ws_bytes=b.value):
        return S._lib.smetric_attend(dtype, C.addressof(c or cache()), bt, n_q, q, out, None, scale, max_new, window, plan,
                                     plan_bytes, ws, ws_bytes, None, None)
    assert call(bt=batch(n_tokens=0)) == S.OK
    for how in (dict(dtype=1), dict(n_q=3), dict(n_q=1), dict(q=None), dict(out=heads(token=4)), dict(scale=0.0),
                dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(max_new=0), dict(window=-1),
                dict(plan=None), dict(plan=FAKE + 64), dict(ws=FAKE + 64), dict(bt=batch(n_tokens=1 << 30))):
        assert call(**how) == S.EINVAL, how
    for how in (dict(plan_bytes=a.value - 1), dict(ws_bytes=b.value - 1), dict(ws=None)):
        assert call(**how) == S.EWORKSPACE, how

    def make(q_off=FAKE, kv_len=FAKE, n_req=2, n_tokens=3, max_new=1, window=0, plan=FAKE, plan_bytes=a.value):
        return S._lib.smetric_attend_plan(q_off, kv_len, n_req, n_tokens, 4, 2, 64, max_new, window, plan, plan_bytes, None,
                                          None)
    for how in (dict(q_off=None), dict(kv_len=None), dict(n_req=0), dict(max_new=0), dict(window=-1), dict(plan=None),
                dict(plan=FAKE + 128)):
        assert make(**how) == S.EINVAL, how
    assert make(plan_bytes=a.value - 1) == S.EWORKSPACE


@pytest.mark.parametrize("bad", [None, "x"])
def test_binding_wants_tensors(bad):
    with pytest.raises(TypeError):
        kv.PagedCache(bad, bad)
    with pytest.raises(TypeError):
        kv.qk_rotate(bad, bad, None)
