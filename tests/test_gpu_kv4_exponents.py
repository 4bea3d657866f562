"""Attention over 4-bit groups at both ends of the exponents that the append enters, where they decide the output."""
import pytest
import torch

from tests import kv4_reference as ref4

pytestmark = pytest.mark.gpu
BF, FH = torch.bfloat16, torch.float16


@pytest.fixture(autouse=True)
def _gpu(dev):
    yield


def _kv():
    from paper_2607_08565_amd import kv
    return kv


def enter(c, side, places, code, e):
    """Codes [n, heads, dim] with exponents e at places of the first request, in its pages and for the reference."""
    for i, place in enumerate(places):
        at = (int(c.table[0, place // 16]), slice(None), place % 16)
        (c.cache.k, c.cache.v)[side].view(torch.uint8)[at] = ref4.pack(code[i]).cuda()
        (c.cache.k_exp, c.cache.v_exp)[side].view(torch.uint8)[at] = 127 + e
        c.kv[0][side][place] = ref4.values(code[i], torch.full((2, 2), 127 + e))


def codes(n, most, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(1, most + 1, (n, 2, 64), generator=g) + 8 * torch.randint(0, 2, (n, 2, 64), generator=g)


@pytest.mark.parametrize("dtype", [BF, FH])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("how", [{}, dict(cap=10.0), dict(cap=100.0), dict(slopes=True)])
def test_largest_values(dtype, new, how):
    """BF16: two tokens with up to 2^125, of which the sums hold a weight of 1 each (cap 10: 2^3.5 above a
    fixed maximum's, where the promised range ends at 2^100); F16 all codes, up to 6 x 2^13."""
    c = ref4.Batch(_kv(), [(100, new)], 4, 2, 64, dtype, "fp4", seed=12, sharp=1.0, **how)
    hi = 100 - 3 if dtype == BF and c.cap == 10.0 else ref4.RANGE[dtype][1]
    for place, e in ((3, hi), (5, hi - 1)):
        enter(c, 1, [place], codes(1, 2 if dtype == BF else 7, place), e)
    out, _ = c.check()
    assert float(out.float().abs().max()) > 2.0 ** (hi - 10)


@pytest.mark.parametrize("dtype", [BF, FH])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("how", [{}, dict(cap=10.0), dict(cap=100.0), dict(slopes=True)])
def test_largest_keys(dtype, new, how):
    """Queries so small that scores are of ordinary size: 64 products of 2^-122 and up to 2^125 (F16 2^-13, 6 x 2^13)."""
    c = ref4.Batch(_kv(), [(100, new)], 4, 2, 64, dtype, "fp4", seed=13, **how)
    hi = ref4.RANGE[dtype][1]
    places = [2, 30, 31, 47, 59]
    enter(c, 0, places[:3], codes(3, 2, 1), hi)
    enter(c, 0, places[3:], codes(2, 2, 2), hi - 1)
    c.q = (torch.sign(c.q.float()) * 2.0 ** (3 - hi if dtype == BF else -hi)).to(dtype)
    _, lse = c.check()
    zero = ref4.Batch(_kv(), [(100, new)], 4, 2, 64, dtype, "fp4", seed=13, **how)
    zero.q = c.q * 0
    # they are seen: five keys of 100 with scores of some 0.8 (F16) and more change lse by some 0.02, and
    # its bound is (5 + 4) 8 + 8 x 64 units of 2^-24, 3.5e-5
    assert float((lse - zero.run()[1]).abs().max()) > 1e-3


@pytest.mark.parametrize("dtype", [BF, FH])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("how", [{}, dict(cap=10.0), dict(cap=100.0), dict(slopes=True)])
def test_smallest_values(dtype, new, how):
    """All groups at the low end: what comes out is of their size, not zero.  (With a fixed maximum, cap 10,
    at the end of the promised range, 2^-100.)"""
    c = ref4.Batch(_kv(), [(100, new)], 4, 2, 64, dtype, "fp4", seed=14, sharp=1.0, **how)
    lo = -98 if dtype == BF and c.cap == 10.0 else ref4.RANGE[dtype][0]
    enter(c, 1, range(100), codes(100, 7, 3), lo)
    out, _ = c.check()
    assert float(out.float().abs().max()) > 2.0 ** lo and bool((out != 0).any(-1).all())
