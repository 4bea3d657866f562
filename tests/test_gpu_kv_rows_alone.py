"""Attention's rows that share a tile: what one of them does not see changes not a bit of its output."""
import math

import pytest
import torch

from tests.test_gpu_kv_attend import BF, FH, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(dev):
    yield


def put(c, request, place, k=None, v=None):
    """The key and the value of a place, in the cache: [kv heads, head_dim], or one number."""
    page, slot = int(c.table[request, place // c.page]), place % c.page
    for pages, x in ((c.cache.k, k), (c.cache.v, v)):
        if x is not None:
            word = pages[page, :, slot]
            x = torch.as_tensor(x, dtype=torch.float32).expand(word.shape)
            pages[page, :, slot] = x.to(pages.dtype).cuda()


# (cached, new tokens), heads: a wavefront's rows in one tile, several tiles, pieces of cut tiles, few rows
SHAPES = [([(96, 32)], 1, 1), ([(200, 33)], 4, 2), ([(700, 80)], 4, 1), ([(5000, 40)], 4, 4), ([(150, 5), (90, 30)], 2, 2)]


@pytest.mark.parametrize("lens,Hq,H", SHAPES)
@pytest.mark.parametrize("D,dtype,fp8", [(64, BF, False), (128, FH, False), (128, BF, True), (256, BF, False)])
@pytest.mark.parametrize("max_new", [None, 1])
def test_a_large_finite_score_of_a_later_token(lens, Hq, H, D, dtype, fp8, max_new):
    """The last token's own key gives it a score of thousands: the other rows' running maxima, which grow a
    little in the same step, are what they were."""
    c = Case(lens, Hq, H, D, dtype, fp8, seed=20, max_new=max_new)
    out, lse = c.check()
    L, n = lens[-1]
    q = c.q[-1].float().view(H, Hq // H, D)[:, 0]
    put(c, len(lens) - 1, L - 1, k=q.sign() * 448)
    got, lse2 = c.run()
    assert torch.equal(got[:-1], out[:-1]) and torch.equal(lse2[:-1], lse[:-1])
    assert bool((lse2[-1] != lse[-1]).any())


ODD = [([(40, 4)], 2, 2), ([(40, 40)], 4, 1), ([(300, 200)], 4, 1), ([(530, 3)], 4, 4), ([(2000, 33)], 2, 2), ([(90, 30)], 6, 3)]


@pytest.mark.parametrize("lens,Hq,H", ODD)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("window", [0, 16])
@pytest.mark.parametrize("D,dtype,fp8", [(64, BF, False), (64, FH, False), (128, BF, False), (256, FH, False), (128, FH, True)])
def test_what_is_not_finite_and_not_seen(lens, Hq, H, bad, window, D, dtype, fp8):
    """The last two places' keys and values, and with a window those before it, are not finite: the
    rows that do not see them are what they were, to the bit."""
    c = Case(lens, Hq, H, D, dtype, fp8, seed=25, window=window)
    out, lse = c.check()
    L, n = lens[0]
    before = (0, 1) if window and L - n - window >= 1 else ()
    for place in (L - 2, L - 1) + before:
        put(c, 0, place, math.nan if fp8 else bad, math.nan if fp8 else bad)
    got, lse2 = c.run()
    assert torch.equal(got[:n - 2], out[:n - 2]) and torch.equal(lse2[:n - 2], lse[:n - 2])
    assert not bool(torch.isfinite(got[n - 2:]).any())


@pytest.mark.parametrize("lens,Hq,H", ODD)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("D,dtype,fp8", [(64, BF, False), (128, FH, False), (256, BF, False), (128, BF, True)])
def test_components_that_are_not_finite(lens, Hq, H, bad, D, dtype, fp8):
    """Some components of the last but one place's value are not finite: they come through in the rows
    that see them and change nothing else."""
    c = Case(lens, Hq, H, D, dtype, fp8, seed=26)
    L, n = lens[0]
    bad, at = math.nan if fp8 else bad, [3, D // 2, D - 1]
    page, slot = int(c.table[0, (L - 2) // 16]), (L - 2) % 16
    for i in at:
        c.cache.v[page, :, slot, i] = 0.0
    out, lse = c.run()
    for i in at:
        c.cache.v[page, :, slot, i] = bad
    got, lse2 = c.run()
    assert torch.equal(lse2, lse) and torch.equal(got[:n - 2], out[:n - 2])
    rest = [i for i in range(D) if i not in at]
    assert torch.equal(got[n - 2:, :, rest], out[n - 2:, :, rest])
    seen = got[n - 2:, :, at]
    # a weight may be too small for the product with infinity to be infinite: it is NaN then
    assert not bool(torch.isfinite(seen).any()) and (math.isnan(bad) or bool(((seen == bad) | torch.isnan(seen)).all()))
    assert math.isnan(bad) or bool((seen == bad).float().mean() > 0.9)
