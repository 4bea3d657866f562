"""Attention over 8-bit pages with scales of any sign, of zero, and without scales."""
import math

import pytest
import torch

from tests.test_gpu_kv_attend import BF, CHUNKS, DECODE, FH, Case, _kv

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(dev):
    yield


def rescale(c, k_scale, v_scale):
    """The same pages with other scales (None: a stored x stands for itself)."""
    new = [torch.ones(c.H) if s is None else torch.tensor(s) for s in (k_scale, v_scale)]
    c.kv = [[x / old.double()[:, None] * s.double()[:, None] for x, old, s in zip(mine, c.scales, new)] for mine in c.kv]
    c.scales = new
    given = [] if k_scale is None else [s.cuda() for s in new]
    c.cache = _kv().PagedCache(c.cache.k, c.cache.v, *given)
    return c


@pytest.mark.parametrize("lens", [CHUNKS, DECODE])
@pytest.mark.parametrize("D,dtype", [(64, FH), (128, BF), (256, BF)])
@pytest.mark.parametrize("window", [0, 50])
@pytest.mark.parametrize("k_scale,v_scale", [((0.0, -0.02, 0.015), (0.02, 0.01, -0.03)), ((-0.01, -0.0, 1e-30), (0.0, -1.5, 2.0)),
                                             ((-0.3, 0.25, 0.0), (1.0, 1.0, 1.0))])
def test_any_scale(lens, D, dtype, window, k_scale, v_scale):
    rescale(Case(lens, 6, 3, D, dtype, True, window=window, seed=21), k_scale, v_scale).check()


@pytest.mark.parametrize("lens", [CHUNKS, DECODE])
def test_without_scales(lens):
    """A stored x stands for itself; queries small enough for scores of tens."""
    rescale(Case(lens, 6, 3, 128, BF, True, seed=22, sharp=0.03), None, None).check()


@pytest.mark.parametrize("lens", [[(40, 40), (3, 5)], [(3, 5), (0, 1), (300, 2)]])
@pytest.mark.parametrize("max_new", [1, 1000])
def test_scales_that_are_not_numbers(lens, max_new):
    """A head whose keys or values stand for NaN has NaN where something is seen, zeros elsewhere; the
    other heads are what they were.  A zero scale times a query that is not finite is NaN."""
    c = Case(lens, 3, 3, 64, BF, True, seed=23, max_new=max_new)
    want, want_lse = c.check()
    place = torch.cat([torch.arange(L - n, L) for L, n in lens])
    sees = (place >= 0).cuda()
    for side in range(2):
        scales = [s.clone() for s in c.scales]
        scales[side][1] = math.nan
        c.cache = _kv().PagedCache(c.cache.k, c.cache.v, *[s.cuda() for s in scales])
        out, lse = c.run()
        assert torch.equal(out[:, ::2], want[:, ::2]) and torch.equal(lse[:, ::2], want_lse[:, ::2])
        assert bool(torch.isnan(out[sees, 1]).all()) and bool((out[~sees, 1] == 0).all())
        assert bool((lse[~sees, 1] == -math.inf).all())
        assert torch.equal(lse, want_lse) if side else bool(torch.isnan(lse[sees, 1]).all())
    ks = c.scales[0].clone()
    ks[1] = 0.0
    c.cache = _kv().PagedCache(c.cache.k, c.cache.v, ks.cuda(), c.scales[1].cuda())
    c.q[-1, 1, 7] = math.inf
    out, lse = c.run()
    assert bool(torch.isnan(out[-1, 1]).all()) and bool(torch.isfinite(out[:-1]).all())
