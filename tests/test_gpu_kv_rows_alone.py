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
