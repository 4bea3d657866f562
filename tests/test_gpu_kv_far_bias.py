"""A bias by distance over long contexts, of either sign: with slopes below zero the keys that count most
are the farthest, whose bias is the largest, and the others' differences from it are what weights them."""

import pytest
import torch

from tests import kv4_reference as ref4
from tests import kv_reference as ref

pytestmark = pytest.mark.gpu
BF, FH = torch.bfloat16, torch.float16


@pytest.fixture(autouse=True)
def _gpu(dev):
    yield


def _kv():
    from paper_2607_08565_amd import kv
    return kv


@pytest.mark.parametrize("slopes", [(-0.5, 0.5), (-0.03, -2.0), (0.01, -2.0 ** -9)])
@pytest.mark.parametrize("how", [dict(cap=0.0), dict(cap=20.0), dict(cap=70.0)])
@pytest.mark.parametrize("D,dtype,pages,new,window", [(256, FH, "same", 1, 0), (256, FH, "same", 9, 0), (256, BF, "fp4", 9, 0),
                                                      (64, FH, "fp4", 2, 30000), (128, FH, "same", 12, 30000), (128, FH, "fp8", 9, 0)])
def test_far_keys_with_a_bias(slopes, how, D, dtype, pages, new, window):
    """Scores are off by dim units of 2^-24 of the products' sum, caps by 49 of the score (12 of caps up to 64), and
    (dim / 16 + 8) of the bias less the row's largest; the output by the weights' mean of that, twice (its
    numerator and its denominator), and a rounding of the weights; lse by that mean, and four float32
    roundings of its own size (the bias taken off, its factor, the sum and the last product), twice as many allowed."""
    L = 40000
    c = ref4.Batch(_kv(), [(L, new)], 2, 1, D, dtype, pages, seed=91, sharp=1.0, window=window, slopes=True, **how)
    c.slopes = torch.tensor(slopes)
    out, lse = c.run()
    k, v = (x[:, 0] for x in c.kv[0])
    for i in range(new):
        place = L - new + i
        lo = max(0, place - window + 1) if window else 0
        j = torch.arange(lo, place + 1)
        for h in range(2):
            q = c.q[i, h].double()
            s = c.scale * (k[lo:place + 1] @ q)
            off = c.scale * (k[lo:place + 1].abs() @ q.abs()) * ref.F32 * D
            if c.cap:
                off = off + ref.F32 * (c.cap * 12 if c.cap <= 64 else 49 * s.abs())
                s = c.cap * torch.tanh(s / c.cap)
            bias = c.slopes[h].double() * (j - place)
            s, off = s + bias, off + (bias.max() - bias) * (D / 16 + 8) * ref.F32
            want = torch.logsumexp(s, 0)
            p = torch.exp(s - want)
            vv = v[lo:place + 1]
            mean = p @ off + 2.0 ** -17  # (and what the weights' sums round)
            assert float(mean) < 2.0 ** -10
            size = p @ vv.abs()
            # weights rounded to the type, divided by their own sum: 1.01 of a unit of |v| and of |out|
            slack = ((p * off) @ vv.abs()) + mean * size + ref.UNIT[dtype] * 1.01 * (size + (p @ vv).abs())
            ref.close(out[i, h], p @ vv, slack, dtype)
            assert abs(float(lse[i, h]) - float(want)) <= float(mean) + (abs(float(want)) + 4) * 8 * ref.F32
    assert bool(torch.isfinite(out).all())
