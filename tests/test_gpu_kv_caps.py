"""Capped scores from the smallest cap to the largest, with bounds below a rounding of the weights."""
import pytest
import torch

from tests import kv4_reference as ref4
from tests import kv_reference as ref

pytestmark = pytest.mark.gpu
BF, FH = torch.bfloat16, torch.float16
FEW, MANY = [(200, 1), (33, 1), (0, 1), (70, 2)], [(200, 60), (33, 33), (5, 9), (130, 130)]


@pytest.fixture(autouse=True)
def _gpu(dev):
    yield


def _kv():
    from paper_2607_08565_amd import kv
    return kv


def check(c):
    """As kv4_reference.close_scores, with a cap's own share of a score's error: 12 units of 2^-24 of caps
    up to 64 (derived there); of larger ones, as far as the score is a quarter of the cap or more,
    which tanh(1/4) = 0.245 of it is, 12 / 0.245 = 49 units of the score, else below 8: the factor's two
    roundings, u's three and those of the series' last sum and product, which are small beside it."""
    out, lse = c.run()
    o, l, mag, big, _ = c.want()
    more = c.cap * 12 * ref.F32 if c.cap <= 64 else big * 49 * ref.F32
    if c.slopes is not None:  # (here at most 0.5 x 200)
        more = more + 100 * (c.D / 16 + 8) * ref.F32
    score = big * c.D * ref.F32 + more
    most = float(score.max())
    assert most < 2.0 ** -8
    ref4.close_scores(out, lse, (o, l, mag, big, torch.as_tensor(more).expand_as(big)), c.D, c.dtype)
    return out, lse


@pytest.mark.parametrize("cap", [2.0 ** -20, 0.3, 50.0, 63.9, 64.1, 100.0, 1000.0, 2.0 ** 15, 2.0 ** 18, 2.0 ** 20])
@pytest.mark.parametrize("lens", [FEW, MANY])
@pytest.mark.parametrize("D,dtype,pages", [(64, BF, "same"), (128, FH, "same"), (128, BF, "fp8"), (64, FH, "fp4"), (256, BF, "fp4")])
def test_caps_of_all_sizes(cap, lens, D, dtype, pages):
    check(ref4.Batch(_kv(), lens, 4, 2, D, dtype, pages, seed=81, cap=cap))


@pytest.mark.parametrize("lens", [FEW, MANY])
@pytest.mark.parametrize("dtype", [BF, FH])
@pytest.mark.parametrize("slopes", [False, True])
def test_scores_around_a_quarter_of_a_large_cap(lens, dtype, slopes):
    """Where one form of the capped score takes over from the other, and far beyond; pages that end inside 16 keys."""
    for sharp in (3.0, 12.0, 50.0):
        check(ref4.Batch(_kv(), lens, 4, 2, 64, dtype, "same", 7, seed=82, cap=70.0, sharp=sharp, slopes=slopes))


@pytest.mark.parametrize("lens", [FEW, MANY])
def test_a_large_cap_is_next_to_none(lens):
    """At a cap of 2^20 scores of at most 20 are off by 20 (20 / 2^20)^2 / 3 < 2^-28: attention without it."""
    c = ref4.Batch(_kv(), lens, 4, 2, 128, BF, "same", seed=83)
    plain, with_cap = c.run(), c.run(cap=2.0 ** 20)
    o, l, mag, big, more = c.want()
    assert float(big.max()) < 20
    ref4.close_scores(*with_cap, (o, l, mag, big, more * 0 + 20 * 49 * ref.F32), 128, BF)
    assert torch.equal(torch.isinf(plain[1]), torch.isinf(with_cap[1]))


@pytest.mark.parametrize("lens", [FEW, MANY])
@pytest.mark.parametrize("how", [{}, dict(cap=2.0 ** -20), dict(cap=50.0), dict(cap=1000.0), dict(slopes=True)])
@pytest.mark.parametrize("pages", ["same", "fp8"])
def test_the_largest_scale_of_a_score_of_zero(lens, how, pages):
    """A query of zeros has scores of zero whatever they are multiplied by, float32's largest number too."""
    c = ref4.Batch(_kv(), lens, 4, 2, 64, BF, pages, seed=84, **how)
    c.q = torch.zeros_like(c.q)
    want = c.want()
    if pages == "fp8":
        c.cache.k_scale.fill_(3e38)
    out, lse = c.run(scale=3.4e38)
    ref4.close_scores(out, lse, want, 64, BF)


def test_caps_that_float32_holds_as_zero_are_refused():
    from paper_2607_08565_amd.smetric import SmetricError
    c = ref4.Batch(_kv(), [(20, 1)], 4, 2, 64, BF, "same", seed=85)
    for cap in (1e-50, -1e-50, 5e-324):
        with pytest.raises(SmetricError):
            c.run(cap=cap)
    assert torch.equal(c.run(cap=-0.0)[0], c.run()[0])
