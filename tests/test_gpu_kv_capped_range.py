"""Capped scores of BF16 chunks, weighted without a running maximum: values at both ends of the range that
is promised for them, where all of a row's scores are at either end of the cap."""
import math

import pytest
import torch

from tests import kv4_reference as ref4

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(autouse=True)
def _gpu(dev):
    yield


def _kv():
    from paper_2607_08565_amd import kv
    return kv


@pytest.mark.parametrize("cap", [1.0, 5.0, 20.0, 30.0, 50.0, 50.4])
@pytest.mark.parametrize("end", [-1, 1])
@pytest.mark.parametrize("D,pages", [(64, "same"), (128, "same"), (256, "same"), (64, "fp4")])
def test_values_at_the_ends_of_their_range(cap, end, D, pages):
    """Values of 1/2 to 6 times a power of two, as far from 1 as the range allows: 2^(115 - cap log2(e)) less
    what 6 and the sums take (they are of some 70 keys, 2^6.2, at both sides).  A first token sees one key."""
    x = 115 - 1.443 * cap
    e = math.floor(x) - 3 if end > 0 else -math.floor(x) + 2
    lens = [(70, 70), (3, 3), (60, 20)]
    c = ref4.Batch(_kv(), lens, 4, 2, D, BF, pages, seed=95, sharp=1.0, cap=cap)
    g = torch.Generator().manual_seed(D)
    c.q = c.q * 0
    c.q[..., 0] = 3e4 * (1 - 2 * (torch.arange(4) % 2)).to(BF)  # (keys of either sign: rows with scores at one end, the other, both)
    code = torch.randint(1, 8, (80, 2, D), generator=g) + 8 * torch.randint(0, 2, (80, 2, D), generator=g)
    v = ref4.values(code, torch.full((80, 2, D // 32), 127 + e))
    assert float(v.abs().max()) < 2.0 ** x and float(v.abs().min()) > 2.0 ** -x
    for i, (L, _) in enumerate(lens):
        for p in range(0, L, 16):
            n, at = min(16, L - p), int(c.table[i, p // 16])
            if pages == "fp4":
                c.cache.v.view(torch.uint8)[at, :, :n] = ref4.pack(code[p:p + n]).transpose(0, 1).cuda()
                c.cache.v_exp.view(torch.uint8)[at, :, :n] = 127 + e
            else:
                c.cache.v[at, :, :n] = v[p:p + n].to(BF).transpose(0, 1).cuda()
        c.kv[i][1] = v[:L]
    out, lse = c.check()
    sees = torch.isfinite(lse)
    assert bool(sees.all()) and bool(torch.isfinite(out).all()) and bool((out != 0).any(-1).all())
