"""Attention where one key outweighs the others by far and has a value of zero: what the others add
is the output, whose bound is relative to it."""
import math

import pytest
import torch

from tests import kv_reference as ref
from tests.test_gpu_kv_attend import BF, FH, Case, _kv

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(dev):
    yield


# 16 bits of F16 hold weights of 29 powers of two in full; chunks spend 8 of them on a maximum that lags
@pytest.mark.parametrize("dtype", [BF, FH])
@pytest.mark.parametrize("new,below", [(1, 16), (1, 20), (1, 24), (1, 29), (20, 16), (20, 20), (20, 21)])
def test_small_weights_of_many_keys(dtype, new, below):
    """All keys but the first have the same weight, 2^-below the first's and nearly half a step of
    8 bits more: rounded to fewer bits than the type's they would all be off alike.  So many
    requests that none is split: a part's weights are relative to its own maximum."""
    L, R = 400, 300
    c = Case([(L, new)] * R, 2, 1, 64, dtype, seed=24)
    c.q = torch.zeros_like(c.q)
    c.q[..., :2] = 8.0  # with the scale of 1/8 a score is the sum of the key's first two components
    score = torch.tensor(math.log(2.0 ** -below * (1 + 0.49 * 2.0 ** -8)), dtype=torch.float64)
    k, v = torch.zeros(L, 1, 64).to(dtype), torch.full((L, 1, 64), 2.0 ** 13).to(dtype)
    k[1:, 0, 0] = score.to(dtype)
    k[1:, 0, 1] = (score - score.to(dtype).double()).to(dtype)
    v[1::2] = 2.0 ** 14
    v[0] = 0.0
    for p in range(L // 16):
        at = c.table[:, p].long()
        c.cache.k[at], c.cache.v[at] = (x[16 * p:16 * p + 16].transpose(0, 1).cuda() for x in (k, v))
    plan, lse = c.plan().make(c.q_off, c.kv_len), torch.empty(c.T, 2, device="cuda")
    out = _kv().attend(c.q.cuda(), c.cache, c.table, plan, scale=c.scale, lse=lse)
    want = ref.attend(c.q[:new].double(), k.double(), v.double(), 1, c.scale, 0, L, new)
    ref.close_attend(out, lse, [torch.cat([x] * R) for x in want], 64, dtype)
