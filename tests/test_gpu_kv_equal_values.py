"""A softmax's weights sum to one: where all the values that a row sees are the same number, that number
comes out, whatever the scores -- the weights of the products and those of their sum are the same ones."""
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


FEW, MANY = [(700, 1), (33, 1), (5, 2), (1, 1), (400, 1)], [(300, 300), (33, 33), (700, 90), (5, 9), (1, 1)]
SPLIT = [[(9000, 1)], [(5000, 60)]]


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype,pages", [(BF, "same"), (FH, "same"), (BF, "fp8"), (FH, "fp8"), (BF, "fp4"), (FH, "fp4")])
@pytest.mark.parametrize("how", [{}, dict(cap=5.0), dict(cap=50.0), dict(cap=60.0), dict(slopes=True), dict(cap=20.0, slopes=True)])
def test_equal_values_come_out_as_they_are(D, dtype, pages, how):
    """Each head and component has one of E2M1's numbers at every place, exact in every type.  Beside the
    weights, which cancel, out has the float32 sums' roundings: of n keys n / 16 in either sum, 2^-24 each,
    2 x 9000 / 16 x 2^-24 < 2^-13 at most, the quotient's and the joining's few.  Of a number that the type
    holds, half of a step is at least 2^-12 (F16), so the number itself is what out is rounded to."""
    for i, lens in enumerate([FEW, MANY, *SPLIT]):
        c = ref4.Batch(_kv(), lens, 6, 2, D, dtype, pages, seed=60 + i, sharp=4.0, **how)
        g = torch.Generator().manual_seed(i)
        code = torch.randint(1, 8, (2, D), generator=g) + 8 * torch.randint(0, 2, (2, D), generator=g)
        want = ref4.values(code, torch.full((2, D // 32), 127))
        v = c.cache.v
        if pages == "fp4":
            v.view(torch.uint8).copy_(ref4.pack(code).cuda()[:, None].expand(v.shape))
            c.cache.v_exp.view(torch.uint8).fill_(127)
        else:
            v.view(torch.uint8 if pages == "fp8" else torch.int16).copy_(
                want.to(v.dtype).view(torch.uint8 if pages == "fp8" else torch.int16).cuda()[:, None].expand(v.shape))
        if pages == "fp8":
            c.cache.v_scale.fill_(0.5)
            want = want / 2
        out, lse = c.run()
        sees = torch.isfinite(lse).cpu()
        assert int(sees.sum()) >= (c.T - 4) * 6
        rows = want.repeat_interleave(3, 0).expand(c.T, 6, D)
        got = out.double().cpu()
        assert torch.equal(got[sees], rows[sees]), float(((got - rows) / rows)[sees].abs().max())
        assert bool((got[~sees] == 0).all())


@pytest.mark.parametrize("new", [1, 20])
@pytest.mark.parametrize("dtype", [BF, FH])
@pytest.mark.parametrize("how", [{}, dict(cap=4.0), dict(cap=60.0)])
def test_weights_that_are_all_rounded_alike(new, dtype, how):
    """Keys whose weights are all nearly half a step above what the type holds, beside one with the largest:
    rounded they are all off to one side, and so has to be their sum."""
    L = 300
    c = ref4.Batch(_kv(), [(L, new)], 2, 1, 64, dtype, "same", seed=70, **how)
    c.q = torch.zeros_like(c.q)
    c.q[..., :2] = 8.0  # with the scale of 1/8 a score is the sum of the key's first two components
    weight = torch.tensor(0.5 * (1 + 0.49 * torch.finfo(dtype).eps), dtype=torch.float64).log()
    k = torch.zeros(L, 1, 64).to(dtype)
    k[1:, 0, 0] = weight.to(dtype)
    k[1:, 0, 1] = (weight - weight.to(dtype).double()).to(dtype)
    for p in range(-(-L // 16)):
        n = min(16, L - 16 * p)
        c.cache.k[int(c.table[0, p]), :, :n] = k[16 * p:16 * p + n].transpose(0, 1).cuda()
    c.cache.v.fill_(64.0)
    c.kv = [[k.double(), torch.full((L, 1, 64), 64.0).double()]]
    out, _ = c.check()
    assert bool((out == 64.0).all())
