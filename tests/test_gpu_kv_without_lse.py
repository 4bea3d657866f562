"""Attention that is not asked for lse gives the same output, bit for bit, as where it is."""
import pytest
import torch

from tests import kv4_reference as ref4

pytestmark = pytest.mark.gpu
BF, FH = torch.bfloat16, torch.float16
FEW, MANY = [(300, 1), (33, 1), (0, 1), (2, 2)], [(150, 150), (33, 33), (300, 90), (5, 9), (1, 1)]


@pytest.fixture(autouse=True)
def _gpu(dev):
    yield


def _kv():
    from paper_2607_08565_amd import kv
    return kv


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF, FH])
@pytest.mark.parametrize("pages", ["same", "fp8", "fp4"])
@pytest.mark.parametrize("page", [16, 7])
@pytest.mark.parametrize("how", [{}, dict(slopes=True), dict(cap=20.0), dict(cap=20.0, slopes=True), dict(cap=100.0), dict(window=40)])
def test_the_same_output(D, dtype, pages, page, how):
    kv = _kv()
    for lens in (FEW, MANY, [(2500, 1)], [(2000, 60)]):
        c = ref4.Batch(kv, lens, 6, 2, D, dtype, pages, page, seed=101, **how)
        want, _ = c.run()
        plan = c.plan().make(c.q_off, c.kv_len)
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = torch.full_like(want, 7.0)
        kv.attend(c.q.cuda(), c.cache, c.table, plan, out=out, cap=c.cap, slopes=None if c.slopes is None else c.slopes.cuda(),
                  status=st)
        assert torch.equal(out, want) and st.item() == 0


@pytest.mark.parametrize("lens", [FEW, MANY])
@pytest.mark.parametrize("how", [{}, dict(cap=20.0), dict(slopes=True)])
def test_unseen_and_visible_nan(lens, how):
    """A value of NaN at the last place reaches the last token's rows alone, also without lse."""
    kv, c = _kv(), ref4.Batch(_kv(), lens, 4, 2, 64, BF, "same", seed=102, **how)
    L, n = lens[0]
    run = lambda: kv.attend(c.q.cuda(), c.cache, c.table, c.plan().make(c.q_off, c.kv_len), cap=c.cap,  # noqa: E731
                            slopes=None if c.slopes is None else c.slopes.cuda())
    before = run()
    c.cache.v[int(c.table[0, (L - 1) // 16]), :, (L - 1) % 16] = float("nan")
    after = run()
    assert bool(torch.isnan(after[n - 1]).all())
    after[n - 1] = before[n - 1]
    assert torch.equal(after, before)


def test_captured_and_replayed():
    kv = _kv()
    for lens, how in ((FEW, {}), (MANY, dict(cap=20.0)), ([(4000, 60)], dict(slopes=True))):
        c = ref4.Batch(kv, lens, 4, 2, 128, BF, "fp4", seed=103, **how)
        q, slopes = c.q.cuda(), None if c.slopes is None else c.slopes.cuda()
        plan, out = c.plan(), torch.empty(c.T, 4, 128, dtype=BF, device="cuda")
        step = lambda: kv.attend(q, c.cache, c.table, plan.make(c.q_off, c.kv_len), out=out, cap=c.cap, slopes=slopes)  # noqa: E731
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            step()
        for i in range(3):
            q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(i)).to(BF))
            want, _ = c.run(q=q)
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
