"""Attention over 4-bit pages, and with capped or biased scores over pages of every type, against the
64-bit form on ragged batches."""
import math

import pytest
import torch

from tests import kv4_reference as ref4
from tests.test_gpu_kv_attend import CHUNKS, DECODE

pytestmark = pytest.mark.gpu
BF, FH = torch.bfloat16, torch.float16


@pytest.fixture(autouse=True)
def _gpu(dev):
    yield


def _kv():
    from paper_2607_08565_amd import kv
    return kv


def batch(*a, **k):
    return ref4.Batch(_kv(), *a, **k)


ALL = [(64, BF), (64, FH), (128, BF), (128, FH), (256, BF), (256, FH)]


@pytest.mark.parametrize("D,dtype", ALL)
@pytest.mark.parametrize("Hq,H", [(1, 1), (8, 1), (14, 2), (16, 1), (6, 2)])
def test_decode(D, dtype, Hq, H):
    batch(DECODE, Hq, H, D, dtype, seed=1).check()


@pytest.mark.parametrize("D,dtype", ALL)
@pytest.mark.parametrize("Hq,H", [(2, 2), (7, 1), (16, 1)])
def test_chunks(D, dtype, Hq, H):
    batch(CHUNKS, Hq, H, D, dtype, seed=2).check()


@pytest.mark.parametrize("page,order", [(16, "pthd"), (48, "phtd"), (128, "phtd"), (1, "phtd"), (5, "pthd"), (24, "phtd")])
@pytest.mark.parametrize("window", [0, 1, 20, 300])
def test_pages_and_windows(page, order, window):
    batch(DECODE, 8, 2, 128, BF, "fp4", page, order, window, seed=3).check()
    batch([(3, 3), (70, 2), (2, 3), (200, 1), (40, 4), (513, 4)], 8, 2, 64, FH, "fp4", page, order, window, seed=4).check()
    batch([(3, 3), (90, 40), (2, 3), (200, 1), (140, 77), (500, 33)], 8, 2, 128, BF, "fp4", page, order, window, seed=5).check()


@pytest.mark.parametrize("lens", [[(5000, 1)], [(9001, 4)], [(6000, 100)], [(4097, 1), (130, 1), (0, 1)], [(3000, 300), (50, 1)]])
@pytest.mark.parametrize("how", [{}, dict(cap=30.0), dict(slopes=True)])
@pytest.mark.parametrize("pages", ["fp4", "same"])
def test_long_requests_are_split(lens, how, pages):
    c = batch(lens, 8, 4, 128, BF, pages, seed=6, sharp=3.0, **how)
    out, lse = c.check()
    again, lse2 = c.run()
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("D,dtype", ALL)
@pytest.mark.parametrize("pages", ["same", "fp8", "fp4"])
@pytest.mark.parametrize("how", [dict(cap=5.0, sharp=6.0), dict(slopes=True), dict(cap=20.0, slopes=True, window=50, sharp=6.0)])
def test_scores(D, dtype, pages, how):
    for lens in (DECODE[:12] + [(300, 1)], CHUNKS):
        for page in (16, 7):
            batch(lens, 6, 2, D, dtype, pages, page, seed=7, **how).check()


@pytest.mark.parametrize("cap", [2.0 ** -20, 0.01, 1.0, 50.0, 2.0 ** 20])
@pytest.mark.parametrize("lens", [[(200, 1), (33, 1)], [(200, 60), (33, 33)]])
def test_caps_from_end_to_end(cap, lens):
    """Small caps make all scores alike, large ones leave them; scores far beyond a cap saturate at it."""
    batch(lens, 4, 2, 64, BF, "same", seed=8, cap=cap).check()
    c = batch(lens, 4, 2, 64, BF, "same", seed=8, cap=min(cap, 50.0), sharp=2000.0)
    c.check()


def test_no_cap_and_no_slopes_is_attention():
    for lens in (DECODE, CHUNKS):
        c = batch(lens, 4, 2, 128, BF, "same", seed=9)
        a, b = c.run(), c.run(cap=0.0, slopes=None)
        zeros = c.run(slopes=torch.zeros(4, device="cuda"))
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        ref4.close_scores(*zeros, c.want(), 128, BF)


@pytest.mark.parametrize("lens,Hq,H", [([(40, 4)], 2, 2), ([(40, 40)], 4, 1), ([(300, 200)], 4, 1), ([(530, 3)], 4, 4)])
@pytest.mark.parametrize("window", [0, 16])
@pytest.mark.parametrize("dtype,pages,how", [(BF, "fp4", {}), (FH, "fp4", {}), (FH, "fp4", dict(cap=10.0)), (BF, "same", dict(cap=10.0)),
                                             (FH, "same", dict(slopes=True)), (BF, "fp8", dict(cap=10.0, slopes=True))])
def test_what_a_row_does_not_see_changes_nothing(lens, Hq, H, window, dtype, pages, how):
    """The last two places hold NaN (4 bits: exponents of 255): only the last two tokens' rows change."""
    c = batch(lens, Hq, H, 64, dtype, pages, seed=10, window=window, **how)
    out, lse = c.check()
    L, n = lens[0]
    for place in (L - 2, L - 1) + ((0, 1) if window and L - n - window >= 1 else ()):
        at = (int(c.table[0, place // 16]), slice(None), place % 16)
        for x in ((c.cache.k_exp, c.cache.v_exp) if pages == "fp4" else (c.cache.k, c.cache.v)):
            x.view(torch.uint8)[at] = 255 if pages != "fp8" else 127  # (all bits: a NaN of 16 bits)
    got, lse2 = c.run()
    assert torch.equal(got[:n - 2], out[:n - 2]) and torch.equal(lse2[:n - 2], lse[:n - 2])
    assert bool(torch.isnan(got[n - 1]).all())


def test_visible_groups_that_are_not_numbers_come_through():
    """A value group of NaN reaches its 32 components of the rows that see it, and nothing else."""
    for lens in ([(50, 3)], [(50, 20)]):
        c = batch(lens, 4, 2, 128, BF, "fp4", seed=11)
        out, _ = c.run()
        c.cache.v_exp.view(torch.uint8)[int(c.table[0, 47 // 16]), 1, 47 % 16, 2] = 255
        got, lse = c.run()
        n = lens[0][1]
        assert bool(torch.isnan(got[n - 3:, 2:, 64:96]).all()) and bool(torch.isfinite(lse).all())
        got[n - 3:, 2:, 64:96] = out[n - 3:, 2:, 64:96] = 0
        assert torch.equal(got[:n - 3], out[:n - 3]) and bool(torch.isfinite(got).all())


@pytest.mark.parametrize("dtype", [BF, FH])
@pytest.mark.parametrize("new", [1, 40])
def test_extreme_exponents(dtype, new):
    """Groups at both ends of what the append enters, beside ordinary ones."""
    c = batch([(100, new)], 4, 2, 64, dtype, "fp4", seed=12)
    lo, hi = ref4.RANGE[dtype]
    small = 127 + lo
    for place, e in ((3, small), (50, small + 1), (70, small)):
        at = (int(c.table[0, place // 16]), slice(None), place % 16)
        for s, x in enumerate((c.cache.k_exp, c.cache.v_exp)):
            x.view(torch.uint8)[at] = e
            ce = ref4.quantise(c.kv[0][s][place], dtype)[0]
            c.kv[0][s][place] = ref4.values(ref4.unpack((c.cache.k, c.cache.v)[s].view(torch.uint8)[at].cpu()),
                                            torch.full((2, 2), e)) if ce is not None else None
    c.check()


def test_strides_and_other_lengths_of_slopes():
    for lens in ([(70, 1), (33, 1)], [(70, 50), (33, 9)]):
        c = batch(lens, 8, 2, 128, BF, "fp4", seed=13, cap=20.0, slopes=True)
        fused = torch.full((c.T, 12, 136), math.nan, dtype=BF, device="cuda")
        fused[:, :8, :128] = c.q.cuda()
        out = torch.zeros(8, c.T, 128, dtype=BF, device="cuda").transpose(0, 1)
        a, _ = c.run(q=fused[:, :8, :128], out=out)
        b, _ = c.run()
        assert a.data_ptr() == out.data_ptr() and torch.equal(a, b)
        with pytest.raises(ValueError):
            c.run(slopes=torch.zeros(2, device="cuda"))
        with pytest.raises(TypeError):
            c.run(slopes=torch.zeros(16, device="cuda")[::2])
        from paper_2607_08565_amd.smetric import SmetricError
        for cap in (-1.0, math.inf, math.nan, 1e-9, 1e9):
            with pytest.raises(SmetricError):
                c.run(cap=cap)


def test_a_step_together():
    """Append in 4 bits, attention with a cap and a bias, reading back: on a side stream, captured and
    replayed on new inputs and lengths, against the eager calls."""
    kv = _kv()
    H, Hq, D, P = 2, 8, 128, 16
    for new in ([1, 1, 1], [40, 1, 130]):
        T, g = sum(new), torch.Generator().manual_seed(14)
        lens = [500, 77, 1300]
        q_off = torch.tensor([0] + new).cumsum(0).cuda()
        kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        table = torch.arange(3 * 90, dtype=torch.int32, device="cuda").view(3, 90)
        make = lambda: kv.PagedCache.empty(270, H, D, P, ref4.F4)  # noqa: E731
        mine, other = make(), make()
        every = torch.tensor([0] + lens).cumsum(0).cuda()
        past = torch.randn(sum(lens), 2 * H, D, generator=g).to(BF).cuda()
        x = torch.randn(T, Hq + 2 * H, D, generator=g).to(BF).cuda()
        slopes = torch.linspace(0.01, 0.4, Hq, device="cuda")
        outs = [torch.empty(T, n, D, dtype=BF, device="cuda") for n in (Hq, H, H)]
        plan, lse = kv.Plan(3, T, Hq, H, D, max(new)), torch.empty(T, Hq, device="cuda")

        def step(c, plan, out, k, v, lse):
            plan.make(q_off, kv_len)
            kv.append(c, table, q_off, kv_len, x[:, Hq:Hq + H], x[:, Hq + H:])
            kv.attend(x[:, :Hq], c, table, plan, out=out, lse=lse, cap=30.0, slopes=slopes)
            kv.read(c, table, q_off, kv_len, k_out=k, v_out=v)

        def eager():
            for c in (mine, other):
                kv.append(c, table, every, torch.tensor(lens, dtype=torch.int32, device="cuda"), past[:, :H], past[:, H:])
            o = [torch.empty_like(t) for t in outs] + [torch.empty_like(lse)]
            step(other, kv.Plan(3, T, Hq, H, D, max(new)), *o)
            torch.cuda.synchronize()
            return o

        def same(o):
            torch.cuda.synchronize()
            for a, b in zip([*outs, lse], o):
                assert torch.equal(a, b)
            for n in ("k", "v", "k_exp", "v_exp"):
                a, b = (getattr(c, n).view(torch.uint8)[:180] for c in (mine, other))
                used = torch.zeros(180, dtype=torch.bool)
                used[:31], used[90:94] = True, True  # whole pages
                assert torch.equal(a[used.cuda()], b[used.cuda()])

        want = eager()
        ref_out = want[0].clone()
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            step(mine, plan, *outs, lse)
        same(want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step(mine, plan, *outs, lse)
        for i in range(4):
            x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(i)).to(BF))
            if i == 2:
                kv_len -= 3
            want = eager()
            graph.replay()
            same(want)
        assert not torch.equal(want[0], ref_out)
        # what was read back is what the attention saw
        keys = [mine_ for mine_ in (outs[1], outs[2])]
        c, e = ref4.quantise(x[:, Hq:Hq + H].double().cpu(), BF)
        assert torch.equal(keys[0].double().cpu(), ref4.values(c, e))
