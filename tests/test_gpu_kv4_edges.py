"""Reading back rows of many heads; capped and biased scores at the ends of their factors' ranges."""
import math

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


def batch(*a, **k):
    return ref4.Batch(_kv(), *a, **k)


@pytest.mark.parametrize("H,D", [(32, 128), (32, 256), (33, 64), (31, 64), (21, 128), (16, 128), (127, 64)])
@pytest.mark.parametrize("pages", ["same", "fp8", "fp4"])
def test_read_rows_of_many_heads(H, D, pages):
    """Tokens of fewer and of more pieces than a workgroup has threads, and of a number that does not divide them."""
    b = batch([(9, 9), (20, 3), (0, 2), (37, 36)], H, H, D, BF, pages, seed=31)
    k, v = _kv().read(b.cache, b.table, b.q_off, b.kv_len, b.T, BF)
    a = 0
    for (L, n), mine in zip(b.lens, b.kv):
        for s, out in enumerate((k, v)):
            got, pad = out[a:a + n].double().cpu(), max(0, n - L)
            assert bool((got[:pad] == 0).all())
            y = mine[s][L - (n - pad):]
            ref.close(got[pad:], y, ref.F32 * y.abs(), BF)
        a += n


@pytest.mark.parametrize("scale", [1e-12, 1e-22, 1e-30, 1e-38])
@pytest.mark.parametrize("dtype", [BF, FH])
@pytest.mark.parametrize("lens", [FEW, MANY])
def test_a_bias_beside_next_to_no_score(scale, dtype, lens):
    for pages in ("same", "fp4"):
        c = batch(lens, 4, 2, 64, dtype, pages, seed=32, slopes=True)
        c.scale = scale
        c.check(scale=scale)


@pytest.mark.parametrize("k_scale", [0.0, -0.02, 1e-30, 0.03])
@pytest.mark.parametrize("how", [dict(cap=10.0), dict(cap=60.0), dict(slopes=True), dict(cap=10.0, slopes=True)])
@pytest.mark.parametrize("dtype", [BF, FH])
@pytest.mark.parametrize("lens", [FEW, MANY])
def test_key_scales_of_any_kind(k_scale, how, dtype, lens):
    """8-bit pages' key scales of zero, below zero and next to nothing give what the formula gives."""
    c = batch(lens, 4, 2, 64, dtype, "fp8", seed=33, **how)
    old = c.cache.k_scale.double().cpu()
    c.cache.k_scale.fill_(k_scale)
    new = c.cache.k_scale.double().cpu()
    for mine in c.kv:
        mine[0] = mine[0] / old[:, None] * new[:, None]
    c.check()


@pytest.mark.parametrize("cap", [29.0, 30.0, 50.4, 50.7, 200.0])
@pytest.mark.parametrize("dtype,pages", [(BF, "same"), (BF, "fp4"), (FH, "same")])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_scores_at_both_ends_of_a_cap(cap, dtype, pages, D):
    """Rows all of whose scores are at -cap, at +cap, or at both: a prompt's first token sees one key only."""
    c = batch([(70, 70), (3, 3)], 4, 2, D, dtype, pages, seed=34, cap=cap, sharp=1.0)
    c.q = c.q * 0
    c.q[..., 0] = 3e4 * (1 - 2 * (torch.arange(4) % 2)).to(dtype)
    out, lse = c.check()
    assert bool(torch.isfinite(out).all()) and float(lse.abs().max()) <= cap + math.log(80)


@pytest.mark.parametrize("how", [{}, dict(cap=20.0), dict(slopes=True), dict(cap=20.0, slopes=True)])
@pytest.mark.parametrize("lens", [FEW, MANY])
def test_queries_that_are_not_finite(how, lens):
    """A query of NaN makes its own row NaN and no other one different."""
    c = batch(lens, 4, 2, 64, BF, "fp4", seed=35, **how)
    out, lse = c.check()
    c.q[0, 1, 5] = math.nan
    got, lse2 = c.run()
    assert bool(torch.isnan(got[0, 1]).all())
    got[0, 1], lse2[0, 1] = out[0, 1], lse[0, 1]
    assert torch.equal(got, out) and torch.equal(lse2, lse)


@pytest.mark.parametrize("side", [0, 1])
def test_read_one_side(side):
    """Through the C entry point one side may be left out: it is not written, the other is what both give."""
    import ctypes as C
    import struct
    from paper_2607_08565_amd import smetric as S
    b = batch([(40, 40), (7, 9)], 2, 2, 64, BF, "fp4", seed=36)
    both = _kv().read(b.cache, b.table, b.q_off, b.kv_len, b.T, BF)
    out = torch.full((b.T, 2, 64), 5.0, dtype=BF, device="cuda")
    heads = struct.pack("Pqq", out.data_ptr(), 128, 64)
    where = struct.pack("PqiiPPq", b.table.data_ptr(), b.table.stride(0), b.table.shape[1], 2, b.q_off.data_ptr(),
                        b.kv_len.data_ptr(), b.T)
    stream = C.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert S._lib.smetric_kv_read(0, b.cache.ref, where, *((heads, None) if side == 0 else (None, heads)), None, stream) == S.OK
    assert torch.equal(out, both[side])


@pytest.mark.parametrize("pages", ["same", "fp8", "fp4"])
@pytest.mark.parametrize("how", [{}, dict(cap=20.0), dict(slopes=True)])
@pytest.mark.parametrize("lens", [[(40, 2), (50, 1)], [(40, 40), (50, 33)]])
def test_bad_batches(pages, how, lens):
    """A page outside the cache, a request longer than its row, a plan of other lengths: status, no access
    out of bounds, and the other request's rows as they were."""
    kv, c = _kv(), batch(lens, 4, 2, 64, BF, pages, seed=37, **how)
    slopes = None if c.slopes is None else c.slopes.cuda()
    n, q, (good, good_lse) = lens[0][1], c.q.cuda(), c.run()
    st = torch.zeros(1, dtype=torch.int32, device="cuda")

    def run(table, kv_len, q_off=c.q_off):
        st.zero_()
        lse = torch.zeros(c.T, 4, device="cuda")
        plan = c.plan().make(q_off, kv_len)
        out = kv.attend(q, c.cache, table, plan, lse=lse, status=st, cap=c.cap, slopes=slopes)
        assert st.item() == -1
        return out, lse
    bad = c.table.clone()
    bad[0, 1] = -1
    out, lse = run(bad, c.kv_len)
    assert torch.equal(out[n:], good[n:]) and torch.equal(lse[n:], good_lse[n:])
    out, lse = run(c.table, torch.tensor([65, 50], dtype=torch.int32, device="cuda"))
    assert bool((out[:n] == 0).all()) and bool((lse[:n] == -math.inf).all()) and torch.equal(out[n:], good[n:])
    out, lse = run(c.table, torch.tensor([-1, 50], dtype=torch.int32, device="cuda"))
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


def test_streams_at_once():
    """Steps with caches, plans and streams of their own, enqueued together, give what they give alone."""
    kv, many = _kv(), []
    for i, (lens, how) in enumerate(((FEW, dict(cap=20.0)), (MANY, dict(slopes=True)), (MANY, dict(cap=30.0)), (FEW, {}))):
        c = batch(lens, 8, 2, 128, BF, "fp4", seed=40 + i, **how)
        many.append((c, c.run(), kv.read(c.cache, c.table, c.q_off, c.kv_len, c.T), torch.cuda.Stream(), c.plan(), c.q.cuda(),
                     torch.empty(c.T, 8, 128, dtype=BF, device="cuda"), torch.empty(c.T, 8, device="cuda"),
                     None if c.slopes is None else c.slopes.cuda()))
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for c, _, _, s, plan, q, out, lse, slopes in many:
            with torch.cuda.stream(s):
                plan.make(c.q_off, c.kv_len)
                kv.attend(q, c.cache, c.table, plan, out=out, lse=lse, cap=c.cap, slopes=slopes)
                got.append(kv.read(c.cache, c.table, c.q_off, c.kv_len, c.T))
        torch.cuda.synchronize()
        for (c, want, rows, *_, out, lse, _), back in zip(many, got):
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
            assert torch.equal(back[0], rows[0]) and torch.equal(back[1], rows[1])
