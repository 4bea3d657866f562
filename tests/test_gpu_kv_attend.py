"""Attention over the paged cache against the 64-bit form, on ragged batches."""
import math

import pytest
import torch

from tests import kv_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(dev):
    yield


def _kv():
    from paper_2607_08565_amd import kv
    return kv


class Case:
    """A batch: lens = (kv_len, new tokens) per request; what no request's place holds is NaN."""

    def __init__(self, lens, Hq, H, D, dtype, fp8=False, page=16, order="phtd", window=0, seed=0, sharp=1.5, max_new=None):
        g = torch.Generator().manual_seed(seed * 1000 + D + page + Hq)
        self.lens, self.Hq, self.H, self.D, self.dtype, self.page, self.window = lens, Hq, H, D, dtype, page, window
        R, T = len(lens), sum(n for _, n in lens)
        self.T = T
        need = [-(-L // page) for L, _ in lens]
        n_pages = sum(need) + 1
        perm = torch.randperm(n_pages, generator=g).int()
        width = max(need + [1])
        table = torch.full((R, width), 1 << 30, dtype=torch.int32)
        self.scales = [0.01 + 0.02 * torch.rand(H, generator=g) for _ in "kv"] if fp8 else [None, None]
        ct = ref.FP8 if fp8 else dtype
        pages = [torch.full((n_pages, H, page, D), math.nan).to(ct) for _ in "kv"]
        self.kv = []
        at = 0
        for i, (L, _) in enumerate(lens):
            table[i, :need[i]] = perm[at:at + need[i]]
            at += need[i]
            mine = []
            for s in range(2):
                x = ((60 if fp8 else 1) * torch.randn(need[i] * page, H, D, generator=g)).to(ct)
                x.view(torch.uint8 if fp8 else torch.int16)[L:] = pages[0].view(torch.uint8 if fp8 else torch.int16)[0, 0, 0, 0]
                b = x.view(torch.uint8 if fp8 else torch.int16).view(need[i], page, H, D).transpose(1, 2)
                pages[s].view(torch.uint8 if fp8 else torch.int16)[table[i, :need[i]].long()] = b
                y = x[:L].float().double()
                mine.append(y * self.scales[s].double()[:, None] if fp8 else y)
            self.kv.append(mine)
        def dev(x):
            x = x.cuda()
            return x if order == "phtd" else x.transpose(1, 2).contiguous().transpose(1, 2)
        self.cache = _kv().PagedCache(dev(pages[0]), dev(pages[1]), *[None if s is None else s.cuda() for s in self.scales])
        self.table = table.cuda()
        self.q = (sharp * torch.randn(T, Hq, D, generator=g)).to(dtype)
        self.q_off = torch.tensor([0] + [n for _, n in lens]).cumsum(0).cuda()
        self.kv_len = torch.tensor([L for L, _ in lens], dtype=torch.int32, device="cuda")
        self.max_new = max_new or max([n for _, n in lens] + [1])
        self.scale = 1 / math.sqrt(D)

    def plan(self):
        return _kv().Plan(len(self.lens), self.T, self.Hq, self.H, self.D, self.max_new, self.window)

    def run(self, plan=None, q=None, out=None, status=None):
        plan = (plan or self.plan()).make(self.q_off, self.kv_len)
        lse = torch.full((self.T, self.Hq), 7.0, device="cuda")
        out = _kv().attend(self.q.cuda() if q is None else q, self.cache, self.table, plan, lse=lse, out=out, status=status)
        return out, lse

    def want(self):
        parts, a = [], 0
        for (L, n), (k, v) in zip(self.lens, self.kv):
            parts.append(ref.attend(self.q[a:a + n].double(), k, v, self.H, self.scale, self.window, L, n))
            a += n
        return [torch.cat([p[i] for p in parts]) for i in range(4)]

    def check(self, **how):
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        out, lse = self.run(status=st, **how)
        ref.close_attend(out, lse, self.want(), self.D, self.dtype)
        assert st.item() == 0
        return out, lse


BF, FH = torch.bfloat16, torch.float16
# one token each: a lone one, page and step ends, padding, a request without new tokens, splits
DECODE = [(1, 1), (15, 1), (16, 1), (17, 1), (0, 1), (50, 0), (31, 1), (32, 1), (33, 1), (63, 1), (64, 1), (65, 1),
          (127, 1), (129, 1), (1000, 1)]
HEADS = [(1, 1), (4, 4), (8, 1), (14, 2), (16, 1), (6, 2)]


@pytest.mark.parametrize("D,dtype,fp8", [(64, BF, False), (128, BF, False), (256, BF, False), (64, FH, True), (128, FH, False),
                                         (128, BF, True), (256, FH, True)])
@pytest.mark.parametrize("Hq,H", HEADS)
def test_decode(D, dtype, fp8, Hq, H):
    Case(DECODE, Hq, H, D, dtype, fp8, seed=1).check()


@pytest.mark.parametrize("page,order", [(16, "pthd"), (48, "phtd"), (128, "phtd"), (1, "phtd"), (5, "pthd"), (24, "phtd")])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("window", [0, 1, 20, 300])
def test_pages_and_windows(page, order, fp8, window):
    Case(DECODE, 8, 2, 128, BF, fp8, page, order, window, seed=2).check()
    Case([(3, 3), (70, 2), (2, 3), (200, 1), (40, 4), (513, 4)], 8, 2, 64, FH, fp8, page, order, window, seed=3).check()
    Case([(3, 3), (90, 40), (2, 3), (200, 1), (140, 77), (500, 33)], 8, 2, 128, BF, fp8, page, order, window, seed=4).check()


@pytest.mark.parametrize("window", [(1 << 24) - 1, 1 << 24, (1 << 31) - 1])
@pytest.mark.parametrize("max_new", [1, 1000])
def test_windows_longer_than_any_request(window, max_new):
    """Also for tokens whose place is negative."""
    lens = [(2, 5), (0, 3), (3, 40), (70, 9)]
    a = Case(lens, 4, 2, 64, BF, seed=16, window=window, max_new=max_new)
    out, lse = a.check()
    b, lse2 = Case(lens, 4, 2, 64, BF, seed=16, max_new=max_new).run()
    assert torch.equal(out, b) and torch.equal(lse, lse2)


# chunks: whole prompts, ends inside tiles and steps, fewer places than tokens, single tokens among them
CHUNKS = [(1, 1), (32, 32), (33, 33), (64, 64), (100, 65), (0, 1), (20, 30), (300, 1), (700, 40), (90, 0), (129, 128), (257, 19)]


@pytest.mark.parametrize("D,dtype,fp8", [(64, BF, False), (128, BF, False), (256, BF, False), (64, FH, True), (128, FH, False),
                                         (128, BF, True), (256, FH, True), (128, FH, True), (256, BF, True)])
@pytest.mark.parametrize("Hq,H", [(2, 2), (6, 2), (7, 1), (16, 1)])
def test_chunks(D, dtype, fp8, Hq, H):
    Case(CHUNKS, Hq, H, D, dtype, fp8, seed=5).check()


@pytest.mark.parametrize("Hq,H,max_new", [(4, 4, 1), (64, 2, 1), (4, 1, 1000)])
def test_shape_of_the_pieces_is_free(Hq, H, max_new):
    """max_new chooses the kernel; either is right for any request."""
    Case(CHUNKS, Hq, H, 128, BF, seed=6, max_new=max_new).check()


@pytest.mark.parametrize("lens", [[(5000, 1)], [(9001, 4)], [(6000, 100)], [(4097, 1), (130, 1), (0, 1)], [(3000, 300), (50, 1)]])
@pytest.mark.parametrize("fp8", [False, True])
def test_long_requests_are_split(lens, fp8):
    c = Case(lens, 8, 4, 128, BF, fp8, seed=7, sharp=3.0)
    out, lse = c.check()
    again, lse2 = c.run()
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("R,most", [(600, 1), (2100, 1), (600, 9), (2100, 5)])
@pytest.mark.parametrize("window", [0, 7])
def test_many_requests(R, most, window):
    """More requests and tiles than one pass of the plan holds, some without tokens, some longer than the rest."""
    lens = [((i * 37) % 61 + (900 if i % 97 == 5 else 0), 0 if i % 13 == 4 else i % most + 1) for i in range(R)]
    Case(lens, 2, 1, 64, BF, seed=17, window=window).check()
    if most > 1:
        Case(lens, 2, 1, 64, BF, seed=17, window=window, max_new=1000).check()


def test_large_scores():
    """Scores of hundreds, maxima that keep growing along the keys and ones that come first."""
    for sign in (1, -1):
        for lens in ([(700, 1)], [(700, 60)]):
            c = Case(lens, 4, 4, 64, BF, seed=8, sharp=1.0)
            L = 700
            ramp = sign * torch.linspace(-60, 60, L)
            k = ramp[:, None, None] * torch.ones(L, 4, 64)
            c.q = torch.ones_like(c.q) * 2
            kb = k.to(BF)
            for p in range(-(-L // 16)):
                n = min(16, L - 16 * p)
                c.cache.k[c.table[0, p].long(), :, :n] = kb[16 * p:16 * p + n].transpose(0, 1).cuda()
            c.kv[0][0] = kb.double()
            c.check()


@pytest.mark.parametrize("lens,Hq,H", [([(40, 4)], 2, 2), ([(40, 40)], 4, 1), ([(300, 200)], 4, 1), ([(530, 3)], 4, 4)])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("window", [0, 16])
@pytest.mark.parametrize("dtype", [BF, FH])
def test_what_a_row_does_not_see_changes_nothing(lens, Hq, H, bad, window, dtype):
    """The last two keys and values are not finite: only the last two tokens' rows are touched;
    with a window, neither is what lies before it."""
    c = Case(lens, Hq, H, 64, dtype, seed=9, window=window)
    out, lse = c.check()
    L = lens[0][0]
    for place in (L - 2, L - 1) + ((0, 1) if window else ()):
        if window and place < 2 and place > L - lens[0][1] - window:
            continue  # some row sees it
        for pages in (c.cache.k, c.cache.v):
            pages[c.table[0, place // 16].long(), :, place % 16] = bad
    got, lse2 = c.run()
    n = lens[0][1] - 2
    assert torch.equal(got[:n], out[:n]) or _near(got[:n], out[:n], dtype)
    assert torch.equal(lse2[:n], lse[:n])
    assert not bool(torch.isfinite(got[n + 1]).all())


def _near(a, b, dtype):
    # where a step holds values that are not finite the weights are not rounded: two roundings apart
    return bool(((a.double() - b.double()).abs() <= 4 * ref.UNIT[dtype] * (b.double().abs() + 1)).all())


def test_visible_values_that_are_not_finite_come_through():
    c = Case([(50, 1), (50, 20)], 4, 2, 64, BF, seed=10)
    c.cache.v[c.table[0, 1].long(), 0, 3, 5] = math.inf
    c.cache.v[c.table[1, 0].long(), 1, 3, 7] = math.nan
    out, lse = c.run()
    assert bool((out[0, :2, 5] == math.inf).all()) and bool(torch.isnan(out[1:, 2:, 7]).all())
    out[0, :2, 5] = 0
    out[1:, 2:, 7] = 0
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())


def test_strides():
    """Queries as a slice of a fused product, the output's heads before its tokens."""
    for lens in ([(70, 1), (33, 1)], [(70, 50), (33, 9)]):
        c = Case(lens, 8, 2, 128, BF, seed=11)
        fused = torch.full((c.T, 12, 136), math.nan, dtype=BF, device="cuda")
        fused[:, :8, :128] = c.q.cuda()
        out = torch.zeros(8, c.T, 128, dtype=BF, device="cuda").transpose(0, 1)
        a, _ = c.run(q=fused[:, :8, :128], out=out)
        b, _ = c.run()
        assert a.data_ptr() == out.data_ptr() and torch.equal(a, b)


@pytest.mark.parametrize("n", [1, 40])
def test_offsets_beyond_32_bits(n):
    """Pages at the far end of a cache of more than 2^32 bytes a side."""
    kv = _kv()
    H, P, D = 4, 16, 128
    n_pages = (1 << 31) // (H * P * D) + 64  # elements beyond 2^31, bytes beyond 2^32
    k, v = (torch.empty(n_pages, H, P, D, dtype=BF, device="cuda") for _ in "kv")
    c = Case([(100, n)], 8, H, D, BF, seed=12)
    used = c.table[0].long()
    far = torch.arange(n_pages - 7, n_pages, device="cuda")
    k[far], v[far] = c.cache.k[used], c.cache.v[used]
    c.cache, c.table = kv.PagedCache(k, v), far[None].int()
    c.check()
    new = torch.ones(1, H, D, dtype=BF, device="cuda")
    kv.append(c.cache, c.table, torch.tensor([0, 1], device="cuda"), torch.tensor([101], dtype=torch.int32, device="cuda"), new, new)
    assert bool((k[-1, :, 100 % 16] == 1).all()) and bool((v[-1, :, 100 % 16] == 1).all())


def test_bad_batches():
    c = Case([(40, 2), (50, 1)], 4, 2, 64, BF, seed=13)
    kv = _kv()
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = c.q.cuda()
    for q_off, kv_len in ((torch.tensor([0, 2, 4]), i32(40, 50)), (torch.tensor([0, 3, 2]), i32(40, 50)),
                          (torch.tensor([1, 2, 3]), i32(40, 50)), (torch.tensor([0, 2, 3]), i32(-1, 50)),
                          (torch.tensor([0, 2, 3]), i32(40, (1 << 24) + 1))):
        plan = c.plan()
        st.zero_()
        plan.make(q_off.cuda(), kv_len, status=st)
        assert st.item() == -1
        st.zero_()
        lse = torch.zeros(3, 4, device="cuda")
        out = kv.attend(q, c.cache, c.table, plan, lse=lse, status=st)
        assert st.item() == -1 and bool((out == 0).all()) and bool((lse == -math.inf).all())
    # a request longer than its table's row: its rows alone
    plan = c.plan().make(c.q_off, i32(65, 50))
    st.zero_()
    out = kv.attend(q, c.cache, c.table, plan, status=st)
    good, _ = c.run()
    assert st.item() == -1 and bool((out[:2] == 0).all()) and torch.equal(out[2], good[2])
    # a page outside the cache: the other request's rows are what they were
    bad = c.table.clone()
    bad[0, 1] = -1
    st.zero_()
    out = kv.attend(q, c.cache, bad, c.plan().make(c.q_off, c.kv_len), status=st)
    assert st.item() == -1 and torch.equal(out[2], good[2])
    # a plan made for another window
    plan = c.plan().make(c.q_off, c.kv_len)
    plan.window = 5
    st.zero_()
    assert bool((kv.attend(q, c.cache, c.table, plan, status=st) == 0).all()) and st.item() == -1


def test_refusals():
    from paper_2607_08565_amd.smetric import SmetricError
    kv = _kv()
    c = Case([(40, 2), (50, 1)], 4, 2, 64, BF, seed=14)
    plan, q = c.plan().make(c.q_off, c.kv_len), c.q.cuda()
    for scale in (0.0, -1.0, math.inf, math.nan):
        with pytest.raises(SmetricError):
            kv.attend(q, c.cache, c.table, plan, scale=scale)
    for args in ((2, 3, 5, 2, 64, 1), (2, 3, 4, 2, 80, 1), (2, 3, 4, 0, 64, 1), (2, 3, 4, 2, 64, 0), (-1, 3, 4, 2, 64, 1),
                 (0, 3, 4, 2, 64, 1), (1, 1 << 30, 8, 1, 64, 1)):
        with pytest.raises(SmetricError):
            kv.Plan(*args)
    with pytest.raises(SmetricError):
        kv.Plan(2, 3, 4, 2, 64, 1, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(SmetricError):
        kv.Plan(2, 3, 4, 2, 64, 1, window=-1).make(c.q_off, c.kv_len)
    with pytest.raises(SmetricError):
        kv.attend(q.half(), c.cache, c.table, plan)
    with pytest.raises(ValueError):
        kv.attend(q[:2], c.cache, c.table, plan)
    with pytest.raises(ValueError):
        kv.attend(q, c.cache, c.table[:1], plan)
    with pytest.raises(ValueError):
        kv.attend(q, c.cache, c.table, c.plan())  # not made
    with pytest.raises(ValueError):
        kv.attend(q, c.cache, c.table, plan, lse=torch.zeros(3, device="cuda"))
    short = c.plan().make(c.q_off, c.kv_len)
    short.ws_bytes -= 1
    with pytest.raises(SmetricError):
        kv.attend(q, c.cache, c.table, short)
    # nothing to do
    e = kv.Plan(0, 0, 4, 2, 64, 1).make(c.q_off[:1], c.kv_len[:0])
    assert kv.attend(q[:0], c.cache, c.table[:0], e).shape[0] == 0


def test_side_stream_and_graph():
    """A step on another stream, and the same captured and replayed on new inputs."""
    kv = _kv()
    for lens in ([(500, 1), (77, 1), (3000, 1)], [(500, 100), (77, 1), (3000, 20)]):
        c = Case(lens, 8, 2, 128, BF, seed=15)
        want, want_lse = c.check()
        s = torch.cuda.Stream()
        plan, q, out = c.plan(), c.q.cuda(), torch.empty(c.T, 8, 128, dtype=BF, device="cuda")
        lse = torch.empty(c.T, 8, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            plan.make(c.q_off, c.kv_len)
            kv.attend(q, c.cache, c.table, plan, out=out, lse=lse)
        s.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            plan.make(c.q_off, c.kv_len)
            kv.attend(q, c.cache, c.table, plan, out=out, lse=lse)
        for k in range(4):
            c.q = torch.randn(c.q.shape, generator=torch.Generator().manual_seed(k)).to(BF)
            q.copy_(c.q)
            if k == 2:  # other lengths through the same graph
                c.kv_len -= 1
            g.replay()
            torch.cuda.synchronize()
            eager, eager_lse = c.run()
            torch.cuda.synchronize()
            assert torch.equal(out, eager) and torch.equal(lse, eager_lse)
