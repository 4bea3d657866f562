"""Keys and values quantised into 4-bit pages, and pages of every type read back, against 64-bit forms."""
import math

import pytest
import torch

from tests import kv4_reference as ref4
from tests import kv_reference as ref
from tests.test_gpu_kv_append import LENS, rotary

pytestmark = pytest.mark.gpu
BF, FH = torch.bfloat16, torch.float16
F4, E8, U8 = ref4.F4, ref4.E8, torch.uint8


@pytest.fixture(autouse=True)
def _gpu(dev):
    yield


def _kv():
    from paper_2607_08565_amd import kv
    return kv


i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
off = lambda *a: torch.tensor(a, device="cuda")  # noqa: E731


class Pages:
    """A 4-bit cache of random bytes and a table of LENS' requests in it."""

    def __init__(self, g, lens, H, D, page, order="phtd"):
        need = [-(-L // page) for L, _ in lens]
        n = sum(need) + 2
        perm, at = torch.randperm(n, generator=g).int(), 0
        self.table = torch.full((len(lens), max(need) + 2), -5, dtype=torch.int32)
        for i, m in enumerate(need):
            self.table[i, :m] = perm[at:at + m]
            at += m

        def dev(shape, t):
            x = torch.randint(0, 256, shape, generator=g, dtype=U8).cuda()
            return (x if order == "phtd" else x.transpose(1, 2).contiguous().transpose(1, 2)).view(t)
        self.cache = _kv().PagedCache(*[dev((n, H, page, D // 2), F4) for _ in "kv"],
                                      **{s + "_exp": dev((n, H, page, D // 32), E8) for s in "kv"})
        place = torch.cat([torch.arange(L - m, L) for L, m in lens])
        req = torch.cat([torch.full((m,), i) for i, (_, m) in enumerate(lens)])
        self.real, self.place = place >= 0, place
        self.at = (self.table[req[self.real], place[self.real] // page].long(), (place % page)[self.real])
        self.q_off = torch.tensor([0] + [m for _, m in lens]).cumsum(0).cuda()
        self.kv_len = torch.tensor([L for L, _ in lens], dtype=torch.int32).cuda()

    def where(self):
        return self.cache, self.table.cuda(), self.q_off, self.kv_len

    def bytes(self):
        c = self.cache
        return [x.view(U8).cpu().contiguous() for x in (c.k, c.v, c.k_exp, c.v_exp)]

    def rows(self, x):
        return x[self.at[0], :, self.at[1]]

    def untouched(self, before):
        for now, old in zip(self.bytes(), before):
            now, old = now.clone(), old.clone()
            now[self.at[0], :, self.at[1]] = 0
            old[self.at[0], :, self.at[1]] = 0
            assert torch.equal(now, old)


def spread(g, *shape):
    """Normal values whose groups of 32 differ by up to 2^12, with exact borders of the rounding among them."""
    x = torch.randn(*shape, generator=g).unflatten(-1, (-1, 32)) * 2.0 ** torch.randint(-6, 7, (*shape[:-1], shape[-1] // 32, 1), generator=g)
    edge = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7, -0.25, -2.5, -5, -7, 6.9375, 7.0625, 0.0, -0.0])
    some = torch.rand(*shape[:-1], shape[-1] // 32, generator=g) < 0.3
    x[..., 8:24] = torch.where(some[..., None], edge * 2.0 ** -2, x[..., 8:24])
    x[..., :8] = torch.where(some[..., None], x[..., :8].clamp(-1, 1), x[..., :8])
    x[..., 24:] = torch.where(some[..., None], x[..., 24:].clamp(-1, 1), x[..., 24:])
    return x.flatten(-2)


@pytest.mark.parametrize("D,dtype", [(64, BF), (64, FH), (128, BF), (128, FH), (256, BF), (256, FH)])
@pytest.mark.parametrize("page,order", [(16, "phtd"), (24, "pthd"), (7, "phtd"), (1, "pthd")])
@pytest.mark.parametrize("H", [1, 3])
def test_append_codes(D, dtype, page, order, H):
    """Every code and exponent of what is entered as it is, bit for bit; nothing else changes."""
    g = torch.Generator().manual_seed(D + page + H)
    p = Pages(g, LENS, H, D, page, order)
    kv = spread(g, len(p.place), 2 * H, D).to(dtype)
    before, d, st = p.bytes(), kv.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    _kv().append(*p.where(), d[:, :H], d[:, H:], status=st)
    got = p.bytes()
    assert st.item() == 0
    for s in range(2):
        c, e = ref4.quantise(kv[p.real, s * H:(s + 1) * H].double(), dtype)
        assert torch.equal(p.rows(got[2 + s]), e.to(U8))
        assert torch.equal(ref4.unpack(p.rows(got[s])), c.long())
    p.untouched(before)
    k, v = _kv().read(*p.where(), n_tokens=len(p.place), dtype=dtype, status=st)
    for out, s in ((k, 0), (v, 1)):
        c, e = ref4.quantise(kv[:, s * H:(s + 1) * H].double(), dtype)
        assert torch.equal(out[p.real.cuda()].double().cpu(), ref4.values(c, e)[p.real])
        assert bool((out[~p.real.cuda()] == 0).all())
    assert st.item() == 0


@pytest.mark.parametrize("D,rot,inter,norm,dtype", [(64, 64, False, True, BF), (64, 48, False, False, FH), (128, 128, False, True, BF),
                                                    (128, 64, True, False, FH), (256, 256, False, True, FH), (256, 16, True, True, BF),
                                                    (128, 0, False, True, FH), (256, 240, False, True, BF), (64, 16, True, True, BF)])
@pytest.mark.parametrize("page", [16, 5])
def test_append_turned(D, rot, inter, norm, dtype, page):
    """Normed and rotated keys: the exponent is that of the float32 result, each component within half
    of its step of it; queries beside them as with other caches."""
    g = torch.Generator().manual_seed(D + rot + page)
    H, Hq = 2, 5
    r, w, t = rotary(g, D, rot, inter, norm, dtype)
    p = Pages(g, LENS, H, D, page)
    x = (2 * torch.randn(len(p.place), Hq + 2 * H, D, generator=g)).to(dtype)
    before, d = p.bytes(), x.cuda()
    q = _kv().append(*p.where(), d[:, Hq:Hq + H], d[:, Hq + H:], q=d[:, :Hq], rotary=r)
    yq, eq = ref.turn(x[:, :Hq], w[0], t, rot, inter, p.place.clamp(min=0))
    ref.close(q[p.real.cuda()], yq[p.real], eq[p.real], dtype)
    assert bool((q[~p.real.cuda()] == 0).all())
    y, slack = ref.turn(x[:, Hq:Hq + H], w[1], t, rot, inter, p.place.clamp(min=0))
    y, slack, got = y[p.real], slack[p.real], p.bytes()
    e, c = p.rows(got[2]).long(), ref4.unpack(p.rows(got[0]))
    group = lambda z: z.unflatten(-1, (-1, 32))  # noqa: E731
    lo = ref4.exponents(group(y.abs() - slack).clamp(min=0), dtype) + 127
    hi = ref4.exponents(group(y.abs() + slack), dtype) + 127
    assert bool(((e >= lo) & (e <= hi)).all()) and bool((lo == hi).float().mean() > 0.9)
    unit = 2.0 ** (e.double() - 127).repeat_interleave(32, -1)
    z = (y.abs() / unit).clamp(max=6)
    half = torch.where(z < 2, 0.25, torch.where(z < 4, 0.5, 1.0))  # (of the larger step at 2 and 4: the slack's)
    near = torch.where(z + slack / unit >= 4, 1.0, torch.where(z + slack / unit >= 2, 0.5, 0.25))
    err = (ref4.values(c, e) - torch.copysign(z * unit, y)).abs()
    assert bool((err <= torch.maximum(half, near) * unit + slack).all())
    cv, ev = ref4.quantise(x[p.real, Hq + H:].double(), dtype)
    assert torch.equal(p.rows(got[3]), ev.to(U8)) and torch.equal(ref4.unpack(p.rows(got[1])), cv.long())
    p.untouched(before)


@pytest.mark.parametrize("dtype", [BF, FH])
def test_append_extremes(dtype):
    """Zeros, NaN, infinities, the type's largest and smallest numbers, beside a neighbour group of ones."""
    D, big = 128, torch.finfo(dtype).max
    rows = [[0.0], [-0.0], [math.nan], [math.inf], [-math.inf, 1.0], [big, -big / 2], [torch.finfo(dtype).tiny],
            [torch.finfo(dtype).smallest_normal / 64], [math.nan, math.inf], [7 * 2.0 ** 13, 2.0 ** 13], [7.0, 0.25]]
    x = torch.zeros(len(rows), 1, D)
    for i, row in enumerate(rows):
        for g in (0, 3):
            x[i, 0, 32 * g + 5:32 * g + 5 + len(row)] = torch.tensor(row)
        x[i, 0, 32:64] = 1.0
    x = x.to(dtype)
    z = torch.zeros(1, 1, 16, D // 2, dtype=U8, device="cuda")
    e = torch.zeros(1, 1, 16, D // 32, dtype=U8, device="cuda")
    c = _kv().PagedCache(z.view(F4), z.clone().view(F4), k_exp=e.view(E8), v_exp=e.clone().view(E8))
    n = len(rows)
    _kv().append(c, i32(0)[None], off(0, n), i32(n), x.cuda(), x.cuda())
    wc, we = ref4.quantise(x[:, 0].double(), dtype)
    for data, exps in ((c.k, c.k_exp), (c.v, c.v_exp)):
        got_e = exps.view(U8)[0, 0, :n].cpu().long()
        assert torch.equal(got_e, we.long())
        got = ref4.values(ref4.unpack(data.view(U8)[0, 0, :n].cpu()), got_e)
        assert torch.equal(torch.nan_to_num(got, nan=77.0), torch.nan_to_num(ref4.values(wc, we), nan=77.0))
    k, v = _kv().read(c, i32(0)[None], off(0, n), i32(n), n, dtype)
    for out in (k, v):
        want = ref4.values(wc, we)
        assert torch.equal(torch.nan_to_num(out[:, 0].double().cpu(), nan=77.0), torch.nan_to_num(want, nan=77.0))
        assert bool(torch.isfinite(out[:, 0, 32:64]).all())


@pytest.mark.parametrize("dtype", [BF, FH])
def test_read_every_byte(dtype):
    """All 256 bytes under all 256 exponents: what they stand for, rounded once to the activations' type."""
    e = torch.arange(256, dtype=U8)[:, None].expand(256, 4)
    b = torch.arange(256, dtype=U8).view(4, 64).repeat(64, 1)  # page p, token p: bytes of p % 4
    cache = []
    for half in range(4):
        cache.append(b[half].expand(256, 64))
    for half in range(4):
        pages = cache[half].reshape(16, 1, 16, 64).contiguous().cuda()
        exps = e.reshape(16, 1, 16, 4).contiguous().cuda()
        c = _kv().PagedCache(pages.view(F4), pages.view(F4), k_exp=exps.view(E8), v_exp=exps.view(E8))
        k, v = _kv().read(c, torch.arange(16, dtype=torch.int32, device="cuda")[None], off(0, 256), i32(256), 256, dtype)
        want = ref4.values(ref4.unpack(cache[half]), e.long())
        got = k[:, 0].cpu()
        assert torch.equal(torch.nan_to_num(got, nan=3.0, posinf=4.0, neginf=5.0),
                           torch.nan_to_num(want.to(dtype), nan=3.0, posinf=4.0, neginf=5.0))
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(v[:, 0].view(torch.int16).cpu(), got.view(torch.int16))


SHAPES = [[(1, 1)], [(40, 7), (0, 3), (5, 0), (2, 5), (33, 33), (64, 16)], [(300, 299), (17, 16), (16, 16)]]


@pytest.mark.parametrize("D,dtype,pages", [(64, BF, "same"), (128, FH, "same"), (256, BF, "same"), (64, FH, "fp8"), (128, BF, "fp8"),
                                           (256, FH, "fp8"), (64, BF, "fp4"), (128, FH, "fp4"), (256, BF, "fp4")])
@pytest.mark.parametrize("H,page,order", [(1, 16, "phtd"), (3, 16, "pthd"), (5, 24, "phtd"), (2, 1, "phtd")])
@pytest.mark.parametrize("lens", SHAPES)
def test_read(D, dtype, pages, H, page, order, lens):
    b = ref4.Batch(_kv(), lens, H, H, D, dtype, pages, page, order, seed=21)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    fused = torch.full((b.T, 2 * H + 1, D + 8), 9.0, dtype=dtype, device="cuda")  # outputs of other strides
    k, v = _kv().read(b.cache, b.table, b.q_off, b.kv_len, k_out=fused[:, :H, :D], v_out=fused[:, H:2 * H, :D], status=st)
    assert st.item() == 0
    a = 0
    for (L, n), mine in zip(lens, b.kv):
        for s, out in enumerate((k, v)):
            got = out[a:a + n].double().cpu()
            pad = max(0, n - L)
            assert bool((got[:pad] == 0).all())
            y = mine[s][L - (n - pad):]
            ref.close(got[pad:], y, ref.F32 * y.abs() if pages == "fp8" else 0 * y, dtype)
            if pages != "fp8":
                assert torch.equal(got[pad:], y)
        a += n
    assert bool((fused[:, 2 * H] == 9).all()) and bool((fused[..., D:] == 9).all())
    again = _kv().read(b.cache, b.table, b.q_off, b.kv_len, b.T, dtype)
    assert torch.equal(again[0], k) and torch.equal(again[1], v)


@pytest.mark.parametrize("pages", ["same", "fp8", "fp4"])
def test_read_bad_inputs_are_zeros(pages):
    b = ref4.Batch(_kv(), [(20, 4), (9, 2)], 2, 2, 64, BF, pages, seed=22)
    good = _kv().read(b.cache, b.table, b.q_off, b.kv_len, b.T, BF)
    bad = b.table.clone()
    bad[0, 1] = b.cache.n_pages
    for table, q_off, kv_len, zero in ((bad, b.q_off, b.kv_len, slice(0, 4)), (b.table, b.q_off, i32(33, 9), slice(0, 4)),
                                       (b.table, b.q_off, i32(-1, 9), slice(0, 4)), (b.table, off(2, 4, 6), b.kv_len, slice(0, 2)),
                                       (b.table, off(0, 4, 5), b.kv_len, slice(5, 6))):
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = _kv().read(b.cache, table, q_off, kv_len, b.T, BF, status=st)
        assert st.item() == -1
        for x in out:
            assert bool((x[zero] == 0).all())
        if zero == slice(0, 4):
            assert torch.equal(out[0][4:], good[0][4:]) and torch.equal(out[1][4:], good[1][4:])
    e = _kv().read(b.cache, b.table[:0], b.q_off[:1], b.kv_len[:0], 0, BF)
    assert e[0].shape == (0, 2, 64)


def test_read_many_requests_with_empty_ones_between():
    R, D, P = 3000, 64, 16
    g = torch.Generator().manual_seed(4)
    n = (torch.rand(R, generator=g) < 0.1).long() * torch.randint(1, 16, (R,), generator=g)
    q_off = torch.cat([torch.zeros(1).long(), n.cumsum(0)])
    z = torch.randn(R, 2, P, D, generator=g).bfloat16()
    c = _kv().PagedCache(z.cuda(), -z.cuda())
    k, v = _kv().read(c, torch.arange(R, dtype=torch.int32, device="cuda")[:, None], q_off.cuda(), n.int().cuda(), int(q_off[-1]))
    want = torch.cat([z[r, :, :int(n[r])].transpose(0, 1) for r in range(R)])
    assert torch.equal(k.cpu(), want) and torch.equal(v.cpu(), -want)


def test_offsets_beyond_32_bits():
    """4-bit pages at the far end of more than 2^32 bytes a side, exponents beyond 2^28."""
    kv = _kv()
    H, P, D = 4, 16, 128
    n_pages = (1 << 32) // (H * P * D // 2) + 64
    c = kv.PagedCache.empty(n_pages, H, D, P, F4)
    far = torch.arange(n_pages - 5, n_pages, device="cuda", dtype=torch.int32)[None]
    x = torch.randn(70, 2 * H, D, generator=torch.Generator().manual_seed(5)).bfloat16()
    kv.append(c, far, off(0, 70), i32(70), x[:, :H].cuda(), x[:, H:].cuda())
    k, v = kv.read(c, far, off(0, 70), i32(70), 70)
    for out, y in ((k, x[:, :H]), (v, x[:, H:])):
        assert torch.equal(out.double().cpu(), ref4.values(*ref4.quantise(y.double(), BF)))
    q = torch.randn(70, 8, D, generator=torch.Generator().manual_seed(6)).bfloat16()
    for new in (1, 70):
        plan = kv.Plan(1, new, 8, H, D, new).make(off(0, new), i32(70))
        out = kv.attend(q[:new].cuda(), c, far, plan)
        keys, vals = (ref4.values(*ref4.quantise(y.double(), BF)) for y in (x[:, :H], x[:, H:]))
        ref4.close_scores(out, None, ref4.attend(q[:new].double(), keys, vals, H, D ** -0.5, 0, 70, new), D, BF)
