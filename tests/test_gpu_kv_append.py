"""Norms, rotation and the append to the paged cache against 64-bit forms."""
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


def table_of(n, rot):
    f = 1e4 ** (-torch.arange(rot // 2).double() * 2 / max(rot, 1))
    a = torch.arange(n).double()[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def rotary(g, D, rot, inter, norm, dtype, n=400):
    w = [(1 + 0.3 * torch.randn(D, generator=g)).to(dtype) if norm else None for _ in "qk"]
    t = table_of(n, rot) if rot else None
    dev = lambda x: None if x is None else x.cuda()  # noqa: E731
    return _kv().Rotary(dev(t), rot, inter, dev(w[0]), dev(w[1])), w, t


TURNS = [(64, 64, False, True, torch.bfloat16), (128, 128, False, True, torch.bfloat16),
         (128, 64, True, False, torch.float16), (256, 256, False, True, torch.float16),
         (256, 16, True, True, torch.bfloat16), (128, 0, False, True, torch.float16), (64, 48, False, False, torch.float16)]


@pytest.mark.parametrize("D,rot,inter,norm,dtype", TURNS)
@pytest.mark.parametrize("T,Hq,H", [(1, 1, 1), (5, 7, 2), (67, 32, 4)])
def test_rotate(D, rot, inter, norm, dtype, T, Hq, H):
    g = torch.Generator().manual_seed(T * D + rot)
    r, w, t = rotary(g, D, rot, inter, norm, dtype)
    qkv = (2 * torch.randn(T, Hq + 2 * H, D, generator=g)).to(dtype)
    pos = torch.randint(0, 400, (T,), generator=g, dtype=torch.int32)
    d = qkv.cuda()
    q, k = _kv().qk_rotate(d[:, :Hq], d[:, Hq:Hq + H], r, pos.cuda())
    for got, x, wt in ((q, qkv[:, :Hq], w[0]), (k, qkv[:, Hq:Hq + H], w[1])):
        ref.close(got, *ref.turn(x, wt, t, rot, inter, pos.long()), dtype)
    # in place, other strides
    _kv().qk_rotate(d[:, :Hq], d[:, Hq:Hq + H], r, pos.cuda(), q_out=d[:, :Hq], k_out=d[:, Hq:Hq + H])
    assert torch.equal(d[:, :Hq], q) and torch.equal(d[:, Hq:Hq + H], k)
    assert torch.equal(d[:, Hq + H:].cpu(), qkv[:, Hq + H:])


def test_rotate_bad_position_and_empty():
    g = torch.Generator().manual_seed(3)
    r, w, t = rotary(g, 128, 128, False, True, torch.bfloat16, n=10)
    q, k = torch.randn(4, 3, 128).bfloat16().cuda(), torch.randn(4, 1, 128).bfloat16().cuda()
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    pos = torch.tensor([0, -1, 10, 9], dtype=torch.int32, device="cuda")
    a, b = _kv().qk_rotate(q, k, r, pos, status=st)
    assert st.item() == -1
    assert bool((a[1:3] == 0).all()) and bool((b[1:3] == 0).all())
    ref.close(a[[0, 3]], *ref.turn(q.cpu()[[0, 3]], w[0], t, 128, False, torch.tensor([0, 9])), torch.bfloat16)
    e, f = _kv().qk_rotate(q[:0], k[:0], r, pos[:0])
    assert e.shape[0] == 0 and f.shape[0] == 0


# (kv_len, new tokens) per request: nothing new, padding, shorter than its new tokens, page ends
LENS = [(1, 1), (16, 1), (17, 3), (0, 1), (40, 0), (33, 33), (2, 5), (130, 70), (48, 16)]


@pytest.mark.parametrize("D,rot,inter,norm,dtype", TURNS)
@pytest.mark.parametrize("cache,page,order", [("same", 16, "phtd"), ("fp8", 16, "phtd"), ("same", 24, "pthd"), ("fp8", 7, "pthd")])
def test_append(D, rot, inter, norm, dtype, cache, page, order):
    g = torch.Generator().manual_seed(D + rot + page)
    Hq, H = 6, 3
    kv = _kv()
    r, w, t = rotary(g, D, rot, inter, norm, dtype)
    T, R = sum(n for _, n in LENS), len(LENS)
    ct = ref.FP8 if cache == "fp8" else dtype
    width = max(-(-L // page) for L, _ in LENS) + 2
    need = [-(-L // page) for L, _ in LENS]
    n_pages = sum(need) + 2
    perm = torch.randperm(n_pages, generator=g).int()
    table = torch.full((R, width), -5, dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = perm[at:at + n]
        at += n
    shape = (n_pages, H, page, D)
    def pages():
        x = torch.randn(shape, generator=g).to(ct).cuda()
        return x if order == "phtd" else x.transpose(1, 2).contiguous().transpose(1, 2)
    sc = [0.01 + 0.02 * torch.rand(H, generator=g) for _ in "kv"] if cache == "fp8" else [None, None]
    c = kv.PagedCache(pages(), pages(), *[None if s is None else s.cuda() for s in sc])
    before = [c.k.clone(), c.v.clone()]
    q_off = torch.tensor([0] + [n for _, n in LENS]).cumsum(0)
    kv_len = torch.tensor([L for L, _ in LENS], dtype=torch.int32)
    qkv = (2 * torch.randn(T, Hq + 2 * H, D, generator=g)).to(dtype)
    d = qkv.cuda()
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = kv.append(c, table.cuda(), q_off.cuda(), kv_len.cuda(), d[:, Hq:Hq + H], d[:, Hq + H:], q=d[:, :Hq], rotary=r, status=st)
    assert st.item() == 0
    place = torch.cat([torch.arange(L - n, L) for L, n in LENS])
    req = torch.cat([torch.full((n,), i) for i, (_, n) in enumerate(LENS)])
    real = place >= 0
    yq, eq = ref.turn(qkv[:, :Hq], w[0], t, rot, inter, place.clamp(min=0))
    ref.close(q[real.cuda()], yq[real], eq[real], dtype)
    assert bool((q[~real.cuda()] == 0).all())
    yk, ek = ref.turn(qkv[:, Hq:Hq + H], w[1], t, rot, inter, place.clamp(min=0))
    yv = qkv[:, Hq + H:].double()
    pg, slot = table[req[real], place[real] // page].long(), (place % page)[real]
    word = torch.uint8 if cache == "fp8" else torch.int16
    take = lambda x: x.contiguous().view(word)[pg.cuda(), :, slot.cuda()].view(ct)  # noqa: E731
    if cache == "fp8":
        ref.close_e4m3(take(c.k), yk[real] / sc[0].double()[:, None], ek[real] / sc[0].double()[:, None])
        ref.close_e4m3(take(c.v), yv[real] / sc[1].double()[:, None], 4 * ref.F32 * yv[real].abs() / sc[1].double()[:, None])
    else:
        ref.close(take(c.k), yk[real], ek[real], dtype)
        assert torch.equal(take(c.v).cpu(), qkv[:, Hq + H:][real])
    # nothing else in the cache changed
    for now, old in zip((c.k, c.v), before):
        now, old = now.contiguous().view(word).clone(), old.contiguous().view(word).clone()
        now[pg.cuda(), :, slot.cuda()] = 0
        old[pg.cuda(), :, slot.cuda()] = 0
        assert torch.equal(now, old)


def test_append_many_requests_with_empty_ones_between():
    """Tokens find their requests among thousands, most of which have none."""
    kv = _kv()
    R, D, P = 5000, 64, 16
    g = torch.Generator().manual_seed(1)
    n = (torch.rand(R, generator=g) < 0.1).long() * torch.randint(1, 4, (R,), generator=g)
    q_off = torch.cat([torch.zeros(1).long(), n.cumsum(0)])
    T = int(q_off[-1])
    kv_len = (n + torch.randint(0, 13, (R,), generator=g)).int()
    table = torch.arange(R, dtype=torch.int32)[:, None]
    z = torch.zeros(R, 1, P, D, dtype=torch.bfloat16, device="cuda")
    c = kv.PagedCache(z, z.clone())
    x = torch.randn(T, 2, D, generator=g).bfloat16()
    kv.append(c, table.cuda(), q_off.cuda(), kv_len.cuda(), x[:, :1].cuda(), x[:, 1:].cuda())
    want = torch.zeros(R, P, D, dtype=torch.bfloat16)
    for r in range(R):
        a, z_ = int(q_off[r]), int(q_off[r + 1])
        want[r, int(kv_len[r]) - (z_ - a):int(kv_len[r])] = x[a:z_, 0]
    assert torch.equal(c.k[:, 0].cpu(), want)


def test_append_saturates_and_keeps_nan():
    kv = _kv()
    z = torch.zeros(1, 1, 16, 64, dtype=ref.FP8, device="cuda")
    one = torch.ones(1, device="cuda")
    c = kv.PagedCache(z, z.clone(), one, one)
    x = torch.zeros(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    x[0, 0, :6] = torch.tensor([1000.0, -1000.0, float("nan"), float("inf"), 448.0, 2.0 ** -10])
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    kv.append(c, i32(0)[None], torch.tensor([0, 1], device="cuda"), i32(1), x, x)
    got = c.v[0, 0, 0, :6].float().cpu()
    assert got[0] == 448 and got[1] == -448 and torch.isnan(got[2]) and got[3] == 448 and got[4] == 448 and got[5] == 0


def test_append_bad_inputs_write_nothing():
    kv = _kv()
    D, P = 64, 16
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    off = lambda *a: torch.tensor(a, device="cuda")  # noqa: E731
    x = torch.ones(2, 1, D, dtype=torch.bfloat16, device="cuda")
    for table, q_off, kv_len in ((i32(7, 0), off(0, 1, 2), i32(1, 1)),   # a page outside the cache
                                 (i32(-1, 0), off(0, 1, 2), i32(1, 1)),
                                 (i32(1, 0), off(0, 1, 2), i32(17, 1)),  # longer than the table's row
                                 (i32(1, 0), off(1, 1, 2), i32(1, 1)),   # token 0 belongs to nobody
                                 (i32(1, 0), off(0, 1, 2), i32(-3, 1))):
        z = torch.zeros(4, 1, P, D, dtype=torch.bfloat16, device="cuda")
        c = kv.PagedCache(z, z.clone())
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        q = kv.append(c, table[:, None], q_off, kv_len, x, x, q=x, status=st)
        assert st.item() == -1
        # the second request's token is entered, the first's is not
        assert bool((c.k[0, 0, 0] == 1).all()) and float(c.k.float().sum()) == D and float(c.v.float().sum()) == D
        assert bool((q[0] == 0).all()) and bool((q[1] == 1).all())


def test_padding_is_zeros_without_eps():
    """Where eps is 0 a token of zeros has no norm; what padding and bad positions leave is zeros all the same."""
    kv = _kv()
    D = 64
    w = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    r = kv.Rotary(table_of(8, D).cuda(), q_weight=w, k_weight=w, eps=0.0)
    x = torch.ones(2, 3, D, dtype=torch.bfloat16, device="cuda")
    z = torch.zeros(1, 1, 16, D, dtype=torch.bfloat16, device="cuda")
    c = kv.PagedCache(z, z.clone())
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    q = kv.append(c, i32(0, 0)[:, None], torch.tensor([0, 1, 2], device="cuda"), i32(0, 1), x[:, :1], x[:, 1:2], q=x, rotary=r)
    assert bool((q[0] == 0).all()) and bool((q[1] == 1).all())
    a, b = kv.qk_rotate(x, x[:, :1], r, i32(8, 0))
    assert bool((a[0] == 0).all()) and bool((b[0] == 0).all()) and bool((a[1] == 1).all()) and bool((b[1] == 1).all())


def test_refusals():
    kv = _kv()
    from paper_2607_08565_amd.smetric import SmetricError
    bf = torch.bfloat16
    q = torch.zeros(2, 2, 64, dtype=bf, device="cuda")
    r = kv.Rotary(table_of(8, 64).cuda())
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(SmetricError):
        kv.qk_rotate(torch.zeros(2, 2, 96, dtype=bf, device="cuda"), torch.zeros(2, 2, 96, dtype=bf, device="cuda"), r, pos)
    with pytest.raises(SmetricError):
        kv.qk_rotate(q, q, r)  # no positions
    with pytest.raises(SmetricError):
        kv.qk_rotate(q, q, kv.Rotary(table_of(8, 24).cuda()), pos)  # rot_dim not of 16
    with pytest.raises(SmetricError):
        kv.qk_rotate(q, q, kv.Rotary(table_of(8, 128).cuda()), pos)  # longer than the head
    with pytest.raises(SmetricError):  # heads not 16-byte aligned
        kv.qk_rotate(torch.zeros(2, 2, 68, dtype=bf, device="cuda")[..., 4:], q, r, pos)
    with pytest.raises(TypeError):
        kv.qk_rotate(q.float(), q, r, pos)
    with pytest.raises(TypeError):
        kv.qk_rotate(q, q.half(), r, pos)
    with pytest.raises(ValueError):
        kv.qk_rotate(q, q[:1], r, pos)
    with pytest.raises(ValueError):
        kv.qk_rotate(q, q, kv.Rotary(q_weight=torch.ones(32, dtype=bf, device="cuda")))
    z = torch.zeros(2, 1, 16, 64, dtype=bf, device="cuda")
    c = kv.PagedCache(z, z)
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    off = torch.tensor([0, 2], device="cuda")
    with pytest.raises(SmetricError):  # a cache of another 16-bit type
        kv.append(c, i32(0)[None], off, i32(2), q[:, :1].half(), q[:, :1].half())
    with pytest.raises(ValueError):
        kv.append(c, i32(0)[None], off, i32(2), q, q)  # two heads into one
    with pytest.raises(ValueError):
        kv.append(c, i32(0)[None], off[:1], i32(2), q[:, :1], q[:, :1])
    with pytest.raises(TypeError):
        kv.append(c, i32(0)[None].long(), off, i32(2), q[:, :1], q[:, :1])
    with pytest.raises(ValueError):
        kv.PagedCache(z, z, torch.ones(1, device="cuda"), torch.ones(1, device="cuda"))  # scales of a 16-bit cache
    with pytest.raises(TypeError):
        kv.PagedCache(z.float(), z.float())
