"""The append with positions of its own, and the values it enters among thousands of requests."""
import pytest
import torch

from tests import kv_reference as ref
from tests.test_gpu_kv_append import LENS, TURNS, _kv, rotary

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu(dev):
    yield


def batch(g, D, page, dtype, Hq=4, H=2):
    """A ragged batch with padding tokens: cache, tables, activations, each token's request and place."""
    need = [-(-L // page) for L, _ in LENS]
    table = torch.full((len(LENS), max(need) + 1), -5, dtype=torch.int32)
    perm, at = torch.randperm(sum(need) + 1, generator=g).int(), 0
    for i, n in enumerate(need):
        table[i, :n] = perm[at:at + n]
        at += n
    z = torch.zeros(sum(need) + 1, H, page, D, dtype=dtype, device="cuda")
    q_off = torch.tensor([0] + [n for _, n in LENS]).cumsum(0)
    kv_len = torch.tensor([L for L, _ in LENS], dtype=torch.int32)
    place = torch.cat([torch.arange(L - n, L) for L, n in LENS])
    req = torch.cat([torch.full((n,), i) for i, (_, n) in enumerate(LENS)])
    x = (2 * torch.randn(len(place), Hq + 2 * H, D, generator=g)).to(dtype)
    return _kv().PagedCache(z, z.clone()), table, q_off, kv_len, place, req, x.split([Hq, H, H], 1)


def append(c, table, q_off, kv_len, q, k, v, **how):
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    return _kv().append(c, table.cuda(), q_off.cuda(), kv_len.cuda(), k.cuda(), v.cuda(), q=q.cuda(), status=st, **how), st.item()


@pytest.mark.parametrize("D,rot,inter,norm,dtype", TURNS)
@pytest.mark.parametrize("page", [16, 7])
def test_positions_other_than_places(D, rot, inter, norm, dtype, page):
    """Rotated to the positions, entered at the places; padding tokens' positions may be anything."""
    g = torch.Generator().manual_seed(D + rot + page)
    r, w, t = rotary(g, D, rot, inter, norm, dtype)
    c, table, q_off, kv_len, place, req, (q, k, v) = batch(g, D, page, dtype)
    real = place >= 0
    pos = torch.randint(0, 400, place.shape, generator=g, dtype=torch.int32)
    given = torch.where(real, pos, torch.tensor([-1, 400, 1 << 30], dtype=torch.int32)[torch.arange(len(pos)) % 3])
    out, status = append(c, table, q_off, kv_len, q, k, v, rotary=r, positions=given.cuda())
    assert status == 0
    y, e = ref.turn(q, w[0], t, rot, inter, pos.long())
    ref.close(out[real.cuda()], y[real], e[real], dtype)
    assert bool((out[~real.cuda()] == 0).all())
    y, e = ref.turn(k, w[1], t, rot, inter, pos.long())
    page_of, slot = table[req[real], place[real] // page].long().cuda(), (place % page)[real].cuda()
    ref.close(c.k[page_of, :, slot], y[real], e[real], dtype)
    assert torch.equal(c.v[page_of, :, slot].cpu(), v[real])
    for pages in (c.k, c.v):  # and nowhere else
        pages[page_of, :, slot] = 0
        assert bool((pages == 0).all())


@pytest.mark.parametrize("bad", [-1, 400, -(1 << 31)])
def test_a_position_outside_the_table(bad):
    """Its token enters neither key nor value and has zeros for queries; the others are what they were."""
    g = torch.Generator().manual_seed(5)
    D, page = 64, 16
    r, _, _ = rotary(g, D, D, False, True, torch.bfloat16)
    c, table, q_off, kv_len, place, req, (q, k, v) = batch(g, D, page, torch.bfloat16)
    pos = torch.randint(0, 400, place.shape, generator=g, dtype=torch.int32)
    want, status = append(c, table, q_off, kv_len, q, k, v, rotary=r, positions=pos.cuda())
    assert status == 0
    k_pages, v_pages = c.k.clone(), c.v.clone()
    for x in (c.k, c.v):
        x.zero_()
    t = int((place >= 0).nonzero()[7])
    pos[t] = bad
    out, status = append(c, table, q_off, kv_len, q, k, v, rotary=r, positions=pos.cuda())
    assert status == -1
    at, slot = int(table[req[t], place[t] // page]), int(place[t] % page)
    for x in (k_pages, v_pages):
        assert bool((x[at, :, slot] != 0).any())
        x[at, :, slot] = 0
    want[t] = 0
    assert torch.equal(c.k, k_pages) and torch.equal(c.v, v_pages) and torch.equal(out, want)


def test_values_of_many_requests():
    """Keys and values each at their own places where most requests have no new token."""
    R, D, P = 5000, 64, 16
    g = torch.Generator().manual_seed(2)
    n = (torch.rand(R, generator=g) < 0.1).long() * torch.randint(1, 4, (R,), generator=g)
    q_off = torch.cat([torch.zeros(1).long(), n.cumsum(0)])
    kv_len = (n + torch.randint(0, 13, (R,), generator=g)).int()
    z = torch.zeros(R, 1, P, D, dtype=torch.bfloat16, device="cuda")
    c = _kv().PagedCache(z, z.clone())
    x = torch.randn(int(q_off[-1]), 2, D, generator=g).bfloat16()
    _kv().append(c, torch.arange(R, dtype=torch.int32)[:, None].cuda(), q_off.cuda(), kv_len.cuda(), x[:, :1].cuda(), x[:, 1:].cuda())
    want = torch.zeros(2, R, P, D, dtype=torch.bfloat16)
    for r in n.nonzero()[:, 0].tolist():
        a, b, L = int(q_off[r]), int(q_off[r + 1]), int(kv_len[r])
        want[:, r, L - (b - a):L] = x[a:b].transpose(0, 1)
    assert torch.equal(c.k[:, 0].cpu(), want[0]) and torch.equal(c.v[:, 0].cpu(), want[1])
