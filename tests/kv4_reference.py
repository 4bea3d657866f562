"""Plain 64-bit forms, on the CPU, of 4-bit pages (E2M1 codes, an exponent per 32 components) and of
attention with capped or biased scores, and batches over pages of any type for their tests."""
import math

import torch

from tests import kv_reference as ref

F4, E8 = torch.float4_e2m1fn_x2, torch.float8_e8m0fnu
LEVELS = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
RANGE = {torch.bfloat16: (-125, 125), torch.float16: (-23, 13)}


def exponents(x, dtype):
    """The smallest k in the type's range with |x| <= 7 2^k, of float64 groups [..., 32]."""
    top = x.abs().amax(-1)
    k = torch.full(top.shape, RANGE[dtype][1])
    for c in range(RANGE[dtype][1] - 1, RANGE[dtype][0] - 1, -1):
        k = torch.where(top <= 7 * 2.0 ** c, torch.full_like(k, c), k)
    return k


def codes(y):
    """Of float64 y in units of its group's power of two: nearest, ties to the even code, saturated."""
    d = (y.abs().clamp(max=6)[..., None] - LEVELS).abs()
    best = d.amin(-1, keepdim=True)
    odd = torch.arange(8) % 2
    c = torch.where(d == best, torch.arange(8) + 100 * odd, torch.full((8,), 1000)).amin(-1) % 100  # even ones first
    return c + 8 * torch.signbit(y)


def quantise(x, dtype):
    """(codes, exponent bytes) of float64 x [..., dim]; 255 where a group holds a NaN."""
    g = x.unflatten(-1, (-1, 32))
    nan = torch.isnan(g).any(-1)
    g = torch.nan_to_num(g, nan=0.0, posinf=1e300, neginf=-1e300)
    k = exponents(g, dtype)
    c = codes(g / 2.0 ** k.double()[..., None]).flatten(-2)
    return c, torch.where(nan, torch.full_like(k, 255), k + 127)


def values(c, e):
    """float64 of codes [..., dim] and exponent bytes [..., dim / 32]."""
    v = torch.where(c >= 8, -LEVELS[c % 8], LEVELS[c % 8]).unflatten(-1, (-1, 32))
    s = torch.where(e == 255, torch.full(e.shape, math.nan).double(), 2.0 ** (e.double() - 127))
    return (v * s[..., None]).flatten(-2)


def pack(c):
    return (c[..., 0::2] + 16 * c[..., 1::2]).to(torch.uint8)


def unpack(b):
    b = b.long()
    return torch.stack([b % 16, b // 16], -1).flatten(-2)


def attend(q, keys, values_, n_kv, scale, window, kv_len, n_new, cap=0.0, slopes=None):
    """kv_reference.attend's outputs and, per row, how far float32 may take a score: cap's and bias's
    share (their derivation beside close_scores)."""
    n_q, D = q.shape[1:]
    G = n_q // n_kv
    out, mag = torch.zeros(n_new, n_q, D).double(), torch.zeros(n_new, n_q, D).double()
    lse = torch.full((n_new, n_q), -math.inf).double()
    big, more = torch.zeros(n_new, n_q).double(), torch.zeros(n_new, n_q).double()
    for i in range(n_new):
        place = kv_len - n_new + i
        lo = max(0, place - window + 1) if window else 0
        if place + 1 <= lo:
            continue
        k, v = keys[lo:place + 1], values_[lo:place + 1]
        j = torch.arange(lo, place + 1)
        for h in range(n_q):
            kk, vv = k[:, h // G], v[:, h // G]
            s = scale * (kk @ q[i, h])
            if cap:
                s = cap * torch.tanh(s / cap)
            if slopes is not None:
                s = s + slopes[h].double() * (j - place)
            lse[i, h] = torch.logsumexp(s, 0)
            p = torch.exp(s - lse[i, h])
            out[i, h], mag[i, h] = p @ vv, p @ vv.abs()
            big[i, h] = scale * (kk.abs() @ q[i, h].abs()).max()
            bias = 0 if slopes is None else slopes[h].double().abs() * (place - lo)
            more[i, h] = cap * 2.0 ** -20 + bias * (D / 16 + 8) * ref.F32
    return out, lse, mag, big, more


def close_scores(out, lse, want, dim, dtype):
    """As kv_reference.close_attend, with what a cap and a bias add to a score's error.

    A cap: t = 1 - 2 / (1 + e), e = 2^y.  y has five roundings, y 2^-24 each, which reach t through
    2 e / (1 + e)^2 y ln 2 <= 0.45: 2.3 units of 2^-24; e's own last place 1, the sum 1, the reciprocal's
    last place 4, the last product and sum 2, the factors log2(e) 1: below 12, 2^-20 has 16.
    A bias: slope log2(e), that divided by the score's factor, the product with the first key's distance,
    the sum with the key's own, the factor's and the last product's and sum's roundings: 8 of at most the
    bias, 2^-24 each.  In chunks it is where the sum of the products begins, dim / 16 matrix
    products, each of which rounds the sum so far: as many more."""
    o, l, mag, big, more = want
    # products of dim terms and, beside them, what the running maximum's subtraction rounds
    score = big * dim * ref.F32 + more
    rel = 2 * score + 2.0 ** -16
    ref.close(out, o, mag * (ref.UNIT[dtype] * 1.01 + rel[..., None]), dtype)
    if lse is not None:
        got = lse.double().cpu()
        assert torch.equal(torch.isinf(got), torch.isinf(l))
        fine = torch.isfinite(l)
        err = (got - l)[fine].abs()
        assert bool((err <= (score + (l.abs() + 4) * 8 * ref.F32)[fine]).all()), float(err.max())


class Batch:
    """lens = (kv_len, new tokens) per request over pages of a type ("same", "fp8", "fp4"); what no
    request's place holds is NaN (in 4 bits: exponents of 255)."""

    def __init__(self, kv, lens, Hq, H, D, dtype, pages="fp4", page=16, order="phtd", window=0, seed=0, sharp=1.5,
                 max_new=None, cap=0.0, slopes=False):
        g = torch.Generator().manual_seed(seed * 1000 + D + page + Hq)
        self.mod, self.lens, self.Hq, self.H, self.D, self.dtype, self.page, self.window = kv, lens, Hq, H, D, dtype, page, window
        self.kind, self.cap = pages, cap
        self.T = sum(n for _, n in lens)
        need = [-(-L // page) for L, _ in lens]
        n_pages = sum(need) + 1
        perm = torch.randperm(n_pages, generator=g).int()
        table = torch.full((len(lens), max(need + [1])), 1 << 30, dtype=torch.int32)
        scales = [0.01 + 0.02 * torch.rand(H, generator=g) for _ in "kv"] if pages == "fp8" else [None, None]
        ct = ref.FP8 if pages == "fp8" else dtype
        word = torch.uint8 if pages != "same" else torch.int16
        shape = (n_pages, H, page, D)
        if pages == "fp4":
            data = [torch.randint(0, 256, (*shape[:3], D // 2), generator=g, dtype=torch.uint8) for _ in "kv"]
            exps = [torch.full((*shape[:3], D // 32), 255, dtype=torch.uint8) for _ in "kv"]
        else:
            data = [torch.full(shape, math.nan).to(ct).view(word) for _ in "kv"]
        self.kv, at = [], 0
        for i, (L, _) in enumerate(lens):
            table[i, :need[i]] = perm[at:at + need[i]]
            at += need[i]
            mine = []
            for s in range(2):
                x = torch.randn(L, H, D, generator=g) * (0.3 + torch.rand(L, H, D // 32, generator=g)).repeat_interleave(32, -1)
                if pages == "fp4":
                    c, e = quantise(x.double(), dtype)
                    self._enter(data[s], pack(c), table[i], page)
                    self._enter(exps[s], e.to(torch.uint8), table[i], page)
                    mine.append(values(c, e))
                else:
                    x = ((60 if pages == "fp8" else 1) * x).to(ct)
                    self._enter(data[s], x.view(word), table[i], page)
                    y = x.float().double()
                    mine.append(y * scales[s].double()[:, None] if pages == "fp8" else y)
            self.kv.append(mine)

        def dev(x, t):
            x = x.cuda()
            return (x if order == "phtd" else x.transpose(1, 2).contiguous().transpose(1, 2)).view(t)
        if pages == "fp4":
            self.cache = kv.PagedCache(dev(data[0], F4), dev(data[1], F4), k_exp=dev(exps[0], E8), v_exp=dev(exps[1], E8))
        else:
            self.cache = kv.PagedCache(dev(data[0], ct), dev(data[1], ct), *[None if s is None else s.cuda() for s in scales])
        self.table = table.cuda()
        self.q = (sharp * torch.randn(self.T, Hq, D, generator=g)).to(dtype)
        self.slopes = (2.0 ** -(1 + 7 * torch.rand(Hq, generator=g))) * (1 - 2 * (torch.rand(Hq, generator=g) < 0.3)) if slopes else None
        self.q_off = torch.tensor([0] + [n for _, n in lens]).cumsum(0).cuda()
        self.kv_len = torch.tensor([L for L, _ in lens], dtype=torch.int32, device="cuda")
        self.max_new = max_new or max([n for _, n in lens] + [1])
        self.scale = 1 / math.sqrt(D)

    @staticmethod
    def _enter(pages, rows, table, page):
        for p in range(0, rows.shape[0], page):
            n = min(page, rows.shape[0] - p)
            pages[int(table[p // page]), :, :n] = rows[p:p + n].transpose(0, 1)

    def plan(self):
        return self.mod.Plan(len(self.lens), self.T, self.Hq, self.H, self.D, self.max_new, self.window)

    def run(self, plan=None, q=None, out=None, status=None, lse=None, **how):
        plan = (plan or self.plan()).make(self.q_off, self.kv_len)
        lse = torch.full((self.T, self.Hq), 7.0, device="cuda") if lse is None else lse
        how = dict(dict(cap=self.cap, slopes=None if self.slopes is None else self.slopes.cuda()), **how)
        out = self.mod.attend(self.q.cuda() if q is None else q, self.cache, self.table, plan, lse=lse, out=out, status=status, **how)
        return out, lse

    def want(self):
        parts, a = [], 0
        for (L, n), (k, v) in zip(self.lens, self.kv):
            parts.append(attend(self.q[a:a + n].double(), k, v, self.H, self.scale, self.window, L, n, self.cap, self.slopes))
            a += n
        return [torch.cat([p[i] for p in parts]) for i in range(5)]

    def check(self, **how):
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        out, lse = self.run(status=st, **how)
        close_scores(out, lse, self.want(), self.D, self.dtype)
        assert st.item() == 0
        return out, lse
