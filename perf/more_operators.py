"""Operators of the paged cache in 4 bits, of its reading back, and of attention with capped or
biased scores, as they are timed.

A case is a dict of plain values with a `kind`:
  store    the new tokens' keys and values quantised into 4-bit pages (kv.append) and read back as
           activations (kv.read), as a prefilling instance does that hands them on
  read     cached tokens of pages of any type read back as activations (kv.read)
  attend   a ragged batch of new tokens over the paged cache (kv.attend with the step's plan): 4-bit
           pages, scores capped (`cap`), scores with a bias by distance (`bias`), or several of these
  layer    a step's first layer over 4-bit pages whole: plan, append, attention, and the new tokens
           read back for the instance that decodes

4-bit pages ("fp4") hold E2M1 values, 32 neighbouring components of a head with one exponent.  Keys
come rotated, so that what is quantised is the same number on every side: two roundings of one
rotation could lie on two sides of a border between 4-bit values.  The batch's shape follows from the
case alone; the seed draws values, the order of the pages and the scales.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "fp8": torch.float8_e4m3fn}
FP8_MAX = 448.0
GROUP = 32  # components with one exponent
LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
# exponents whose 4-bit values the activations' type holds exactly
EXPONENTS = {"bf16": (-125, 125), "f16": (-23, 13)}


def _kv():
    from paper_2607_08565_amd import kv
    return kv


def listed():
    return [
        # the smallest call: one agent's next token
        dict(name="store_token", kind="store", requests=1, new=1, ragged=False, ctx=1024, sigma=0.0, cap_len=65536, pad=0,
             kv_heads=4, dim=128, dtype="bf16", cache="fp4", page=16),
        # prompts prefilled together: what is left of each after its hit
        dict(name="store_chunks", kind="store", requests=16, new=2048, ragged=True, ctx=1024, sigma=0.6, cap_len=65536,
             pad=0, kv_heads=8, dim=128, dtype="bf16", cache="fp4", page=64),
        # a long session's cache handed to another instance
        dict(name="read_session", kind="read", requests=1, ctx=16384, sigma=0.0, cap_len=16384, pad=0, kv_heads=4, dim=128,
             dtype="bf16", cache="fp4", page=16),
        # what an instance holds of 24 sessions, 8-bit pages, heads of 64
        dict(name="read_sessions", kind="read", requests=24, ctx=3000, sigma=0.8, cap_len=16384, pad=3, kv_heads=16, dim=64,
             dtype="f16", cache="fp8", page=16),
        # one agent's next token after a prompt of 1,024, 4-bit pages
        dict(name="attend_token_4bit", kind="attend", requests=1, new=1, ragged=False, ctx=1024, sigma=0.0, cap_len=65536,
             pad=0, q_heads=32, kv_heads=4, dim=128, dtype="bf16", cache="fp4", page=16, window=0, cap=0.0, bias=False),
        # a decoding step of 32 requests of the throughput configuration's lengths, 4-bit pages
        dict(name="attend_decode_4bit", kind="attend", requests=32, new=1, ragged=False, ctx=24576, sigma=0.6,
             cap_len=65536, pad=0, q_heads=32, kv_heads=4, dim=128, dtype="bf16", cache="fp4", page=16, window=0, cap=0.0,
             bias=False),
        # a 16,384-token prompt of which 12,288 tokens were cached, 4-bit pages
        dict(name="attend_chunk_4bit", kind="attend", requests=1, new=4096, ragged=False, ctx=12288, sigma=0.0,
             cap_len=16384, pad=0, q_heads=32, kv_heads=4, dim=128, dtype="bf16", cache="fp4", page=16, window=0, cap=0.0,
             bias=False),
        # decoding requests and prompts' chunks in one batch, heads of 64 with a sliding window, 4-bit pages
        dict(name="attend_mixed_4bit", kind="attend", requests=24, new=1000, ragged=True, ctx=3000, sigma=0.8,
             cap_len=16384, pad=3, q_heads=16, kv_heads=16, dim=64, dtype="f16", cache="fp4", page=16, window=2048, cap=0.0,
             bias=False),
        # a decoding step of a model that caps its scores, heads of 256
        dict(name="attend_decode_capped", kind="attend", requests=16, new=1, ragged=False, ctx=8192, sigma=0.6,
             cap_len=32768, pad=0, q_heads=16, kv_heads=8, dim=256, dtype="bf16", cache="bf16", page=16, window=0, cap=50.0,
             bias=False),
        # a prompt's chunk in such a model
        dict(name="attend_chunk_capped", kind="attend", requests=1, new=2048, ragged=False, ctx=6000, sigma=0.0,
             cap_len=16384, pad=0, q_heads=32, kv_heads=16, dim=128, dtype="bf16", cache="bf16", page=64, window=4096,
             cap=50.0, bias=False),
        # decoding requests and chunks of a model whose positions are a bias by distance, 8-bit pages
        dict(name="attend_mixed_biased", kind="attend", requests=13, new=700, ragged=True, ctx=2000, sigma=0.8,
             cap_len=8192, pad=1, q_heads=32, kv_heads=32, dim=128, dtype="f16", cache="fp8", page=32, window=0, cap=0.0,
             bias=True),
        # one layer of a step: follow-up turns that add a few hundred tokens to their sessions, capped scores
        dict(name="layer_turns_4bit", kind="layer", requests=8, new=512, ragged=True, ctx=4096, sigma=0.6, cap_len=32768,
             pad=0, q_heads=32, kv_heads=4, dim=128, dtype="bf16", cache="fp4", page=16, window=0, cap=30.0, bias=False),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["store", "read", "attend", "layer"], [2, 2, 6, 1])[0]
    dim = rng.choice([64, 128, 128, 128, 256])
    kv_heads = rng.choice([1, 2, 4, 4, 8, 8, 16])
    dtype, page = rng.choice(["bf16", "bf16", "f16"]), rng.choice([16, 16, 16, 32, 64, 48, 128])
    common = dict(kv_heads=kv_heads, dim=dim, dtype=dtype, page=page, sigma=rng.choice([0.0, 0.6]))
    if kind == "store":
        new = rng.choice([1, 1, _logint(rng, 1, 2048)])
        requests = _logint(rng, 1, max(1, min(256, 24576 // new)))
        while requests * new * kv_heads * dim > 2.5e7:
            requests, new = max(1, requests // 2), max(1, new * 2 // 3)
        return dict(kind=kind, requests=requests, new=new, ragged=rng.random() < 0.6, cap_len=16384,
                    ctx=_logint(rng, 64, max(64, 16384 // requests)), pad=rng.choice([0, 0, 3]), cache="fp4", **common)
    if kind == "read":
        requests, ctx = _logint(rng, 1, 48), _logint(rng, 1, 16384)
        while requests * ctx * kv_heads * dim > 1e8:
            requests, ctx = max(1, requests // 2), max(1, ctx * 2 // 3)
        return dict(kind=kind, requests=requests, ctx=ctx, cap_len=32768, pad=rng.choice([0, 0, 3]),
                    cache=rng.choice(["fp4", "fp4", "fp8", dtype]), **common)
    q_heads = kv_heads * rng.choice([1, 2, 4, 8]) if kv_heads > 4 else kv_heads * rng.choice([1, 2, 4, 7, 8, 16])
    q_heads = max(kv_heads, min(q_heads, 8192 // dim // kv_heads * kv_heads))
    cap, bias = rng.choice([0.0, 0.0, 20.0, 30.0, 50.0]), rng.random() < 0.3
    cache = "fp4" if kind == "layer" or (not cap and not bias) else rng.choice(["fp4", "fp8", dtype, dtype])
    new = rng.choice([1, 1, _logint(rng, 2, 16), _logint(rng, 16, 2000)])
    if kind == "layer":
        new = min(new, 512)
    requests = _logint(rng, 1, 64 if new <= 16 else 12)
    ctx = _logint(rng, 16, 65536 if requests * kv_heads * dim <= 2048 and new <= 16 else 16384 if new <= 16 else 8192)
    cap_len = min(131072, max(2 * ctx, 256)) + new
    # padded scores of the plain form stay within a few GB, the cache within half the largest listed one's
    while requests * new * q_heads * cap_len > 1.5e9 or requests * cap_len * kv_heads * dim > 4e8 or new > cap_len:
        requests, cap_len, ctx = max(1, requests * 2 // 3), max(new, cap_len * 3 // 4), max(1, ctx * 3 // 4)
        if requests == 1 and new > 16:
            new = new * 3 // 4
    return dict(kind=kind, requests=requests, new=new, ragged=rng.random() < 0.5, ctx=ctx, cap_len=cap_len,
                pad=rng.choice([0, 0, 2]), q_heads=q_heads, cache=cache, window=rng.choice([0, 0, 0, _logint(rng, 16, 4096)]),
                cap=cap, bias=bias, **common)


# ---------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------
def _lengths(case):
    """(cached tokens before the step, new tokens) of each request, from the case alone; what is
    read back are all of a session's tokens.  Padding requests, the last `pad`, have one token
    each and nothing in the cache."""
    shape = np.random.default_rng([0x4B17] + [int(v) if isinstance(v, (bool, int, float)) else len(v)
                                              for k, v in sorted(case.items()) if k != "name"])
    n = case["requests"]
    ctx = np.full(n, case["ctx"])
    if case["sigma"]:
        ctx = np.rint(shape.lognormal(math.log(case["ctx"]), case["sigma"], n)).astype(np.int64)
    if case["kind"] == "read":
        new = np.clip(ctx, 1, case["cap_len"])
        ctx = np.zeros(n, np.int64)
    else:
        new = np.full(n, case["new"], np.int64)
        if case["ragged"] and case["new"] > 1:
            new = np.rint(np.exp(shape.uniform(0, math.log(case["new"]), n))).astype(np.int64)
            new[0] = case["new"]
        if case["ragged"] and n > 2:
            ctx[1] = 0  # a first turn: nothing cached
        ctx = np.minimum(ctx, case["cap_len"] - new)
    return np.concatenate([ctx, np.full(case["pad"], -1)]), np.concatenate([new, np.ones(case["pad"], np.int64)])


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _normal(g, shape, dtype, scale=1.0):
    """Normal values, in pieces so that a large cache needs no second one beside it."""
    out = torch.empty(shape, dtype=dtype, device=DEV)
    flat = out.view(torch.uint8).view(-1).view(dtype)
    for part in flat.split(1 << 26):
        x = torch.randn(part.shape, generator=g, device=DEV)
        part.copy_((x * scale).clamp_(-FP8_MAX, FP8_MAX) if dtype == TYPES["fp8"] else x * scale)
    return out


def _exponent(x, kind):
    """The smallest k with |x| <= 7 * 2^k for a group's components: none is further from its 4-bit
    value than half of the largest step."""
    top = x.abs().amax(-1)
    m, e = torch.frexp(top)
    return torch.where(top > 0, e - 3 + (m > 0.875), -127).clamp(*EXPONENTS[kind])


def _quantised(x, kind):
    """Codes (one a byte) and exponents of float32 x [..., dim]: to nearest, ties to the even code."""
    x = x.unflatten(-1, (-1, GROUP))
    k = _exponent(x, kind)
    y = torch.ldexp(x.abs(), -k[..., None]).clamp(max=6.0)
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
    y = torch.round(y / step) * step
    code = torch.where(y < 2, 2 * y, torch.where(y < 4, y + 2, y / 2 + 4)).to(torch.uint8)
    return (code | torch.signbit(x).to(torch.uint8) << 3).flatten(-2), k


def _values(code, k):
    """What codes and exponents stand for, float32."""
    v = torch.tensor(LEVELS + [-x for x in LEVELS], device=DEV)[code.long()]
    return torch.ldexp(v.unflatten(-1, (-1, GROUP)), k[..., None]).flatten(-2)


def _packed(code):
    return code[..., 0::2] | code[..., 1::2] << 4


def _unpacked(b):
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)


def _pages4(g, shape, kind):
    """4-bit pages of normal values: keys and values [pages, heads, page, dim / 2] and their exponents
    [pages, heads, page, dim / 32], the two exponents of a page's head beside each other."""
    n, H, P, D = shape
    sides, exps = [], torch.empty((n, H, 2, P, D // GROUP), dtype=torch.uint8, device=DEV)
    for s in range(2):
        side = torch.empty((n, H, P, D // 2), dtype=torch.uint8, device=DEV)
        step = max(1, (1 << 25) // (H * P * D))
        for a in range(0, n, step):
            m = min(step, n - a)
            # heads differ in size, as they do in earnest
            x = torch.randn((m, H, P, D), generator=g, device=DEV) * (0.5 + torch.arange(H, device=DEV)[:, None, None] / H)
            code, k = _quantised(x, kind)
            side[a:a + m], exps[a:a + m, :, s] = _packed(code), (k + 127).to(torch.uint8)
        sides.append(side)
    return sides, [exps[:, :, 0], exps[:, :, 1]]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed) * 2 + 1)
    kind, t, H, D, P = case["kind"], TYPES[case["dtype"]], case["kv_heads"], case["dim"], case["page"]
    ctx, new = _lengths(case)
    R = len(new)
    kv_len = np.where(ctx < 0, 0, ctx + new)
    off = np.zeros(R + 1, np.int64)
    np.cumsum(new, out=off[1:])
    T, pages = int(off[-1]), -(-kv_len // P)
    width = max(1, int(pages.max()))
    n_pages = int(pages.sum()) + 3
    # the requests' pages lie anywhere in the cache; what a table does not need is -1
    order = np.random.default_rng([0x9A6E, int(seed)]).permutation(n_pages).astype(np.int32)
    inside = np.arange(width) < pages[:, None]
    table = np.full((R, width), -1, np.int32)
    table[inside] = order[:int(pages.sum())]
    st = dict(case=case, page_table=_dev(table), q_off=_dev(off), kv_len=_dev(kv_len.astype(np.int32)), tokens=T,
              max_kv=int(kv_len.max()), max_new=int(new.max()), scale=1.0 / math.sqrt(D), scales=[None, None], exps=[None, None])
    if case["cache"] == "fp4":
        st["pages"], st["exps"] = _pages4(g, (n_pages, H, P, D), case["dtype"])
    else:
        ct = TYPES[case["cache"]]
        if case["cache"] == "fp8":
            st["scales"] = [0.02 + 0.01 * torch.rand(H, generator=g, device=DEV) for _ in "kv"]
        st["pages"] = [_normal(g, (n_pages, H, P, D), ct, 40.0 if case["cache"] == "fp8" else 1.0) for _ in "kv"]
    if kind in ("store", "layer"):
        # one product gives queries, keys and values of a token side by side
        Hq = case.get("q_heads", 0)
        qkv = _normal(g, (T, Hq + 2 * H, D), t, 2.0)
        st.update(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + H], v=qkv[:, Hq + H:])
    elif kind == "attend":
        # scores that a cap bends
        st["q"] = _normal(g, (T, case["q_heads"], D), t, 8.0 if case["cap"] else 2.0)
    if kind in ("attend", "layer"):
        # the usual slopes: a geometric sequence from 2^(-8 / heads) to 2^-8
        n = case["q_heads"]
        st["slopes"] = _dev((2.0 ** (-8.0 * (np.arange(n) + 1) / n)).astype(np.float32)) if case["bias"] else None
    if own:
        kv = _kv()
        k, v = st["pages"]
        if case["cache"] == "fp4":
            f4, e8 = torch.float4_e2m1fn_x2, torch.float8_e8m0fnu
            st["cache"] = kv.PagedCache(k.view(f4), v.view(f4), k_exp=st["exps"][0].view(e8), v_exp=st["exps"][1].view(e8))
        else:
            st["cache"] = kv.PagedCache(k, v, k_scale=st["scales"][0], v_scale=st["scales"][1])
        if kind != "attend":
            st.update(k_out=torch.empty((T, H, D), dtype=t, device=DEV), v_out=torch.empty((T, H, D), dtype=t, device=DEV))
        if kind in ("attend", "layer"):
            Hq = case["q_heads"]
            st.update(plan=kv.Plan(R, T, Hq, H, D, max_new=st["max_new"], window=case["window"]),
                      out=torch.empty((T, Hq, D), dtype=t, device=DEV),
                      lse=torch.empty((T, Hq), dtype=torch.float32, device=DEV))
            if kind == "attend":
                st["plan"].make(st["q_off"], st["kv_len"])
    return st


# ---------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------
def run(st):
    kind = st["case"]["kind"]
    if not own:
        return {"store": _plain_store, "read": _plain_read, "attend": _plain_attend, "layer": _plain_layer}[kind](st)
    kv, where, got = _kv(), (st["cache"], st["page_table"], st["q_off"], st["kv_len"]), {}
    if kind == "layer":
        st["plan"].make(st["q_off"], st["kv_len"])
    if kind in ("store", "layer"):
        kv.append(*where, st["k"], st["v"])
    if kind in ("attend", "layer"):
        got["out"] = kv.attend(st["q"], st["cache"], st["page_table"], st["plan"], scale=st["scale"], out=st["out"],
                               lse=st["lse"], cap=st["case"]["cap"], slopes=st["slopes"])
        got["lse"] = st["lse"]
    if kind != "attend":
        got["k"], got["v"] = kv.read(*where, k_out=st["k_out"], v_out=st["v_out"])
    return got


def _places(st):
    """Request and place in its request (negative: padding) of every new token."""
    token = torch.arange(st["tokens"], device=DEV)
    r = torch.searchsorted(st["q_off"][1:], token, right=True)
    return r, st["kv_len"].long()[r] - (st["q_off"][r + 1] - token)


def _where(st):
    """Page and slot of every new token, and whether it is in the cache."""
    r, at = _places(st)
    real, at, P = at >= 0, at.clamp(min=0), st["case"]["page"]
    return st["page_table"][r, at // P].long().clamp(min=0), at % P, real


def _plain_enter(st):
    page, slot, real = _where(st)
    for x, pages, exps in zip((st["k"], st["v"]), st["pages"], st["exps"]):
        code, k = _quantised(x[real].float(), st["case"]["dtype"])
        pages[page[real], :, slot[real]] = _packed(code)
        exps[page[real], :, slot[real]] = (k + 127).to(torch.uint8)


def _side(st, side, index):
    """float32 values of the cache's keys (0) or values (1) at an index of pages, heads, slots."""
    if st["case"]["cache"] == "fp4":
        return _values(_unpacked(st["pages"][side][index]), st["exps"][side][index].int() - 127)
    pages, t = st["pages"][side], st["pages"][side].dtype
    # bytes are moved as whole numbers: torch indexes no 8-bit floats
    return pages.view(torch.uint8)[index].view(t).float() if t == TYPES["fp8"] else pages[index].float()


def _plain_read(st):
    page, slot, real = _where(st)
    got = {}
    for s, name in enumerate("kv"):
        x = _side(st, s, (page, slice(None), slot))
        if st["scales"][s] is not None:
            x = x * st["scales"][s][:, None]
        got[name] = torch.where(real[:, None, None], x, 0.0).to(TYPES[st["case"]["dtype"]])
    return got


def _plain_store(st):
    _plain_enter(st)
    return _plain_read(st)


def _gathered(st, side, width):
    """float32 [requests, kv_heads, width * page, dim] of the requests' pages."""
    x = _side(st, side, st["page_table"][:, :width].clamp(min=0).long())
    if st["scales"][side] is not None:
        x = x * st["scales"][side][:, None, None]
    return x.permute(0, 2, 1, 3, 4).flatten(2, 3)


def _plain_attend(st):
    c, q = st["case"], st["q"]
    H, D, G = c["kv_heads"], c["dim"], c["q_heads"] // c["kv_heads"]
    r, at = _places(st)
    i = torch.arange(q.shape[0], device=DEV) - st["q_off"][r]
    R, N = st["kv_len"].numel(), st["max_new"]
    width = max(1, -(-st["max_kv"] // c["page"]))
    qp = torch.zeros((R, N, H, G, D), device=DEV)
    qp[r, i] = q.float().view(-1, H, G, D)
    place = torch.full((R, N), -1, dtype=torch.long, device=DEV)
    place[r, i] = at
    s = torch.matmul(qp.permute(0, 2, 3, 1, 4).reshape(R, H, G * N, D), _gathered(st, 0, width).transpose(-1, -2))
    s = s.view(R, H, G, N, -1)
    s *= st["scale"]
    j = torch.arange(s.shape[-1], device=DEV)
    if c["cap"]:
        s.div_(c["cap"]).tanh_().mul_(c["cap"])
    if st["slopes"] is not None:
        s.addcmul_(st["slopes"].view(H, G, 1, 1), (j - place[..., None])[:, None, None].float())
    hidden = j > place[..., None]
    if c["window"]:
        hidden |= j <= place[..., None] - c["window"]
    s.masked_fill_(hidden[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    s.sub_(m).exp_()
    l = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(R, H, G * N, -1), _gathered(st, 1, width)).view(R, H, G, N, D)
    o = o / torch.where(l == 0, torch.ones_like(l), l)
    lse = (m + l.log()).squeeze(-1)
    return dict(out=o.permute(0, 3, 1, 2, 4)[r, i].reshape(-1, H * G, D).to(q.dtype),
                lse=lse.permute(0, 3, 1, 2)[r, i].reshape(-1, H * G))


def _plain_layer(st):
    new = _plain_store(st)
    return dict(new, **_plain_attend(st))


# ---------------------------------------------------------------------------------------
# The same from the definitions, in 64 bits and one request after another
# ---------------------------------------------------------------------------------------
def _exact_group(x, kind):
    """What groups of 32 numbers [..., 32] become in 4 bits: the nearest of the sixteen multiples, of
    two equally near ones that with the even code."""
    top = x.abs().amax(-1, keepdim=True)
    lo, hi = EXPONENTS[kind]
    unit = torch.full_like(top, 2.0 ** lo)
    for k in range(lo, hi):
        unit = torch.where(top > 7 * 2.0 ** k, 2.0 ** (k + 1), unit)
    y, best, far = x.abs() / unit, torch.zeros_like(x), torch.full_like(x, math.inf)
    for code in (0, 2, 4, 6, 1, 3, 5, 7):  # even ones first: an odd one has to be nearer
        v = code / 2 if code < 4 else (2 + code % 2) * 2.0 ** (code // 2 - 2)
        d = (y - v).abs()
        best, far = torch.where(d < far, v, best), torch.minimum(d, far)
    return torch.copysign(best, x) * unit


def _exact_side(st, side, pages, head):
    """float64 [tokens, dim] of a head's rows in the given pages."""
    x = st["pages"][side][pages, head] if st["case"]["cache"] != "fp8" else \
        st["pages"][side].view(torch.uint8)[pages, head].view(TYPES["fp8"])
    if st["case"]["cache"] != "fp4":
        x = x.double()
        return (x if st["scales"][side] is None else x * st["scales"][side][head].double()).flatten(0, 1)
    out = torch.empty((*x.shape[:-1], st["case"]["dim"]), dtype=torch.float64, device=DEV)
    for nibble in range(2):
        c = (x >> 4 * nibble & 15).int()
        top, frac = c >> 1 & 3, (c & 1).double() / 2
        v = torch.where(top == 0, frac, (1 + frac) * torch.exp2((top - 1).double()))
        out[..., nibble::2] = torch.where(c >= 8, -v, v)
    e = torch.exp2(st["exps"][side][pages, head].double() - 127).repeat_interleave(GROUP, -1)
    return (out * e).flatten(0, 1)


def exact(case, seed):
    st = prepare(case, seed)
    off, lens, table = st["q_off"].tolist(), st["kv_len"].tolist(), st["page_table"].long()
    P, H, D, T = case["page"], case["kv_heads"], case["dim"], st["tokens"]
    got = {}
    if case["kind"] in ("store", "layer"):
        in_cache = torch.zeros(T, dtype=torch.bool, device=DEV)
        for r, L in enumerate(lens):
            in_cache[max(off[r], off[r + 1] - L):off[r + 1]] = True
        for n in "kv":
            x = torch.cat([_exact_group(part.double().unflatten(-1, (-1, GROUP)), case["dtype"]).flatten(-2)
                           for part in st[n].split(max(1, (1 << 23) // (H * D)))])
            got[n] = torch.where(in_cache[:, None, None], x, 0.0)
    if case["kind"] == "store":
        return got
    if case["kind"] == "read":
        for s, n in enumerate("kv"):
            got[n] = torch.zeros((T, H, D), dtype=torch.float64, device=DEV)
            for r, L in enumerate(lens):
                for h in range(H if L else 0):
                    got[n][off[r]:off[r + 1], h] = _exact_side(st, s, table[r, :-(-L // P)], h)[:L]
        return got
    G = case["q_heads"] // H
    out = torch.zeros((T, H, G, D), dtype=torch.float64, device=DEV)
    lse = torch.full((T, H, G), -math.inf, dtype=torch.float64, device=DEV)
    for r, L in enumerate(lens):
        a, z = off[r], off[r + 1]
        if L == 0 or a == z:
            continue
        at = L - (z - torch.arange(a, z, device=DEV))
        key = torch.arange(L, device=DEV)
        seen = key[None] <= at[:, None]
        if case["window"]:
            seen &= key[None] > at[:, None] - case["window"]
        for h in range(H):
            k, v = (_exact_side(st, s, table[r, :-(-L // P)], h)[:L] for s in range(2))
            if case["kind"] == "layer":  # the step's own tokens are in the cache by then
                first = max(a, z - L)
                k[L - (z - first):], v[L - (z - first):] = got["k"][first:z, h], got["v"][first:z, h]
            for g in range(G):
                s = st["q"][a:z, h * G + g].double() @ k.t() * st["scale"]
                if case["cap"]:
                    s = case["cap"] * torch.tanh(s / case["cap"])
                if st["slopes"] is not None:
                    s = s - st["slopes"][h * G + g].double() * (at[:, None] - key[None])
                s = torch.where(seen, s, -math.inf)
                lse[a:z, h, g] = torch.logsumexp(s, -1)
                out[a:z, h, g] = torch.nan_to_num(torch.exp(s - lse[a:z, h, g][:, None]), nan=0.0) @ v
    return dict(got, out=out.view(T, H * G, D), lse=lse.view(T, H * G))


# ---------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------
def work(case):
    H, D = case["kv_heads"], case["dim"]
    ctx, new = _lengths(case)
    kv_len, T, R = np.where(ctx < 0, 0, ctx + new), int(new.sum()), len(new)
    row = {"fp4": D // 2 + D // GROUP, "fp8": D}.get(case["cache"], 2 * D)  # of one head's keys or values
    pages = lambda tokens: 4 * int((-(-tokens // case["page"])).sum())  # noqa: E731
    nbytes, flops = 12 * R, 0
    if case["kind"] == "read":
        return dict(bytes=nbytes + pages(kv_len) + T * 2 * H * (row + 2 * D), flops=T * 2 * H * D)
    if case["kind"] in ("store", "layer"):
        # activations in, 4-bit rows out, activations out: what is read back has just been written
        nbytes += pages(new) + T * 2 * H * (2 * D + row + 2 * D)
        flops += T * 2 * H * D * 4
    if case["kind"] in ("attend", "layer"):
        Hq = case["q_heads"]
        # pairs of a token and a key that it sees; keys that any token of a request sees
        pairs, keys = 0, 0
        for L, n in zip(kv_len.tolist(), new.tolist()):
            at = np.arange(L - n, L)
            sees = np.maximum(0, at + 1 if not case["window"] else np.minimum(at + 1, case["window"]))
            pairs += int(sees.sum())
            keys += L if not case["window"] else min(L, case["window"] + n - 1)
        flops += 4 * pairs * Hq * D
        nbytes += pages(kv_len) + keys * 2 * H * row + T * Hq * (4 * D + 4)
    return dict(bytes=nbytes, flops=flops)
