"""Plain 64-bit forms of the paged-cache operators, on the CPU, with the bounds that their
float32 computation and its roundings allow."""
import math

import torch

FP8 = torch.float8_e4m3fn
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # largest relative error of one rounding to 8, 11 bits
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}  # half the smallest value's distance to zero
F32 = 2.0 ** -24


def turn(x, weight, table, rot, interleaved, pos, eps=1e-6):
    """(y, bound on the float32 computation's error) of x [tokens, heads, dim] in float64."""
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps) * weight.double()
    size = y.abs().clone()
    if rot:
        n = rot // 2
        a = torch.arange(n)
        b = a + n
        if interleaved:
            a, b = 2 * torch.arange(n), 2 * torch.arange(n) + 1
        cos, sin = table.double()[pos][:, None].split(n, -1)
        ya, yb = y[..., a], y[..., b]
        out = y.clone()
        out[..., a], out[..., b] = ya * cos - yb * sin, yb * cos + ya * sin
        s = size.clone()
        size[..., a] = size[..., b] = s[..., a] + s[..., b]
        y = out
    # the mean square's sum (dim terms), root, quotient and two products, then the rotation's three
    return y, size * F32 * (x.shape[-1] / 16 + 16)


def close(got, want, slack, dtype):
    """got (rounded once to dtype) within one rounding of want and the computation's slack."""
    err = (got.double().cpu() - want).abs()
    bound = UNIT[dtype] * (want.abs() + slack) + slack + TINY[dtype]
    assert bool((err <= bound).all()), float((err - bound).max())


def close_e4m3(got, want, slack):
    """got within half a step of want / scale saturated: 3 fraction bits, steps of 2^-9 below 2^-6."""
    want = want.clamp(-448, 448)
    err = (got.float().double().cpu() - want).abs()
    bound = torch.maximum((want.abs() + slack) * 2.0 ** -4, torch.full_like(want, 2.0 ** -10)) + slack
    assert bool((err <= bound).all()), float((err - bound).max())


def attend(q, keys, values, n_kv, scale, window, kv_len, n_new):
    """One request: q [n_new, n_q, dim], keys and values [kv_len, n_kv, dim] (what the cache
    stands for), all float64.  (out, lse, sum of p |v|, largest sum of |q k|)."""
    n_q, D = q.shape[1:]
    G = n_q // n_kv
    out, mag = torch.zeros(n_new, n_q, D).double(), torch.zeros(n_new, n_q, D).double()
    lse, big = torch.full((n_new, n_q), -math.inf).double(), torch.zeros(n_new, n_q).double()
    for i in range(n_new):
        place = kv_len - n_new + i
        lo = max(0, place - window + 1) if window else 0
        if place + 1 <= lo:
            continue
        k, v = keys[lo:place + 1], values[lo:place + 1]
        for h in range(n_q):
            kk, vv = k[:, h // G], v[:, h // G]
            s = scale * (kk @ q[i, h])
            lse[i, h] = torch.logsumexp(s, 0)
            p = torch.exp(s - lse[i, h])
            out[i, h], mag[i, h] = p @ vv, p @ vv.abs()
            big[i, h] = scale * (kk.abs() @ q[i, h].abs()).max()
    return out, lse, mag, big


def close_attend(out, lse, want, dim, dtype):
    o, l, mag, big = want
    # a score is off by at most dim roundings of its products' sum, a weight by that and its own
    # rounding to dtype, the weights' float32 sum by as little
    rel = 2 * big * dim * F32 + 2.0 ** -16
    slack = mag * (UNIT[dtype] * 1.01 + rel[..., None])
    close(out, o, slack, dtype)
    if lse is not None:
        got = lse.double().cpu()
        assert torch.equal(torch.isinf(got), torch.isinf(l))
        fine = torch.isfinite(l)
        err = (got - l)[fine].abs()
        assert bool((err <= (big * dim * F32 + (l.abs() + 4) * 8 * F32)[fine]).all()), float(err.max())
