"""The instance's side of a routed request: the paged KV cache and what writes and reads it.

A thin binding of include/smetric_kv.h (the calls themselves in csrc/kv_calls.cpp).  A step of a
model's layer on a batch of requests, each with one new token or a chunk of them:

    plan.make(q_off, kv_len)                                    # once per step
    q = kv.append(cache, table, q_off, kv_len, k, v, q=q, rotary=rotary)  # per layer
    out = kv.attend(q, cache, table, plan)

and, for an instance that hands a request's tokens on, kv.read of what the pages hold.  Tensors go
in by data pointer on torch's current stream of the current device, which has to be theirs; there is
no CPU fallback.
"""
from __future__ import annotations

import collections
import ctypes as C

import torch

from .smetric import EINVAL, SmetricError, _check, _dev, _lib

try:
    from . import _kv_calls
except ImportError as e:
    raise RuntimeError("_kv_calls.so is missing or does not fit: build it first (__graft_entry__.build())") from e

# two components a byte; a group's exponent (None where torch has no such type: no 4-bit caches then)
_E2M1, _E8M0 = getattr(torch, "float4_e2m1fn_x2", None), getattr(torch, "float8_e8m0fnu", None)
_DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float8_e4m3fn: 2, **({} if _E2M1 is None else {_E2M1: 3})}
GROUP = 32  # components of a 4-bit cache with one exponent


class _Kept:
    """Structures that callers of the library's entry points pass by address, also of one that was
    made for that call alone: C.addressof(_Cache(...)).  ctypes would free it before the call, so the
    last 64 stay, each with the structures that it points to (held).  The calls of this module hold
    theirs themselves."""
    _last: collections.deque = collections.deque(maxlen=64)
    held: tuple = ()

    def __init__(self, *fields, **named):
        super().__init__(*fields, **named)
        self._last.append(self)


class _Exps(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_stride", C.c_int64 * 3), ("v_stride", C.c_int64 * 3)]


class _Cache(_Kept, C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("n_pages", C.c_int64), ("k_stride", C.c_int64 * 3),
                ("v_stride", C.c_int64 * 3), ("page_size", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int32), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("exps", C.c_void_p)]


class _Rotary(_Kept, C.Structure):
    _fields_ = [("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("table", C.c_void_p), ("n_pos", C.c_int64),
                ("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("eps", C.c_float)]


def _opt(t: torch.Tensor | None, dtype: torch.dtype, name: str):
    return None if t is None else _dev(t, dtype, name)


def _device(*tensors: torch.Tensor | None) -> int:
    """The index of the device that all of them are on, -1 if there are none."""
    on = {t.get_device() for t in tensors if t is not None}
    if len(on) > 1:
        raise ValueError("tensors on different devices")
    return on.pop() if on else -1


class PagedCache:
    """Keys and values in pages: two tensors [n_pages, n_kv_heads, page_size, head_dim] of any
    strides with contiguous components (a view of another order is one), bfloat16, float16,
    float8_e4m3fn -- then with float32 scales per head: a stored x stands for x * scale -- or
    float4_e2m1fn_x2, whose last dimension is head_dim / 2 bytes of two components, with exponents
    k_exp and v_exp, float8_e8m0fnu [n_pages, n_kv_heads, page_size, head_dim / 32]: a stored x
    stands for x * 2^(e - 127)."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor | None = None,
                 v_scale: torch.Tensor | None = None, k_exp: torch.Tensor | None = None, v_exp: torch.Tensor | None = None):
        for t, name in ((k, "k"), (v, "v")):
            if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in _DTYPES or t.dim() != 4:
                raise TypeError(f"{name}: expected a CUDA tensor [pages, heads, page_size, head_dim] of 16, 8 or 4 bits")
            if t.stride(3) != 1:
                raise ValueError(f"{name}: components must be contiguous")
        if k.shape != v.shape or k.dtype != v.dtype:
            raise ValueError("k and v differ in shape or type")
        if (k_scale is None) != (v_scale is None):
            raise ValueError("k_scale and v_scale go together")
        if k_scale is not None and (k.dtype != torch.float8_e4m3fn or k_scale.numel() != k.shape[1] or
                                    v_scale.numel() != k.shape[1]):
            raise ValueError("scales: one per head of a float8_e4m3fn cache")
        per = 2 if k.dtype == _E2M1 else 1  # components of an element of the tensor
        exps = ((k_exp, "k_exp"), (v_exp, "v_exp"))
        for t, name in exps:
            if (t is None) == (per == 2):
                raise ValueError("k_exp and v_exp: both with a float4_e2m1fn_x2 cache, neither with another one")
            if t is not None and (not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != _E8M0):
                raise TypeError(f"{name}: expected a float8_e8m0fnu CUDA tensor")
            if t is not None and (t.shape != (*k.shape[:3], 2 * k.shape[3] // GROUP) or t.stride(3) != 1):
                raise ValueError(f"{name}: expected one per {GROUP} components, those of a token contiguous")
        self.k, self.v, self.k_scale, self.v_scale, self.k_exp, self.v_exp = k, v, k_scale, v_scale, k_exp, v_exp
        self.n_pages, self.n_kv_heads, self.page_size = k.shape[:3]
        self.head_dim = per * k.shape[3]
        self.dtype = k.dtype
        strides = lambda t, n: (C.c_int64 * 3)(*[n * x for x in t.stride()[:3]])  # noqa: E731
        self.c = _Cache(k.data_ptr(), v.data_ptr(), self.n_pages, strides(k, per), strides(v, per), self.page_size,
                        self.n_kv_heads, self.head_dim, _DTYPES[k.dtype], _opt(k_scale, torch.float32, "k_scale"),
                        _opt(v_scale, torch.float32, "v_scale"))
        if per == 2:
            self.exps = _Exps(k_exp.data_ptr(), v_exp.data_ptr(), strides(k_exp, 1), strides(v_exp, 1))
            self.c.exps, self.c.held = C.addressof(self.exps), (self.exps,)
        self.device = _device(k, v, k_scale, v_scale, k_exp, v_exp)
        self.ref = C.addressof(self.c)

    @classmethod
    def empty(cls, n_pages: int, n_kv_heads: int, head_dim: int, page_size: int = 16,
              dtype: torch.dtype = torch.bfloat16, device="cuda", **scales) -> "PagedCache":
        shape = (n_pages, n_kv_heads, page_size, head_dim)
        if _E2M1 is not None and dtype == _E2M1:
            # a page's two exponents of a head beside each other: at heads of 128 and pages of 16 one line of memory
            e = torch.empty((n_pages, n_kv_heads, 2, page_size, head_dim // GROUP), dtype=_E8M0, device=device)
            shape = (*shape[:3], head_dim // 2)
            scales = dict(scales, k_exp=e[:, :, 0], v_exp=e[:, :, 1])
        return cls(torch.empty(shape, dtype=dtype, device=device), torch.empty(shape, dtype=dtype, device=device), **scales)


class Rotary:
    """Norm weights (or None) and the table of angles: float32 [positions, rot_dim], a row the
    cosines then the sines of a position's rot_dim / 2 angles."""

    def __init__(self, table: torch.Tensor | None = None, rot_dim: int | None = None, interleaved: bool = False,
                 q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None, eps: float = 1e-6):
        rot_dim = (0 if table is None else table.shape[1]) if rot_dim is None else int(rot_dim)
        if rot_dim and (table is None or table.dim() != 2 or table.shape[1] != rot_dim):
            raise ValueError(f"table: expected [positions, {rot_dim}]")
        self.table, self.q_weight, self.k_weight, self.rot_dim = table, q_weight, k_weight, rot_dim
        w = [None if x is None else _dev(x, x.dtype, n) for x, n in ((q_weight, "q_weight"), (k_weight, "k_weight"))]
        self.c = _Rotary(w[0], w[1], _opt(table, torch.float32, "table") if rot_dim else None,
                         table.shape[0] if rot_dim else 0, rot_dim, int(interleaved), eps)
        self.device = _device(table if rot_dim else None, q_weight, k_weight)
        self.ref = C.addressof(self.c)


def _new(t: torch.Tensor, name: str) -> torch.Tensor:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a bfloat16 or float16 CUDA tensor [tokens, heads, head_dim]")
    return torch.empty(t.shape, dtype=t.dtype, device=t.device)


def qk_rotate(q: torch.Tensor, k: torch.Tensor, rotary: Rotary, positions: torch.Tensor | None = None,
              q_out: torch.Tensor | None = None, k_out: torch.Tensor | None = None, status: torch.Tensor | None = None):
    """smetric_qk_rotate: queries and keys [tokens, heads, head_dim] normed and rotated to
    their positions (int32).  Outputs may be the inputs.  Returns (q_out, k_out)."""
    q_out = _new(q, "q") if q_out is None else q_out
    k_out = _new(k, "k") if k_out is None else k_out
    rc = _kv_calls.qk_rotate(q, k, rotary.ref, rotary.q_weight, rotary.k_weight, positions, q_out, k_out, status,
                            rotary.device)
    if rc:
        raise SmetricError("smetric_qk_rotate", rc)
    return q_out, k_out


def append(cache: PagedCache, page_table: torch.Tensor, q_off: torch.Tensor, kv_len: torch.Tensor, k: torch.Tensor,
           v: torch.Tensor, q: torch.Tensor | None = None, q_out: torch.Tensor | None = None,
           rotary: Rotary | None = None, positions: torch.Tensor | None = None, status: torch.Tensor | None = None):
    """smetric_kv_append: the new tokens' keys (normed and rotated) and values into the pages, quantised
    where these hold 8 or 4 bits; kv_len counts the new tokens already.  With q its queries normed and rotated are
    returned (q_out, may be q)."""
    if q is not None and q_out is None:
        q_out = _new(q, "q")
    r = (0, None, None) if rotary is None else (rotary.ref, rotary.q_weight, rotary.k_weight)
    rc = _kv_calls.append(cache.ref, page_table, q_off, kv_len, k, v, q, q_out, *r, positions, status, cache.device,
                          -1 if rotary is None else rotary.device)
    if rc:
        raise SmetricError("smetric_kv_append", rc)
    return q_out if q is not None else None


def read(cache: PagedCache, page_table: torch.Tensor, q_off: torch.Tensor, kv_len: torch.Tensor,
         n_tokens: int | None = None, dtype: torch.dtype | None = None, k_out: torch.Tensor | None = None,
         v_out: torch.Tensor | None = None, status: torch.Tensor | None = None):
    """smetric_kv_read: the last q_off[r+1] - q_off[r] of request r's kv_len[r] cached tokens read
    back as activations, n_tokens = q_off[-1] of all requests.  Returns (k_out, v_out)
    [n_tokens, heads, head_dim], made of `dtype` (a 16-bit cache's own, else bfloat16) where not
    given; n_tokens and dtype are not needed beside one that is."""
    given = k_out if k_out is not None else v_out
    if given is None and n_tokens is None:
        raise ValueError("n_tokens: expected with no output given")
    if given is None or k_out is None or v_out is None:
        if dtype is None:
            dtype = given.dtype if given is not None else cache.dtype if cache.dtype.itemsize == 2 else torch.bfloat16
        n = given.shape[0] if given is not None else n_tokens
        make = lambda: torch.empty((n, cache.n_kv_heads, cache.head_dim), dtype=dtype, device=cache.k.device)  # noqa: E731
        k_out, v_out = make() if k_out is None else k_out, make() if v_out is None else v_out
    rc = _kv_calls.read(cache.ref, page_table, q_off, kv_len, k_out, v_out, status, cache.device)
    if rc:
        raise SmetricError("smetric_kv_read", rc)
    return k_out, v_out


class Plan:
    """How a step's attention is split over the GPU: made once per step from the lengths, used
    by every layer.  The buffers (plan and workspace) are kept; a plan serves any batch of the
    same n_req and n_tokens after another make().  They belong to the stream that is current
    here: work on another one has to end before the plan is dropped, as torch then hands
    their memory out again.  workspace: a contiguous uint8 tensor of ws_bytes, 256-byte
    aligned, which plans used in turn on one stream may share."""

    def __init__(self, n_req: int, n_tokens: int, n_q_heads: int, n_kv_heads: int, head_dim: int, max_new: int,
                 window: int = 0, device="cuda", workspace: torch.Tensor | None = None):
        self.args = (n_req, n_tokens, n_q_heads, n_kv_heads, head_dim, max_new)
        self.window = int(window)
        a, b = C.c_uint64(), C.c_uint64()
        _check("smetric_attend_plan_bytes", _lib.smetric_attend_plan_bytes(*self.args, C.byref(a), C.byref(b)))
        self.plan_bytes, self.ws_bytes = int(a.value), int(b.value)
        if torch.device(device).type != "cuda":
            raise TypeError("device: expected a CUDA device")
        if workspace is not None:
            _dev(workspace, torch.uint8, "workspace")
            if workspace.numel() < self.ws_bytes:
                raise SmetricError("smetric_attend_plan_bytes", EINVAL)
        self.mem = torch.empty(self.plan_bytes, dtype=torch.uint8, device=device)
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device) if workspace is None else workspace
        self.device = _device(self.mem, self.workspace)
        self.plan_ptr, self.ws_ptr = self.mem.data_ptr(), self.workspace.data_ptr()
        self.q_off = self.kv_len = None

    def make(self, q_off: torch.Tensor, kv_len: torch.Tensor, status: torch.Tensor | None = None) -> "Plan":
        """smetric_attend_plan for these lengths (device tensors, read on the current stream)."""
        rc = _kv_calls.make_plan(q_off, kv_len, *self.args, self.window, self.plan_ptr, self.plan_bytes, status,
                                 self.device)
        if rc:
            raise SmetricError("smetric_attend_plan", rc)
        self.q_off, self.kv_len = q_off, kv_len
        return self


def attend(q: torch.Tensor, cache: PagedCache, page_table: torch.Tensor, plan: Plan, scale: float | None = None,
           out: torch.Tensor | None = None, lse: torch.Tensor | None = None, status: torch.Tensor | None = None,
           cap: float = 0.0, slopes: torch.Tensor | None = None):
    """smetric_attend: the new tokens' attention over the pages, as `plan` (made for the batch)
    splits it.  scale: 1 / sqrt(head_dim) by default; lse (float32 [tokens, heads]) is
    filled if given.  cap: scores become cap * tanh(score / cap); slopes (float32 [heads]): they get a
    bias slopes[head] * (key's place - token's place) (smetric_attend_scores).  With bfloat16 and a cap up
    to 50.5, without slopes, values in the cache have to be 0 or between 2^-x and 2^x in magnitude, x =
    115 - 1.443 cap (2^42 at a cap of 50): others may count as 0 or infinite.  Returns out
    [tokens, heads, head_dim]."""
    if plan.kv_len is None:
        raise ValueError("plan: make() it for the batch first")
    _, T, Hq, H, D, max_new = plan.args
    if H != cache.n_kv_heads or D != cache.head_dim:
        raise ValueError("plan and cache differ in heads or head_dim")
    out = _new(q, "q") if out is None else out
    rc = _kv_calls.attend(q, out, lse, cache.ref, page_table, plan.q_off, plan.kv_len, T, Hq,
                          D ** -0.5 if scale is None else scale, max_new, plan.window, plan.plan_ptr, plan.plan_bytes,
                          plan.ws_ptr, plan.ws_bytes, status, cache.device, plan.device, cap, slopes)
    if rc:
        raise SmetricError("smetric_attend" if cap == 0 and slopes is None else "smetric_attend_scores", rc)
    return out
