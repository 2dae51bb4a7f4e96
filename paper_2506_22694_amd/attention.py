"""The attention of a drafter's layer: binding over include/vocabtrim_attention.h.

Norms of queries and keys with the position rotation (and their gradients), a paged key-value cache in 16, 8 or 4 bits,
and the attention of new tokens over it, with a sliding window and sinks where the layer has them.  As in binding.py, tensors supply memory and the current
stream; every step runs in the library's kernels, and what it refuses is raised.

Tensors of heads are [n, heads, head_dim]: rows may lie apart (views of one projection's output), a row's heads and
values may not.
"""
from __future__ import annotations

import ctypes

import torch
from torch.autograd import forward_ad

from . import binding
from .binding import VT_I32, VT_I64, _check, _dtype_code, _ptr, _require_cuda, _scratch, _stream, load_library

VT_E4M3, VT_E2M1 = 2, 4
GROUP = 32      # values of a 4-bit row that share a scale
VT_ROPE_HALVES, VT_ROPE_NEIGHBOURS = 0, 1


def rope_table(positions: int, rotary_dim: int, base: float = 10000.0, device="cuda",
               frequencies: torch.Tensor | None = None) -> torch.Tensor:
    """float32 [positions, rotary_dim]: cosines of every position's angles, then their sines.

    Angles are products in 64 bits: far positions keep theirs.  `frequencies` ([rotary_dim / 2], per position) replaces
    base^(-2 i / rotary_dim)."""
    if frequencies is None:
        frequencies = base ** (-torch.arange(0, rotary_dim, 2, dtype=torch.float64, device=device) / rotary_dim)
    elif tuple(frequencies.shape) != (rotary_dim // 2,):
        raise ValueError("frequencies must be [rotary_dim / 2]")
    angle = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * frequencies.to(device=device, dtype=torch.float64)
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


# --------------------------------------------------------------------------- arguments
# The native way (csrc/vt_bind.cpp) checks, makes the results and calls; it answers None to a call that is not plain, which goes on below.
def _got(got):
    if type(got) is int:
        _check(got)
    return got


def _no_tangent(*tensors) -> None:
    """Refuses dual tensors: no call here has a derivative in forward mode."""
    if getattr(forward_ad, "_current_level", 0) < 0:      # (most often: no level is open, so there are none; 2.8 us a call to ask the tensors)
        return
    if any(isinstance(t, torch.Tensor) and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise ValueError("no tangent comes back from here: there is no derivative in forward mode")


def _no_gradient(*tensors) -> None:
    """Refuses what a gradient is asked for of, where there would be none."""
    _no_tangent(*tensors)
    if torch.is_grad_enabled() and any(isinstance(t, torch.Tensor) and t.requires_grad for t in tensors):
        raise ValueError("no gradient comes back from here: detach what requires one, or call under torch.no_grad() (qk_norm_rope has gradients of q, k and "
                         "the weights)")


def _heads(t: torch.Tensor, n: int, heads: int, D: int, dtype) -> int:
    """The row stride of a tensor of heads, checked."""
    if not t.is_cuda or t.dtype != dtype or t.dim() != 3 or tuple(t.shape) != (n, heads, D):
        raise ValueError(f"expected a device tensor [{n}, {heads}, {D}] of {dtype}, got {list(t.shape)} of {t.dtype}")
    row, head, one = t.stride()
    if (D > 1 and one != 1) or (heads > 1 and head != D):
        raise ValueError("a row's heads and values must be contiguous")
    return row if n > 1 else heads * D


def _index(t: torch.Tensor, n: int, what: str) -> int:
    if t.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"{what} must be int32 or int64")
    if t.numel() != n or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous device tensor of {n} values")
    return VT_I32 if t.dtype == torch.int32 else VT_I64


def _norm_arguments(q, n, D, positions, table, q_weight, k_weight, eps, interleaved):
    """The arguments that the forward, the backward and the cache's calls share: weights to positions."""
    if (q_weight is None) != (k_weight is None):
        raise ValueError("give both weights or neither")
    if (table is None) != (positions is None):
        raise ValueError("give both positions and table or neither")
    for w in (q_weight, k_weight):
        if w is not None and (not w.is_cuda or not w.is_contiguous() or w.dtype != q.dtype or w.numel() != D):
            raise ValueError("weights must be contiguous device tensors [head_dim] of the element type")
    rows, rot, pos_type = 0, 0, VT_I32
    if table is not None:
        if not table.is_cuda or not table.is_contiguous() or table.dtype != torch.float32 or table.dim() != 2:
            raise ValueError("table must be a contiguous float32 device tensor [positions, rotary_dim]")
        rows, rot = table.shape
        pos_type = _index(positions, n, "positions")
    return (_ptr(q_weight), _ptr(k_weight), eps, _ptr(table), rows, rot, VT_ROPE_NEIGHBOURS if interleaved else VT_ROPE_HALVES,
            _ptr(positions), pos_type)


# --------------------------------------------------------------------------- norm and rotation
def _own_rows(g: torch.Tensor) -> torch.Tensor:
    """A gradient as the library takes it: those of sums and broadcasts have no rows of their own, pieces of one may begin anywhere."""
    g = g.contiguous()
    return g if g.data_ptr() % 16 == 0 else g.clone()


class _QkNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, positions, table, q_weight, k_weight, eps, interleaved):
        ctx.save_for_backward(q, k, positions, table, q_weight, k_weight)
        ctx.eps, ctx.interleaved = eps, interleaved
        return _qk_norm_rope(q, k, positions, table, q_weight, k_weight, eps, interleaved, None, None)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gq, gk):
        q, k, positions, table, q_weight, k_weight = ctx.saved_tensors
        dq, dk, dqw, dkw = qk_norm_rope_backward(_own_rows(gq), _own_rows(gk), q, k, positions, table, q_weight, k_weight, ctx.eps, ctx.interleaved)
        if dqw is not None:
            dqw, dkw = dqw.view_as(q_weight).to(q_weight.dtype), dkw.view_as(k_weight).to(k_weight.dtype)
        return dq, dk, None, None, dqw, dkw, None, None


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor | None = None, table: torch.Tensor | None = None,
                 q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None, eps: float = 1e-6,
                 interleaved: bool = False, q_out: torch.Tensor | None = None, k_out: torch.Tensor | None = None):
    """Norm of each head of q [n, q_heads, D] and k [n, k_heads, D], then the rotation of its first table.shape[1] values at
    the row's position: (q', k') in their type.  Without weights no norm, without a table no rotation.

    `q_out` / `k_out` supply the results (q and k themselves, say).  Where a gradient is asked for, it comes from
    qk_norm_rope_backward (there is no forward mode); a program that captures its backward pass in a graph calls that itself."""
    if binding._bind is not None:
        got = binding._bind.norm(q, k, positions, table, q_weight, k_weight, eps, interleaved, q_out, k_out)
        if got is not None:
            return _got(got)
    _no_gradient(table, q_out, k_out)
    _no_tangent(q, k, q_weight, k_weight)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (q, k, q_weight, k_weight)):
        if q_out is not None or k_out is not None:
            raise ValueError("q_out and k_out are for calls without gradients")
        return _QkNormRope.apply(q, k, positions, table, q_weight, k_weight, eps, interleaved)
    return _qk_norm_rope(q, k, positions, table, q_weight, k_weight, eps, interleaved, q_out, k_out)


def _qk_norm_rope(q, k, positions, table, q_weight, k_weight, eps, interleaved, q_out, k_out):
    L = load_library()
    n, hq, D = q.shape
    hk = k.shape[1]
    qs, ks = _heads(q, n, hq, D, q.dtype), _heads(k, n, hk, D, q.dtype)
    norm = _norm_arguments(q, n, D, positions, table, q_weight, k_weight, eps, interleaved)
    if q_out is None:
        q_out = torch.empty((n, hq, D), dtype=q.dtype, device=q.device)
    if k_out is None:
        k_out = torch.empty((n, hk, D), dtype=q.dtype, device=q.device)
    _check(L.vt_qk_norm_rope(_ptr(q), qs, _ptr(k), ks, _dtype_code(q), n, hq, hk, D, *norm, _ptr(q_out), _heads(q_out, n, hq, D, q.dtype),
                             _ptr(k_out), _heads(k_out, n, hk, D, q.dtype), _stream(q.device)))
    return q_out, k_out


def qk_norm_rope_backward(gq: torch.Tensor, gk: torch.Tensor, q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor | None = None,
                          table: torch.Tensor | None = None, q_weight: torch.Tensor | None = None,
                          k_weight: torch.Tensor | None = None, eps: float = 1e-6, interleaved: bool = False,
                          dq: torch.Tensor | None = None, dk: torch.Tensor | None = None, ws: torch.Tensor | None = None):
    """Gradients of qk_norm_rope from those of its results, (dq, dk, dq_weight, dk_weight): the weights' in float32 [D] (None
    without weights).  `dq` / `dk` supply the results (gq and gk themselves, say).  They are numbers: no graph leads through here."""
    L = load_library()
    if binding._bind is not None and dq is None and dk is None and ws is None:
        got = binding._bind.norm_backward(gq, gk, q, k, positions, table, q_weight, k_weight, eps, interleaved)
        if got is not None:
            return _got(got)
    _no_tangent(gq, gk, q, k, table, q_weight, k_weight, dq, dk)
    n, hq, D = q.shape
    hk = k.shape[1]
    qs, ks = _heads(q, n, hq, D, q.dtype), _heads(k, n, hk, D, q.dtype)
    gqs, gks = _heads(gq, n, hq, D, q.dtype), _heads(gk, n, hk, D, q.dtype)
    norm = _norm_arguments(q, n, D, positions, table, q_weight, k_weight, eps, interleaved)
    dev = q.device
    if dq is None:
        dq = torch.empty((n, hq, D), dtype=q.dtype, device=dev)
    if dk is None:
        dk = torch.empty((n, hk, D), dtype=q.dtype, device=dev)
    dqw = dkw = None
    if q_weight is not None:
        dqw, dkw = torch.empty((2, D), dtype=torch.float32, device=dev).unbind(0)
        if ws is None:
            ws = _scratch(L.vt_qk_norm_rope_backward_ws_bytes(n, D), dev)
    _require_cuda(ws)
    _check(L.vt_qk_norm_rope_backward(_ptr(gq), gqs, _ptr(gk), gks, _ptr(q), qs, _ptr(k), ks, _dtype_code(q), n, hq, hk, D, *norm,
                                      _ptr(dq), _heads(dq, n, hq, D, q.dtype), _ptr(dk), _heads(dk, n, hk, D, q.dtype), _ptr(dqw),
                                      _ptr(dkw), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(), _stream(dev)))
    return dq, dk, dqw, dkw


# --------------------------------------------------------------------------- the cache
class _CacheStruct(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("type", ctypes.c_int32), ("pages", ctypes.c_int64), ("heads", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("head_dim", ctypes.c_int32)]


class KVCache:
    """A paged key-value cache on the device: k and v [pages, heads, page_size, head_dim], bfloat16 or float8_e4m3fn with the
    exponents of its scales [pages, heads, page_size] (uint8).  In 4 bits, float4_e2m1fn_x2 (two values to a byte, the first in
    its lower half), k and v are [pages, heads, page_size, head_dim / 2], head_dim a multiple of 32, and the scales' exponents
    [pages, heads, head_dim / 32, page_size].  Its memory needs no initialisation.  A slot is page * page_size + place."""

    def __init__(self, pages: int, page_size: int, heads: int, head_dim: int, dtype: torch.dtype = torch.bfloat16, device="cuda"):
        four = dtype == torch.float4_e2m1fn_x2
        if four and head_dim % GROUP:
            raise ValueError("head_dim of a 4-bit cache must be a multiple of 32")

        def held():
            return torch.empty((pages, heads, page_size, head_dim // 2 if four else head_dim), dtype=dtype, device=device)

        def scale():
            if dtype == torch.bfloat16:
                return None
            return torch.empty((pages, heads, head_dim // GROUP, page_size) if four else (pages, heads, page_size), dtype=torch.uint8, device=device)

        self._set(held(), held(), scale(), scale())

    @classmethod
    def of(cls, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor | None = None, v_scale: torch.Tensor | None = None) -> "KVCache":
        """A cache in the caller's tensors."""
        cache = cls.__new__(cls)
        cache._set(k, v, k_scale, v_scale)
        return cache

    def _set(self, k, v, k_scale, v_scale):
        held = {torch.bfloat16: 1, torch.float8_e4m3fn: VT_E4M3, torch.float4_e2m1fn_x2: VT_E2M1}.get(k.dtype)
        if held is None:
            raise TypeError(f"unsupported element type of a cache {k.dtype}")
        if k.dim() != 4 or v.shape != k.shape or v.dtype != k.dtype:
            raise ValueError("k and v must be [pages, heads, page_size, head_dim] of one type")
        pages, heads, page_size, head_dim = k.shape
        scales = (pages, heads, page_size)
        if held == VT_E2M1:
            head_dim *= 2
            scales = (pages, heads, head_dim // GROUP, page_size)
        for s in (k_scale, v_scale):
            if (s is not None) != (held != 1) or (s is not None and (tuple(s.shape) != scales or s.dtype != torch.uint8)):
                raise ValueError("k_scale and v_scale must be uint8 [pages, heads, page_size] of an 8-bit cache, [pages, heads, head_dim / 32, page_size] of a "
                                 "4-bit one, and are not of a 16-bit one")
        _no_gradient(k, v)
        _require_cuda(k, v, k_scale, v_scale)
        self._tensors = (k, v, k_scale, v_scale)
        self._struct = _CacheStruct(_ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale), held, pages, heads, page_size, head_dim)
        self._address = ctypes.addressof(self._struct)

    k = property(lambda self: self._tensors[0])
    v = property(lambda self: self._tensors[1])
    k_scale = property(lambda self: self._tensors[2])
    v_scale = property(lambda self: self._tensors[3])
    pages = property(lambda self: self._struct.pages)
    heads = property(lambda self: self._struct.heads)
    page_size = property(lambda self: self._struct.page_size)
    head_dim = property(lambda self: self._struct.head_dim)

    def slots(self, page_table: torch.Tensor, request: torch.Tensor, token: torch.Tensor) -> torch.Tensor:
        """Slots (int64) of tokens `token` of requests `request`, by a page table [requests, pages of each]."""
        page = page_table[request.long(), torch.div(token, self.page_size, rounding_mode="floor").long()].long()
        return page * self.page_size + token % self.page_size


def qkv_to_cache(q: torch.Tensor | None, k: torch.Tensor, v: torch.Tensor, cache: KVCache, slots: torch.Tensor,
                 positions: torch.Tensor | None = None, table: torch.Tensor | None = None, q_weight: torch.Tensor | None = None,
                 k_weight: torch.Tensor | None = None, eps: float = 1e-6, interleaved: bool = False,
                 q_out: torch.Tensor | None = None):
    """qk_norm_rope on q and k, with k and v written to the cache at `slots` (outside it: not written), in one launch.
    Returns q' (None without q).  Inputs that require a gradient are refused: none comes back from a cache."""
    L = load_library()
    if binding._bind is not None and q is not None and type(cache) is KVCache:
        got = binding._bind.to_cache(q, k, v, cache._address, slots, positions, table, q_weight, k_weight, eps, interleaved, q_out)
        if got is not None:
            return _got(got)
    _no_gradient(q, k, v, table, q_weight, k_weight, q_out)
    n, hk, D = k.shape
    if hk != cache.heads or D != cache.head_dim:
        raise ValueError("k and v must have the cache's heads")
    ks, vs = _heads(k, n, hk, D, k.dtype), _heads(v, n, hk, D, k.dtype)
    hq = qs = qos = 0
    if q is not None:
        hq = q.shape[1]
        qs = _heads(q, n, hq, D, k.dtype)
        if q_out is None:
            q_out = torch.empty((n, hq, D), dtype=q.dtype, device=q.device)
        qos = _heads(q_out, n, hq, D, k.dtype)
    elif q_out is not None:
        raise ValueError("q_out without q")
    norm = _norm_arguments(k, n, D, positions, table, q_weight, k_weight, eps, interleaved)
    _check(L.vt_qkv_to_cache(_ptr(q), qs, _ptr(k), ks, _ptr(v), vs, _dtype_code(k), n, hq, *norm, _ptr(q_out), qos, cache._address,
                             _ptr(slots), _index(slots, n, "slots"), _stream(k.device)))
    return q_out


def kv_cache_write(cache: KVCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor) -> None:
    """k and v [n, heads, head_dim] into the cache as they are, at `slots` (outside it: not written)."""
    qkv_to_cache(None, k, v, cache, slots)


def kv_cache_read(cache: KVCache, slots: torch.Tensor, dtype: torch.dtype = torch.bfloat16, k_out: torch.Tensor | None = None,
                  v_out: torch.Tensor | None = None):
    """The cache's rows at `slots` as values, (k, v) [n, heads, head_dim]; zeros for slots outside it."""
    L = load_library()
    if binding._bind is not None and k_out is None and v_out is None and type(cache) is KVCache and dtype in (torch.bfloat16, torch.float32):
        got = binding._bind.cache_read(cache._address, slots, dtype == torch.float32)
        if got is not None:
            return _got(got)
    _no_gradient(k_out, v_out)
    n = slots.numel()
    shape = (n, cache.heads, cache.head_dim)
    if k_out is None:
        k_out = torch.empty(shape, dtype=dtype, device=slots.device)
    if v_out is None:
        v_out = torch.empty(shape, dtype=dtype, device=slots.device)
    _require_cuda(k_out, v_out)
    for t in (k_out, v_out):
        if tuple(t.shape) != shape or t.dtype != k_out.dtype:
            raise ValueError("k_out and v_out must be [n, heads, head_dim] of one type")
    _check(L.vt_kv_cache_read(cache._address, _ptr(slots), _index(slots, n, "slots"), n, _ptr(k_out), _ptr(v_out), _dtype_code(k_out),
                              _stream(slots.device)))
    return k_out, v_out


# --------------------------------------------------------------------------- attention
class AttentionWorkspace:
    """Device scratch of paged_attention: allocated once (no initialisation needed), for calls of up to these sizes."""

    def __init__(self, n: int, q_heads: int, kv_heads: int, head_dim: int, requests: int, max_rows: int, max_length: int, device):
        self.buf = _scratch(load_library().vt_paged_attention_ws_bytes(n, q_heads, kv_heads, head_dim, requests, max_rows, max_length), device)

    @property
    def nbytes(self) -> int:
        return self.buf.numel()


def paged_attention(q: torch.Tensor, cache: KVCache, page_table: torch.Tensor, lengths: torch.Tensor,
                    row_start: torch.Tensor | None = None, max_rows: int | None = None, tail_mask: torch.Tensor | None = None,
                    max_length: int | None = None, scale: float | None = None, ws: AttentionWorkspace | None = None,
                    out: torch.Tensor | None = None, return_lse: bool = False, out_lse: torch.Tensor | None = None,
                    window: int | None = None, sinks: int = 0, positions: torch.Tensor | None = None):
    """Attention of q [n, q_heads, head_dim] over the cached tokens of their requests: out like q [, lse float32 [n, q_heads]].

    page_table int32 [requests, pages of each], lengths int32 [requests].  Row i is request i's, or rows
    row_start[b] .. row_start[b + 1] - 1 are request b's, at most max_rows (other rows are not computed).  tail_mask (int64 [n], its bits): which of
    the last 64 tokens a row sees, bit j being token length - 64 + j.  scale: of the scores (head_dim^-1/2).
    max_length: no request is longer (the page table's width, where it isn't given; near the longest is fastest).

    window, sinks: the row at position p sees no tokens but t > p - window and t < sinks, and only those of a request are read that
    some row sees.  A request's rows are its last tokens and, without a tail mask, see none behind themselves: a prompt's chunk
    whose keys are cached.  With a tail mask the nodes of a tree may have `positions` (int32 or int64 [n]; the prompt's length plus
    their depth), which count from the first of the last 64 tokens on.  A window of max_length and more: all tokens up to the row's own.

    Without a window a row sees all cached tokens of its request that no tail mask hides, those of the request's later rows too: a causal
    prompt on a layer without a window is window=max_length.
    A q that requires a gradient is refused: there is none."""
    L = load_library()
    if binding._bind is not None and type(ws) is AttentionWorkspace and type(cache) is KVCache:
        got = binding._bind.attend(q, cache._address, page_table, lengths, row_start, max_rows, tail_mask, max_length, scale, ws.buf, out, return_lse,
                                   out_lse, window, sinks, positions)
        if got is not None:
            return _got(got)
    _no_gradient(q, out, out_lse)
    n, hq, D = q.shape
    _require_cuda(page_table, lengths, row_start, tail_mask, out_lse)
    if page_table.dtype != torch.int32 or page_table.dim() != 2 or lengths.dtype != torch.int32:
        raise ValueError("page_table must be int32 [requests, pages] and lengths int32")
    requests, pages = page_table.shape
    if D != cache.head_dim or lengths.numel() != requests:
        raise ValueError("shape mismatch between q, cache, page_table and lengths")
    if row_start is None:
        if max_rows is None:
            max_rows = 1
    elif max_rows is None:
        raise ValueError("max_rows: the most rows that a request has")
    elif row_start.dtype != torch.int32 or row_start.numel() != requests + 1:
        raise ValueError("row_start must be int32 [requests + 1]")
    if tail_mask is not None and (tail_mask.dtype not in (torch.int64, torch.uint64) or tail_mask.numel() != n):
        raise ValueError("tail_mask must be int64 [n]")
    if window is None and (sinks != 0 or positions is not None):
        raise ValueError("sinks and positions are a window's")
    if positions is not None and tail_mask is None:
        raise ValueError("positions go with a tail mask: without one a request's rows are its last tokens")
    pos_type = VT_I32 if positions is None else _index(positions, n, "positions")
    if max_length is None:
        max_length = pages * cache.page_size
    if scale is None:
        scale = D ** -0.5
    dev = q.device
    if out is None:
        out = torch.empty((n, hq, D), dtype=q.dtype, device=dev)
    if out_lse is not None:
        if out_lse.dtype != torch.float32 or out_lse.numel() != n * hq:
            raise ValueError("out_lse must be float32 [n, q_heads]")
    elif return_lse:
        out_lse = torch.empty((n, hq), dtype=torch.float32, device=dev)
    if ws is None:
        ws = AttentionWorkspace(n, hq, cache.heads, D, requests, max_rows, max_length, dev)
    what = (_ptr(q), _heads(q, n, hq, D, q.dtype), _dtype_code(q), n, hq, cache._address, _ptr(page_table), pages, _ptr(lengths), requests, _ptr(row_start),
            max_rows, _ptr(tail_mask))
    how = (max_length, scale, _ptr(out), _heads(out, n, hq, D, q.dtype), _ptr(out_lse), _ptr(ws.buf), ws.nbytes, _stream(dev))
    if window is None:
        _check(L.vt_paged_attention(*what, *how))
    else:
        _check(L.vt_paged_attention_window(*what, _ptr(positions), pos_type, window, sinks, *how))
    return (out, out_lse) if return_lse else out
