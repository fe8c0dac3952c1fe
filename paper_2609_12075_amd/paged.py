"""Paged key/value cache: ctypes binding of include/vla_paged.h.

Keys and values of a layer live in pages of a pool (``KVPool``); a ``Batch``
says which tokens each request brings, how long its context then is and on
which pages it lies. ``append`` writes a step's keys and values (rotating
queries and keys on the way), ``attention`` attends over the cache and
``shared_attention`` reads a context that all requests begin with once for
the batch. Calls run on the pool's device, on `stream` or that device's
current stream; tensors that a call allocates belong to that stream (use on
another one waits for it, and tells the allocator by record_stream).
"""
from __future__ import annotations

import ctypes
import functools
from typing import Optional, Sequence

import torch

from . import vla

EXPORTS = ["vla_kv_append", "vla_attention_workspace", "vla_paged_attention", "vla_shared_attention",
           "vla_debug_paged_plan"]

_ci, _vp, _i64 = ctypes.c_int, ctypes.c_void_p, ctypes.c_int64


class KVPoolC(ctypes.Structure):
    _fields_ = [("device", _ci), ("dtype", _ci), ("n_kv", _ci), ("head_dim", _ci), ("page_tokens", _ci),
                ("n_pages", _ci), ("k", _vp), ("v", _vp), ("page_stride", _i64), ("head_stride", _i64),
                ("token_stride", _i64)]


class RaggedC(ctypes.Structure):
    _fields_ = [("n_req", _ci), ("n_tok", _ci), ("max_new", _ci), ("max_len", _ci), ("start", _vp), ("kv_len", _vp),
                ("pages", _vp), ("pages_stride", _ci)]


class AppendArgsC(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("k_tok_stride", _i64), ("k_head_stride", _i64), ("v_tok_stride", _i64),
                ("v_head_stride", _i64), ("n_q", _ci), ("q", _vp), ("q_out", _vp), ("q_tok_stride", _i64),
                ("q_head_stride", _i64), ("qo_tok_stride", _i64), ("qo_head_stride", _i64), ("n_axes", _ci),
                ("sections", _ci * 3), ("positions", _vp), ("rope_base", ctypes.c_float)]


class AttentionArgsC(ctypes.Structure):
    _fields_ = [("q", _vp), ("o", _vp), ("q_tok_stride", _i64), ("q_head_stride", _i64), ("o_tok_stride", _i64),
                ("o_head_stride", _i64), ("lse", _vp), ("n_q", _ci), ("scale", ctypes.c_float), ("cap", ctypes.c_float),
                ("causal", _ci), ("window", _ci), ("prefix", _vp), ("ws", _vp), ("ws_bytes", ctypes.c_size_t)]


_L = None


def _lib():
    global _L
    if _L is None:
        L = vla.lib()
        P = ctypes.POINTER
        L.vla_kv_append.argtypes = [P(KVPoolC), P(RaggedC), P(AppendArgsC), _vp]
        L.vla_attention_workspace.argtypes = [P(KVPoolC), P(RaggedC), P(AttentionArgsC), _ci, P(ctypes.c_size_t)]
        L.vla_paged_attention.argtypes = [P(KVPoolC), P(RaggedC), P(AttentionArgsC), _vp]
        L.vla_shared_attention.argtypes = [P(KVPoolC), P(RaggedC), P(AttentionArgsC), _ci, _vp]
        L.vla_debug_paged_plan.argtypes = [P(KVPoolC), P(RaggedC), P(AttentionArgsC), _ci, P(_ci)]
        for n in EXPORTS:
            getattr(L, n).restype = _ci
        _L = L
    return _L


def _dtype(t) -> int:
    if t.dtype == torch.bfloat16:
        return 1
    if t.dtype == torch.float32:
        return 0
    raise TypeError(f"float32 or bfloat16 tensors, not {t.dtype}")


def _i32(t, name, shape, device):
    if t.dtype is not torch.int32 or t.shape != shape or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name} must be a contiguous int32 tensor {shape} on {device}, "
                         f"not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


class KVPool:
    """One layer's pool: k and v [n_pages][n_kv][page_tokens][head_dim] views
    of one layout (any strides of the outer three dimensions, so a pool kept
    token-major or layer-interleaved is passed as a view)."""

    def __init__(self, k, v):
        if k.dim() != 4 or k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype or k.device != v.device:
            raise ValueError("k and v must be 4-d tensors of one shape, layout, type and device")
        if k.stride(3) != 1 and k.shape[3] > 1:
            raise ValueError("head_dim must be contiguous")
        if not k.is_cuda:
            raise ValueError("the pool must be on a GPU")
        self.k, self.v = k, v
        self.device, self.dtype = k.device, k.dtype
        n, h, p, d = k.shape
        self.index, self.n_kv, self.head_dim = k.device.index, h, d
        self.c = KVPoolC(k.device.index, _dtype(k), h, d, p, n, k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1),
                         k.stride(2))
        self.ref = ctypes.byref(self.c)


class Batch:
    """A ragged batch (vla_ragged): start int32 [n_req + 1], kv_len int32
    [n_req], pages int32 [n_req][entries], all on the pool's device; n_tok rows
    of the token buffers; max_new and max_len bound the tokens a request
    brings and has (the tensors may change within these bounds while captured
    calls are replayed)."""

    def __init__(self, start, kv_len, pages, n_tok: int, max_new: int, max_len: int):
        n = kv_len.shape[0]
        dev = kv_len.device
        if pages.dim() != 2:
            raise ValueError("pages must be 2-d")
        self.start, self.kv_len, self.pages = start, kv_len, pages
        self.device, self.index, self.n_req, self.n_tok = dev, dev.index, n, n_tok
        self.c = RaggedC(n, n_tok, max_new, max_len, _i32(start, "start", (n + 1,), dev),
                         _i32(kv_len, "kv_len", (n,), dev), _i32(pages, "pages", (n, pages.shape[1]), dev),
                         pages.shape[1])
        self.ref = ctypes.byref(self.c)


# A call's kernels take a few microseconds where the batch is one token, so
# the host's part is kept short: sizes compared as tuples, argument structures
# built at once, the stream's handle without a stream object around it.
def _rows(t, name, pool: KVPool, batch: Batch, heads: int):
    """Checks a token buffer [n_tok][heads][head_dim] and returns (address, token stride, head stride)."""
    if t.shape != (batch.n_tok, heads, pool.head_dim):
        raise ValueError(f"{name} must be [{batch.n_tok}, {heads}, {pool.head_dim}], not {tuple(t.shape)}")
    if t.dtype is not pool.dtype or t.get_device() != pool.index:
        raise ValueError(f"{name} must be {pool.dtype} on {pool.device}, not {t.dtype} on {t.device}")
    ts, hs, ds = t.stride()
    if ds != 1 and pool.head_dim > 1:
        raise ValueError(f"{name} must have contiguous rows")
    return t.data_ptr(), ts, hs


def _heads(q):
    if q.dim() != 3:
        raise ValueError(f"q must be 3-d, not {tuple(q.shape)}")
    return q.shape[1]


def _same_device(pool: KVPool, batch: Batch):
    if batch.index != pool.index:
        raise ValueError(f"the batch is on {batch.device}, the pool on {pool.device}")


def _stream(pool: KVPool, stream):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(pool.index)
    return vla._stream(stream)


def _empty(shape, dtype, pool: KVPool, stream):
    """A tensor for a call on `stream`, from that stream's own memory: what the
    current stream's pool gives may still be in use by its earlier work."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=pool.device)
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream), device=pool.device) if int(stream) else \
            torch.cuda.default_stream(pool.device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=pool.device)


@functools.lru_cache(maxsize=64)
def _sections(s):
    return (_ci * 3)(*s)


def append(pool: KVPool, batch: Batch, k, v, q=None, q_out=None, positions=None, sections: Sequence[int] = (),
           rope_base: float = 10000.0, stream=None):
    """vla_kv_append. k, v [n_tok][n_kv][head_dim], q [n_tok][n_q][head_dim]
    (views with contiguous rows); sections: the pairs that each axis turns
    (empty: no rotation); positions int32 [n_tok][len(sections)] or None (one
    axis: the tokens' places). Returns q_out (allocated unless given)."""
    _same_device(pool, batch)
    n = len(sections)
    if n > 3:
        raise ValueError("at most three axes")
    n_q, qr, qo = 0, (None, 0, 0), (None, 0, 0)
    if q is not None:
        n_q = _heads(q)
        qr = _rows(q, "q", pool, batch, n_q)
        if q_out is None:
            q_out = _empty(q.shape, q.dtype, pool, stream)
        qo = _rows(q_out, "q_out", pool, batch, n_q)
    elif q_out is not None:
        raise ValueError("q_out without q")
    kp, kt, kh = _rows(k, "k", pool, batch, pool.n_kv)
    vp, vt, vh = _rows(v, "v", pool, batch, pool.n_kv)
    pos = None if positions is None else _i32(positions, "positions", (batch.n_tok, n), pool.device)
    a = AppendArgsC(kp, vp, kt, kh, vt, vh, n_q, qr[0], qo[0], qr[1], qr[2], qo[1], qo[2], n, _sections(tuple(sections)),
                    pos, rope_base)
    vla._check((_L or _lib()).vla_kv_append(pool.ref, batch.ref, ctypes.byref(a), _stream(pool, stream)))
    return q_out


def _attend(pool, batch, q, shared_len, out, lse, scale, cap, causal, window, prefix, ws, stream):
    _same_device(pool, batch)
    L = _L or _lib()
    n_q = _heads(q)
    qp, qt, qh = _rows(q, "q", pool, batch, n_q)
    if out is None:
        out = _empty(q.shape, q.dtype, pool, stream)
    op, ot, oh = _rows(out, "out", pool, batch, n_q)
    lp = None
    if lse is not None:
        if lse.dtype != torch.float32 or lse.shape != (batch.n_tok, n_q) or not lse.is_contiguous() \
                or lse.device != pool.device:
            raise ValueError(f"lse must be a contiguous float32 tensor [{batch.n_tok}, {n_q}] on {pool.device}")
        lp = lse.data_ptr()
    pf = None if prefix is None else _i32(prefix, "prefix", (batch.n_req,), pool.device)
    a = AttentionArgsC(qp, op, qt, qh, ot, oh, lp, n_q, scale, cap, 1 if causal else 0, window, pf, None, 0)
    r = ctypes.byref(a)
    if ws is None:
        need = ctypes.c_size_t()
        vla._check(L.vla_attention_workspace(pool.ref, batch.ref, r, shared_len or 0, ctypes.byref(need)))
        if need.value:
            ws = _empty((need.value,), torch.uint8, pool, stream)
    elif ws.device != pool.device or not ws.is_contiguous():
        raise ValueError(f"ws must be a contiguous tensor on {pool.device}")
    if ws is not None:
        a.ws, a.ws_bytes = ws.data_ptr(), ws.numel() * ws.element_size()
    s = _stream(pool, stream)
    if shared_len is None:
        vla._check(L.vla_paged_attention(pool.ref, batch.ref, r, s))
    else:
        vla._check(L.vla_shared_attention(pool.ref, batch.ref, r, shared_len, s))
    return out


def attention(pool: KVPool, batch: Batch, q, out=None, lse=None, scale: float = 0.0, cap: float = 0.0,
              causal: bool = True, window: int = 0, prefix=None, ws=None, stream=None):
    """vla_paged_attention. q [n_tok][n_q][head_dim] (a view with contiguous
    rows); lse float32 [n_tok][n_q] or None; prefix int32 [n_req] or None; ws:
    a tensor of workspace_bytes(...) bytes or None (allocated for the call).
    Returns out (allocated unless given; rows behind the last request are not
    written)."""
    return _attend(pool, batch, q, None, out, lse, scale, cap, causal, window, prefix, ws, stream)


def shared_attention(pool: KVPool, batch: Batch, q, shared_len: int, out=None, lse=None, scale: float = 0.0,
                     cap: float = 0.0, causal: bool = True, window: int = 0, prefix=None, ws=None, stream=None):
    """vla_shared_attention: as attention, for a batch whose requests have
    their first shared_len tokens (whole pages) on the same pages."""
    return _attend(pool, batch, q, int(shared_len), out, lse, scale, cap, causal, window, prefix, ws, stream)


def workspace_bytes(pool: KVPool, batch: Batch, n_q: int, shared_len: int = 0, causal: bool = True, window: int = 0,
                    cap: Optional[float] = None, prefix=None) -> int:
    """vla_attention_workspace: scratch bytes of such an attention (host only).
    A capped call may need more than another one, and so may one with a
    prefix: cap and prefix are those of the call (prefix False: none); with
    either left out, what is told suffices with and without it."""
    caps = (0.0, 1.0) if cap is None else (cap,)
    prefixes = (False, causal) if prefix is None else (prefix is not False,)
    most = 0
    for c in caps:
        for p in prefixes:
            # (of the prefix only whether there is one is looked at)
            a = AttentionArgsC(n_q=n_q, causal=int(bool(causal)), window=window, cap=c, prefix=64 if p else None)
            need = ctypes.c_size_t()
            vla._check((_L or _lib()).vla_attention_workspace(pool.ref, batch.ref, ctypes.byref(a), shared_len,
                                                              ctypes.byref(need)))
            most = max(most, need.value)
    return most


def attention_plan(n_req: int, n_tok: int, max_new: int, max_len: int, n_q: int, n_kv: int, head_dim: int, page: int = 16,
                   shared_len: int = 0, bf16: bool = True, causal: bool = True, window: int = 0, prefix: bool = False,
                   cap: float = 0.0) -> dict:
    """vla_debug_paged_plan: how an attention of such sizes is launched (host
    only): the padded head dim and, a part each, (kernel, row tiles, key tiles a
    range, ranges)."""
    pool = KVPoolC(0, 1 if bf16 else 0, n_kv, head_dim, page, 1, None, None, 0, page * head_dim, head_dim)
    batch = RaggedC(n_req, n_tok, max_new, max_len, None, None, None, -(-max_len // page))
    a = AttentionArgsC(n_q=n_q, causal=1 if causal else 0, window=window, prefix=64 if prefix else None, cap=cap)
    plan = (_ci * 9)()
    vla._check(_lib().vla_debug_paged_plan(ctypes.byref(pool), ctypes.byref(batch), ctypes.byref(a), shared_len, plan))
    parts = [tuple(plan[1 + 4 * i:5 + 4 * i]) for i in range(2) if plan[1 + 4 * i] >= 0]
    return {"hdp": plan[0], "parts": [(("keys", "rows", "f32", "rows2", "rows8", "f32_rows")[p[0]],) + p[1:] for p in parts]}
