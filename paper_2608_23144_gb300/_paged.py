"""The paged 8-bit cache of keys and values and the attention over it: argument
checks and marshalling only, as in ``_binding``. The cache and the step's batch
are handles, made once and passed to the calls of every layer and step."""
from __future__ import annotations

import ctypes as ct
from typing import Optional

import torch

from ._binding import AwsrcError, _check, _require, lib
from ._binding import _stream as _stream_of

# The current stream's handle without a torch.cuda.Stream object: the object
# alone costs 3 of a short call's 15 us.
_raw_stream = torch._C._cuda_getCurrentRawStream


_current_device = torch._C._cuda_getDevice


def _stream(stream, device: torch.device) -> int:
    return _raw_stream(device.index) if stream is None else _stream_of(stream)


def _on(device: torch.device, call, *args) -> int:
    """call(*args) with `device` current: the library launches on the current
    device, and the default stream's handle does not name one."""
    if _current_device() == device.index:
        return call(*args)
    with torch.cuda.device(device):
        return call(*args)


PAGE_SIZES = (16, 32, 64, 128)
HEAD_DIMS = (64, 128)
EXP_NAN = -128  # exponent of a block that received a non-finite value

_DTYPES = {torch.float32: 0, torch.bfloat16: 1}


class _Cache(ct.Structure):
    _fields_ = [("n_pages", ct.c_int32), ("page", ct.c_int32), ("n_kv_heads", ct.c_int32), ("head_dim", ct.c_int32),
                ("k", ct.c_void_p), ("v", ct.c_void_p), ("k_exp", ct.c_void_p), ("v_exp", ct.c_void_p)]


class _Batch(ct.Structure):
    _fields_ = [("n_seq", ct.c_int32), ("n_tok", ct.c_int32), ("max_new", ct.c_int32), ("max_kv", ct.c_int32),
                ("table_stride", ct.c_int32), ("pad_", ct.c_int32), ("q_start", ct.c_void_p), ("kv_len", ct.c_void_p),
                ("page_table", ct.c_void_p)]


class _Rows(ct.Structure):
    _fields_ = [("p", ct.c_void_p), ("tok_stride", ct.c_int64), ("head_stride", ct.c_int64), ("dtype", ct.c_int32),
                ("pad_", ct.c_int32)]


def _declare():
    P, vp, sz, i32, st = ct.POINTER, ct.c_void_p, ct.c_size_t, ct.c_int32, ct.c_int
    lib.awsrc_attention_workspace_bytes.restype = st
    lib.awsrc_attention_workspace_bytes.argtypes = [P(_Cache), i32, P(sz)]
    lib.awsrc_attention_workspace_init.restype = st
    lib.awsrc_attention_workspace_init.argtypes = [P(_Cache), i32, vp, sz, vp]
    lib.awsrc_kv_append.restype = st
    lib.awsrc_kv_append.argtypes = [P(_Cache), P(_Batch), i32, P(_Rows), P(_Rows), P(_Rows), P(_Rows), vp, vp, i32,
                                    i32, i32, vp, sz, vp]
    lib.awsrc_paged_attention.restype = st
    lib.awsrc_paged_attention.argtypes = [P(_Cache), P(_Batch), i32, P(_Rows), P(_Rows), vp, ct.c_float, i32, vp, sz,
                                          vp]


_declare()


class KvCache:
    """A paged cache held in 8 bits (include/awsrc.h has the layout):
    ``k`` [pages, kv_heads, dim / 16, page, 16] and ``v`` [pages, kv_heads, page / 16, dim, 16]
    float8_e4m3fn codes, ``k_exp`` and ``v_exp`` [pages, kv_heads] int8: a code
    stands for code * 2**exp of its (page, kv head)."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_exp: torch.Tensor, v_exp: torch.Tensor):
        _require(k, "k", dtype=torch.float8_e4m3fn)
        if k.dim() != 5 or k.shape[4] != 16:
            raise ValueError(f"k must be [pages, kv_heads, dim / 16, page, 16], not {tuple(k.shape)}")
        pages, heads, runs, page, _ = k.shape
        self.pages, self.kv_heads, self.head_dim, self.page = int(pages), int(heads), 16 * int(runs), int(page)
        if self.head_dim not in HEAD_DIMS or self.page not in PAGE_SIZES:
            raise ValueError(f"head_dim {self.head_dim} must be one of {HEAD_DIMS}, page {self.page} of {PAGE_SIZES}")
        self.device = k.device
        _require(v, "v", dtype=torch.float8_e4m3fn, shape=(pages, heads, page // 16, self.head_dim, 16), device=k.device)
        for name, t in (("k_exp", k_exp), ("v_exp", v_exp)):
            _require(t, name, dtype=torch.int8, shape=(pages, heads), device=k.device)
        self.k, self.v, self.k_exp, self.v_exp = k, v, k_exp, v_exp
        for name in ("k", "v", "k_exp", "v_exp"):
            if not getattr(self, name).is_contiguous():
                raise ValueError(f"{name} must be contiguous")
        self._c = _Cache(self.pages, self.page, self.kv_heads, self.head_dim, k.data_ptr(), v.data_ptr(),
                         k_exp.data_ptr(), v_exp.data_ptr())
        self._ref = ct.byref(self._c)


class KvBatch:
    """The sequences of one step: new tokens q_start[b] .. q_start[b + 1] of
    sequence b are the last of its kv_len[b] tokens, token p of it in page
    page_table[b, p // page]. int32 device tensors, read by the kernels when
    they run; max_new and max_kv (the most new tokens and kv_len they may hold)
    choose launch shapes."""

    def __init__(self, q_start: torch.Tensor, kv_len: torch.Tensor, page_table: torch.Tensor, n_tok: int, max_new: int,
                 max_kv: int):
        _require(kv_len, "kv_len", dtype=torch.int32)
        if kv_len.dim() != 1:
            raise ValueError(f"kv_len must be 1-D, not {kv_len.dim()}-D")
        n = kv_len.shape[0]
        _require(q_start, "q_start", dtype=torch.int32, shape=(n + 1,), device=kv_len.device)
        _require(page_table, "page_table", dtype=torch.int32, device=kv_len.device)
        if page_table.dim() != 2 or page_table.shape[0] != n or page_table.shape[1] < 1:
            raise ValueError(f"page_table has shape {tuple(page_table.shape)}, expected ({n}, at least 1)")
        if not (q_start.is_contiguous() and kv_len.is_contiguous() and page_table.is_contiguous()):
            raise ValueError("q_start, kv_len and page_table must be contiguous")
        if min(n_tok, max_new, max_kv) < 0:
            raise ValueError("n_tok, max_new and max_kv must not be negative")
        self.q_start, self.kv_len, self.page_table = q_start, kv_len, page_table
        self.n_tok, self.device = int(n_tok), kv_len.device
        # a 0-size tensor has no address; such a batch is a no-op
        ptr = [t.data_ptr() or q_start.data_ptr() for t in (q_start, kv_len, page_table)]
        self._c = _Batch(n, self.n_tok, int(max_new), int(max_kv), page_table.shape[1], 0, *ptr)
        self._ref = ct.byref(self._c)


def awsrc_kv_cache(k: torch.Tensor, v: torch.Tensor, k_exp: torch.Tensor, v_exp: torch.Tensor) -> KvCache:
    """Handle of a paged cache in the given tensors."""
    return KvCache(k, v, k_exp, v_exp)


def awsrc_kv_cache_alloc(n_pages: int, n_kv_heads: int, head_dim: int, page: int = 64, device="cuda") -> KvCache:
    """A new paged cache of n_pages pages of `page` tokens."""
    def e4m3(*shape):
        return torch.zeros(shape, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)

    exps = [torch.zeros(n_pages, n_kv_heads, dtype=torch.int8, device=device) for _ in range(2)]
    return KvCache(e4m3(n_pages, n_kv_heads, head_dim // 16, page, 16),
                   e4m3(n_pages, n_kv_heads, page // 16, head_dim, 16), *exps)


def awsrc_kv_batch(q_start: torch.Tensor, kv_len: torch.Tensor, page_table: torch.Tensor, n_tok: int, max_new: int,
                   max_kv: int) -> KvBatch:
    """Handle of one step's sequences, shared by the calls of all layers."""
    return KvBatch(q_start, kv_len, page_table, n_tok, max_new, max_kv)


def awsrc_attention_workspace(cache: KvCache, n_heads: int, stream=None) -> torch.Tensor:
    """A workspace for awsrc_kv_append and awsrc_paged_attention calls on this
    cache, ready for use: any batch, one stream at a time."""
    n = ct.c_size_t()
    _check(lib.awsrc_attention_workspace_bytes(cache._ref, n_heads, ct.byref(n)), "attention_workspace_bytes")
    ws = torch.empty(n.value, dtype=torch.uint8, device=cache.device)
    _check(_on(ws.device, lib.awsrc_attention_workspace_init, cache._ref, n_heads, ws.data_ptr(), n.value,
               _stream(stream, ws.device)),
           "attention_workspace_init")
    return ws


_EMPTY = 16  # stands for the address of an empty tensor, which no kernel reads


def _rows(t: torch.Tensor, name: str, shape, dtype, device) -> _Rows:
    """Checks a [n_tok, heads, dim] tensor of any strides but dims in a row."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor, not {type(t).__name__}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    ts, hs, ds = t.stride()
    if ds != 1:
        raise ValueError(f"{name} must have its dims in a row (last stride 1, not {ds})")
    return _Rows(t.data_ptr() or _EMPTY, ts, hs, _DTYPES[dtype], 0)


def _common(cache: KvCache, batch: KvBatch, q: torch.Tensor, workspace: torch.Tensor):
    """Checks what both calls take; returns (device, q's shape)."""
    if not isinstance(cache, KvCache) or not isinstance(batch, KvBatch):
        raise TypeError("cache and batch must come from awsrc_kv_cache and awsrc_kv_batch")
    if not isinstance(q, torch.Tensor) or q.dtype not in _DTYPES:
        raise TypeError("q must be a float32 or bfloat16 tensor")
    shape = q.shape
    if len(shape) != 3 or shape[0] != batch.n_tok or shape[1] < 1 or shape[1] % cache.kv_heads != 0 or shape[2] != cache.head_dim:
        raise ValueError(f"q has shape {tuple(shape)}, expected ({batch.n_tok}, a multiple of {cache.kv_heads}, "
                         f"{cache.head_dim})")
    dev = cache.device
    if dev.type != "cuda" or batch.device != dev:
        raise ValueError(f"the cache is on {dev}, the batch on {batch.device}: one CUDA device is needed")
    if workspace.dtype is not torch.uint8 or workspace.device != dev or not workspace.is_contiguous():
        raise ValueError("workspace must come from awsrc_attention_workspace")
    return dev, shape


def awsrc_kv_append(cache: KvCache, batch: KvBatch, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                    cos: Optional[torch.Tensor], sin: Optional[torch.Tensor], workspace: torch.Tensor,
                    interleaved: bool = False, q_out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Writes the batch's keys and values [n_tok, kv_heads, dim] into the cache
    and rotates q [n_tok, heads, dim] and k by position on the way; returns the
    rotated q (in `q_out`, which may be q). cos and sin are float32 [positions,
    rotary_dim / 2] tables (None: no rotation). Batch entries that cannot be
    right are skipped and reported by awsrc_workspace_status(workspace)."""
    dev, shape = _common(cache, batch, q, workspace)
    dt = q.dtype
    if q_out is None:
        q_out = torch.empty(shape, dtype=dt, device=dev)
    kv_shape = (shape[0], cache.kv_heads, shape[2])
    rq = _rows(q, "q", shape, dt, dev)
    rk = _rows(k, "k", kv_shape, dt, dev)
    rv = _rows(v, "v", kv_shape, dt, dev)
    ro = _rows(q_out, "q_out", shape, dt, dev)
    if cos is None and sin is None:
        cp = sp = None
        rows = half = 0
    else:
        _require(cos, "cos", dtype=torch.float32, device=dev)
        if cos.dim() != 2:
            raise ValueError(f"cos must be 2-D (positions x rotary_dim / 2), not {cos.dim()}-D")
        _require(sin, "sin", dtype=torch.float32, shape=cos.shape, device=dev)
        if not (cos.is_contiguous() and sin.is_contiguous()):
            raise ValueError("cos and sin must be contiguous")
        cp, sp, (rows, half) = cos.data_ptr(), sin.data_ptr(), cos.shape
    st = _on(dev, lib.awsrc_kv_append, cache._ref, batch._ref, shape[1], rq, rk, rv, ro, cp, sp, rows, 2 * half,
             bool(interleaved), workspace.data_ptr(), workspace.numel(), _stream(stream, dev))
    if st:
        _check(st, "kv_append")
    return q_out


def awsrc_paged_attention(cache: KvCache, batch: KvBatch, q: torch.Tensor, workspace: torch.Tensor,
                          sm_scale: Optional[float] = None, causal: bool = True, out: Optional[torch.Tensor] = None,
                          lse: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Attention of the batch's (rotated) queries [n_tok, heads, dim] over their
    sequences' cached tokens, to `out` (same shape and dtype; not q) and, when
    given, the float32 [n_tok, heads] `lse` (natural log of the softmax sum).
    sm_scale defaults to dim ** -0.5. causal: query i of a sequence sees the
    tokens up to its own; else all. A query that sees none gets 0 and -inf."""
    dev, shape = _common(cache, batch, q, workspace)
    dt = q.dtype
    if out is None:
        out = torch.empty(shape, dtype=dt, device=dev)
    rq = _rows(q, "q", shape, dt, dev)
    ro = _rows(out, "out", shape, dt, dev)
    lp = None
    if lse is not None:
        _require(lse, "lse", dtype=torch.float32, shape=shape[:2], device=dev)
        if not lse.is_contiguous():
            raise ValueError("lse must be contiguous")
        lp = lse.data_ptr()
    st = _on(dev, lib.awsrc_paged_attention, cache._ref, batch._ref, shape[1], rq, ro, lp,
             shape[2] ** -0.5 if sm_scale is None else sm_scale, bool(causal), workspace.data_ptr(), workspace.numel(),
             _stream(stream, dev))
    if st:
        _check(st, "paged_attention")
    return out


__all__ = ["EXP_NAN", "HEAD_DIMS", "PAGE_SIZES", "AwsrcError", "KvBatch", "KvCache", "awsrc_attention_workspace",
           "awsrc_kv_append", "awsrc_kv_batch", "awsrc_kv_cache", "awsrc_kv_cache_alloc", "awsrc_paged_attention"]
