"""Serving steps around the paged cache: the step's tables from the requests'
lengths, products of matrices held in 8 bits, and the verification of drafted
tokens. Argument checks and marshalling only, as in ``_binding``."""
from __future__ import annotations

import ctypes as ct
from typing import Optional

import torch

from ._binding import _check, _made_for, _require, lib
from ._paged import _DTYPES, _EMPTY, PAGE_SIZES, KvCache, _on, _stream


class _Pool(ct.Structure):
    _fields_ = [("n_pages", ct.c_int32), ("page", ct.c_int32), ("n_seq", ct.c_int32), ("table_stride", ct.c_int32),
                ("page_table", ct.c_void_p), ("kv_len", ct.c_void_p), ("free_pages", ct.c_void_p),
                ("free_count", ct.c_void_p)]


class _Probs(ct.Structure):
    _fields_ = [("p", ct.c_void_p), ("stride", ct.c_int64), ("dtype", ct.c_int32), ("pad_", ct.c_int32)]


class _Fp8(ct.Structure):
    _fields_ = [("rows", ct.c_int32), ("cols", ct.c_int32), ("codes", ct.c_void_p), ("exps", ct.c_void_p)]


def _declare():
    P, vp, sz, i32, i64, st = ct.POINTER, ct.c_void_p, ct.c_size_t, ct.c_int32, ct.c_int64, ct.c_int
    for name, args in (
            ("step_workspace_bytes", [P(sz)]),
            ("step_workspace_init", [vp, sz, vp]),
            ("kv_plan", [P(_Pool), vp, vp, i32, vp, vp, vp, vp, vp, sz, vp]),
            ("verify_drafts", [i32, i32, i32, i32, vp, vp, P(_Probs), P(_Probs), vp, vp, vp, vp, vp, vp, vp, sz, vp]),
            ("fp8_matrix_bytes", [i32, i32, P(sz), P(sz)]),
            ("fp8_quantize", [vp, i32, i64, P(_Fp8), vp]),
            ("fp8_gemm", [P(_Fp8), P(_Fp8), vp, i32, i64, vp, sz, vp]),
            ("fp8_linear", [vp, i32, i64, P(_Fp8), P(_Fp8), vp, i32, i64, vp, sz, vp])):
        f = getattr(lib, "awsrc_" + name)
        f.restype, f.argtypes = st, args


_declare()


_Tensor = torch.Tensor
_I32, _I64, _F32, _U8 = torch.int32, torch.int64, torch.float32, torch.uint8
_INT = (1 << 31) - 1  # what the library's lengths hold: ctypes would cut them off


# The checks are a small call's largest part: each looks at a tensor once and only
# then finds out what is wrong with it.
def _ints(t, name: str, shape, device, dtype=_I32) -> int:
    """Checks a contiguous tensor of one dtype and returns its address."""
    if not (isinstance(t, _Tensor) and t.dtype is dtype and t.shape == shape and t.device == device and t.is_contiguous()):
        _require(t, name, dtype=dtype, shape=shape, device=device)
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr() or _EMPTY


def _cuda(device: torch.device, what: str):
    if device.type != "cuda":
        raise ValueError(f"{what} is on {device}: a CUDA device is needed")


def _workspace(t, device) -> torch.Tensor:
    if not (isinstance(t, _Tensor) and t.dtype is _U8 and t.device == device and t.is_contiguous()):
        _require(t, "workspace", dtype=_U8, device=device)
        raise ValueError("workspace must come from awsrc_step_workspace")
    return t


def awsrc_step_workspace(device="cuda", stream=None) -> torch.Tensor:
    """A workspace for awsrc_kv_plan, awsrc_verify_drafts, awsrc_fp8_gemm and
    awsrc_fp8_linear, ready for use; one stream at a time."""
    n = ct.c_size_t()
    _check(lib.awsrc_step_workspace_bytes(ct.byref(n)), "step_workspace_bytes")
    ws = _made_for(stream, torch.empty, n.value, dtype=torch.uint8, device=device)
    _check(_on(ws.device, lib.awsrc_step_workspace_init, ws.data_ptr(), n.value, _stream(stream, ws.device)),
           "step_workspace_init")
    return ws


# ------------------------------------------------------------------ the plan


class KvPool:
    """Pages of a cache and who holds them, int32 tensors on the device:
    sequence b holds the first ceil(kv_len[b] / page) entries of page_table[b];
    free_pages is a stack of free_count[0] pages that nobody holds."""

    def __init__(self, page_table: torch.Tensor, kv_len: torch.Tensor, free_pages: torch.Tensor,
                 free_count: torch.Tensor, page: int):
        _require(kv_len, "kv_len", dtype=torch.int32)
        if kv_len.dim() != 1:
            raise ValueError(f"kv_len must be 1-D, not {kv_len.dim()}-D")
        n, self.device = kv_len.shape[0], kv_len.device
        _require(page_table, "page_table")
        if page_table.dim() != 2 or page_table.shape[0] != n or page_table.shape[1] < 1:
            raise ValueError(f"page_table has shape {tuple(page_table.shape)}, expected ({n}, at least 1)")
        _require(free_pages, "free_pages")
        if free_pages.dim() != 1 or free_pages.shape[0] < 1:
            raise ValueError(f"free_pages has shape {tuple(free_pages.shape)}, expected (pages of the cache,)")
        if page not in PAGE_SIZES:
            raise ValueError(f"page {page} must be one of {PAGE_SIZES}")
        if max(n, page_table.shape[1], free_pages.shape[0]) > _INT:
            raise ValueError("a pool has 2^31 - 1 entries of a kind at most")
        ptr = [_ints(page_table, "page_table", page_table.shape, self.device), _ints(kv_len, "kv_len", (n,), self.device),
               _ints(free_pages, "free_pages", free_pages.shape, self.device),
               _ints(free_count, "free_count", (1,), self.device)]
        self.page_table, self.kv_len, self.free_pages, self.free_count = page_table, kv_len, free_pages, free_count
        self.page, self.n_seq = int(page), int(n)
        self._c = _Pool(free_pages.shape[0], self.page, n, page_table.shape[1], *ptr)
        self._ref = ct.byref(self._c)


def awsrc_kv_pool(page_table: torch.Tensor, kv_len: torch.Tensor, free_pages: torch.Tensor, free_count: torch.Tensor,
                  page: int) -> KvPool:
    """Handle of a cache's pages in the given tensors."""
    return KvPool(page_table, kv_len, free_pages, free_count, page)


def awsrc_kv_pool_alloc(cache: KvCache, n_seq: int, max_len: int) -> KvPool:
    """A pool of all pages of `cache`, free, for n_seq sequences of up to max_len tokens."""
    if not isinstance(cache, KvCache):
        raise TypeError("cache must come from awsrc_kv_cache")
    kw = dict(dtype=torch.int32, device=cache.device)
    return KvPool(torch.full((n_seq, max(1, -(-max_len // cache.page))), -1, **kw), torch.zeros(n_seq, **kw),
                  torch.arange(cache.pages - 1, -1, -1, **kw), torch.full((1,), cache.pages, **kw), cache.page)


def awsrc_kv_plan(pool: KvPool, keep: Optional[torch.Tensor], add: torch.Tensor, workspace: torch.Tensor,
                  n_tok: Optional[int] = None, q_start: Optional[torch.Tensor] = None,
                  tok_seq: Optional[torch.Tensor] = None, tok_pos: Optional[torch.Tensor] = None,
                  tok_slot: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """The next step's tables, on the device: every sequence keeps its first
    keep[b] tokens (None: all; not pool.kv_len itself) and gets add[b] new ones if pages and the n_tok
    rows of the step have room for them; the pool's kv_len, page_table and stack
    are brought up to date. Returns q_start (int32 [n_seq + 1]); with it, kv_len
    and page_table are awsrc_kv_batch's arguments. tok_seq, tok_pos (int32) and
    tok_slot (int64), [n_tok] each, receive every new token's sequence, position
    and page * page size + row, -1 behind the last. n_tok defaults to their
    length. awsrc_workspace_status(workspace): 8 an entry that cannot be right
    (its sequence was left as it is), 16 a sequence that found no room: it has no
    rows in q_start and holds up those behind it that need pages."""
    if not isinstance(pool, KvPool):
        raise TypeError("pool must come from awsrc_kv_pool")
    dev, n = pool.device, pool.n_seq
    if n_tok is None:
        for some in (tok_slot, tok_pos, tok_seq):
            if isinstance(some, _Tensor):
                n_tok = some.numel()
                break
        else:
            raise ValueError("n_tok is needed without tok_seq, tok_pos and tok_slot")
    if not 0 <= n_tok <= _INT:
        raise ValueError(f"n_tok must not be {'negative' if n_tok < 0 else 'above 2^31 - 1'}")
    seqs, toks = (n,), (n_tok,)
    kp = None if keep is None else _ints(keep, "keep", seqs, dev)
    ap = _ints(add, "add", seqs, dev)
    tp = None if tok_seq is None else _ints(tok_seq, "tok_seq", toks, dev)
    pp = None if tok_pos is None else _ints(tok_pos, "tok_pos", toks, dev)
    sp = None if tok_slot is None else _ints(tok_slot, "tok_slot", toks, dev, _I64)
    _workspace(workspace, dev)
    if dev.type != "cuda":
        _cuda(dev, "the pool")
    if q_start is None:
        q_start = _made_for(stream, torch.empty, n + 1, dtype=_I32, device=dev)
    qp = _ints(q_start, "q_start", (n + 1,), dev)
    st = _on(dev, lib.awsrc_kv_plan, pool._ref, kp, ap, n_tok, qp, tp, pp, sp, workspace.data_ptr(), workspace.numel(),
             _stream(stream, dev))
    if st:
        _check(st, "kv_plan")
    return q_start


# ---------------------------------------------------------- drafted tokens


def _probs(t, name: str, shape, device) -> _Probs:
    if isinstance(t, _Tensor) and t.shape == shape and t.device == device:
        dtype, (stride, one) = _DTYPES.get(t.dtype), t.stride()
        if dtype is not None and (one == 1 or shape[1] == 1):
            return _Probs(t.data_ptr() or _EMPTY, stride, dtype, 0)
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor, not {type(t).__name__}")
    if t.dtype not in _DTYPES:
        raise TypeError(f"{name} must be float32 or bfloat16, not {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    raise ValueError(f"{name} must have its rows' elements in a row (last stride 1, not {t.stride(1)})")


def awsrc_verify_drafts(row_start: torch.Tensor, ids: torch.Tensor, target: torch.Tensor, draft: Optional[torch.Tensor],
                        u: torch.Tensor, r: torch.Tensor, workspace: torch.Tensor, max_draft: Optional[int] = None,
                        kv_len: Optional[torch.Tensor] = None, accepted: Optional[torch.Tensor] = None,
                        tokens: Optional[torch.Tensor] = None, keep: Optional[torch.Tensor] = None, stream=None):
    """Which drafted tokens the target accepts and the token that follows them.
    Sequence b has the rows row_start[b] .. row_start[b + 1] (int32): ids (int32)
    of its last token and its drafts; `target` [rows, vocab] probabilities after
    each, `draft` those each draft ids[t + 1] was drawn from (None: drafts of
    certainty), float32 or bfloat16; u [rows] and r [n_seq] float32 random numbers
    in [0, 1). Returns (accepted [n_seq], tokens [n_seq, max_draft + 1]: the
    accepted drafts, the token, -1 behind), int32. With kv_len (int32 [n_seq]),
    `keep` receives it less the drafts not accepted, as awsrc_kv_plan takes it;
    keep may be kv_len, but not a pool's: awsrc_kv_plan has to find there what the
    sequences hold. A sequence without rows gets tokens of -1: one that the plan
    left out goes on with the token it had, torch.where(row_start[1:] >
    row_start[:-1], next, had). max_draft defaults to that of `tokens`."""
    if not isinstance(row_start, _Tensor) or row_start.dim() != 1 or row_start.shape[0] < 1:
        _require(row_start, "row_start", dtype=_I32)
        raise ValueError(f"row_start has shape {tuple(row_start.shape)}, expected (n_seq + 1,)")
    n, dev = row_start.shape[0] - 1, row_start.device
    sp = _ints(row_start, "row_start", (n + 1,), dev)
    if not isinstance(target, _Tensor) or target.dim() != 2 or target.shape[1] < 1:
        raise ValueError("target must be a 2-D tensor (rows x vocab)")
    shape = target.shape
    rows, vocab = shape
    if rows > _INT or vocab > _INT:
        raise ValueError(f"target of {rows} rows and a vocab of {vocab}: 2^31 - 1 at most")
    tp = _probs(target, "target", shape, dev)
    dp = None if draft is None else _probs(draft, "draft", shape, dev)
    seqs, all_rows = (n,), (rows,)
    ip = _ints(ids, "ids", all_rows, dev)
    up = _ints(u, "u", all_rows, dev, _F32)
    rp = _ints(r, "r", seqs, dev, _F32)
    if tokens is not None:
        if not isinstance(tokens, _Tensor) or tokens.dim() != 2 or tokens.shape[1] < 1:
            _require(tokens, "tokens")
            raise ValueError(f"tokens has shape {tuple(tokens.shape)}, expected ({n}, max_draft + 1)")
        max_draft = tokens.shape[1] - 1 if max_draft is None else max_draft
    if max_draft is None or not 0 <= max_draft <= _INT:
        raise ValueError("max_draft (the most drafts of a sequence, from 0 to 2^31 - 1) is needed without tokens")
    if keep is not None and kv_len is None:
        raise ValueError("keep needs kv_len")
    _workspace(workspace, dev)
    if dev.type != "cuda":
        _cuda(dev, "row_start")
    if accepted is None:
        accepted = _made_for(stream, torch.empty, n, dtype=_I32, device=dev)
    if tokens is None:
        tokens = _made_for(stream, torch.empty, n, max_draft + 1, dtype=_I32, device=dev)
    cp, op = _ints(accepted, "accepted", seqs, dev), _ints(tokens, "tokens", (n, max_draft + 1), dev)
    lp = kp = None
    if keep is not None:
        kp = _ints(keep, "keep", seqs, dev)
        lp = kp if kv_len is keep else _ints(kv_len, "kv_len", seqs, dev)
    st = _on(dev, lib.awsrc_verify_drafts, n, rows, vocab, max_draft, sp, ip, tp, dp, up, rp, lp, cp, op, kp,
             workspace.data_ptr(), workspace.numel(), _stream(stream, dev))
    if st:
        _check(st, "verify_drafts")
    return accepted, tokens


# ------------------------------------------------ matrices held in 8 bits


class Fp8Matrix:
    """A rows x cols matrix held in e4m3 codes with one power-of-two scale per
    row and 128 columns, in the tensor cores' operand order (include/awsrc.h):
    ``codes`` float8_e4m3fn [ceil(cols / 128), rows up to 8s, 128], ``exps``
    uint8 [ceil(cols / 512), ceil(rows / 128), 32, 4, 4]."""

    def __init__(self, rows: int, cols: int, codes: torch.Tensor, exps: torch.Tensor):
        rows, cols = int(rows), int(cols)
        if rows < 0 or cols < 1 or rows > 1 << 30 or cols > 1 << 24:
            raise ValueError(f"a matrix of {rows} x {cols} cannot be held (0 to 2^30 rows, 1 to 2^24 columns)")
        blocks = -(-cols // 128)
        _require(codes, "codes", dtype=torch.float8_e4m3fn, shape=(blocks, -(-rows // 8) * 8, 128))
        _require(exps, "exps", dtype=torch.uint8, shape=(-(-blocks // 4), -(-rows // 128), 32, 4, 4), device=codes.device)
        if not (codes.is_contiguous() and exps.is_contiguous()):
            raise ValueError("codes and exps must be contiguous")
        self.rows, self.cols, self.codes, self.exps, self.device = rows, cols, codes, exps, codes.device
        self._c = _Fp8(rows, cols, codes.data_ptr() or 128, exps.data_ptr() or 128)
        self._ref = ct.byref(self._c)

    def values(self) -> torch.Tensor:
        """The matrix that the codes and scales stand for, float32 [rows, cols]."""
        blocks, rows8, _ = self.codes.shape
        if self.rows == 0:
            return torch.empty(0, self.cols, device=self.device)
        r = torch.arange(8, device=self.device)
        c = self.codes.view(torch.uint8).view(blocks, rows8 // 8, 8, 8, 16)
        c = c[:, :, r[:, None], r[:, None] ^ r].view(blocks, rows8, 128)  # a row's pieces back in their order
        c = c.view(torch.float8_e4m3fn).transpose(0, 1)[:self.rows].float()
        e = self.exps.permute(1, 3, 2, 0, 4).reshape(-1, 4 * self.exps.shape[0])[:self.rows, :blocks]
        scale = (e.int() << 23).view(torch.float32)  # 2^(e - 127)
        return (c * scale[..., None]).flatten(1)[:, :self.cols]


def awsrc_fp8_matrix(rows: int, cols: int, device="cuda", stream=None) -> Fp8Matrix:
    """A new matrix of zeros held in 8 bits, filled on `stream` (None: the current one)."""
    blocks = -(-cols // 128)
    codes = _made_for(stream, torch.zeros, max(0, blocks), max(0, -(-rows // 8) * 8), 128, dtype=torch.uint8, device=device)
    exps = _made_for(stream, torch.zeros, max(0, -(-blocks // 4)), max(0, -(-rows // 128)), 32, 4, 4, dtype=torch.uint8,
                     device=device)
    return Fp8Matrix(rows, cols, codes.view(torch.float8_e4m3fn), exps)


def _matrix(x, name: str, device=None):
    """Checks a 2-D float32 or bfloat16 tensor of any row stride: (address, dtype, stride)."""
    if isinstance(x, _Tensor) and x.dim() == 2 and (device is None or x.device == device):
        dtype, (stride, one) = _DTYPES.get(x.dtype), x.stride()
        if dtype is not None and (one == 1 or x.shape[1] <= 1):
            return x.data_ptr() or _EMPTY, dtype, stride
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor, not {type(x).__name__}")
    if x.dtype not in _DTYPES:
        raise TypeError(f"{name} must be float32 or bfloat16, not {x.dtype}")
    if x.dim() != 2:
        raise ValueError(f"{name} must be 2-D, not {x.dim()}-D")
    if device is not None and x.device != device:
        raise ValueError(f"{name} is on {x.device}, expected {device}")
    raise ValueError(f"{name} must have its rows' elements in a row (last stride 1, not {x.stride(1)})")


def _fp8(m, name: str, device=None) -> Fp8Matrix:
    if not isinstance(m, Fp8Matrix):
        raise TypeError(f"{name} must come from awsrc_fp8_quantize or awsrc_fp8_matrix")
    if device is not None and m.device != device:
        raise ValueError(f"{name} is on {m.device}, expected {device}")
    return m


def awsrc_fp8_quantize(x: torch.Tensor, out: Optional[Fp8Matrix] = None, stream=None) -> Fp8Matrix:
    """x (2-D, float32 or bfloat16, any row stride) in 8 bits; `out` reuses a matrix of its shape."""
    p, dt, stride = _matrix(x, "x")
    dev = x.device
    if dev.type != "cuda":
        _cuda(dev, "x")
    if out is None:
        out = awsrc_fp8_matrix(x.shape[0], x.shape[1], dev, stream)
    _fp8(out, "out", dev)
    if (out.rows, out.cols) != tuple(x.shape):
        raise ValueError(f"out is {out.rows} x {out.cols}, x {x.shape[0]} x {x.shape[1]}")
    st = _on(dev, lib.awsrc_fp8_quantize, p, dt, stride, out._ref, _stream(stream, dev))
    if st:
        _check(st, "fp8_quantize")
    return out


def _product(x_rows: int, x_cols: int, w: Fp8Matrix, out, out_dtype, dev, stream=None):
    if x_cols != w.cols:
        raise ValueError(f"x has {x_cols} columns, w {w.cols}")
    if out is None:
        out = _made_for(stream, torch.empty, x_rows, w.rows, dtype=out_dtype, device=dev)
    res = _matrix(out, "out", dev)
    if tuple(out.shape) != (x_rows, w.rows):
        raise ValueError(f"out has shape {tuple(out.shape)}, expected ({x_rows}, {w.rows})")
    return (out, *res)


def awsrc_fp8_gemm(x: Fp8Matrix, w: Fp8Matrix, workspace: torch.Tensor, out: Optional[torch.Tensor] = None,
                   out_dtype=torch.float32, stream=None) -> torch.Tensor:
    """x w^T of two matrices held in 8 bits: float32 or bfloat16 [x.rows, w.rows],
    in `out` (any row stride) or a new tensor of out_dtype."""
    dev = _fp8(w, "w").device
    _fp8(x, "x", dev)
    _workspace(workspace, dev)
    if dev.type != "cuda":
        _cuda(dev, "w")
    out, yp, dt, ys = _product(x.rows, x.cols, w, out, out_dtype, dev, stream)
    st = _on(dev, lib.awsrc_fp8_gemm, x._ref, w._ref, yp, dt, ys, workspace.data_ptr(), workspace.numel(),
             _stream(stream, dev))
    if st:
        _check(st, "fp8_gemm")
    return out


def awsrc_fp8_linear(x: torch.Tensor, w: Fp8Matrix, x8: Fp8Matrix, workspace: torch.Tensor,
                     out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """x w^T for activations x (2-D, float32 or bfloat16, any row stride), which
    are held in 8 bits in x8 (a matrix of x's shape) on the way; the result has
    x's dtype unless `out` says otherwise. `out` shares no elements with x. While a
    call is made, no other host thread queues work on its stream that writes w."""
    xp, xt, xs = _matrix(x, "x")
    dev = x.device
    _fp8(x8, "x8", dev)
    _fp8(w, "w", dev)
    if (x8.rows, x8.cols) != tuple(x.shape):
        raise ValueError(f"x8 is {x8.rows} x {x8.cols}, x {x.shape[0]} x {x.shape[1]}")
    _workspace(workspace, dev)
    if dev.type != "cuda":
        _cuda(dev, "x")
    out, yp, yt, ys = _product(x.shape[0], x.shape[1], w, out, x.dtype, dev, stream)
    st = _on(dev, lib.awsrc_fp8_linear, xp, xt, xs, x8._ref, w._ref, yp, yt, ys, workspace.data_ptr(), workspace.numel(),
             _stream(stream, dev))
    if st:
        _check(st, "fp8_linear")
    return out


__all__ = ["Fp8Matrix", "KvPool", "awsrc_fp8_gemm", "awsrc_fp8_linear", "awsrc_fp8_matrix", "awsrc_fp8_quantize",
           "awsrc_kv_plan", "awsrc_kv_pool", "awsrc_kv_pool_alloc", "awsrc_step_workspace", "awsrc_verify_drafts"]
