"""Paged cache of uncompressed keys and values: rotary positions, append, decode attention, page
copies and gather (the ``aatc_paged_*``, ``aatc_rotate`` and ``aatc_pages_copy`` calls of
``include/aatc.h``).

`Pages` is the device memory, `Rotary` the frequencies; the functions are the operators.  A sequence
is a row of a block table: its token i is in page ``table[row, i // page_size]``.  The bookkeeping of
a pool (which sequence owns which page) is in `paper_2608_14191_gb300.paged_cache`.

As for the packed cache the binding only checks what the library cannot see behind a pointer and
marshals; every call is asynchronous on the current stream.
"""
from __future__ import annotations

import ctypes

import numpy as np
import torch

from . import HEAD_DIM, _arg_error, _check, _dev_tensor, _on_device, _stream, load

_TYPES = {torch.bfloat16: 0, torch.float16: 1}
_I32T, _F32T = torch.int32, torch.float32
_SCALINGS = {"plain": (0, ()), "linear": (1, ()), "ntk": (2, ()), "ramp": (3, ("fast", "slow")),
             "banded": (4, ("low", "high"))}


class _Desc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("n_pages", ctypes.c_int32)]


class _Rotary(ctypes.Structure):
    _fields_ = [("turns", ctypes.c_void_p), ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("factor", ctypes.c_float)]


class _Heads(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class _Decode(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("cap", ctypes.c_float), ("window", ctypes.c_int32),
                ("slopes", ctypes.c_void_p), ("prior_out", ctypes.c_void_p), ("prior_lse", ctypes.c_void_p)]


class Rotary:
    """Rotary frequencies on a device.  rot_dim: how many of the 128 dimensions turn (a multiple of
    16); layout: "half" (dimension i pairs with i + rot_dim / 2) or "interleaved" (2 i with 2 i + 1).
    scaling: None, or a dict with `kind` and `factor`, and what the kind needs (aatc_rotary_frequencies):
      dict(kind="linear" | "ntk", factor=s)
      dict(kind="ramp", factor=s, original=tokens, fast=32.0, slow=1.0)
      dict(kind="banded", factor=s, original=tokens, low=1.0, high=4.0)
    `frequencies` (fp64, radians per position) and `factor` (on the turned values) are what came out."""

    def __init__(self, rot_dim: int = HEAD_DIM, base: float = 10000.0, layout: str = "half", scaling: dict | None = None,
                 device="cuda"):
        if layout not in ("half", "interleaved"):
            _arg_error("Rotary", f"layout must be half or interleaved, not {layout}")
        s = dict(scaling or {"kind": "plain"})
        kind = s.pop("kind", None)
        if kind not in _SCALINGS:
            _arg_error("Rotary", f"unknown scaling {kind}")
        code, ends = _SCALINGS[kind]
        scale, original = float(s.pop("factor", 1.0)), int(s.pop("original", 0))
        p = [float(s.pop(e, float("nan"))) for e in ends] + [0.0] * (2 - len(ends))
        if s:
            _arg_error("Rotary", f"{kind} scaling has no {sorted(s)}")
        if not 0 < int(rot_dim) <= HEAD_DIM:
            _arg_error("Rotary", "rot_dim must be a multiple of 16 up to 128")
        lib = load()
        freq, factor = np.zeros(max(1, rot_dim // 2)), ctypes.c_double()
        _check(lib.aatc_rotary_frequencies(int(rot_dim), float(base), code, scale, original, p[0], p[1],
                                           freq.ctypes.data, ctypes.byref(factor)), "aatc_rotary_frequencies")
        turns = np.empty(rot_dim // 2, np.uint64)
        _check(lib.aatc_rotary_turns(freq.ctypes.data, turns.size, turns.ctypes.data), "aatc_rotary_turns")
        self.rot_dim, self.layout, self.frequencies, self.factor = int(rot_dim), layout, freq, factor.value
        self.turns = torch.from_numpy(turns.view(np.int64)).to(device)
        self._arg = _Rotary(self.turns.data_ptr(), self.rot_dim, int(layout == "interleaved"), self.factor)
        self._ref = ctypes.byref(self._arg)


class Pages:
    """Device memory of a page pool: [n_layers][n_pages][keys | values][n_kv_heads][page_size][128]."""

    def __init__(self, n_layers: int, n_pages: int, n_kv_heads: int, page_size: int, dtype=torch.bfloat16, device="cuda"):
        self._take(torch.empty((n_layers, n_pages, 2, n_kv_heads, page_size, HEAD_DIM), dtype=dtype, device=device))

    @classmethod
    def of(cls, data):
        """The pool that lies in a tensor of the shape above."""
        self = cls.__new__(cls)
        self._take(data)
        return self

    def _take(self, data):
        _dev_tensor(data, "Pages", "data", None, 6, (None, None, 2, None, None, HEAD_DIM))
        if data.dtype not in _TYPES or not data.is_contiguous():
            _arg_error("Pages", "data must be contiguous, of torch.bfloat16 or torch.float16")
        self.data, self.dtype, self.device = data, data.dtype, data.device
        self.n_layers, self.n_pages, _, self.n_kv_heads, self.page_size, _ = data.shape
        self._desc = _Desc(_TYPES[data.dtype], self.n_kv_heads, self.page_size, self.n_pages)
        self._ref = ctypes.byref(self._desc)
        n = ctypes.c_size_t()
        self._lib = load()
        _check(self._lib.aatc_pages_bytes(self._ref, ctypes.byref(n)), "aatc_pages_bytes")
        self.layer_bytes = n.value
        self._layers = [data.data_ptr() + i * n.value for i in range(self.n_layers)]
        self.flags = torch.zeros(1, dtype=_I32T, device=data.device)
        self._flags = self.flags.data_ptr()
        self._needs = {}

    def layer(self, i: int, where: str) -> int:
        if not 0 <= i < self.n_layers:
            _arg_error(where, f"layer must be in 0 .. {self.n_layers - 1}")
        return self._layers[i]

    def decode_workspace_bytes(self, n_q_heads: int) -> int:
        n = self._needs.get(n_q_heads)
        if n is None:
            got = ctypes.c_size_t()
            _check(self._lib.aatc_paged_decode_workspace_bytes(self._ref, int(n_q_heads), ctypes.byref(got)),
                   "aatc_paged_decode_workspace_bytes")
            n = self._needs[n_q_heads] = got.value
        return n

    def decode_workspace(self, n_q_heads: int):
        """A workspace for decode_attention: enough for any batch and any lengths."""
        return torch.empty(max(4, self.decode_workspace_bytes(n_q_heads) // 4), dtype=_F32T, device=self.device)

    def device_error(self, clear: bool = False) -> int:
        """Flags that kernels raised (2: a bounded wait timed out, 4: a page id outside the pool, 8: a row,
        index or length outside the table).  Synchronizes."""
        f = int(self.flags.item())
        if clear:
            self.flags.zero_()
        return f


# Every call first checks all its arguments in one expression of cheap attribute reads, and only where that fails
# goes through them one by one for the message (a call of a step costs the host as much as the GPU).

def _heads(t, where: str, name: str, dtype, n_heads=None, n_tokens=None):
    """Checks a [tokens][heads][128] argument."""
    _dev_tensor(t, where, name, dtype, 3, (n_tokens, n_heads, HEAD_DIM))
    if t.stride()[2] != 1:
        _arg_error(where, f"the 128 values of a head of {name} must be contiguous")


def _ints(t, where: str, name: str, n: int):
    """Checks a contiguous int32 vector of n entries."""
    if not _on_device(t) or t.dtype != _I32T or t.shape != (n,) or not t.is_contiguous():
        _arg_error(where, f"{name} must be a contiguous device int32 tensor of {n} entries")


def _floats(t, where: str, name: str, shape):
    if not _on_device(t) or t.dtype != _F32T or t.shape != shape or not t.is_contiguous():
        _arg_error(where, f"{name} must be a contiguous device float32 tensor of shape {tuple(shape)}")


def _table(t, where: str, n_rows=None):
    """Checks a block table [rows][max_pages]."""
    if not _on_device(t) or t.dtype != _I32T or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        _arg_error(where, "table must be a device int32 tensor [rows][max_pages], rows contiguous")
    if n_rows is not None and t.shape[0] != n_rows:
        _arg_error(where, f"table must have {n_rows} rows, not {t.shape[0]}")


def rotate(rope: Rotary, x, positions, out=None, backward: bool = False, stream=None):
    """aatc_rotate: x [tokens][heads][128] (bf16 or f16, strided) turned by positions (int32 [tokens]).
    out: None for a new tensor, or x itself.  backward: the gradient with respect to x, given out's."""
    try:
        n, h, d = x.shape
        dtype = x.dtype
        if out is None:
            out = torch.empty((n, h, d), dtype=dtype, device=x.device)
        xs, os = x.stride(), out.stride()
        fine = (d == HEAD_DIM and x.is_cuda and dtype in _TYPES and xs[2] == 1 and out.is_cuda and out.dtype is dtype and
                out.shape == x.shape and os[2] == 1 and positions.is_cuda and positions.dtype is _I32T and
                positions.shape == (n,) and positions.is_contiguous() and isinstance(rope, Rotary))
    except (AttributeError, ValueError, TypeError, IndexError):
        fine = False
    if not fine:
        _check_rotate(rope, x, positions, out)
    _check(load().aatc_rotate(rope._ref, _TYPES[dtype], x.data_ptr(), xs[0], xs[1], positions.data_ptr(), n, h,
                              1 if backward else 0, out.data_ptr(), os[0], os[1], _stream(stream)), "aatc_rotate")
    return out


def _check_rotate(rope, x, positions, out):
    where = "aatc_rotate"
    if not isinstance(rope, Rotary):
        _arg_error(where, "rope must be a Rotary")
    if not _on_device(x) or x.dtype not in _TYPES:
        _arg_error(where, "x must be a device tensor of torch.bfloat16 or torch.float16")
    _heads(x, where, "x", None)
    _heads(out, where, "out", x.dtype, x.shape[1], x.shape[0])
    _ints(positions, where, "positions", x.shape[0])


def append(pages: Pages, layer: int, k, v, table, index, rows=None, positions=None, rope: Rotary | None = None, q=None,
           q_out=None, stream=None):
    """aatc_paged_append: keys and values [tokens][n_kv_heads][128] of new tokens to their pages, the
    keys turned by rope; index int32 [tokens] in the sequence (negative: padding, nothing is written),
    rows int32 [tokens] of the table (None: token t in row t), positions int32 [tokens] for the rotation
    (None: the index).  q [tokens][n_q_heads][128] is turned along; returns q_out (None without q)."""
    dtype, n_q, qh, ro, op = pages.dtype, 0, None, None, None
    try:
        n, n_kv, d = k.shape
        tn, tm = table.shape
        one = (n,)
        ks, vs, ts = k.stride(), v.stride(), table.stride()
        fine = (d == HEAD_DIM and n_kv == pages.n_kv_heads and k.is_cuda and k.dtype is dtype and ks[2] == 1 and v.is_cuda and
                v.dtype is dtype and v.shape == k.shape and vs[2] == 1 and table.is_cuda and table.dtype is _I32T and
                (ts[1] == 1 or tm <= 1) and index.is_cuda and index.dtype is _I32T and index.shape == one and
                index.is_contiguous())
        if rows is None:
            fine = fine and n <= tn
        else:
            fine = fine and rows.is_cuda and rows.dtype is _I32T and rows.shape == one and rows.is_contiguous()
        if positions is not None:
            fine = (fine and positions.is_cuda and positions.dtype is _I32T and positions.shape == one and
                    positions.is_contiguous())
        if q is not None:
            n_q = q.shape[1]
            if q_out is None:
                q_out = torch.empty((n, n_q, HEAD_DIM), dtype=dtype, device=q.device)
            qs = q.stride()
            fine = (fine and rope is not None and q.is_cuda and q.dtype is dtype and q.shape == (n, n_q, HEAD_DIM) and
                    qs[2] == 1 and (q_out is q or (q_out.is_cuda and q_out.dtype is dtype and q_out.shape == q.shape and
                                                   q_out.is_contiguous())))
            qh, op = ctypes.byref(_Heads(q.data_ptr(), qs[0], qs[1])), q_out.data_ptr()
        elif q_out is not None:
            fine = False
        if rope is not None:
            ro = rope._ref
    except (AttributeError, ValueError, TypeError, IndexError):
        fine = False
    if not fine:
        _check_append(pages, k, v, table, index, rows, positions, rope, q, q_out)
    _check(pages._lib.aatc_paged_append(pages._ref, pages.layer(layer, "aatc_paged_append"), table.data_ptr(), tn,
                                        ts[0] if tn > 1 else tm, tm, None if rows is None else rows.data_ptr(),
                                        index.data_ptr(), None if positions is None else positions.data_ptr(), n,
                                        ctypes.byref(_Heads(k.data_ptr(), ks[0], ks[1])),
                                        ctypes.byref(_Heads(v.data_ptr(), vs[0], vs[1])), ro, qh, n_q, op, pages._flags,
                                        _stream(stream)), "aatc_paged_append")
    return q_out


def _check_append(pages, k, v, table, index, rows, positions, rope, q, q_out):
    where, dtype = "aatc_paged_append", pages.dtype
    _heads(k, where, "k", dtype, pages.n_kv_heads)
    n = k.shape[0]
    _heads(v, where, "v", dtype, pages.n_kv_heads, n)
    _table(table, where)
    _ints(index, where, "index", n)
    if rows is not None:
        _ints(rows, where, "rows", n)
    elif table.shape[0] < n:
        _arg_error(where, f"table has {table.shape[0]} rows for {n} tokens: give rows")
    if positions is not None:
        _ints(positions, where, "positions", n)
    if rope is not None and not isinstance(rope, Rotary):
        _arg_error(where, "rope must be a Rotary")
    if q is not None:
        if rope is None:
            _arg_error(where, "q without rope")
        _heads(q, where, "q", dtype, None, n)
        if q_out is not q:
            _heads(q_out, where, "q_out", dtype, q.shape[1], n)
            if not q_out.is_contiguous():
                _arg_error(where, "q_out must be contiguous, or q itself")
    elif q_out is not None:
        _arg_error(where, "q_out without q")


def decode_attention(pages: Pages, layer: int, q, table, lens, out=None, lse=None, prior=None, scale: float | None = None,
                     cap: float = 0.0, window: int = 0, slopes=None, workspace=None, stream=None):
    """aatc_paged_decode_attention: q [batch][n_q_heads][128] (the pages' type) over the first lens[b]
    tokens (int32 [batch]) of each row of the table -> fp32 [batch][n_q_heads][128].  lse: fp32
    [batch][n_q_heads], written; prior: (out, lse) of another set of tokens that joins the softmax; scale:
    1 / sqrt(128) by default; cap: scores become cap tanh(score / cap); window: only the last ones; slopes:
    fp32 [n_q_heads], slope (t - (len - 1)) is added to the score of token t."""
    try:
        batch, n_q, d = q.shape
        tn, tm = table.shape
        if out is None:
            out = torch.empty((batch, n_q, HEAD_DIM), dtype=_F32T, device=q.device)
        qs, ts = q.stride(), table.stride()
        fine = (d == HEAD_DIM and q.is_cuda and q.dtype is pages.dtype and qs[2] == 1 and table.is_cuda and
                table.dtype is _I32T and tn == batch and (ts[1] == 1 or tm <= 1) and lens.is_cuda and lens.dtype is _I32T and
                lens.shape == (batch,) and lens.is_contiguous() and out.is_cuda and out.dtype is _F32T and
                out.shape == q.shape and out.is_contiguous() and
                (workspace is None or (workspace.is_cuda and workspace.is_contiguous())))
        how = _Decode(0.08838834764831845 if scale is None else scale, cap, window)
        ep = None
        if lse is not None:
            fine = fine and lse.is_cuda and lse.dtype is _F32T and lse.shape == (batch, n_q) and lse.is_contiguous()
            ep = lse.data_ptr()
        if slopes is not None:
            fine = fine and slopes.is_cuda and slopes.dtype is _F32T and slopes.shape == (n_q,) and slopes.is_contiguous()
            how.slopes = slopes.data_ptr()
        if prior is not None:
            po, pl = prior
            fine = (fine and po.is_cuda and po.dtype is _F32T and po.shape == q.shape and po.is_contiguous() and pl.is_cuda and
                    pl.dtype is _F32T and pl.shape == (batch, n_q) and pl.is_contiguous())
            how.prior_out, how.prior_lse = po.data_ptr(), pl.data_ptr()
    except (AttributeError, ValueError, TypeError, IndexError):
        fine = False
    if not fine:
        _check_decode(pages, q, table, lens, out, lse, prior, slopes, workspace)
    base = pages.layer(layer, "aatc_paged_decode_attention")
    if batch == 0:
        return out
    if workspace is None:                 # (the library refuses one that is too small)
        workspace = pages.decode_workspace(n_q)
    _check(pages._lib.aatc_paged_decode_attention(pages._ref, base, table.data_ptr(), ts[0] if tn > 1 else tm, tm,
                                                  lens.data_ptr(), batch, ctypes.byref(_Heads(q.data_ptr(), qs[0], qs[1])),
                                                  n_q, ctypes.byref(how), out.data_ptr(), ep, workspace.data_ptr(),
                                                  workspace.nbytes, pages._flags, _stream(stream)),
           "aatc_paged_decode_attention")
    return out


def _check_decode(pages, q, table, lens, out, lse, prior, slopes, workspace):
    where = "aatc_paged_decode_attention"
    _heads(q, where, "q", pages.dtype)
    batch, n_q = q.shape[0], q.shape[1]
    _table(table, where, batch)
    _ints(lens, where, "lens", batch)
    _floats(out, where, "out", (batch, n_q, HEAD_DIM))
    if lse is not None:
        _floats(lse, where, "lse", (batch, n_q))
    if slopes is not None:
        _floats(slopes, where, "slopes", (n_q,))
    if prior is not None:
        if not isinstance(prior, (tuple, list)) or len(prior) != 2:
            _arg_error(where, "prior must be (out, lse)")
        _floats(prior[0], where, "prior[0]", (batch, n_q, HEAD_DIM))
        _floats(prior[1], where, "prior[1]", (batch, n_q))
    if workspace is not None and (not _on_device(workspace) or not workspace.is_contiguous()):
        _arg_error(where, "workspace must be a contiguous device tensor")


def copy_pages(pages: Pages, pairs, stream=None):
    """aatc_pages_copy: page pairs[i][0] to page pairs[i][1] in every layer; pairs int32 [n][2] on the
    host.  No page may be written twice, or be both read and written."""
    p = pairs
    if not isinstance(p, np.ndarray) or p.dtype != np.int32 or not p.flags.c_contiguous:
        p = np.ascontiguousarray(pairs, dtype=np.int32)
    if p.size == 0:
        return
    if p.ndim != 2 or p.shape[1] != 2:
        _arg_error("aatc_pages_copy", "pairs must be [n][2]")
    _check(pages._lib.aatc_pages_copy(pages._ref, pages._layers[0], pages.n_layers, pages.layer_bytes,
                                      p.__array_interface__["data"][0], p.shape[0], _stream(stream)), "aatc_pages_copy")


def gather(pages: Pages, layer: int, table, first: int, n_tokens: int, lens=None, out=None, stream=None):
    """aatc_paged_gather: tokens [first, first + n_tokens) of every row of the table, contiguous:
    (K, V), each [rows][n_tokens][n_kv_heads][128] as aatc_encode takes them.  lens: int32 [rows];
    tokens past their sequence's length come out as zeros."""
    try:
        tn, tm = table.shape
        ts, dtype = table.stride(), pages.dtype
        shape = (tn, n_tokens, pages.n_kv_heads, HEAD_DIM)
        fine = table.is_cuda and table.dtype is _I32T and (ts[1] == 1 or tm <= 1) and n_tokens >= 0
        if out is not None:
            k, v = out
            fine = (fine and k.is_cuda and k.dtype is dtype and k.shape == shape and k.is_contiguous() and v.is_cuda and
                    v.dtype is dtype and v.shape == shape and v.is_contiguous())
        elif fine:
            k, v = pages.data.new_empty(shape), pages.data.new_empty(shape)
        if lens is not None:
            fine = fine and lens.is_cuda and lens.dtype is _I32T and lens.shape == (tn,) and lens.is_contiguous()
    except (AttributeError, ValueError, TypeError, IndexError):
        fine = False
    if not fine:
        k, v = _check_gather(pages, table, n_tokens, lens, out)
    _check(pages._lib.aatc_paged_gather(pages._ref, pages.layer(layer, "aatc_paged_gather"), table.data_ptr(), tn,
                                        ts[0] if tn > 1 else tm, tm, first, n_tokens,
                                        None if lens is None else lens.data_ptr(), k.data_ptr(), v.data_ptr(),
                                        pages._flags, _stream(stream)), "aatc_paged_gather")
    return k, v


def _check_gather(pages, table, n_tokens, lens, out):
    where = "aatc_paged_gather"
    _table(table, where)
    shape = (table.shape[0], n_tokens, pages.n_kv_heads, HEAD_DIM)
    if n_tokens < 0:
        _arg_error(where, "n_tokens must not be negative")
    if out is None:
        out = pages.data.new_empty(shape), pages.data.new_empty(shape)
    if not isinstance(out, (tuple, list)) or len(out) != 2:
        _arg_error(where, "out must be (K, V)")
    for t in out:
        if not _on_device(t) or t.dtype != pages.dtype or t.shape != shape or not t.is_contiguous():
            _arg_error(where, f"out must be two contiguous device tensors of the pages' type, {shape}")
    if lens is not None:
        _ints(lens, where, "lens", table.shape[0])
    return out
