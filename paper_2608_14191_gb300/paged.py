"""Paged cache of uncompressed keys and values: rotary positions, append, decode attention, attention of drafted trees,
attention weights and the tokens that are kept by them, page copies and gather (the ``aatc_paged_*``, ``aatc_rotate``,
``aatc_choose_tokens`` and ``aatc_pages_copy`` calls of ``include/aatc.h``).

`Pages` is the device memory, `Rotary` the frequencies; the functions are the operators.  A sequence
is a row of a block table: its token i is in page ``table[row, i // page_size]``.  The bookkeeping of
a pool (which sequence owns which page) is in `paper_2608_14191_gb300.paged_cache`.

As for the packed cache the binding only checks what the library cannot see behind a pointer and
marshals; every call is asynchronous on the current stream.
"""
from __future__ import annotations

import ctypes
import operator

import numpy as np
import torch

from . import HEAD_DIM, _arg_error, _check, _dev_tensor, _on_device, _stream, load

load()                  # (the extension is linked to the library)
try:
    from . import _calls  # noqa: E402
except ImportError as e:
    raise ImportError("the extension _calls is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'` "
                      "(it needs Python's headers)") from e

_calls.setup(torch.int32, torch.float32, torch.bfloat16, torch.float16, torch._C._cuda_getCurrentRawStream,
             torch._C._cuda_getDevice)
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
        self._addr = ctypes.addressof(self._arg)


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
        self._addr = ctypes.addressof(self._desc)
        n = ctypes.c_size_t()
        self._lib = load()
        _check(self._lib.aatc_pages_bytes(self._addr, ctypes.byref(n)), "aatc_pages_bytes")
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
            _check(self._lib.aatc_paged_decode_workspace_bytes(self._addr, int(n_q_heads), ctypes.byref(got)),
                   "aatc_paged_decode_workspace_bytes")
            n = self._needs[n_q_heads] = got.value
        return n

    def decode_workspace(self, n_q_heads: int, stream=None):
        """A workspace for decode_attention: enough for any batch and any lengths."""
        return _made((max(4, self.decode_workspace_bytes(n_q_heads) // 4),), _F32T, self.device, stream)

    def tree_workspace_bytes(self, n_q_heads: int) -> int:
        got = ctypes.c_size_t()
        _check(self._lib.aatc_paged_tree_workspace_bytes(self._addr, int(n_q_heads), ctypes.byref(got)),
               "aatc_paged_tree_workspace_bytes")
        return got.value

    def tree_workspace(self, n_q_heads: int, stream=None):
        """A workspace for tree_attention: enough for any batch and any lengths."""
        return _made((max(4, self.tree_workspace_bytes(n_q_heads) // 4),), _F32T, self.device, stream)

    def device_error(self, clear: bool = False) -> int:
        """Flags that kernels raised (2: a bounded wait timed out, 4: a page id outside the pool, 8: a row,
        index or length outside the table).  Synchronizes."""
        f = int(self.flags.item())
        if clear:
            self.flags.zero_()
        return f


# Every call first goes the short way, through the extension, which checks the common kinds of arguments and makes the
# call; where it takes one of them for something else (None), the long way checks them one by one, with a
# message for what is wrong, and makes the call through ctypes.

def _heads(t, where: str, name: str, dtype, n_heads=None, n_tokens=None):
    """Checks a [tokens][heads][128] argument; its pointer and strides (0 where there is one of them)."""
    _dev_tensor(t, where, name, dtype, 3, (n_tokens, n_heads, HEAD_DIM))
    s = t.stride()
    if s[2] != 1:
        _arg_error(where, f"the 128 values of a head of {name} must be contiguous")
    return _Heads(t.data_ptr(), s[0] if t.shape[0] > 1 else 0, s[1] if t.shape[1] > 1 else 0)


def _ints(t, where: str, name: str, n: int) -> int:
    """Checks a contiguous int32 vector of n entries."""
    if not _on_device(t) or t.dtype != _I32T or t.shape != (n,) or not t.is_contiguous():
        _arg_error(where, f"{name} must be a contiguous device int32 tensor of {n} entries")
    return t.data_ptr()


def _floats(t, where: str, name: str, shape) -> int:
    if not _on_device(t) or t.dtype != _F32T or t.shape != shape or not t.is_contiguous():
        _arg_error(where, f"{name} must be a contiguous device float32 tensor of shape {tuple(shape)}")
    return t.data_ptr()


def _table(t, where: str, n_rows=None):
    """Checks a block table [rows][max_pages]; (pointer, rows, row stride, max_pages)."""
    if not _on_device(t) or t.dtype != _I32T or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        _arg_error(where, "table must be a device int32 tensor [rows][max_pages], rows contiguous")
    n, m = t.shape
    if n_rows is not None and n != n_rows:
        _arg_error(where, f"table must have {n_rows} rows, not {n}")
    return t.data_ptr(), n, t.stride(0) if n > 1 else m, m


def _made(shape, dtype, device, stream):
    """An empty tensor for a call on `stream` (None: the current one).  Its memory is that stream's: a block that the
    current stream got back may still be in use by what is queued there, which `stream` does not wait for.  And the
    caller may use the tensor on the current stream, so it is not given away again before that is done with it."""
    if stream is None or device.type != "cuda":
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(torch.cuda.current_stream(device))
    return t


def _pages(pages, where: str):
    if not isinstance(pages, Pages):
        _arg_error(where, "pages must be a Pages")


def rotate(rope: Rotary, x, positions, out=None, backward: bool = False, stream=None):
    """aatc_rotate: x [tokens][heads][128] (bf16 or f16, strided) turned by positions (int32 [tokens]).
    out: None for a new tensor, x itself, or another tensor of its type whose heads do not overlap.  backward: the
    gradient with respect to x, given out's; autograd does not record the call."""
    where = "aatc_rotate"
    if not isinstance(rope, Rotary):
        _arg_error(where, "rope must be a Rotary")
    if out is None and isinstance(x, torch.Tensor):
        out = _made(x.shape, x.dtype, x.device, stream)
    st = _calls.rotate(rope._addr, x, positions, out, backward, None if stream is None else stream.cuda_stream)
    if st is None:
        if not _on_device(x) or x.dtype not in _TYPES:
            _arg_error(where, "x must be a device tensor of torch.bfloat16 or torch.float16")
        a = _heads(x, where, "x", None)
        n, h = x.shape[0], x.shape[1]
        b = _heads(out, where, "out", x.dtype, h, n)
        st = load().aatc_rotate(rope._addr, _TYPES[x.dtype], a.x, a.token_stride, a.head_stride,
                                _ints(positions, where, "positions", n), n, h, int(bool(backward)), b.x, b.token_stride,
                                b.head_stride, _stream(stream))
    if st:
        _check(st, where)
    return out


def append(pages: Pages, layer: int, k, v, table, index, rows=None, positions=None, rope: Rotary | None = None, q=None,
           q_out=None, stream=None):
    """aatc_paged_append: keys and values [tokens][n_kv_heads][128] of new tokens to their pages, the
    keys turned by rope; index int32 [tokens] in the sequence (negative: padding, nothing is written),
    rows int32 [tokens] of the table (None: token t in row t), positions int32 [tokens] for the rotation
    (None: the index).  q [tokens][n_q_heads][128] is turned along; returns q_out (None without q)."""
    where = "aatc_paged_append"
    _pages(pages, where)
    if rope is not None and not isinstance(rope, Rotary):
        _arg_error(where, "rope must be a Rotary")
    if q is not None and q_out is None and _on_device(q):
        q_out = _made(q.shape, q.dtype, q.device, stream)
    base, ro = pages.layer(layer, where), None if rope is None else rope._addr
    st = _calls.append(pages._addr, base, pages._flags, pages.dtype, pages.n_kv_heads, k, v, table, index, rows, positions, ro,
                       q, q_out, None if stream is None else stream.cuda_stream)
    if st is None:
        dtype = pages.dtype
        kh = _heads(k, where, "k", dtype, pages.n_kv_heads)
        n = k.shape[0]
        vh = _heads(v, where, "v", dtype, pages.n_kv_heads, n)
        tp, tn, ts, tm = _table(table, where)
        ip = _ints(index, where, "index", n)
        rp = None if rows is None else _ints(rows, where, "rows", n)
        if rows is None and tn < n:
            _arg_error(where, f"table has {tn} rows for {n} tokens: give rows")
        pp = None if positions is None else _ints(positions, where, "positions", n)
        qh, n_q, op = None, 0, None
        if q is not None:
            if rope is None:
                _arg_error(where, "q without rope")
            qh = _heads(q, where, "q", dtype, None, n)
            n_q = q.shape[1]
            op = q_out.data_ptr() if q_out is q else _heads(q_out, where, "q_out", dtype, n_q, n).x
            if q_out is not q and not q_out.is_contiguous():
                _arg_error(where, "q_out must be contiguous, or q itself")
            qh = ctypes.byref(qh)
        elif q_out is not None:
            _arg_error(where, "q_out without q")
        st = pages._lib.aatc_paged_append(pages._addr, base, tp, tn, ts, tm, rp, ip, pp, n, ctypes.byref(kh),
                                          ctypes.byref(vh), ro, qh, n_q, op, pages._flags, _stream(stream))
    if st:
        _check(st, where)
    return q_out


def decode_attention(pages: Pages, layer: int, q, table, lens, out=None, lse=None, prior=None, scale: float | None = None,
                     cap: float = 0.0, window: int = 0, slopes=None, workspace=None, stream=None):
    """aatc_paged_decode_attention: q [batch][n_q_heads][128] (the pages' type) over the first lens[b]
    tokens (int32 [batch]) of each row of the table -> fp32 [batch][n_q_heads][128].  lse: fp32
    [batch][n_q_heads], written; prior: (out, lse) of another set of tokens that joins the softmax, taken with the
    same scores (the packed decode has the default scale, and no cap and no slopes); scale: 1 / sqrt(128) by default; cap: scores become cap tanh(score / cap); window: only the last ones; slopes:
    fp32 [n_q_heads], slope (t - (len - 1)) is added to the score of token t."""
    where = "aatc_paged_decode_attention"
    _pages(pages, where)
    base = pages.layer(layer, where)
    if out is None and _on_device(q):
        out = _made(q.shape, _F32T, q.device, stream)
    if prior is None:
        prior = (None, None)
    elif not isinstance(prior, (tuple, list)) or len(prior) != 2 or prior[0] is None or prior[1] is None:
        _arg_error(where, "prior must be (out, lse)")
    if scale is None:
        scale = 0.08838834764831845       # 1 / sqrt(128)
    st = None
    if workspace is not None:
        st = _calls.decode(pages._addr, base, pages._flags, pages.dtype, q, table, lens, out, lse, prior[0], prior[1], scale,
                           cap, window, slopes, workspace, None if stream is None else stream.cuda_stream)
    if st is None:
        qh = _heads(q, where, "q", pages.dtype)
        batch, n_q = q.shape[0], q.shape[1]
        tp, _, ts, tm = _table(table, where, batch)
        lp = _ints(lens, where, "lens", batch)
        op = _floats(out, where, "out", (batch, n_q, HEAD_DIM))
        ep = None if lse is None else _floats(lse, where, "lse", (batch, n_q))
        if not 0 <= window < 1 << 31:
            _arg_error(where, "window must be in 0 .. 2^31 - 1")
        how = _Decode(scale, cap, window)
        if slopes is not None:
            how.slopes = _floats(slopes, where, "slopes", (n_q,))
        if prior[0] is not None:
            how.prior_out = _floats(prior[0], where, "prior[0]", (batch, n_q, HEAD_DIM))
            how.prior_lse = _floats(prior[1], where, "prior[1]", (batch, n_q))
        if batch == 0:
            return out
        if workspace is None:             # (the library refuses one that is too small)
            workspace = pages.decode_workspace(n_q, stream)
        elif not _on_device(workspace) or not workspace.is_contiguous():
            _arg_error(where, "workspace must be a contiguous device tensor")
        st = pages._lib.aatc_paged_decode_attention(pages._addr, base, tp, ts, tm, lp, batch, ctypes.byref(qh), n_q,
                                                    ctypes.byref(how), op, ep, workspace.data_ptr(), workspace.nbytes,
                                                    pages._flags, _stream(stream))
    if st:
        _check(st, where)
    return out


def tree_masks(parents, starts=None, words: int | None = None):
    """The masks of drafted trees, as tree_attention takes them (numpy int32 [tokens][words], to be moved to the device):
    parents: for every drafted token the number of its parent among its sequence's drafted tokens, which comes before
    it, or -1; starts: where the sequences begin, and the end (None: one sequence)."""
    where = "tree_masks"
    p = np.asarray(parents)
    s = np.array([0, p.size]) if starts is None else np.asarray(starts)
    if p.ndim != 1 or (p.size and p.dtype.kind not in "iu") or s.ndim != 1 or s.size < 1 or s.dtype.kind not in "iu":
        _arg_error(where, "parents and starts must be whole numbers in one dimension")
    if s[0] != 0 or s[-1] != p.size or np.any(s[1:] < s[:-1]):
        _arg_error(where, f"starts must ascend from 0 to {p.size}")
    most = int(np.max(s[1:] - s[:-1], initial=0))
    least = max(1, -(-most // 32))
    if words is not None and words < least:
        _arg_error(where, f"{most} drafted tokens need {least} words")
    words = least if words is None else int(words)
    bits = np.zeros((p.size, words), np.uint32)
    for i0, i1 in zip(s[:-1].tolist(), s[1:].tolist()):
        for i in range(i1 - i0):
            j = int(p[i0 + i])
            if not -1 <= j < i:
                _arg_error(where, f"the parent of drafted token {i} must be -1 or come before it, not {j}")
            if j >= 0:
                bits[i0 + i] = bits[i0 + j]
            bits[i0 + i, i // 32] |= np.uint32(1 << i % 32)
    return bits.view(np.int32)


def _tree_args(pages, where: str, q, table, lens, starts, mask):
    """Checks what tree_attention and attention_weights have in common, for the library's call: (the first part, then q's
    descriptor, which has to live as long)."""
    _dev_tensor(q, where, "q", pages.dtype, 3, (None, None, HEAD_DIM))
    qh = _heads(q, where, "q", pages.dtype) if q.shape[0] else _Heads()      # (without tokens the strides mean nothing)
    n, n_q = q.shape[0], q.shape[1]
    tp, batch, ts, tm = _table(table, where)
    lp = _ints(lens, where, "lens", batch)
    if starts is None and n != batch:
        _arg_error(where, f"{n} queries of {batch} sequences: give starts")
    sp = None if starts is None else _ints(starts, where, "starts", batch + 1)
    mp, words = None, 0
    if mask is not None:
        if not _on_device(mask) or mask.dtype != _I32T or mask.dim() != 2 or mask.shape[0] != n or not mask.is_contiguous():
            _arg_error(where, f"mask must be a contiguous device int32 tensor [{n}][words]")
        mp, words = mask.data_ptr(), mask.shape[1]
        if n and not words:
            _arg_error(where, "mask has no words")
        if not n:
            mp, words = None, 0
    return (tp, ts, tm, lp, batch, sp, ctypes.byref(qh), n, n_q, mp, words), qh


def tree_attention(pages: Pages, layer: int, q, table, lens, starts=None, mask=None, out=None, lse=None,
                   scale: float | None = None, cap: float = 0.0, workspace=None, stream=None):
    """aatc_paged_tree_attention: attention of every sequence's last tokens, whose keys and values are in its pages.
    q [tokens][n_q_heads][128] (the pages' type), sequence b's are tokens starts[b] .. starts[b + 1] (int32 [batch + 1];
    None: one of each sequence, with results of 0 and -infinity where a length is 0); lens int32 [batch] with them; mask int32 [tokens][words]: which of its sequence's drafted tokens
    each one sees (`tree_masks`), None: those up to itself.  -> out [tokens][n_q_heads][128] of the pages' type; lse: fp32
    [tokens][n_q_heads], written; scale, cap: as decode_attention's."""
    where = "aatc_paged_tree_attention"
    _pages(pages, where)
    base = pages.layer(layer, where)
    if out is None and _on_device(q):
        out = _made(q.shape, pages.dtype, q.device, stream)
    if scale is None:
        scale = 0.08838834764831845       # 1 / sqrt(128)
    st = None
    if workspace is not None:
        st = _calls.tree(pages._addr, base, pages._flags, pages.dtype, q, table, lens, starts, mask, out, lse, scale, cap,
                         workspace, None if stream is None else stream.cuda_stream)
    if st is None:
        args, qh = _tree_args(pages, where, q, table, lens, starts, mask)
        if not _on_device(out) or out.dtype != pages.dtype or out.shape != q.shape or not out.is_contiguous():
            _arg_error(where, f"out must be a contiguous device tensor of the pages' type of shape {tuple(q.shape)}")
        ep = None if lse is None else _floats(lse, where, "lse", q.shape[:2])
        if q.shape[0] == 0:
            return out
        if workspace is None:             # (the library refuses one that is too small)
            workspace = pages.tree_workspace(q.shape[1], stream)
        elif not _on_device(workspace) or not workspace.is_contiguous():
            _arg_error(where, "workspace must be a contiguous device tensor")
        st = pages._lib.aatc_paged_tree_attention(pages._addr, base, *args, scale, cap, out.data_ptr(), ep,
                                                  workspace.data_ptr(), workspace.nbytes, pages._flags, _stream(stream))
    if st:
        _check(st, where)
    return out


def attention_weights(pages: Pages, layer: int, q, table, lens, starts, lse, weights, mask=None, scale: float | None = None,
                      cap: float = 0.0, decay: float = 1.0, stream=None):
    """aatc_paged_attention_weights: what every token got in the attention of these queries (as tree_attention takes them, with
    the lse that it wrote; or decode_attention's, with starts None, of a call with the same scale and cap and without window and
    slopes, which are not known here; with a prior the weights are shares of both sets) is added to weights, fp32
    [batch][n_kv_heads][width], which are returned; decay: the factor on what was there (0: nothing is read)."""
    where = "aatc_paged_attention_weights"
    _pages(pages, where)
    base = pages.layer(layer, where)
    if scale is None:
        scale = 0.08838834764831845       # 1 / sqrt(128)
    st = _calls.weights(pages._addr, base, pages._flags, pages.dtype, pages.n_kv_heads, q, table, lens, starts, mask, lse, scale,
                        cap, decay, weights, None if stream is None else stream.cuda_stream)
    if st is None:
        args, qh = _tree_args(pages, where, q, table, lens, starts, mask)
        ep = _floats(lse, where, "lse", q.shape[:2])
        width = weights.shape[2] if isinstance(weights, torch.Tensor) and weights.dim() == 3 else 0
        wp = _floats(weights, where, "weights", (args[4], pages.n_kv_heads, width))
        if args[4] == 0:
            return weights
        st = pages._lib.aatc_paged_attention_weights(pages._addr, base, *args, ep, scale, cap, decay, wp, width,
                                                     pages._flags, _stream(stream))
    if st:
        _check(st, where)
    return weights


def choose_tokens(weights, lens, keep: int, first: int = 0, last: int = 0, kept=None, stream=None):
    """aatc_choose_tokens: of weights fp32 [batch][heads][width] and lens int32 [batch] the indexes of the `keep` tokens of every
    sequence and head that stay, int32 [batch][heads][keep], ascending, -1 behind the end of shorter ones: the first `first`,
    the last `last`, and those of most weight between."""
    where = "aatc_choose_tokens"
    try:
        keep, first, last = (operator.index(x) for x in (keep, first, last))
    except TypeError:
        _arg_error(where, "keep, first and last must be whole numbers")
    if kept is None and _on_device(weights) and weights.dim() == 3 and keep >= 0:
        kept = _made((weights.shape[0], weights.shape[1], keep), _I32T, weights.device, stream)
    st = _calls.choose(weights, lens, keep, first, last, kept, None if stream is None else stream.cuda_stream)
    if st is None:
        shape = tuple(weights.shape) if isinstance(weights, torch.Tensor) and weights.dim() == 3 else (0, 0, 0)
        wp = _floats(weights, where, "weights", shape)
        lp = _ints(lens, where, "lens", shape[0])
        if not all(0 <= x < 1 << 31 for x in (keep, first, last)):
            _arg_error(where, "keep, first and last must be in 0 .. 2^31 - 1")
        want = (shape[0], shape[1], keep)
        if not _on_device(kept) or kept.dtype != _I32T or kept.shape != want or not kept.is_contiguous():
            _arg_error(where, f"kept must be a contiguous device int32 tensor of shape {want}")
        st = load().aatc_choose_tokens(wp, *shape, lp, keep, first, last, kept.data_ptr(), _stream(stream))
    if st:
        _check(st, where)
    return kept


def keep_tokens(pages: Pages, layer: int | None, table, lens, kept, first=None, weights=None, stream=None):
    """aatc_paged_keep_tokens: in one layer (None: in every one) token first[b] + kept[b][j] of sequence b moves to the place of
    token first[b] + j.  kept: int32 [batch][n], or [batch][n_kv_heads][n] with other tokens in every kv-head (choose_tokens),
    ascending, negative behind the last one; lens: int32 [batch], before the call; first: int32 [batch] (None: 0);
    weights: fp32 [batch][n_kv_heads][width], moved along, with zeros behind."""
    where = "aatc_paged_keep_tokens"
    _pages(pages, where)
    if layer is None and weights is not None:
        _arg_error(where, "weights are those of one layer: give it")
    base, layers = (pages.layer(0, where), pages.n_layers) if layer is None else (pages.layer(layer, where), 1)
    st = _calls.keep(pages._addr, base, pages._flags, pages.n_kv_heads, layers, pages.layer_bytes, table, lens, kept, first,
                     weights, None if stream is None else stream.cuda_stream)
    if st is None:
        tp, batch, ts, tm = _table(table, where)
        lp = _ints(lens, where, "lens", batch)
        fp = None if first is None else _ints(first, where, "first", batch)
        if not _on_device(kept) or kept.dtype != _I32T or kept.dim() not in (2, 3) or not kept.is_contiguous() or \
                tuple(kept.shape[:-1]) != (batch, pages.n_kv_heads)[:kept.dim() - 1]:
            _arg_error(where, f"kept must be a contiguous device int32 tensor [{batch}][n] or [{batch}][{pages.n_kv_heads}][n]")
        width = weights.shape[2] if isinstance(weights, torch.Tensor) and weights.dim() == 3 else 0
        wp = None if weights is None else _floats(weights, where, "weights", (batch, pages.n_kv_heads, width))
        if weights is not None and width < 1:
            _arg_error(where, "weights has no room for a token")
        if batch == 0:
            return
        st = pages._lib.aatc_paged_keep_tokens(pages._addr, base, layers, pages.layer_bytes, tp, ts, tm, lp, batch, fp,
                                               kept.data_ptr(), kept.shape[-1], int(kept.dim() == 3), wp, width, pages._flags,
                                               _stream(stream))
    if st:
        _check(st, where)


def copy_pages(pages: Pages, pairs, stream=None):
    """aatc_pages_copy: page pairs[i][0] to page pairs[i][1] in every layer; pairs int32 (or equal whole
    numbers) [n][2] on the host.  No page may be written twice, or be both read and written."""
    where = "aatc_pages_copy"
    _pages(pages, where)
    st = _calls.copy(pages._addr, pages._layers[0], pages.n_layers, pages.layer_bytes, pairs,
                     None if stream is None else stream.cuda_stream)
    if st is None:
        given = np.asarray(pairs)
        if given.size == 0:
            return
        if given.ndim != 2 or given.shape[1] != 2:
            _arg_error(where, "pairs must be [n][2]")
        if given.dtype.kind not in "biuf":
            _arg_error(where, "pairs must be whole numbers")
        with np.errstate(invalid="ignore"):
            p = np.ascontiguousarray(given.astype(np.int32))
        if not np.array_equal(p, given):      # (the conversion cuts fractions off and wraps what int32 cannot hold)
            _arg_error(where, "pairs must be page ids: whole numbers of 32 bits")
        st = pages._lib.aatc_pages_copy(pages._addr, pages._layers[0], pages.n_layers, pages.layer_bytes, p.ctypes.data,
                                        p.shape[0], _stream(stream))
    if st:
        _check(st, where)


def gather(pages: Pages, layer: int, table, first: int, n_tokens: int, lens=None, out=None, stream=None):
    """aatc_paged_gather: tokens [first, first + n_tokens) of every row of the table, contiguous:
    (K, V), each [rows][n_tokens][n_kv_heads][128] (bf16 pages: as aatc_encode takes them; f16 it does not take).
    lens: int32 [rows]; tokens past their sequence's length come out as zeros."""
    where = "aatc_paged_gather"
    _pages(pages, where)
    base = pages.layer(layer, where)
    if out is None:
        if not _on_device(table) or n_tokens < 0:
            _arg_error(where, "table must be a device tensor, n_tokens not negative")
        shape = (table.shape[0], n_tokens, pages.n_kv_heads, HEAD_DIM)
        k = _made(shape, pages.dtype, pages.device, stream)
        v = _made(shape, pages.dtype, pages.device, stream)
    elif isinstance(out, (tuple, list)) and len(out) == 2:
        k, v = out
    else:
        _arg_error(where, "out must be (K, V)")
    st = _calls.gather(pages._addr, base, pages._flags, pages.dtype, pages.n_kv_heads, table, first, n_tokens, lens, k, v,
                       None if stream is None else stream.cuda_stream)
    if st is None:
        tp, tn, ts, tm = _table(table, where)
        if not (0 <= first < 1 << 31 and 0 <= n_tokens < 1 << 31):
            _arg_error(where, "first and n_tokens must be in 0 .. 2^31 - 1")
        shape = (tn, int(n_tokens), pages.n_kv_heads, HEAD_DIM)
        for t in (k, v):
            if not _on_device(t) or t.dtype != pages.dtype or t.shape != shape or not t.is_contiguous():
                _arg_error(where, f"out must be two contiguous device tensors of the pages' type, {shape}")
        lp = None if lens is None else _ints(lens, where, "lens", tn)
        st = pages._lib.aatc_paged_gather(pages._addr, base, tp, tn, ts, tm, int(first), int(n_tokens), lp, k.data_ptr(),
                                          v.data_ptr(), pages._flags, _stream(stream))
    if st:
        _check(st, where)
    return k, v
