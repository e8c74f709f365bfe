"""Bookkeeping of a page pool, and sequences whose old tokens are packed and whose new ones are paged.

`PagedSequences` keeps on the host which sequence has which pages: pages are counted references, so a fork
shares all its pages with its origin and the first of the two that writes into a shared page gets its own
copy.  `PagedTailCache` serves a batch of sequences of different lengths from both caches: the first
`coded` tokens of every sequence (one number for the batch, as the packed decode has one context length)
transform-coded, the rest in pages, and one softmax over both.  It is the counterpart of
`sink_window.SinkWindowCache` for sequences that do not grow in step.

Everything here runs on the current stream.
"""
from __future__ import annotations

import operator

import numpy as np
import torch

from . import HEAD_DIM, decode_attention_sw, encode
from .paged import Pages, append, choose_tokens, copy_pages, decode_attention, gather, keep_tokens


class PoolExhausted(RuntimeError):
    """The pool has fewer free pages than the call needs; nothing has changed."""


class PagedSequences:
    """Sequences in the rows of a block table over `pages`.  `table` (int32 [max_seqs][max_pages]) and
    `lens` (int32 [max_seqs]) are on the device for the operators; a row without a sequence has length 0.
    Token i of a sequence is the i-th one kept: `drop_front` takes whole pages of old tokens away."""

    def __init__(self, pages: Pages, max_seqs: int, max_tokens: int):
        if max_seqs < 1 or max_tokens < 1:
            raise ValueError("max_seqs, max_tokens >= 1 required")
        self.pages, self.page_size = pages, pages.page_size
        self.max_pages = -(-max_tokens // self.page_size)
        self.refs = np.zeros(pages.n_pages, np.int32)
        self._free = list(range(pages.n_pages - 1, -1, -1))
        self._table = np.zeros((max_seqs, self.max_pages), np.int32)
        self._lens = np.zeros(max_seqs, np.int32)
        self._used = np.zeros(max_seqs, bool)
        self.table = torch.zeros((max_seqs, self.max_pages), dtype=torch.int32, device=pages.device)
        self.lens = torch.zeros(max_seqs, dtype=torch.int32, device=pages.device)

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def length(self, row: int) -> int:
        return int(self._lens[self._row(row)])

    def pages_of(self, row: int) -> np.ndarray:
        return self._table[row, :-(-self.length(row) // self.page_size)]

    def _row(self, row: int) -> int:
        if not 0 <= row < len(self._used) or not self._used[row]:
            raise ValueError(f"row {row} has no sequence")
        return row

    def _new_row(self, row) -> int:
        if row is None:
            free = np.flatnonzero(~self._used)
            if not len(free):
                raise ValueError("every row has a sequence")
            return int(free[0])
        if not 0 <= row < len(self._used) or self._used[row]:
            raise ValueError(f"row {row} has a sequence, or is none")
        return row

    def _staged(self, array):
        """A snapshot of a host array that a copy to the device may read after this call has returned: pinned memory,
        which torch keeps until the copy is done.  (Plain memory may be read by the device in place, later.)"""
        t = torch.from_numpy(np.ascontiguousarray(array, np.int32))
        return t.pin_memory() if self.pages.device.type == "cuda" else t

    def _push(self, table: bool):
        if table:
            self.table.copy_(self._staged(self._table), non_blocking=True)
        self.lens.copy_(self._staged(self._lens), non_blocking=True)

    def _release(self, ids):
        np.subtract.at(self.refs, ids, 1)
        self._free.extend(int(i) for i in ids if self.refs[i] == 0)

    def add(self, row: int | None = None) -> int:
        """A new sequence of no tokens, in the given free row or in the first one."""
        row = self._new_row(row)
        self._used[row] = True
        return row

    def fork(self, row: int, to: int | None = None) -> int:
        """A sequence of the same tokens that shares all pages."""
        ids = self.pages_of(row)
        new = self._new_row(to)
        self._used[new] = True
        self._table[new, :len(ids)] = ids
        self._lens[new] = self._lens[row]
        np.add.at(self.refs, ids, 1)
        self._push(True)
        return new

    def free(self, row: int):
        ids = self.pages_of(row)
        self._release(ids)
        self._lens[row], self._used[row] = 0, False
        self._push(False)

    def grow(self, counts: dict):
        """Room for counts[row] more tokens of every row, with copies of shared pages that they will write
        into.  Returns (rows, index), device int32: where `append` puts the new tokens, packed by
        row in the order of `counts`."""
        P, need, copies, take = self.page_size, 0, [], []
        for row, n in counts.items():
            old = int(self._lens[self._row(row)])
            if n < 0 or old + n > self.max_pages * P:
                raise ValueError(f"row {row}: {n} tokens after {old} do not fit its table")
            new = -(-(old + n) // P) - -(-old // P)
            take.append((row, old, new))
            need += new
        # of the rows that write into one shared page, all but the last need a copy of it (the last keeps it if
        # no other sequence has it)
        left = {}
        for row, old, _ in take:
            if counts[row] and old % P:
                page = int(self._table[row, old // P])
                left[page] = left.get(page, int(self.refs[page]))
                if left[page] > 1:
                    left[page] -= 1
                    copies.append((row, old // P, page))
        need += len(copies)
        if need > len(self._free):
            raise PoolExhausted(f"{need} pages needed, {len(self._free)} free")
        pairs = []
        for row, at, page in copies:
            own = self._free.pop()
            pairs.append((page, own))
            self.refs[page] -= 1
            self.refs[own] = 1
            self._table[row, at] = own
        for row, old, new in take:
            first = -(-old // P)
            for i in range(first, first + new):
                self._table[row, i] = own = self._free.pop()
                self.refs[own] = 1
            self._lens[row] += counts[row]
        if pairs:
            copy_pages(self.pages, np.array(pairs, np.int32))
        self._push(need > 0)
        rows = np.repeat(np.fromiter(counts, np.int32, len(counts)), list(counts.values()))
        index = [np.arange(old, old + counts[row], dtype=np.int32) for row, old, _ in take]
        index = np.concatenate(index) if index else np.zeros(0, np.int32)
        return tuple(self._staged(x).to(self.pages.device, non_blocking=True) for x in (rows, index))

    def drop_front(self, row: int, tokens: int):
        """Takes the first `tokens` tokens (whole pages) away from a sequence."""
        if tokens % self.page_size or not 0 <= tokens <= self.length(row):
            raise ValueError("whole pages of tokens that the sequence has")
        n, ids = tokens // self.page_size, self.pages_of(row).copy()
        self._release(ids[:n])
        self._table[row, :len(ids) - n] = ids[n:]
        self._lens[row] -= tokens
        self._push(True)

    def _own(self, ranges):
        """Copies of the shared pages that (row, first token, end) will write into; all or PoolExhausted."""
        shared, left, P = [], {}, self.page_size
        for row, t0, t1 in ranges:
            for at in range(t0 // P, -(-t1 // P) if t1 > t0 else t0 // P):
                page = int(self._table[row, at])
                left[page] = left.get(page, int(self.refs[page]))
                if left[page] > 1:                   # (the last row that writes into a page keeps it, if no other sequence has it)
                    left[page] -= 1
                    shared.append((row, at, page))
        if len(shared) > len(self._free):
            raise PoolExhausted(f"{len(shared)} pages needed, {len(self._free)} free")
        pairs = []
        for row, at, page in shared:
            own = self._free.pop()
            pairs.append((page, own))
            self.refs[page] -= 1
            self.refs[own] = 1
            self._table[row, at] = own
        if pairs:
            copy_pages(self.pages, np.array(pairs, np.int32))
            self._push(True)

    def _shorten(self, lengths: dict):
        for row, n in lengths.items():
            ids, keep = self.pages_of(row).copy(), -(-n // self.page_size)
            self._release(ids[keep:])
            self._lens[row] = n
        self._push(False)

    def _check_weights(self, weights):
        """All that the operators would refuse, of every layer: once the first layer's tokens have moved it is too late."""
        if weights is None:
            return
        if len(weights) != self.pages.n_layers:
            raise ValueError(f"weights of {self.pages.n_layers} layers needed")
        rows, heads, most = len(self._lens), self.pages.n_kv_heads, max(1, int(self._lens.max()))
        for i, w in enumerate(weights):
            if not isinstance(w, torch.Tensor) or w.device != self.pages.device or w.dtype != torch.float32 or w.dim() != 3 or \
                    tuple(w.shape[:2]) != (rows, heads) or not most <= w.shape[2] < 1 << 31 or not w.is_contiguous():
                raise ValueError(f"layer {i}'s weights must be a contiguous float32 tensor [{rows}][{heads}][{most} or more] on {self.pages.device}")
        spans = sorted((w.data_ptr(), w.nbytes) for w in weights)
        if any(at + n > after for (at, n), (after, _) in zip(spans, spans[1:])):
            raise ValueError("layers share weights, which move with every layer's tokens: give each its own")

    def accept(self, drafted: dict, kept: dict, weights=None):
        """Of the last drafted[row] tokens of every row, in every layer, the ones with the numbers kept[row] (ascending, 0 the first
        drafted one) stay and move together, the others are gone: a verified tree's path.  Keys keep the positions that they were
        turned by.  weights: as evict's, moved with their tokens (those of the tokens that are gone become 0)."""
        self._check_weights(weights)
        paths = {}
        for row, n in drafted.items():
            path = np.asarray(kept.get(row, ()))
            if not 0 <= n <= self.length(row):
                raise ValueError(f"row {row} has no {n} drafted tokens")
            if path.ndim != 1 or (path.size and (path.dtype.kind not in "iu" or path[0] < 0 or path[-1] >= n or np.any(path[1:] <= path[:-1]))):
                raise ValueError(f"row {row}: the kept ones must be ascending numbers below {n}")
            paths[row] = path.astype(np.int32)
        if any(row not in drafted for row in kept):
            raise ValueError("kept without drafted")
        begin = {row: self.length(row) - n for row, n in drafted.items()}
        # (the first of a path that stay where they are need no copy of their page)
        moved = {row: int(np.argmax(p != np.arange(len(p)))) if np.any(p != np.arange(len(p))) else len(p) for row, p in paths.items()}
        self._own([(row, begin[row] + moved[row], begin[row] + len(p)) for row, p in paths.items()])
        if paths and (weights is not None or any(moved[row] < len(p) for row, p in paths.items())):
            lists = np.full((len(self._lens), max(1, max(len(p) for p in paths.values()))), -1, np.int32)
            first = self._lens.copy()                    # (nothing of the other rows)
            for row, p in paths.items():
                lists[row, :len(p)], first[row] = p, begin[row]
            lists, first = (self._staged(x).to(self.pages.device, non_blocking=True) for x in (lists, first))
            if weights is None:
                keep_tokens(self.pages, None, self.table, self.lens, lists, first=first)
            else:
                for layer, w in enumerate(weights):
                    keep_tokens(self.pages, layer, self.table, self.lens, lists, first=first, weights=w)
        self._shorten({row: begin[row] + len(p) for row, p in paths.items()})

    def evict(self, weights, keep: int, first: int = 0, last: int = 0):
        """Every sequence of more than `keep` tokens is cut to that many: in each layer and kv-head the first `first`, the last `last`
        and those of most weight between (weights: of every layer its own fp32 [max_seqs][n_kv_heads][width], as
        attention_weights adds them up; they move with their tokens).  Keys keep the positions that they were turned by, so
        `append` needs positions from then on."""
        if weights is None:
            raise ValueError("weights needed")
        self._check_weights(weights)
        keep, first, last = (operator.index(x) for x in (keep, first, last))
        if not 0 <= first + last <= keep or min(first, last) < 0:
            raise ValueError("0 <= first + last <= keep required")
        cut = [int(r) for r in np.flatnonzero(self._lens > keep)]
        if not cut:
            return
        # (one list for all layers: between the moves nothing is allocated that could fail)
        kept = torch.empty((len(self._lens), self.pages.n_kv_heads, keep), dtype=torch.int32, device=self.pages.device)
        self._own([(row, min(first, keep), keep) for row in cut])
        for layer, w in enumerate(weights):
            kept = choose_tokens(w, self.lens, keep, first, last, kept=kept)
            keep_tokens(self.pages, layer, self.table, self.lens, kept, weights=w)
        self._shorten({row: keep for row in cut})

    def compact(self) -> int:
        """Moves pages so that those in use are the first ones; returns how many they are."""
        used = np.flatnonzero(self.refs)
        n = len(used)
        holes, far = np.flatnonzero(self.refs[:n] == 0), used[used >= n]
        if len(far):
            pairs = np.stack([far, holes], 1).astype(np.int32)
            copy_pages(self.pages, pairs)
            place = np.arange(len(self.refs), dtype=np.int32)
            place[far] = holes
            for row in np.flatnonzero(self._used):
                ids = self.pages_of(row)
                ids[:] = place[ids]
            self.refs[holes], self.refs[far] = self.refs[far], 0
            self._free = list(range(len(self.refs) - 1, n - 1, -1))
            self._push(True)
        return n


class PagedTailCache:
    """The layers of a model for `batch` sequences: `coded` first tokens of each packed, the others paged.

    A step: `begin` (how many new tokens each sequence has), then for every layer `append` and, where each sequence
    has one new token, `attend`, then `end`, which codes old tokens.  A sequence keeps at least `window` tokens in
    full precision; whenever all have `step` more, the oldest `step` of each go to the packed cache.
    rope: a `paged.Rotary` for the model's positions, or None where keys and queries come turned already.
    Scores have the packed decode's scale, no cap and no slopes, and keys and values are bf16.  `coded` is one number:
    a row without tokens keeps everything from being coded, and rows do not leave or enter once it is above 0."""

    def __init__(self, plan, batch: int, max_tokens: int, device="cuda", window: int = 128, step: int = 16,
                 page_size: int = 16, tail_tokens: int | None = None, n_pages: int | None = None, rope=None):
        if step < 1 or step % page_size or window < 0:
            raise ValueError("step must be whole pages, window >= 0")
        self.plan, self.batch, self.max_tokens, self.window, self.step, self.rope = plan, batch, max_tokens, window, step, rope
        dm = plan.dims
        tail = max_tokens if tail_tokens is None else tail_tokens
        if n_pages is None:
            n_pages = batch * -(-tail // page_size)
        self.pages = Pages(dm.n_layers, n_pages, dm.n_kv_heads, page_size, torch.bfloat16, device)
        self.seqs = PagedSequences(self.pages, batch, tail)
        for row in range(batch):
            self.seqs.add(row)
        self.caches = [plan.new_cache(batch, max_tokens, device) for _ in range(dm.n_layers)]
        self.coded = 0
        self.out = torch.empty((2, batch, dm.n_q_heads, HEAD_DIM), dtype=torch.float32, device=device)
        self.lse = torch.empty((batch, dm.n_q_heads), dtype=torch.float32, device=device)
        self.workspace = self.pages.decode_workspace(dm.n_q_heads)
        self.packed_workspace = torch.empty(max(1, plan.workspace_bytes(batch, max_tokens) // 4), device=device)
        self._rows = self._index = self._positions = None

    def length(self, row: int) -> int:
        return self.coded + self.seqs.length(row)

    def begin(self, counts):
        """counts: the number of new tokens of every sequence (their keys, values and queries follow packed,
        sequence after sequence)."""
        if len(counts) != self.batch:
            raise ValueError(f"{self.batch} counts needed")
        if any(self.length(r) + n > self.max_tokens for r, n in enumerate(counts)):
            raise ValueError("packed cache capacity exceeded")
        self._rows, self._index = self.seqs.grow({r: int(n) for r, n in enumerate(counts)})
        self._positions = self._index + self.coded

    def append(self, layer: int, k, v, q=None):
        """k, v bf16 [tokens][n_kv_heads][128] and q [tokens][n_q_heads][128] of the step's tokens; returns the
        turned queries (q itself without a rope)."""
        turn = self.rope is not None
        got = append(self.pages, layer, k, v, self.seqs.table, self._index, rows=self._rows, positions=self._positions,
                     rope=self.rope, q=q if turn else None)
        return got if turn else q

    def attend(self, layer: int, q):
        """Attention of one query row per sequence, turned, over all its tokens: q bf16 [batch][n_q_heads][128] ->
        fp32 [batch][n_q_heads][128] (overwritten by the next call)."""
        prior = None
        if self.coded:
            decode_attention_sw(self.plan, layer, q, self.caches[layer], 0, self.coded, self.max_tokens, out=self.out[0],
                                lse=self.lse, workspace=self.packed_workspace)
            prior = (self.out[0], self.lse)
        return decode_attention(self.pages, layer, q, self.seqs.table, self.seqs.lens, out=self.out[1], prior=prior,
                                workspace=self.workspace)

    def end(self) -> int:
        """Codes as many tokens of every sequence as the window allows; returns their number."""
        least = min(self.seqs.length(r) for r in range(self.batch))
        n = self.step * max(0, (least - self.window) // self.step)
        if n:
            for layer, cache in enumerate(self.caches):
                k, v = gather(self.pages, layer, self.seqs.table, 0, n)
                encode(self.plan, layer, k, v, cache, self.coded, self.max_tokens)
            for row in range(self.batch):
                self.seqs.drop_front(row, n)
            self.coded += n
        return n

    def fork(self, row: int, to: int):
        """Sequence `to` becomes a copy of `row`: its pages are shared, its packed tokens copied."""
        if not 0 <= row < self.batch or not 0 <= to < self.batch:
            raise ValueError(f"rows 0 .. {self.batch - 1}")
        if row == to:
            return
        self.seqs.free(to)
        self.seqs.fork(row, to)
        tiles = -(-self.max_tokens // 128)
        words = self.batch * self.plan.dims.n_kv_heads * 2 * tiles * self.plan.n_words * 128
        for cache in self.caches:
            for part in (cache[:words], cache[words:]):
                per_seq = part.view(self.batch, -1)
                per_seq[to] = per_seq[row]
