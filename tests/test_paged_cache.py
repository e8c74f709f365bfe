"""Bookkeeping of the page pool against a token-by-token model (no GPU: pages on the CPU, copies by torch),
and, on the GPU, the tail cache and the example that runs all the paged operators together."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Books:
    """Sequences as lists of token numbers, written into the pages through what the bookkeeping says."""

    def __init__(self, module, paged, n_pages, max_seqs, max_tokens, page):
        self.pages = paged.Pages(1, n_pages, 1, page, torch.float16, "cpu")
        self.s = module.PagedSequences(self.pages, max_seqs, max_tokens)
        self.tokens, self.next, self.page = {}, 1, page

    def grow(self, counts):
        rows, index = (x.tolist() for x in self.s.grow(counts))
        assert rows == [r for r, n in counts.items() for _ in range(n)]
        for r, i in zip(rows, index):
            assert i == len(self.tokens[r])
            self.tokens[r].append(self.next)
            self.pages.data[0, int(self.s.table[r, i // self.page]), 0, 0, i % self.page, 0] = self.next
            self.next = self.next % 2000 + 1                       # (exact in f16)

    def check(self):
        live = np.zeros(self.pages.n_pages, int)
        for r, want in self.tokens.items():
            assert self.s.length(r) == len(want) == int(self.s.lens[r])
            ids = self.s.pages_of(r)
            assert len(ids) == -(-len(want) // self.page) and np.array_equal(ids, self.s.table[r, :len(ids)].numpy())
            live[ids] += 1
            got = self.pages.data[0, torch.from_numpy(ids).long(), 0, 0, :, 0].reshape(-1)[:len(want)]
            assert got.int().tolist() == want
        assert np.array_equal(live, self.s.refs)
        assert sorted(self.s._free) == np.flatnonzero(live == 0).tolist()
        for r in range(len(self.s._used)):
            assert bool(self.s._used[r]) == (r in self.tokens) and (r in self.tokens or int(self.s.lens[r]) == 0)


@pytest.fixture
def books(aatc, monkeypatch):
    monkeypatch.setattr(aatc, "_DEVICE_TYPE", "cpu")
    from paper_2608_14191_gb300 import paged, paged_cache

    def copy(pages, pairs, stream=None):
        pairs = torch.as_tensor(np.asarray(pairs)).long()
        src, dst = pairs[:, 0], pairs[:, 1]
        assert len(set(dst.tolist())) == len(dst) and not set(src.tolist()) & set(dst.tolist())
        pages.data[:, dst] = pages.data[:, src]

    monkeypatch.setattr(paged_cache, "copy_pages", copy)
    return lambda *a: Books(paged_cache, paged, *a)


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("page", [8, 16])
def test_random_histories(books, page, seed):
    from paper_2608_14191_gb300.paged_cache import PoolExhausted
    rng = np.random.default_rng([seed, page])
    b = books(40, 7, 12 * page, page)
    for _ in range(300):
        rows = list(b.tokens)
        act = rng.choice(["add", "grow", "grow", "grow", "fork", "free", "drop", "compact"])
        if act == "add" and len(rows) < 7:
            r = b.s.add()
            assert r not in b.tokens
            b.tokens[r] = []
        elif act == "grow" and rows:
            some = rng.permutation(rows)[:rng.integers(1, len(rows) + 1)]
            counts = {int(r): int(min(rng.choice([0, 1, 1, 3, page + 2]), 12 * page - len(b.tokens[r]))) for r in some}
            try:
                b.grow(counts)
            except PoolExhausted:
                pass                                              # and nothing has changed, which check() sees
        elif act == "fork" and rows and len(rows) < 7:
            r, free = int(rng.choice(rows)), b.s.free_pages
            b.tokens[b.s.fork(r)] = list(b.tokens[r])
            assert b.s.free_pages == free
        elif act == "free" and len(rows) > 2:
            r = int(rng.choice(rows))
            b.s.free(r)
            del b.tokens[r]
        elif act == "drop" and rows:
            r = int(rng.choice(rows))
            n = page * int(rng.integers(0, len(b.tokens[r]) // page + 1))
            b.s.drop_front(r, n)
            b.tokens[r] = b.tokens[r][n:]
        elif act == "compact":
            n = b.s.compact()
            assert n == np.count_nonzero(b.s.refs) and not b.s.refs[n:].any()
        b.check()


def test_copy_on_write_counts(books):
    """A page shared by k rows costs k - 1 copies where all of them write, and k where one more keeps it."""
    b = books(20, 6, 64, 8)
    b.tokens[b.s.add()] = []
    b.grow({0: 5})
    for r in (1, 2, 3):
        assert b.s.fork(0) == r
        b.tokens[r] = list(b.tokens[0])
    assert b.s.free_pages == 19
    b.grow({1: 1, 3: 1})
    assert b.s.free_pages == 17
    b.check()
    b.grow({0: 1, 2: 1})                                          # (each other's page: one copy)
    assert b.s.free_pages == 16
    b.check()
    b.grow({0: 1, 1: 1, 2: 1, 3: 1})
    assert b.s.free_pages == 16
    b.grow({0: 2})
    assert b.s.free_pages == 15
    b.check()


def test_bookkeeping_refusals(books):
    b = books(4, 2, 30, 8)                                        # (a table of four pages)
    with pytest.raises(ValueError):
        b.s.length(0)
    b.s.add()
    b.tokens[0] = []
    for call in (lambda: b.s.add(0), lambda: b.s.add(2), lambda: b.s.fork(1), lambda: b.s.free(-1), lambda: b.s.grow({0: 33}),
                 lambda: b.s.grow({1: 1}), lambda: b.s.grow({0: -1}), lambda: b.s.drop_front(0, 8), lambda: b.s.fork(0, 0)):
        with pytest.raises(ValueError):
            call()
        b.check()
    b.grow({0: 32})
    b.s.add()
    b.tokens[1] = []
    from paper_2608_14191_gb300.paged_cache import PoolExhausted
    with pytest.raises(PoolExhausted):
        b.s.grow({1: 1})
    with pytest.raises(ValueError):
        b.s.add()
    b.s.drop_front(0, 32)
    b.tokens[0] = []
    b.grow({1: 1, 0: 0})
    b.check()


def test_grow_returns_a_pair(books, monkeypatch):
    """(rows, index) are there when the call returns, staged with the call's own uploads, and can be read more than once."""
    b = books(20, 3, 64, 8)
    b.s.add()
    b.s.add()
    staged = []
    monkeypatch.setattr(b.s, "_staged", lambda x, real=b.s._staged: staged.append(len(np.atleast_1d(x))) or real(x))
    got = b.s.grow({0: 3, 1: 2})
    assert len(staged) == 4                                       # table, lengths, rows, index
    assert isinstance(got, tuple) and len(got) == 2
    for _ in range(2):
        rows, index = got
        assert rows.tolist() == [0, 0, 0, 1, 1] and index.tolist() == [0, 1, 2, 0, 1]
        assert rows.dtype == index.dtype == torch.int32


@pytest.mark.gpu
def test_tail_cache(aatc):
    """Ragged sequences, coded as the window allows, forked on the way: every step's attention against 64 bits over
    the decoded coefficients of the coded tokens and the full-precision others, whose tolerance is that of
    the packed decode (1e-4 relative) for the whole."""
    from paper_2608_14191_gb300.paged_cache import PagedTailCache
    from test_gpu_prefill_layouts import random_plan, tokens
    rng = np.random.default_rng(41)
    n_kv, group, batch, dev = 2, 4, 4, "cuda:0"
    plan, basis, _ = random_plan(aatc, rng, n_kv, group, 8, (352, 288))
    cache = PagedTailCache(plan, batch, 400, dev, window=32, step=16, page_size=8, tail_tokens=200, n_pages=90)
    k_all, v_all = tokens(rng, basis, batch, 400, n_kv)
    kept = [(k_all[r, :0], v_all[r, :0]) for r in range(batch)]
    used = [0] * batch

    def take(counts):
        new = []
        for r, n in enumerate(counts):
            new.append((k_all[r, used[r]:used[r] + n], v_all[r, used[r]:used[r] + n]))
            used[r] += n
            kept[r] = tuple(torch.cat([a, b]) for a, b in zip(kept[r], new[r]))
        return torch.cat([a for a, _ in new]).contiguous(), torch.cat([b for _, b in new]).contiguous()

    coded = []
    for step, counts in enumerate([(90, 33, 0, 60), (1, 1, 1, 1)] + [(1, 1, 1, 1)] * 3 + [(0, 20, 70, 5)] + [(1, 1, 1, 1)] * 40):
        if step == 7:
            cache.fork(0, 3)
            kept[3], free = kept[0], cache.seqs.free_pages
            used[3] = max(used[3], 200)
        k, v = take(counts)
        cache.begin(counts)
        cache.append(0, k, v)
        if set(counts) == {1}:
            q = torch.from_numpy(rng.standard_normal((batch, n_kv * group, 128))).to(dev).to(torch.bfloat16)
            out = cache.attend(0, q)
            n = cache.coded
            coef = aatc.dequantize(plan, 0, cache.caches[0], batch, 0, max(n, 1), 400).double()
            u = [torch.from_numpy(basis[0, :, i]).to(dev).double() for i in (0, 1)]
            for r in range(batch):
                assert cache.length(r) == len(kept[r][0])
                kk, vv = (torch.cat([torch.einsum("nhc,hdc->nhd", coef[r, :n, :, i], u[i]), kept[r][i][n:].double()])
                          for i in (0, 1))
                p = torch.softmax(torch.einsum("hd,nhd->hn", q[r].double(), kk.repeat_interleave(group, 1)) / math.sqrt(128), -1)
                ref = torch.einsum("hn,nhd->hd", p, vv.repeat_interleave(group, 1))
                assert (out[r] - ref).norm() <= 1e-4 * ref.norm(), (step, r)
        cache.end()
        coded.append(cache.coded)
        if step == 20:
            cache.seqs.compact()
    assert coded[0] == 0 and coded[-1] >= 48 and all(b >= a for a, b in zip(coded, coded[1:]))
    assert cache.pages.device_error() == 0 and plan.device_error() == 0


@pytest.mark.gpu
def test_example():
    """The example's last step: coding at 4 bits a channel leaves a step of about 2 x 2.6 x 1.2 / 16 = 0.39 standard
    deviations, 0.11 of the values' size in keys and in values each, 0.16 together; the bound is twice that."""
    path = os.path.join(ROOT, "examples", "paged_generation.py")
    spec = importlib.util.spec_from_file_location("paged_generation", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    got = m.generate(steps=60)
    assert got["lengths"] == [n + 60 for p in m.PROMPTS for n in (p, p)]
    assert got["cache"].coded > 0 and 0 < got["worst"] <= 0.32
