"""Attention of drafted trees and attention weights where numbers are large, small or many: caps of any size, values and scores at
the ends of their range, long f16 contexts, free slots of a batch.  On the GPU against the definitions in 64 bits.

Tolerances are those of test_gpu_paged_tokens, with its SCORE for what a score errs by: in these tests scores that come out of
the tensor cores are under 8 before the cap (asserted), 8 * 8 * 2^-23 = 7.6e-6 of truncation, and a capped one errs by
2^-21 of the cap up to 64 (3.1e-5), or by 4e-7 of itself (3.2e-6) past that: 3.9e-5 at most.  Where keys and queries have one
value that is not 0, products are exact, and only the cap's part is left."""
import math

import numpy as np
import pytest
import torch
from test_gpu_paged_tokens import DEV, DTYPES, SCORE, Drafts, Pool, check_tree, check_weights, ints, normal, random_tree, scores_of

from paper_2608_14191_gb300 import paged

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _built(aatc):
    return aatc


# ---------------------------------------------------------------- caps
def one_product(pool, d, keys):
    """Keys and queries whose only value is the first one: with scale 1 the score of a token is its key's."""
    d.q.zero_()
    d.q[..., 0] = 1.0
    for r, x in enumerate(keys):
        pool.k[r].zero_()
        pool.k[r][:, 0, 0] = x
        pool.put(r)


def chain(pool, d, r, s):
    """out, lse and sum p |v| of a chain's queries with scores s [token] in 64 bits, one kv-head."""
    n, c = pool.lens[r], d.counts[r]
    sees = torch.arange(n, device=DEV) <= n - c + torch.arange(c, device=DEV)[:, None]
    s = torch.where(sees, s.double(), -math.inf)
    lse = torch.logsumexp(s, 1)
    p, v = torch.exp(s - lse[:, None]), pool.v[r][:, 0].double()
    return p @ v, lse, p @ v.abs()


@pytest.mark.parametrize("cap", [20.0, 50.0, 64.0, 69.0, 80.0])
@pytest.mark.parametrize("levels,size", [((3.0, 2.5, 2.75), 2.0 ** 100), ((-3.0, -2.5, -2.75), 2.0 ** -100), ((3.0, -3.0, 0.1), 1.0)], ids=str)
@pytest.mark.parametrize("heads", [4, 150])
def test_capped_scores_at_the_cap(heads, levels, size, cap):
    """All scores near the cap or near its negative, with values at the ends of bf16: the weights are of the size that the
    scores' differences give, so results of the values' size come out."""
    rng = np.random.default_rng([int(cap), heads, int(levels[0] + 10)])
    lens, counts = [700, 300, 129], [2, 1, 3]
    pool = Pool(rng, lens, 1, 16, torch.bfloat16)
    for r, n in enumerate(lens):
        pool.v[r].copy_(torch.from_numpy(rng.uniform(0.5, 1.5, (n, 1, 128)) * size).to(DEV))
    d = Drafts(rng, pool, counts, heads)
    one_product(pool, d, [torch.from_numpy(rng.choice(levels, n) * cap).to(DEV) for n in lens])
    lse = torch.empty((6, heads), device=DEV)
    out = paged.tree_attention(pool.pages, 0, d.q, pool.table, pool.device_lens, d.starts, lse=lse, scale=1.0, cap=cap)
    w = paged.attention_weights(pool.pages, 0, d.q, pool.table, pool.device_lens, d.starts, lse, torch.zeros((3, 1, 700), device=DEV),
                                scale=1.0, cap=cap)
    u = 2.0 ** -8
    for r in range(3):
        x = pool.k[r][:, 0, 0].double()
        ref, ref_lse, most = chain(pool, d, r, cap * torch.tanh(x / cap))
        sees = torch.arange(lens[r], device=DEV) <= lens[r] - counts[r] + torch.arange(counts[r], device=DEV)[:, None]
        want = torch.where(sees, torch.exp(cap * torch.tanh(x / cap) - lse[d.of(r)].double().T[:, :, None]), 0.0).sum((0, 1))
        assert torch.all((w[r, 0, :lens[r]].double() - want).abs() <= 6e-5 * want + 1e-30)       # (a sum of 450 rounds less than a score errs)
        off = (out[d.of(r)].double() - ref[:, None]).abs()
        bound = 1.01 * u * (most + ref.abs()) + 2 * SCORE * 1.5 * size
        assert torch.all(off <= bound[:, None]), (r, float((off / bound[:, None]).max()))
        assert torch.all((lse[d.of(r)] - ref_lse[:, None]).abs() <= SCORE)
    assert pool.pages.device_error() == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cap,scale", [(30.0, 0.09), (63.9, 0.09), (64.0, -0.09), (64.1, 0.09), (128.0, 0.09), (400.0, 0.09), (1e3, 0.09),
                                       (1e4, -0.05), (1e6, 0.09), (1e12, 0.09), (1e30, 0.09), (8e37, 0.09)])
def test_caps_of_any_size(cap, scale, dtype):
    """Large caps leave scores as they are, to their own precision: trees, chains, weights."""
    rng = np.random.default_rng([71])
    lens, counts = [1, 100, 101, 640, 2011], [1, 40, 7, 64, 5]
    pool = Pool(rng, lens, 2, 16, dtype, scale=0.7)
    d = Drafts(rng, pool, counts, 6, [random_tree(rng, n) for n in counts])
    assert max(float((lambda s: s[s > -math.inf].abs().max())(scores_of(pool, d, r, scale=scale))) for r in range(5)) < 8
    check_tree(pool, d, cap=cap, scale=scale)
    check_weights(pool, d, 2011, cap=cap, scale=scale)
    d = Drafts(rng, pool, counts, 6)
    check_tree(pool, d, cap=cap, scale=scale)
    check_weights(pool, d, 2011, decay=0.0, cap=cap, scale=scale)


@pytest.mark.parametrize("cap", [30.0, 1e3, 1e6])
def test_caps_as_the_decode_has_them(cap):
    """The decode's log-sums with a cap are those of one drafted token, and give weights that sum to the heads."""
    rng = np.random.default_rng(72)
    pool = Pool(rng, [900, 33, 4001], 2, 16, torch.bfloat16, scale=0.7)
    q = normal(rng, (3, 8, 128), torch.bfloat16)
    step, lse = torch.empty((3, 8), device=DEV), torch.empty((3, 8), device=DEV)
    paged.decode_attention(pool.pages, 0, q, pool.table, pool.device_lens, lse=step, cap=cap)
    paged.tree_attention(pool.pages, 0, q, pool.table, pool.device_lens, lse=lse, cap=cap)
    assert torch.all((step - lse).abs() <= 2 * SCORE)
    w = torch.zeros((3, 2, 4001), device=DEV)
    paged.attention_weights(pool.pages, 0, q, pool.table, pool.device_lens, None, step, w, cap=cap)
    assert torch.all((w.double().sum(2) - 4).abs() <= 2e-4 * 4)


# ---------------------------------------------------------------- long f16 contexts
@pytest.mark.parametrize("heads", [4, 130])
@pytest.mark.parametrize("at", [3, 700000])
def test_small_weights_of_a_long_f16_context(at, heads):
    """2^20 tokens, all of one sequence in one CTA: one of weight 1 and value 0, the others of weight 2^-40 and value 1.  What a weight
    is raised to or rounded by is 2^-34 of the largest one at that length, 2^-14 of a value for all of them."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    n, P = 1 << 20, 256
    pages = paged.Pages(1, 2, 1, P, torch.float16, DEV)
    pages.data.zero_()
    pages.data[0, :, 0, 0, :, 0] = -40 * math.log(2)
    pages.data[0, :, 1] = 1.0
    pages.data[0, 1, :, 0, at % P] = 0.0
    table = torch.zeros((sms, n // P), dtype=torch.int32, device=DEV)
    table[:, at // P] = 1
    q = torch.zeros((sms, heads, 128), dtype=torch.float16, device=DEV)
    q[..., 0] = 1.0
    lse = torch.empty((sms, heads), device=DEV)
    out = paged.tree_attention(pages, 0, q, table, ints([n] * sms), lse=lse, scale=1.0)
    small = (n - 1) * math.exp(float(pages.data[0, 0, 0, 0, 0, 0]))
    ref = small / (1 + small)
    assert (out.double() - ref).abs().max() <= 2.0 ** -14 + 2.0 ** -25 + 2.0 ** -10 * ref
    assert (lse.double() - math.log1p(small)).abs().max() <= SCORE
    assert pages.device_error() == 0


# ---------------------------------------------------------------- free slots
@pytest.mark.parametrize("dtype", DTYPES)
def test_free_slots_without_starts(dtype):
    """A step of one query each in a batch with free slots (length 0): nothing is flagged, their results are 0 and -infinity, as the
    decode's are, and the others' as those with starts; also in a captured call whose lengths change."""
    rng = np.random.default_rng(73)
    for lens in ([0], [5, 0, 700, 0, 1, 0], [0] * 399 + [17]):
        pool = Pool(rng, lens, 2, 16, dtype, scale=1.2)
        n = len(lens)
        q = normal(rng, (n, 6, 128), dtype)
        some = [r for r in range(n) if lens[r]]
        ws = pool.pages.tree_workspace(6)
        out, lse, step = torch.full((n, 6, 128), 7.0, dtype=dtype, device=DEV), torch.full((n, 6), 7.0, device=DEV), torch.empty((n, 6), device=DEV)
        call = lambda: paged.tree_attention(pool.pages, 0, q, pool.table, pool.device_lens, out=out, lse=lse, workspace=ws)  # noqa: E731
        call()
        paged.decode_attention(pool.pages, 0, q, pool.table, pool.device_lens, lse=step)
        w = torch.ones((n, 2, 701), device=DEV)
        paged.attention_weights(pool.pages, 0, q, pool.table, pool.device_lens, None, step, w, decay=0.5)
        assert pool.pages.device_error() == 0
        free = [r for r in range(n) if not lens[r]]
        assert torch.all(out[free] == 0) and torch.all(lse[free] == -math.inf) and torch.all(w[free] == 1)
        assert torch.all((lse[some] - step[some]).abs() <= 2 * SCORE)
        for r in some:
            assert torch.all((w[r, :, :lens[r]].double().sum(1) - 3 - 0.5 * lens[r]).abs() <= 2e-4 * 3 + 2.0 ** -22 * lens[r])
            assert torch.all(w[r, :, lens[r]:] == 1)
        if some:
            d = Drafts(rng, pool, [int(x > 0) for x in lens], 6)
            d.q = q[some].contiguous()
            got, got_lse = check_tree(pool, d)
            assert torch.equal(got, out[some]) and torch.equal(got_lse, lse[some])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        keep = (out.clone(), lse.clone())
        pool.device_lens.zero_()
        out.fill_(7.0)
        g.replay()
        assert torch.all(out == 0) and torch.all(lse == -math.inf)
        pool.device_lens.copy_(ints(lens))
        g.replay()
        assert torch.equal(out, keep[0]) and torch.equal(lse, keep[1])
        paged.tree_attention(pool.pages, 0, q, pool.table, pool.device_lens, out=out.fill_(7.0))
        assert torch.equal(out, keep[0]) and pool.pages.device_error() == 0
        # a length below 0 is none
        pool.device_lens.fill_(-1)
        call()
        assert pool.pages.device_error(clear=True) == 8


# ---------------------------------------------------------------- infinite values of tokens far below the others
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads", [4, 150])
@pytest.mark.parametrize("n,low,strong", [(600, 10, 300), (600, 10, 200), (600, 200, 10), (600, 10, 599), (70001, 10, 69000), (70001, 69000, 10)])
def test_infinite_value_far_below(n, low, strong, heads, dtype):
    """One infinite value of a weight of 2^-200 comes out, wherever the line is cut and whichever token is met first; the other
    dimensions are the strong token's."""
    rng = np.random.default_rng(74)
    pool = Pool(rng, [n], 1, 16, dtype)
    d = Drafts(rng, pool, [1], heads)
    x = torch.full((n,), -200 * math.log(2), device=DEV)
    x[strong] = 0.0
    pool.v[0][low, 0, 7], pool.v[0][low, 0, 9] = math.inf, -math.inf
    one_product(pool, d, [x])
    lse = torch.empty((1, heads), device=DEV)
    out = paged.tree_attention(pool.pages, 0, d.q, pool.table, pool.device_lens, d.starts, lse=lse, scale=1.0)
    assert torch.all(out[..., 7] == math.inf) and torch.all(out[..., 9] == -math.inf)
    rest = [i for i in range(128) if i not in (7, 9)]
    assert torch.all((out[0][:, rest].double() - pool.v[0][strong, 0, rest].double()).abs() <= 2.0 ** -7 * 6)
    assert torch.all(lse.abs() <= SCORE) and pool.pages.device_error() == 0


# ---------------------------------------------------------------- log-sums of two sets of tokens
def test_weights_by_the_log_sum_of_two_sets():
    """A decode joined with another set of tokens has the log-sum of both: weights are shares of that."""
    rng = np.random.default_rng(75)
    pool = Pool(rng, [300, 41], 2, 16, torch.bfloat16, scale=1.2)
    d = Drafts(rng, pool, [1, 1], 8)
    prior = (torch.randn((2, 8, 128), device=DEV), torch.full((2, 8), 6.0, device=DEV))
    lse = torch.empty((2, 8), device=DEV)
    paged.decode_attention(pool.pages, 0, d.q, pool.table, pool.device_lens, lse=lse, prior=prior)
    w = paged.attention_weights(pool.pages, 0, d.q, pool.table, pool.device_lens, None, lse, torch.zeros((2, 2, 300), device=DEV))
    for r, n in enumerate(pool.lens):
        s = scores_of(pool, d, r)[0]
        both = torch.logaddexp(torch.logsumexp(s, 1), torch.tensor(6.0, dtype=torch.float64, device=DEV))
        want = torch.exp(s - both[:, None]).view(2, 4, n).sum(1)
        assert torch.all((w[r, :, :n].double() - want).abs() <= (SCORE + 6e-5) * want + 1e-30)


# ---------------------------------------------------------------- pages outside the pool
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads", [4, 150])
def test_pages_outside_the_pool_in_every_other_tile(heads, dtype):
    """Every other tile of 128 tokens has a page outside the pool (flagged, its tokens drop out) and an infinite value, which comes
    out; the same bits in every run."""
    rng = np.random.default_rng(76)
    n, P = 3200, 32
    pool = Pool(rng, [n], 1, P, dtype, scale=1.2)
    d = Drafts(rng, pool, [1], heads)
    tiles = np.arange(0, n // 128, 2)
    pool.v[0][128 * tiles + 5, 0, tiles] = math.inf
    pool.put(0)
    pool.table[0, torch.from_numpy(4 * tiles + 1).to(DEV)] = pool.pages.n_pages
    left = np.array([t for t in range(n) if not (t // P % 4 == 1 and t // 128 % 2 == 0)])
    s = scores_of(pool, d, 0)[0][:, left]
    p, v = torch.softmax(s, 1), torch.where(torch.isfinite(pool.v[0]), pool.v[0], 0.0)[left, 0].double()
    first = None
    for _ in range(20):
        out = paged.tree_attention(pool.pages, 0, d.q, pool.table, pool.device_lens, d.starts)[0]
        assert pool.pages.device_error(clear=True) == 4
        assert torch.all(out[:, tiles] == math.inf)
        rest = np.setdiff1d(np.arange(128), tiles)
        u = torch.finfo(dtype).eps / 2
        bound = 1.01 * u * (p @ v.abs() + (p @ v).abs()) + 2 * SCORE * 6 + 2.0 ** -25 + n * 2.0 ** -30 * 6
        assert torch.all(((out.double() - p @ v).abs() <= bound)[:, rest])
        first = out if first is None else first
        assert torch.equal(out, first)


# ---------------------------------------------------------------- tables written just before
def test_tables_written_by_the_call_before():
    """Tables, lengths and weights that the call before on the stream writes, over and over: every call sees its own."""
    rng = np.random.default_rng(77)
    pool = Pool(rng, [2000, 300], 2, 16, torch.bfloat16, scale=1.2)
    d = Drafts(rng, pool, [3, 5], 8)
    tables = [pool.table, pool.table.clone()]
    used = pool.host[0, :125]
    tables[1][0, :125] = ints(used[rng.permutation(125)])
    want = []
    for t in tables:
        lse = torch.empty((8, 8), device=DEV)
        out = paged.tree_attention(pool.pages, 0, d.q, t, pool.device_lens, d.starts, lse=lse)
        w = torch.zeros((2, 2, 2000), device=DEV)
        paged.attention_weights(pool.pages, 0, d.q, t, pool.device_lens, d.starts, lse, w)
        want.append((out, lse, w))
    table, ws, got = torch.empty_like(tables[0]), pool.pages.tree_workspace(8), []
    for i in range(60):
        lse, w = torch.empty((8, 8), device=DEV), torch.zeros((2, 2, 2000), device=DEV)
        table.copy_(tables[i % 2])
        out = paged.tree_attention(pool.pages, 0, d.q, table, pool.device_lens, d.starts, lse=lse, workspace=ws)
        table.copy_(tables[i % 2])
        paged.attention_weights(pool.pages, 0, d.q, table, pool.device_lens, d.starts, lse, w)
        got.append((out, lse, w))
    for i, g in enumerate(got):
        assert all(torch.equal(x, y) for x, y in zip(g, want[i % 2])), i
    assert pool.pages.device_error() == 0
