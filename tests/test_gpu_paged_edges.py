"""The paged operators where types, streams and arguments end, on the GPU against their definitions in 64 bits.  Tolerances as
in test_gpu_paged; the ones that are finer are derived at their test."""
import math

import numpy as np
import pytest
import torch

from paper_2608_14191_gb300 import paged
from test_gpu_paged import DEV, DTYPES, SCORE, Pool, attend, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _built(aatc):
    return aatc


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", [8, 16, 64])
def test_decode_infinite_values(page, dtype):
    """Live infinities and NaN among the values come out as the formula has them, whatever the weight: of a token alone, of
    equal weights, of weights 2^-25 and 2^-40 of the largest, in the first unit and in the last one."""
    rng = np.random.default_rng([61, page])
    pool = Pool(rng, [1, 40, 90, 50, 1500, 17], 2, page, dtype)
    q = normal(rng, (6, 6, 128), dtype)
    inf, nan = math.inf, math.nan

    def put(r, t, kind, head, dims, values):
        to = (pool.k, pool.v)[kind][r]
        to[t, head, dims] = torch.tensor(values, dtype=dtype, device=DEV)
        pool.write(r, t, pool.k[r][t:t + 1], pool.v[r][t:t + 1])

    put(0, 0, 1, 0, [9, 77], [inf, -inf])
    q[1] = 0.0
    put(1, 7, 1, 1, [0, 127], [inf, nan])
    for t, values in ((5, [inf, -inf, inf, nan]), (6, [1.0, -inf, -inf, 2.0])):
        put(2, t, 1, 0, [9, 20, 64, 100], values)
    pool.k[3].zero_()
    pool.write(3, 0, pool.k[3], pool.v[3])
    q[3] = 0.0
    q[3, :, 0] = 1.0
    for t, bits in ((33, 25), (49, 40)):
        put(3, t, 0, 0, [0], [-bits * math.log(2) * math.sqrt(128)])
        put(3, t, 1, 0, [t], [inf])
    put(4, 1499, 1, 1, [63], [-inf])
    put(4, 700, 1, 0, [1], [inf])
    put(5, 16, 1, 0, [2], [inf])
    lse = torch.empty((6, 6), device=DEV)
    out = paged.decode_attention(pool.pages, 0, q, pool.table, pool.device_lens, lse=lse).double()
    for b in range(6):
        ref, ref_lse = attend(q[b], pool.k[b], pool.v[b])
        assert not torch.isfinite(ref).all()
        assert torch.equal(torch.isnan(out[b]), torch.isnan(ref)), b
        odd = torch.isinf(ref)
        assert torch.equal(out[b][odd], ref[odd]) and torch.equal(torch.isinf(out[b]), odd), b
        fine = torch.isfinite(ref)
        assert (out[b] - ref)[fine].abs().max() <= 2 * SCORE * 6 and (lse[b] - ref_lse).abs().max() <= SCORE, b
    assert pool.pages.device_error() == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bits", [5, 12, 18, 24, 28.5, 30.5, 33])
def test_decode_small_weights(bits, dtype):
    """Every unit has one token of weight 1 and value 0 beside fifteen of weight 2^-bits and values of 0.5 to 1.5, so the result
    is what the small weights keep.  A weight carries 22 bits, or 2^-42 of the largest where that is more: the scores' SCORE on
    either side as everywhere, and 15 * 1.5 * 2^-42."""
    rng = np.random.default_rng([62, int(2 * bits)])
    n = 1600
    pool = Pool(rng, [n], 1, 16, dtype)
    large = torch.arange(n, device=DEV) % 16 == 3
    pool.k[0].zero_()
    pool.k[0][~large, 0, 0] = -bits * math.log(2)
    pool.v[0].copy_(torch.from_numpy(rng.uniform(0.5, 1.5, (n, 1, 128))).to(DEV))
    pool.v[0][large] = 0.0
    pool.write(0, 0, pool.k[0], pool.v[0])
    q = torch.zeros((1, 4, 128), dtype=dtype, device=DEV)
    q[..., 0] = 1.0
    out = paged.decode_attention(pool.pages, 0, q, pool.table, pool.device_lens, scale=1.0).double()
    ref, _ = attend(q[0], pool.k[0], pool.v[0], scale=1.0)
    assert torch.all((out[0] - ref).abs() <= 2 * SCORE * ref + 15 * 1.5 * 2.0 ** -42)
    assert pool.pages.device_error() == 0


def test_results_of_a_given_stream_are_in_its_own_memory():
    """A result that is made for a call on another stream does not lie in a block that the current stream got back just
    before (what is queued there may still use it), and the values come out with work queued on both."""
    rng = np.random.default_rng(63)
    pool = Pool(rng, [300, 47], 2, 16, torch.bfloat16)
    rope = paged.Rotary(64, 10000.0, device=DEV)
    q = normal(rng, (2, 8, 128), torch.bfloat16)
    x = normal(rng, (4000, 8, 128), torch.bfloat16)
    places = torch.tensor([300, 47], dtype=torch.int32, device=DEV)
    kv = normal(rng, (2, 2, 128), torch.bfloat16)
    far = torch.arange(4000, dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    calls = {
        "rotate": lambda stream: (paged.rotate(rope, x, far, stream=stream),),
        "append": lambda stream: (paged.append(pool.pages, 0, kv, kv, pool.table, places, rope=rope, q=q, stream=stream),),
        "decode": lambda stream: (paged.decode_attention(pool.pages, 0, q, pool.table, pool.device_lens, stream=stream),),
        "gather": lambda stream: paged.gather(pool.pages, 0, pool.table, 0, 40, stream=stream),
    }
    for name, call in calls.items():
        want = call(None)
        shapes = [(w.shape, w.dtype) for w in want]
        torch.cuda.synchronize()
        for _ in range(3):
            held = [torch.empty(s, dtype=d, device=DEV) for s, d in shapes for _ in range(4)]
            blocks = [(h.data_ptr(), h.data_ptr() + h.nbytes) for h in held]
            torch.cuda._sleep(2_000_000)                          # about a millisecond of the current stream's time
            for h in held:
                h.fill_(7.0)
            del held, h
            got = call(side)
            assert not any(a < g.data_ptr() + g.nbytes and g.data_ptr() < b for g in got for a, b in blocks), name
            torch.cuda.synchronize()
            assert all(torch.equal(g, w) for g, w in zip(got, want)), name
    assert pool.pages.device_error() == 0


def test_decode_longer_than_its_waits():
    """A call of some three seconds (65535 sequences that share 896000 places of 64 pages) is not taken for one that stands
    still: its waits are bounded at one and two seconds each, of no progress.  A lane of the kernel adds up to 56000
    weights between 0.01 and 100 one after the other: relative 56000 * 2^-24 of the sum and of the outputs' sums."""
    rng = np.random.default_rng(64)
    batch, places, n_q = 65535, 3500, 2
    pages = paged.Pages(1, 64, 1, 256, torch.bfloat16, DEV)
    pages.data.copy_(torch.from_numpy(rng.standard_normal(pages.data.shape)))
    pages.data[:, :, 1] = pages.data[:, :, 1].clamp(-1, 1) / 2 + 1
    host = rng.integers(0, 64, places)
    table = torch.from_numpy(host).to(DEV, torch.int32)[None].expand(batch, -1)
    q = normal(rng, (1, n_q, 128), torch.bfloat16)
    lens = torch.full((batch,), places * 256, dtype=torch.int32, device=DEV)
    out = torch.full((batch, n_q, 128), math.nan, device=DEV)
    lse = torch.full((batch, n_q), math.nan, device=DEV)
    workspace = pages.decode_workspace(n_q)
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    paged.decode_attention(pages, 0, q.expand(batch, -1, -1), table, lens, out=out, lse=lse, workspace=workspace)
    end.record()
    end.synchronize()
    assert pages.device_error() == 0
    assert begin.elapsed_time(end) > 2000                          # (or it does not reach what it is for)
    k, v = (pages.data[0, :, i, 0].double().reshape(-1, 128) for i in (0, 1))
    times = torch.from_numpy(np.bincount(host, minlength=64)).to(DEV).repeat_interleave(256).double()
    s = q[0].double() @ k.T / math.sqrt(128)
    assert s.abs().max() < math.log(100)
    weights = times * torch.exp(s)
    ref, ref_lse = weights @ v / weights.sum(1, keepdim=True), weights.sum(1).log()
    chain = 56000 * 2.0 ** -24
    assert torch.all((lse - ref_lse).abs() <= SCORE + chain)
    assert torch.all((out - ref).abs() <= (2 * SCORE + 2 * chain) * 1.5)


@pytest.mark.parametrize("n", [1, 40, 5000])
def test_gather_flags_lengths_outside_the_table(n):
    """Lengths below 0 and past the table are flagged, as in the decode; they count as 0 and as the whole table."""
    rng = np.random.default_rng([65, n])
    pool = Pool(rng, [n, n, n], 2, 16, torch.float16)
    table = pool.table[:, :-(-n // 16)].contiguous()              # (no wider than the sequences)
    room = table.shape[1] * 16
    dev = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    for lens, flag in ((dev(n, 0, room), 0), (dev(n, -1, n), 8), (dev(room + 1, 0, n), 8), (dev(0, n, 2**31 - 1), 8), (dev(-2**31, n, n), 8)):
        k, v = paged.gather(pool.pages, 0, table, 0, n, lens=lens)
        assert pool.pages.device_error(clear=True) == flag
        for r, length in enumerate(lens.tolist()):
            live = max(0, min(length, n))
            for got, x in ((k, pool.k), (v, pool.v)):
                assert torch.equal(got[r, :live], x[r][:live]) and torch.all(got[r, live:] == 0)


@pytest.mark.parametrize("batch", [1, 100, 385])
@pytest.mark.parametrize("room,window", [(256, 0), (264, 0), (272, 0), (640, 255), (640, 256), (640, 257), (640, 271), (640, 272), (256, 300)])
def test_decode_around_whole_segments(room, window, batch):
    """Tables and windows of fewer than 272 tokens, whose segments go whole to one CTA, and wider ones, whose pieces go through the
    workspace; the lengths let windows begin anywhere in a unit."""
    rng = np.random.default_rng([66, room, window, batch])
    lens = rng.integers(0, room + 1, batch)
    lens[rng.integers(0, batch)] = room
    pages = paged.Pages(1, batch * room // 8, 2, 8, torch.bfloat16, DEV)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV, torch.int32)  # noqa: E731
    table = dev(rng.permutation(pages.n_pages).reshape(batch, -1))
    index = np.concatenate([np.arange(n) for n in lens])
    k, v = (normal(rng, (len(index), 2, 128), torch.bfloat16) for _ in range(2))
    paged.append(pages, 0, k, v, table, dev(index), rows=dev(np.repeat(np.arange(batch), lens)))
    q = normal(rng, (batch, 6, 128), torch.bfloat16)
    workspace = pages.decode_workspace(6).fill_(-3.0)
    lse = torch.empty((batch, 6), device=DEV)
    out = paged.decode_attention(pages, 0, q, table, dev(lens), lse=lse, window=window, workspace=workspace)
    start = np.concatenate([[0], np.cumsum(lens)])
    for b in range(batch):
        part = slice(int(start[b]), int(start[b + 1]))
        ref, ref_lse = attend(q[b], k[part], v[part], window=window)
        assert (out[b] - ref).abs().max() <= 2 * SCORE * 6, b
        assert lens[b] == 0 or (lse[b] - ref_lse).abs().max() <= SCORE, b
    whole = min(room, window or room) < 272
    pieces = workspace[:-4 * torch.cuda.get_device_properties(0).multi_processor_count]
    assert bool((pieces == -3.0).all()) == whole
    assert pages.device_error() == 0
