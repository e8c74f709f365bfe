"""The paged cache's operators on the GPU against their definitions in 64 bits.

Tolerances.  Rotations: one rounding to p significant bits (bf16 8, f16 11), so 2^-p of the value, and the
fp32 arithmetic before it: an angle within 2^-23, sine and cosine within 2^-22, three roundings, under
2^-20 of |a| + |b|.  Attention: every score here is under 32 in size (asserted), a chain of 8 fp32 sums
of 16 products that may truncate at 2^-23 of the running value errs by under 32 * 8 * 2^-23 = 3.1e-5, so the
log-sum-exp is within SCORE = 4e-5 with its own rounding, and the output, whose weights each move by
that factor at most and are normalised, within 2 SCORE max |v|.  Moved values are compared bit for bit."""
import math

import numpy as np
import pytest
import torch

from paper_2608_14191_gb300 import paged

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SCORE = 4e-5
DTYPES = [torch.bfloat16, torch.float16]
BITS = {torch.bfloat16: 8, torch.float16: 11}


@pytest.fixture(autouse=True)
def _built(aatc):
    return aatc


def normal(rng, shape, dtype, scale=1.0):
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(DEV).to(dtype)


# ---------------------------------------------------------------- rotary positions
def turned(x, positions, rope, backward=False):
    """rope's rotation of x [n][h][128] in 64 bits, and the bound of its fp32 arithmetic."""
    w = torch.from_numpy(rope.frequencies).to(DEV)
    angle = positions.double()[:, None, None] * w
    c, s = angle.cos() * rope.factor, angle.sin() * rope.factor * (-1 if backward else 1)
    y, slack = x.double().clone(), torch.zeros_like(x, dtype=torch.float64)
    r = rope.rot_dim
    pair = (slice(0, r // 2), slice(r // 2, r)) if rope.layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    a, b = (x[..., p].double() for p in pair)
    y[..., pair[0]], y[..., pair[1]] = a * c - b * s, a * s + b * c
    for p in pair:
        slack[..., p] = (a.abs() + b.abs()) * abs(rope.factor) * 2.0 ** -20
    return y, slack


def check_turned(got, x, positions, rope, backward=False):
    y, slack = turned(x, positions, rope, backward)
    bound = y.abs() * 2.0 ** -BITS[x.dtype] + slack + (2.0 ** -25 if x.dtype == torch.float16 else 0.0)
    assert torch.all((got.double() - y).abs() <= bound)
    assert torch.equal(got[..., rope.rot_dim:], x[..., rope.rot_dim:])


SCALINGS = [None, dict(kind="linear", factor=4.0), dict(kind="ntk", factor=2.5),
            dict(kind="ramp", factor=8.0, original=2048, fast=32.0, slow=1.0),
            dict(kind="banded", factor=8.0, original=8192, low=1.0, high=4.0)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rot,scaling,n,heads", [(128, None, 1, 1), (128, SCALINGS[4], 333, 8), (64, SCALINGS[3], 65, 7),
                                                 (96, SCALINGS[1], 130, 3), (16, SCALINGS[2], 1000, 32),
                                                 (112, None, 17, 28), (32, SCALINGS[3], 4097, 12)])
def test_rotate(rot, scaling, n, heads, layout, dtype):
    rng = np.random.default_rng([rot, n])
    rope = paged.Rotary(rot, 500000.0, layout, scaling, DEV)
    x = normal(rng, (n, heads, 128), dtype)
    positions = torch.from_numpy(rng.integers(-5, 1 << 20, n)).to(DEV, torch.int32)
    for backward in (False, True):
        check_turned(paged.rotate(rope, x, positions, backward=backward), x, positions, rope, backward)
    y = x.clone()
    assert paged.rotate(rope, y, positions, out=y) is y
    assert torch.equal(y, paged.rotate(rope, x, positions))


def test_rotate_extreme_positions_and_strides():
    """Positions at both ends of 32 bits keep their angle; heads before tokens, rows inside wider ones."""
    rng = np.random.default_rng(3)
    rope = paged.Rotary(128, 10000.0, device=DEV)
    positions = torch.tensor([0, 1, -1, 2**31 - 1, -2**31, 131071, 7], dtype=torch.int32, device=DEV)
    x = normal(rng, (5, 7, 256), torch.float16)[..., 128:].transpose(0, 1)
    # the angle of the exact turns: position times frequency in 64 bits is off by 2^-53 * 2^31 at most
    got = paged.rotate(rope, x, positions)
    check_turned(got, x, positions, rope)
    out = torch.full((7, 9, 200), 5.0, dtype=torch.float16, device=DEV)
    assert paged.rotate(rope, x, positions, out=out[:, 2:7, 16:144]) is not None
    assert torch.equal(out[:, 2:7, 16:144], got)
    out[:, 2:7, 16:144] = 5.0
    assert torch.all(out == 5.0)


def test_rotate_over_32_bit_offsets():
    rng = np.random.default_rng(4)
    rope = paged.Rotary(64, 10000.0, "interleaved", device=DEV)
    far = torch.empty((1 << 31) + 1024, dtype=torch.bfloat16, device=DEV)
    x = far.as_strided((3, 2, 128), (1 << 30, 128, 1))
    x.copy_(normal(rng, (3, 2, 128), torch.bfloat16))
    want = x.clone()
    positions = torch.tensor([3, 70000, 12], dtype=torch.int32, device=DEV)
    check_turned(paged.rotate(rope, x, positions), want, positions, rope)
    paged.rotate(rope, x, positions, out=x)
    check_turned(x, want, positions, rope)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotate_gradient(layout):
    """backward against the transposed Jacobian by differences: the map is linear, so a difference of any width
    is its derivative up to the roundings of its two ends (2^-11 of values up to 4, over a width of 2)."""
    rng = np.random.default_rng(5)
    rope = paged.Rotary(32, 10000.0, layout, dict(kind="ramp", factor=4.0, original=64, fast=4.0, slow=0.5), DEV)
    positions = torch.full((256,), 37, dtype=torch.int32, device=DEV)
    steps = torch.eye(128, dtype=torch.float16, device=DEV)[:, None].repeat(2, 1, 1)
    steps[128:] *= -1
    ends = paged.rotate(rope, steps, positions).double()[:, 0]
    jacobian = (ends[:128] - ends[128:]) / 2                       # [input][output]
    g = normal(rng, (256, 1, 128), torch.float16)
    got = paged.rotate(rope, g, positions, backward=True)
    want = g.double()[:, 0] @ jacobian.T
    bound = 2 * 2.0 ** -11 * 4 * 2
    assert (got.double()[:, 0] - want).abs().max() <= bound
    check_turned(got, g, positions, rope, backward=True)


# ---------------------------------------------------------------- pages
class Pool:
    """A pool full of NaN, and sequences whose pages lie in it in random order; table entries that no
    token needs are ids outside the pool."""

    def __init__(self, rng, lens, n_kv, page, dtype, scale=1.0, extra=2):
        self.lens, self.page, self.rng = list(lens), page, rng
        per = [-(-n // page) for n in lens]
        self.pages = paged.Pages(1, max(1, sum(per)) + extra, n_kv, page, dtype, DEV)
        self.pages.data.fill_(float("nan"))
        ids = rng.permutation(self.pages.n_pages)[:sum(per)]
        m = max(1, max(per)) + 1
        table = np.full((len(lens), m), 2**31 - 1, np.int64)
        at = 0
        for r, k in enumerate(per):
            table[r, :k] = ids[at:at + k]
            at += k
        self.host = table
        self.table = torch.from_numpy(table).to(DEV, torch.int32)
        self.device_lens = torch.tensor(self.lens, dtype=torch.int32, device=DEV)
        self.k = [normal(rng, (n, n_kv, 128), dtype, scale) for n in lens]
        self.v = [normal(rng, (n, n_kv, 128), dtype) for n in lens]
        for r in range(len(lens)):
            self.write(r, 0, self.k[r], self.v[r])

    def write(self, r, first, k, v):
        for i in range(0, len(k)):
            t = first + i
            where = self.pages.data[0, int(self.host[r, t // self.page])]
            where[0, :, t % self.page], where[1, :, t % self.page] = k[i], v[i]


def attend(q, k, v, scale=1 / math.sqrt(128), cap=0.0, window=0, slopes=None, prior=None):
    """out, lse of one sequence in 64 bits: q [n_q][128], k and v [n][n_kv][128], prior (out0, lse0)."""
    n, group = len(k), q.shape[0] // k.shape[1] if k.shape[1] else 1
    kd, vd = (x.double().repeat_interleave(group, 1) for x in (k, v))
    s = torch.einsum("hd,nhd->hn", q.double(), kd) * scale
    if n:
        fine = s[torch.isfinite(s)]
        assert fine.numel() == 0 or fine.abs().max() < 32
    if cap:
        s = cap * torch.tanh(s / cap)
    if slopes is not None:
        s = s + slopes.double()[:, None] * (torch.arange(n, device=DEV) - (n - 1)).double()
    if window:
        s, vd = s[:, max(0, n - window):], vd[max(0, n - window):]
    if prior is not None:
        s = torch.cat([s, prior[1].double()[:, None]], 1)
        vd = torch.cat([vd, prior[0].double()[None]], 0)
    if s.shape[1] == 0:
        return torch.zeros_like(q, dtype=torch.float64), torch.full((len(q),), -math.inf, device=DEV).double()
    lse = torch.logsumexp(s, 1)
    p = torch.where(lse[:, None] == -math.inf, 0.0, torch.exp(s - lse[:, None]))
    if prior is not None:                                          # (the prior of nothing may hold anything)
        vd = torch.cat([vd[:-1], torch.where(p[:, -1, None] > 0, vd[-1], 0.0)[None]], 0)
    return torch.einsum("hn,nhd->hd", p, vd), lse


def check_decode(pool, q, lse=True, prior=None, **how):
    batch, n_q = q.shape[:2]
    out = torch.full((batch, n_q, 128), float("nan"), device=DEV)
    got_lse = torch.full((batch, n_q), float("nan"), device=DEV) if lse else None
    paged.decode_attention(pool.pages, 0, q, pool.table, pool.device_lens, out=out, lse=got_lse, prior=prior, **how)
    for b in range(batch):
        one = None if prior is None else (prior[0][b], prior[1][b])
        ref, ref_lse = attend(q[b], pool.k[b], pool.v[b], prior=one, **how)
        big = max([1.0] + [float(x.double().abs().max()) for x in (pool.v[b],) + ((prior[0][b],) if prior else ()) if x.numel()])
        assert torch.isfinite(ref).all()
        assert (out[b] - ref).abs().max() <= 2 * SCORE * big, (b, float((out[b] - ref).abs().max()))
        if lse:
            empty = ref_lse == -math.inf
            assert torch.equal(got_lse[b] == -math.inf, empty)
            assert torch.all((got_lse[b] - ref_lse)[~empty].abs() <= SCORE)
    assert pool.pages.device_error() == 0
    return out, got_lse


LENGTHS = [
    [1], [0], [7], [16], [17], [1000], [5, 0, 1, 64, 0, 129], [255, 256, 257], [3] * 40, [0, 0], [4099, 2, 1500],
    list(range(0, 70, 3)),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", [8, 16, 64, 256])
@pytest.mark.parametrize("lens", LENGTHS, ids=lambda x: f"{len(x)}x{max(x)}")
def test_decode_lengths(lens, page, dtype):
    rng = np.random.default_rng([len(lens), max(lens), page])
    pool = Pool(rng, lens, 2, page, dtype, scale=1.5)
    check_decode(pool, normal(rng, (len(lens), 8, 128), dtype))


@pytest.mark.parametrize("n_kv,group", [(1, 1), (8, 1), (8, 4), (4, 7), (2, 8), (3, 5), (1, 12), (2, 17), (1, 32), (5, 2)])
def test_decode_heads(n_kv, group):
    rng = np.random.default_rng([n_kv, group])
    pool = Pool(rng, [300, 1, 47, 1111], n_kv, 32, torch.bfloat16, scale=1.5)
    check_decode(pool, normal(rng, (4, n_kv * group, 128), torch.bfloat16))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("how", [dict(cap=5.0), dict(window=1), dict(window=16), dict(window=100), dict(window=10**6),
                                 dict(scale=0.3), dict(scale=0.0), dict(cap=30.0, window=77, scale=0.2)], ids=str)
def test_decode_options(how, dtype):
    rng = np.random.default_rng([len(str(how))])
    pool = Pool(rng, [0, 1, 100, 101, 640, 2011], 2, 16, dtype, scale=0.7)
    q = normal(rng, (6, 6, 128), dtype)
    check_decode(pool, q, **how)
    slopes = torch.from_numpy(2.0 ** -rng.uniform(0, 9, 6)).to(DEV).float()
    check_decode(pool, q, lse=False, slopes=slopes, **how)


def test_decode_prior():
    """A split context: one part's result joins the other's; parts of nothing; results in the prior's place."""
    rng = np.random.default_rng(11)
    lens = [0, 0, 5, 700, 33, 1500]
    pool = Pool(rng, lens, 2, 16, torch.bfloat16, scale=1.2)
    q = normal(rng, (6, 8, 128), torch.bfloat16)
    out0 = torch.from_numpy(rng.standard_normal((6, 8, 128))).to(DEV).float()
    lse0 = torch.from_numpy(rng.uniform(-3, 9, (6, 8))).to(DEV).float()
    lse0[1], lse0[2], lse0[3, :4], lse0[4] = -math.inf, -math.inf, -math.inf, 31.0
    out0[1], out0[2] = 0.0, float("nan")                           # what a part of no tokens holds is not read
    out, lse = check_decode(pool, q, prior=(out0, lse0))
    assert torch.all(out[1] == 0) and torch.all(lse[1] == -math.inf)
    same = out0.clone(), lse0.clone()
    paged.decode_attention(pool.pages, 0, q, pool.table, pool.device_lens, out=same[0], lse=same[1], prior=same)
    assert torch.equal(same[0], out) and torch.equal(same[1], lse)
    # a sequence cut in two, and whole
    n, cut = 1500, 48 * 16
    table, lens = pool.table[5:, :cut // 16].contiguous(), torch.tensor([cut], dtype=torch.int32, device=DEV)
    first = paged.decode_attention(pool.pages, 0, q[5:], table, lens, lse=lse[5:])
    rest = torch.tensor([n - cut], dtype=torch.int32, device=DEV)
    both = paged.decode_attention(pool.pages, 0, q[5:], pool.table[5:, cut // 16:], rest, prior=(first, lse[5:]))
    ref, _ = attend(q[5], pool.k[5], pool.v[5])
    assert (both[0] - ref).abs().max() <= 2 * SCORE * float(pool.v[5].double().abs().max())


def test_decode_values_outside_the_number_line():
    """Keys that make a score -infinity drop their token; infinities of live values come out; nothing else
    changes.  (Masked places hold NaN in every test: the pools are full of it.)"""
    rng = np.random.default_rng(12)
    pool = Pool(rng, [200, 3, 90], 1, 16, torch.bfloat16)
    q = normal(rng, (3, 4, 128), torch.bfloat16)
    q[:, :, 0] = 1.0
    for r, gone in ((0, [0, 17, 199]), (1, [0, 1, 2])):
        for t in gone:
            pool.k[r][t, 0, 0] = -math.inf
            pool.write(r, t, pool.k[r][t:t + 1], pool.v[r][t:t + 1])
    pool.v[2][5, 0, 9] = math.inf
    pool.write(2, 5, pool.k[2][5:6], pool.v[2][5:6])
    lse = torch.empty((3, 4), device=DEV)
    out = paged.decode_attention(pool.pages, 0, q, pool.table, pool.device_lens, lse=lse)
    left = [t for t in range(200) if t not in (0, 17, 199)]
    ref, ref_lse = attend(q[0], pool.k[0][left], pool.v[0][left])
    assert (out[0] - ref).abs().max() <= 2 * SCORE * 6 and (lse[0] - ref_lse).abs().max() <= SCORE
    assert torch.all(lse[1] == -math.inf) and torch.all(out[1] == 0)
    assert torch.all(out[2, :, 9] == math.inf) and torch.isfinite(out[2, :, :9]).all() and torch.isfinite(out[2, :, 10:]).all()


def test_decode_bad_tables_are_flagged():
    """A page id outside the pool drops that page's tokens, a length past the table is cut; both are flagged."""
    rng = np.random.default_rng(13)
    pool = Pool(rng, [100, 100], 2, 16, torch.bfloat16)
    q = normal(rng, (2, 8, 128), torch.bfloat16)
    table = pool.table.clone()
    table[0, 3] = -1
    out = paged.decode_attention(pool.pages, 0, q, table, pool.device_lens)
    left = [t for t in range(100) if t // 16 != 3]
    ref, _ = attend(q[0], pool.k[0][left], pool.v[0][left])
    assert (out[0] - ref).abs().max() <= 2 * SCORE * 6
    assert (out[1] - attend(q[1], pool.k[1], pool.v[1])[0]).abs().max() <= 2 * SCORE * 6
    assert pool.pages.device_error(clear=True) == 4 and pool.pages.device_error() == 0
    lens = torch.tensor([-3, 2**31 - 1], dtype=torch.int32, device=DEV)
    cut = pool.table[:, :2].contiguous()
    out = paged.decode_attention(pool.pages, 0, q, cut, lens)
    assert torch.all(out[0] == 0)
    assert (out[1] - attend(q[1], pool.k[1][:32], pool.v[1][:32])[0]).abs().max() <= 2 * SCORE * 6
    assert pool.pages.device_error(clear=True) == 8


def test_decode_strides_streams_and_graphs():
    """Queries inside a wider projection, a table inside a wider one; a side stream; a captured call whose
    lengths grow; the same bits every time."""
    rng = np.random.default_rng(14)
    lens = [500, 20, 0, 1301]
    pool = Pool(rng, lens, 2, 16, torch.bfloat16)
    wide = normal(rng, (4, 12, 256), torch.bfloat16)
    q = wide[:, 1:9, 64:192]
    wide_table = torch.full((4, pool.table.shape[1] + 5), -9, dtype=torch.int32, device=DEV)
    wide_table[:, 3:-2] = pool.table
    out, _ = check_decode(pool, q)
    pool.table = wide_table[:, 3:-2]
    again, _ = check_decode(pool, q)
    assert torch.equal(out, again)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = pool.pages.decode_workspace(8)
    with torch.cuda.stream(side):
        on_side = paged.decode_attention(pool.pages, 0, q, pool.table, pool.device_lens, workspace=ws)
    given = paged.decode_attention(pool.pages, 0, q, pool.table, pool.device_lens, stream=side, workspace=ws)
    side.synchronize()
    assert torch.equal(on_side, out) and torch.equal(given, out)
    graph, res = torch.cuda.CUDAGraph(), torch.empty_like(out)
    with torch.cuda.graph(graph):
        paged.decode_attention(pool.pages, 0, q, pool.table, pool.device_lens, out=res, workspace=ws)
    for cut in ([500, 20, 0, 1301], [1, 0, 0, 700]):
        pool.device_lens.copy_(torch.tensor(cut, dtype=torch.int32))
        graph.replay()
        for b, n in enumerate(cut):
            ref, _ = attend(q[b], pool.k[b][:n], pool.v[b][:n])
            assert (res[b] - ref).abs().max() <= 2 * SCORE * 6


@pytest.mark.parametrize("batch,most", [(300, 40), (1, 40000), (33, 2500)])
def test_decode_many_and_long(batch, most):
    """More sequences than SMs, and one sequence over all of them (written by append)."""
    rng = np.random.default_rng([batch, most])
    lens = rng.integers(0, most + 1, batch)
    lens[0] = most
    pages = paged.Pages(1, int(sum(-(-lens // 16))) + 1, 2, 16, torch.bfloat16, DEV)
    per = -(-lens // 16)
    table = torch.zeros((batch, int(per.max())), dtype=torch.int32)
    ids = rng.permutation(pages.n_pages)
    at = np.concatenate([[0], np.cumsum(per)])
    for b in range(batch):
        table[b, :per[b]] = torch.from_numpy(ids[at[b]:at[b + 1]])
    table = table.to(DEV)
    rows = torch.from_numpy(np.repeat(np.arange(batch), lens)).to(DEV, torch.int32)
    index = torch.from_numpy(np.concatenate([np.arange(n) for n in lens])).to(DEV, torch.int32)
    k, v = (normal(rng, (int(lens.sum()), 2, 128), torch.bfloat16) for _ in range(2))
    paged.append(pages, 0, k, v, table, index, rows=rows)
    q = normal(rng, (batch, 8, 128), torch.bfloat16)
    lse = torch.empty((batch, 8), device=DEV)
    out = paged.decode_attention(pages, 0, q, table, torch.from_numpy(lens).to(DEV, torch.int32), lse=lse)
    first = np.concatenate([[0], np.cumsum(lens)])
    for b in range(batch):
        part = slice(int(first[b]), int(first[b + 1]))
        ref, ref_lse = attend(q[b], k[part], v[part])
        assert (out[b] - ref).abs().max() <= 2 * SCORE * 6, b
        if lens[b]:
            assert (lse[b] - ref_lse).abs().max() <= SCORE
    assert pages.device_error() == 0


# ---------------------------------------------------------------- append, gather, copies
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n_kv,group,page,rot,layout", [(8, 4, 16, 128, "half"), (4, 7, 8, 64, "interleaved"),
                                                        (1, 1, 256, 16, "half"), (3, 5, 32, 96, "interleaved")])
def test_append(n_kv, group, page, rot, layout, dtype):
    rng = np.random.default_rng([n_kv, page])
    before = [0, 3, 37, 0, 290]
    new = [1, 30, 0, 45, 270]
    pool = Pool(rng, [a + b for a, b in zip(before, new)], n_kv, page, dtype)
    want = pool.pages.data.clone()
    rows = np.repeat(np.arange(5), new)
    index = np.concatenate([np.arange(a, a + b) for a, b in zip(before, new)])
    order = rng.permutation(len(rows))                             # tokens of a packed batch in any order
    rows, index = rows[order], index[order]
    index[::17] = -1                                               # padding
    n = len(rows)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV, torch.int32)  # noqa: E731
    qkv = normal(rng, (n, (group + 2) * n_kv, 128), dtype)
    q, k, v = qkv[:, :group * n_kv], qkv[:, group * n_kv:(group + 1) * n_kv], qkv[:, (group + 1) * n_kv:]
    rope = paged.Rotary(rot, 10000.0, layout, dict(kind="linear", factor=2.0), DEV)
    positions = dev(rng.integers(0, 100000, n))
    for pos in (None, positions):
        at = dev(index) if pos is None else pos
        pool.pages.data.copy_(want)
        got_q = paged.append(pool.pages, 0, k, v, pool.table, dev(index), rows=dev(rows), positions=pos, rope=rope, q=q)
        check_turned(got_q, q, at, rope)
        turned_k = paged.rotate(rope, k, at)
        check_turned(turned_k, k, at, rope)
        for i in range(n):
            if index[i] < 0:
                continue
            where = (0, int(pool.host[rows[i], index[i] // page]))
            assert torch.equal(pool.pages.data[where][0, :, index[i] % page], turned_k[i])
            assert torch.equal(pool.pages.data[where][1, :, index[i] % page], v[i])
            pool.pages.data[where][:, :, index[i] % page] = want[where][:, :, index[i] % page]
        same = torch.isnan(want) & torch.isnan(pool.pages.data) | (want == pool.pages.data)
        assert torch.all(same)                                     # and nothing else was written
    # without rotation; queries in place
    paged.append(pool.pages, 0, k, v, pool.table, dev(index), rows=dev(rows))
    i = int(np.flatnonzero(index >= 0)[-1])
    assert torch.equal(pool.pages.data[0, int(pool.host[rows[i], index[i] // page]), 0, :, index[i] % page], k[i])
    held = q.clone()
    assert paged.append(pool.pages, 0, k, v, pool.table, dev(index), rows=dev(rows), rope=rope, q=q, q_out=q) is q
    check_turned(q, held, dev(index), rope)
    assert pool.pages.device_error() == 0


def test_append_bad_places_are_flagged():
    rng = np.random.default_rng(22)
    pool = Pool(rng, [40, 40], 2, 16, torch.bfloat16)
    want = pool.pages.data.clone()
    k = normal(rng, (2, 2, 128), torch.bfloat16)
    dev = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    for rows, index, flag in ((dev(0, 2), dev(-1, 0), 8), (dev(-1, 0), dev(0, -7), 8), (dev(0, 1), dev(-1, 16 * 4), 8),
                              (dev(0, 1), dev(-1, 50), 4), (dev(0, 1), dev(-1, 2**31 - 1), 8)):
        paged.append(pool.pages, 0, k, k, pool.table, index, rows=rows)
        assert pool.pages.device_error(clear=True) == flag
    assert torch.all(torch.isnan(want) & torch.isnan(pool.pages.data) | (want == pool.pages.data))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page,n_kv,first,n", [(16, 8, 0, 16), (16, 8, 5, 16), (8, 3, 13, 1), (64, 1, 0, 290), (256, 4, 255, 2),
                                               (32, 2, 31, 200)])
def test_gather(page, n_kv, first, n, dtype):
    rng = np.random.default_rng([page, n])
    lens = [first + n, first + n + 40, max(first, 1), 0, first + (n + 1) // 2]
    pool = Pool(rng, lens, n_kv, page, dtype)
    k, v = paged.gather(pool.pages, 0, pool.table[:2], first, n)
    for r in (0, 1):
        assert torch.equal(k[r], pool.k[r][first:first + n]) and torch.equal(v[r], pool.v[r][first:first + n])
    if first + n > pool.table.shape[1] * page:
        return
    k, v = paged.gather(pool.pages, 0, pool.table, first, n, lens=pool.device_lens)
    for r, length in enumerate(lens):
        live = max(0, min(length - first, n))
        for got, x in ((k, pool.k), (v, pool.v)):
            assert torch.equal(got[r, :live], x[r][first:first + live]) and torch.all(got[r, live:] == 0)
    assert pool.pages.device_error() == 0
    paged.gather(pool.pages, 0, torch.full((1, 40), -1, dtype=torch.int32, device=DEV), first, n, out=(k[:1], v[:1]))
    assert torch.all(k[0] == 0) and pool.pages.device_error() == 4


@pytest.mark.parametrize("layers,n_pages,n_kv,page,n", [(1, 2, 1, 8, 1), (3, 40, 2, 16, 20), (32, 30, 8, 16, 7), (2, 2600, 1, 8, 1300),
                                                        (1, 9, 5, 256, 3)])
def test_copy_pages(layers, n_pages, n_kv, page, n):
    rng = np.random.default_rng([layers, n_pages])
    data = torch.from_numpy(rng.integers(0, 1 << 15, (layers, n_pages, 2, n_kv, page, 128)).astype(np.int16)).to(DEV)
    pages = paged.Pages.of(data.view(torch.float16))
    ids = rng.permutation(n_pages)
    pairs = np.stack([rng.choice(ids[n:], n) if n_pages > n + 1 else ids[n:n + 1], ids[:n]], 1)
    want = data.clone()
    want[:, torch.from_numpy(pairs[:, 1]).to(DEV)] = want[:, torch.from_numpy(pairs[:, 0]).to(DEV)]
    paged.copy_pages(pages, pairs)
    assert torch.equal(data, want)
    paged.copy_pages(pages, np.zeros((0, 2)))
    assert torch.equal(data, want)


def test_pages_over_32_bit_offsets():
    """A pool of more than 2^31 values: its last pages are written, read, moved and gathered."""
    rng = np.random.default_rng(31)
    pages = paged.Pages(1, 66000, 8, 16, torch.bfloat16, DEV)
    ids = [65999, 3, 65537, 65998]
    table = torch.tensor([ids[:3]], dtype=torch.int32, device=DEV)
    k, v = (normal(rng, (40, 8, 128), torch.bfloat16) for _ in range(2))
    index = torch.arange(40, dtype=torch.int32, device=DEV)
    paged.append(pages, 0, k, v, table, index, rows=torch.zeros_like(index))
    assert torch.equal(pages.data[0, 65537, 1, :, 7], v[39])
    paged.copy_pages(pages, [(65537, 65998)])
    table[0, 2] = 65998
    got = paged.gather(pages, 0, table, 0, 40)
    assert torch.equal(got[0][0], k) and torch.equal(got[1][0], v)
    q = normal(rng, (1, 32, 128), torch.bfloat16)
    out = paged.decode_attention(pages, 0, q, table, torch.tensor([40], dtype=torch.int32, device=DEV))
    assert (out[0] - attend(q[0], k, v)[0]).abs().max() <= 2 * SCORE * 6
    assert pages.device_error() == 0


# ---------------------------------------------------------------- the packed cache's part
@pytest.mark.parametrize("batch,n_ctx,n_full", [(1, 300, 0), (3, 1000, 0), (2, 513, 37), (70, 20, 0), (1, 0, 9)])
def test_packed_log_sum(aatc, batch, n_ctx, n_full):
    """aatc_decode_attention_lse: the same output bits as without it, and the log of the softmax's sum; it
    joins a paged part as one softmax over both."""
    from test_gpu_prefill_layouts import random_plan, tokens
    rng = np.random.default_rng([batch, n_ctx])
    n_kv, group = 2, 4
    plan, basis, _ = random_plan(aatc, rng, n_kv, group, 8, (352, 288))
    cap = max(n_ctx, 1) + 5
    cache = plan.new_cache(batch, cap, DEV)
    full = tokens(rng, basis, batch, n_full, n_kv) if n_full else (None, None)
    keys = values = torch.zeros((batch, 0, n_kv, 128), dtype=torch.float64, device=DEV)
    if n_ctx:
        k, v = tokens(rng, basis, batch, n_ctx, n_kv)
        aatc.encode(plan, 0, k, v, cache, 0, cap)
        coef = aatc.dequantize(plan, 0, cache, batch, 0, n_ctx, cap).double()
        keys, values = (torch.einsum("bnhc,hdc->bnhd", coef[:, :, :, i], torch.from_numpy(basis[0, :, i]).to(DEV).double())
                        for i in (0, 1))
    if n_full:
        keys, values = torch.cat([keys, full[0].double()], 1), torch.cat([values, full[1].double()], 1)
    q = normal(rng, (batch, n_kv * group, 128), torch.bfloat16)
    args = (plan, 0, q, cache, 0, n_ctx, cap, full[0], full[1], n_full)
    lse = torch.empty((batch, n_kv * group), device=DEV)
    plain, out = aatc.decode_attention_sw(*args), aatc.decode_attention_sw(*args, lse=lse)
    assert torch.equal(plain, out)
    pool = Pool(rng, rng.integers(0, 90, batch), n_kv, 16, torch.bfloat16)
    joined = paged.decode_attention(pool.pages, 0, q, pool.table, pool.device_lens, prior=(out, lse))
    for b in range(batch):
        s = torch.einsum("hd,nhd->hn", q[b].double(), keys[b].repeat_interleave(group, 1)) / math.sqrt(128)
        # the packed scores are sums of operands of about 22 bits: 2^-20 of scores under 32
        assert (lse[b] - torch.logsumexp(s, 1)).abs().max() <= 32 * 2.0 ** -20 + SCORE
        ref, _ = attend(q[b], torch.cat([keys[b], pool.k[b].double()]), torch.cat([values[b], pool.v[b].double()]))
        assert (joined[b] - ref).abs().max() <= 1e-4 * max(1.0, float(values[b].abs().max()), 6.0)
    assert plan.device_error() == 0


@pytest.mark.parametrize("batch,max_pages", [(2, 8388607), (1000, 20), (1000, 20000), (385, 4)])
def test_decode_wide_tables(batch, max_pages):
    """More sequences than a CTA has threads, and tables whose width takes the places of tokens past 31 bits."""
    rng = np.random.default_rng([batch, max_pages])
    lens = rng.integers(0, 60, batch)
    lens[-1] = 700
    per = -(-lens // 256)
    pages = paged.Pages(1, int(per.sum()), 8, 256, torch.bfloat16, DEV)
    ids = rng.permutation(int(per.sum()))
    first = np.concatenate([[0], np.cumsum(per)])
    table = torch.full((batch, max_pages), -1, dtype=torch.int32, device=DEV)
    host = np.full((batch, 3), -1)
    for b in range(batch):
        host[b, :per[b]] = ids[first[b]:first[b + 1]]
    table[:, :3] = torch.from_numpy(host).to(DEV, torch.int32)
    rows = torch.from_numpy(np.repeat(np.arange(batch), lens)).to(DEV, torch.int32)
    index = torch.from_numpy(np.concatenate([np.arange(n) for n in lens])).to(DEV, torch.int32)
    k, v = (normal(rng, (int(lens.sum()), 8, 128), torch.bfloat16) for _ in range(2))
    paged.append(pages, 0, k, v, table, index, rows=rows)
    q = normal(rng, (batch, 8, 128), torch.bfloat16)
    out = paged.decode_attention(pages, 0, q, table, torch.from_numpy(lens).to(DEV, torch.int32))
    start = np.concatenate([[0], np.cumsum(lens)])
    for b in list(range(0, batch, max(1, batch // 50))) + [batch - 1]:
        part = slice(int(start[b]), int(start[b + 1]))
        ref, _ = attend(q[b], k[part], v[part])
        assert (out[b] - ref).abs().max() <= 2 * SCORE * 6, b
    assert torch.isfinite(out).all() and pages.device_error() == 0


@pytest.mark.parametrize("page", [8, 16, 128])
def test_decode_negative_scale_and_bad_ids_by_page(page):
    """A negative scale under edges and caps; a page outside the pool drops its tokens whatever the page's size."""
    rng = np.random.default_rng([51, page])
    pool = Pool(rng, [150, 9, 0], 2, page, torch.bfloat16, scale=0.7)
    q = normal(rng, (3, 6, 128), torch.bfloat16)
    check_decode(pool, q, scale=-0.3)
    check_decode(pool, q, scale=-0.3, cap=4.0, window=33)
    table = pool.table.clone()
    table[0, 1], table[1, 0] = pool.pages.n_pages, -7
    out = paged.decode_attention(pool.pages, 0, q, table, pool.device_lens)
    left = [t for t in range(150) if t // page != 1]
    ref, _ = attend(q[0], pool.k[0][left], pool.v[0][left])
    assert (out[0] - ref).abs().max() <= 2 * SCORE * 6
    gone = 9 if page > 8 else 8
    ref, _ = attend(q[1], pool.k[1][gone:], pool.v[1][gone:])
    assert (out[1] - ref).abs().max() <= 2 * SCORE * 6 and torch.all(out[2] == 0)
    assert pool.pages.device_error(clear=True) == 4


def test_single_rows_and_broadcasts():
    """One token or one head of any stride; heads and tables that are broadcast; results of a side stream."""
    rng = np.random.default_rng(52)
    rope = paged.Rotary(64, 10000.0, device=DEV)
    x = normal(rng, (8 * 1000,), torch.bfloat16).as_strided((1, 1, 128), (3, 5, 1))
    at = torch.tensor([77], dtype=torch.int32, device=DEV)
    check_turned(paged.rotate(rope, x, at), x, at, rope)
    pool = Pool(rng, [45], 3, 16, torch.bfloat16)
    q = normal(rng, (1, 1, 128), torch.bfloat16).expand(5, 6, 128)
    lens = torch.tensor([45, 0, 16, 31, 1], dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = paged.decode_attention(pool.pages, 0, q, pool.table.expand(5, -1), lens, stream=side)
    k, v = paged.gather(pool.pages, 0, pool.table.expand(5, -1), 3, 40, stream=side)
    side.synchronize()
    for b, n in enumerate(lens.tolist()):
        ref, _ = attend(q[b], pool.k[0][:n], pool.v[0][:n])
        assert (out[b] - ref).abs().max() <= 2 * SCORE * 6
        assert torch.equal(k[b], pool.k[0][3:43]) and torch.equal(v[b], pool.v[0][3:43])
    one = normal(rng, (4, 1, 128), torch.bfloat16)
    pool.pages.data.zero_()
    index = torch.arange(4, dtype=torch.int32, device=DEV)
    paged.append(pool.pages, 0, one.expand(4, 3, 128), one.expand(4, 3, 128), pool.table, index, rows=torch.zeros_like(index))
    got = paged.gather(pool.pages, 0, pool.table, 0, 4)
    assert torch.equal(got[0][0], one.expand(4, 3, 128)) and torch.equal(got[1][0], one.expand(4, 3, 128))
    assert pool.pages.device_error() == 0


def test_gather_of_more_rows_than_a_grid_has():
    rng = np.random.default_rng(53)
    pages = paged.Pages(1, 70, 1, 8, torch.float16, DEV)
    pages.data.copy_(normal(rng, pages.data.shape, torch.float16))
    table = torch.from_numpy(rng.integers(0, 70, (70001, 1))).to(DEV, torch.int32)
    lens = torch.from_numpy(rng.integers(0, 9, 70001)).to(DEV, torch.int32)
    k, v = paged.gather(pages, 0, table, 5, 2, lens=lens)
    for i, got in enumerate((k, v)):
        want = pages.data[0, table[:, 0].long(), i, 0, 5:7][:, :, None]
        want = torch.where((torch.arange(5, 7, device=DEV) < lens[:, None])[:, :, None, None], want, 0)
        assert torch.equal(got, want)
    assert pages.device_error() == 0


@pytest.mark.parametrize("batch", [1, 3, 100, 384, 385])
@pytest.mark.parametrize("cap_tokens", [256, 264])
def test_decode_narrow_tables(batch, cap_tokens):
    """Tables at the width up to which segments stay whole and one past it, by a window too."""
    rng = np.random.default_rng([batch, cap_tokens])
    lens = rng.integers(0, cap_tokens + 1, batch)
    lens[rng.integers(0, batch)] = cap_tokens
    pool = Pool(rng, [0] * batch, 2, 8, torch.bfloat16)
    pages = paged.Pages(1, batch * cap_tokens // 8, 2, 8, torch.bfloat16, DEV)
    ids = rng.permutation(pages.n_pages).reshape(batch, -1)
    table = torch.from_numpy(ids).to(DEV, torch.int32)
    rows = torch.from_numpy(np.repeat(np.arange(batch), lens)).to(DEV, torch.int32)
    index = torch.from_numpy(np.concatenate([np.arange(n) for n in lens])).to(DEV, torch.int32)
    k, v = (normal(rng, (int(lens.sum()), 2, 128), torch.bfloat16) for _ in range(2))
    paged.append(pages, 0, k, v, table, index, rows=rows)
    start = np.concatenate([[0], np.cumsum(lens)])
    pool.pages, pool.table, pool.device_lens = pages, table, torch.from_numpy(lens).to(DEV, torch.int32)
    pool.k, pool.v = ([x[start[b]:start[b + 1]] for b in range(batch)] for x in (k, v))
    q = normal(rng, (batch, 6, 128), torch.bfloat16)
    check_decode(pool, q)
    check_decode(pool, q, window=77, cap=20.0)


@pytest.mark.parametrize("batch", [1535, 1536, 1537, 4000])
@pytest.mark.parametrize("cap_tokens", [64, 512])
def test_decode_more_sequences_than_a_chunk(batch, cap_tokens):
    """Around the number of sequences whose prefix sums a CTA takes at once, with and without the second launch."""
    rng = np.random.default_rng([batch, cap_tokens])
    lens = rng.integers(0, 33, batch)
    lens[[0, batch // 2, batch - 1]] = cap_tokens
    per = -(-lens // 16)
    first = np.concatenate([[0], np.cumsum(per)])
    ids = rng.permutation(int(per.sum()))
    host = np.full((batch, cap_tokens // 16), -1)
    for b in range(batch):
        host[b, :per[b]] = ids[first[b]:first[b + 1]]
    pages = paged.Pages(1, int(per.sum()), 1, 16, torch.float16, DEV)
    table = torch.from_numpy(host).to(DEV, torch.int32)
    rows = torch.from_numpy(np.repeat(np.arange(batch), lens)).to(DEV, torch.int32)
    index = torch.from_numpy(np.concatenate([np.arange(n) for n in lens])).to(DEV, torch.int32)
    k, v = (normal(rng, (int(lens.sum()), 1, 128), torch.float16) for _ in range(2))
    paged.append(pages, 0, k, v, table, index, rows=rows)
    q = normal(rng, (batch, 4, 128), torch.float16)
    lse = torch.empty((batch, 4), device=DEV)
    out = paged.decode_attention(pages, 0, q, table, torch.from_numpy(lens).to(DEV, torch.int32), lse=lse)
    start = np.concatenate([[0], np.cumsum(lens)])
    for b in sorted({0, 1, batch // 2, batch - 2, batch - 1, *range(0, batch, 61), *range(min(batch, 1530), min(batch, 1540))}):
        part = slice(int(start[b]), int(start[b + 1]))
        ref, ref_lse = attend(q[b], k[part], v[part])
        assert (out[b] - ref).abs().max() <= 2 * SCORE * 6, b
        assert lens[b] == 0 or (lse[b] - ref_lse).abs().max() <= SCORE
    assert torch.isfinite(out).all() and torch.all(out[lens == 0] == 0) and pages.device_error() == 0
