"""The paged cache's host side: rotary frequencies and turns against 64-bit formulas, and the refusal of
every bad argument before anything is launched (no GPU: the required device type is the CPU here, and
a call that the binding lets through is refused by the library's own checks)."""
import ctypes
import math
import types
from fractions import Fraction

import numpy as np
import pytest
import torch

bf16, f16, i32 = torch.bfloat16, torch.float16, torch.int32
S = types.SimpleNamespace(cuda_stream=0)


@pytest.fixture
def paged(aatc, monkeypatch):
    monkeypatch.setattr(aatc, "_DEVICE_TYPE", "cpu")
    from paper_2608_14191_gb300 import paged as m
    return m


def refused(aatc_error, call, status=1, what=None):
    with pytest.raises(aatc_error) as e:
        call()
    assert e.value.status == status and (what is None or what in str(e.value)), str(e.value)


@pytest.mark.parametrize("rot", [16, 64, 96, 128])
@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_frequencies(paged, rot, base):
    i = np.arange(rot // 2)
    w = base ** (-2.0 * i / rot)
    close = dict(rtol=1e-14, atol=0)
    got = paged.Rotary(rot, base, device="cpu")
    np.testing.assert_allclose(got.frequencies, w, **close)
    assert got.factor == 1.0
    np.testing.assert_allclose(paged.Rotary(rot, base, scaling=dict(kind="linear", factor=4), device="cpu").frequencies, w / 4, **close)
    ntk = paged.Rotary(rot, base, scaling=dict(kind="ntk", factor=4), device="cpu").frequencies
    assert ntk[0] == 1.0 and abs(ntk[-1] * 4 / w[-1] - 1) < 1e-13       # the fastest as it is, the slowest by 4
    np.testing.assert_allclose(np.diff(np.log(ntk)), np.log(ntk[1]), rtol=1e-12)
    ramp = paged.Rotary(rot, base, scaling=dict(kind="ramp", factor=4, original=4096, fast=32, slow=1), device="cpu")
    assert abs(ramp.factor - (0.1 * math.log(4) + 1)) < 1e-15
    turns = 4096 * w / (2 * math.pi)                                     # over the original context
    assert np.allclose(ramp.frequencies[turns > 32 * base ** (2 / rot)], w[turns > 32 * base ** (2 / rot)], **close)
    assert np.allclose(ramp.frequencies[turns < base ** (-2 / rot)], w[turns < base ** (-2 / rot)] / 4, **close)
    assert np.all(np.diff(ramp.frequencies) < 0) and np.all(ramp.frequencies <= w * (1 + 1e-15))
    band = paged.Rotary(rot, base, scaling=dict(kind="banded", factor=8, original=8192, low=1, high=4), device="cpu")
    turns = 8192 * w / (2 * math.pi)
    for f, x, n in zip(band.frequencies, w, turns):
        want = x if n >= 4 else x / 8 if n <= 1 else ((n - 1) / 3) * x + (1 - (n - 1) / 3) * x / 8
        assert abs(f / want - 1) < 1e-13
    assert band.factor == 1.0


def test_turns(paged, aatc):
    """64-bit fractions of a turn: within 2^-62 + the 2^-53 of the double quotient, negative ones from the other side."""
    pi = Fraction(3141592653589793238462643383279502884197, 10**39)
    freq = np.array([1.0, 0.1, 1e-6, 6.283185307179586, 20.0, 0.0, -1.0, -1e-20])
    out = np.empty(len(freq), np.uint64)
    assert aatc.load().aatc_rotary_turns(freq.ctypes.data, len(freq), out.ctypes.data) == 0
    for f, t in zip(freq, out):
        want = Fraction(float(f)) / (2 * pi)
        off = (Fraction(int(t), 1 << 64) - want) % 1
        assert min(off, 1 - off) <= Fraction(1, 1 << 62) + abs(want) * Fraction(1, 1 << 52)


def test_rotary_refusals(paged, aatc):
    E = aatc.AatcError
    for rot in (0, -16, 8, 100, 144, 256):
        refused(E, lambda: paged.Rotary(rot, device="cpu"))
    for base in (1.0, 0.5, -3.0, math.inf, math.nan):
        refused(E, lambda: paged.Rotary(64, base, device="cpu"))
    refused(E, lambda: paged.Rotary(64, layout="other", device="cpu"), what="layout")
    for s in (dict(kind="none"), dict(factor=2.0), dict(kind="linear", factor=0.5), dict(kind="ntk", factor=math.nan),
              dict(kind="linear", factor=2.0, original=100, fast=3), dict(kind="ramp", factor=2.0, original=100),
              dict(kind="ramp", factor=2.0, original=0, fast=32, slow=1), dict(kind="ramp", factor=2.0, original=9, fast=1, slow=2),
              dict(kind="ramp", factor=2.0, original=9, fast=1, slow=0), dict(kind="banded", factor=2.0, original=9, low=4, high=4)):
        refused(E, lambda: paged.Rotary(64, scaling=s, device="cpu"))
    lib, out = aatc.load(), np.empty(4, np.uint64)
    for f in (np.array([math.nan]), np.array([math.inf])):
        assert lib.aatc_rotary_turns(f.ctypes.data, 1, out.ctypes.data) == 1
    assert lib.aatc_rotary_turns(out.ctypes.data, 0, out.ctypes.data) == 1
    assert lib.aatc_rotary_turns(None, 1, out.ctypes.data) == 1


def test_rotate_refusals(paged, aatc):
    E, rope = aatc.AatcError, paged.Rotary(64, device="cpu")
    x, p = torch.zeros((5, 3, 128), dtype=bf16), torch.zeros(5, dtype=i32)
    odd = torch.zeros(5 * 3 * 128 + 8, dtype=bf16)
    for args in ((None, x, p), (rope, x.float(), p), (rope, x[0], p), (rope, x[..., :64], p), (rope, x, p.long()),
                 (rope, x, p[:4]), (rope, x, torch.zeros(10, dtype=i32)[::2]), (rope, x.transpose(1, 2).contiguous().transpose(1, 2), p),
                 (rope, x, p, x.half()), (rope, x, p, x[:4]), (rope, odd[1:1 + 1920].view(5, 3, 128), p),
                 (rope, odd[:1915 + 4].as_strided((5, 3, 128), (383, 128, 1)), p)):
        refused(E, lambda: paged.rotate(*args, stream=S))
    assert paged.rotate(rope, x[:0], p[:0], stream=S).shape == (0, 3, 128)


def pool(paged, page=16, n_pages=9, n_kv=2, dtype=bf16, layers=2):
    return paged.Pages(layers, n_pages, n_kv, page, dtype, "cpu")


def test_pages_refusals(paged, aatc):
    E = aatc.AatcError
    for page in (1, 4, 12, 512):
        refused(E, lambda: pool(paged, page))
    refused(E, lambda: pool(paged, dtype=torch.float32))
    refused(E, lambda: paged.Pages.of(torch.zeros((2, 3, 2, 2, 16, 64), dtype=bf16)))
    refused(E, lambda: paged.Pages.of(torch.zeros((2, 3, 1, 2, 16, 128), dtype=bf16)))
    refused(E, lambda: paged.Pages.of(torch.zeros((2, 6, 2, 2, 16, 128), dtype=bf16)[:, ::2]))
    p = pool(paged)
    assert p.layer_bytes == 9 * 2 * 2 * 16 * 128 * 2 and p.device_error() == 0
    n = ctypes.c_size_t()
    lib = aatc.load()
    for d in ((0, 2, 16, 0), (0, 0, 16, 4), (2, 2, 16, 4), (-1, 2, 16, 4), (0, 2, 16, (1 << 24) + 1), (0, 4096, 256, 1 << 24)):
        assert lib.aatc_pages_bytes(ctypes.byref(paged._Desc(*d)), ctypes.byref(n)) == 1
    assert lib.aatc_pages_bytes(None, ctypes.byref(n)) == 1


def test_append_refusals(paged, aatc):
    E, p, rope = aatc.AatcError, pool(paged), paged.Rotary(64, device="cpu")
    k, q, t, i = (torch.zeros((3, 2, 128), dtype=bf16), torch.zeros((3, 8, 128), dtype=bf16), torch.zeros((3, 4), dtype=i32),
                  torch.zeros(3, dtype=i32))
    good = dict(pages=p, layer=0, k=k, v=k, table=t, index=i, rope=rope, q=q)
    for bad in (dict(layer=2), dict(layer=-1), dict(k=k.half()), dict(v=k[:2]), dict(k=k[:, :1]), dict(table=t.long()),
                dict(table=t.T), dict(table=t[:2]), dict(index=i[:2]), dict(rows=i[:2]), dict(positions=i.long()), dict(rope=None),
                dict(q=q.half()), dict(q=q[:2]), dict(q=None, q_out=q), dict(q_out=torch.zeros((3, 16, 128), dtype=bf16)[:, ::2]),
                dict(q_out=q[:2]), dict(table=t[:, :0])):
        refused(E, lambda: paged.append(**{**good, **bad}, stream=S))
    assert paged.append(p, 0, k[:0], k[:0], t, i[:0], rows=i[:0], stream=S) is None


def test_decode_refusals(paged, aatc):
    E, p = aatc.AatcError, pool(paged)
    q, t, n = torch.zeros((3, 8, 128), dtype=bf16), torch.zeros((3, 4), dtype=i32), torch.ones(3, dtype=i32)
    f = torch.zeros
    good = dict(pages=p, layer=0, q=q, table=t, lens=n, workspace=f(1 << 20))
    for bad in (dict(layer=2), dict(q=q.half()), dict(q=q[..., :64]), dict(table=t[:2]), dict(table=t.long()), dict(lens=n.long()),
                dict(lens=n[:2]), dict(out=f((3, 8, 128), dtype=bf16)), dict(out=f((3, 4, 128))), dict(lse=f((3, 4))),
                dict(lse=f((8, 3)).T), dict(prior=(f((3, 8, 128)), f((3, 4)))), dict(prior=(f((3, 4, 128)), f((3, 8)))),
                dict(slopes=f(4)), dict(slopes=f(8).double()), dict(cap=-1.0), dict(cap=math.nan), dict(window=-1),
                dict(scale=math.inf), dict(q=q[:, :7]), dict(q=q[:, :1]), dict(workspace=f(8)[::2])):
        refused(E, lambda: paged.decode_attention(**{**good, **bad}, stream=S))
    assert paged.decode_attention(p, 0, q[:0], t[:0], n[:0], stream=S).shape == (0, 8, 128)


def test_copy_refusals(paged, aatc):
    E, p = aatc.AatcError, pool(paged)
    for pairs in ([(0, 9)], [(9, 0)], [(-1, 0)], [(0, -1)], [(0, 1), (2, 1)], [(0, 1), (1, 2)], [(3, 3)], [(1, 2), (0, 1)],
                  [0, 1], [(0, 1, 2)]):
        refused(E, lambda: paged.copy_pages(p, pairs, stream=S))
    paged.copy_pages(p, [], stream=S)


def test_gather_refusals(paged, aatc):
    E, p = aatc.AatcError, pool(paged)
    t, n = torch.zeros((3, 4), dtype=i32), torch.zeros(3, dtype=i32)
    refused(E, lambda: paged.gather(p, 0, t, 0, 65, stream=S), status=3)
    refused(E, lambda: paged.gather(p, 0, t, 60, 5, stream=S), status=3)
    out = torch.zeros((3, 5, 2, 128), dtype=bf16)
    for call in (lambda: paged.gather(p, 2, t, 0, 5, stream=S), lambda: paged.gather(p, 0, t, -1, 5, stream=S),
                 lambda: paged.gather(p, 0, t, 0, -1, stream=S), lambda: paged.gather(p, 0, t.long(), 0, 5, stream=S),
                 lambda: paged.gather(p, 0, t, 0, 5, lens=n[:2], stream=S),
                 lambda: paged.gather(p, 0, t, 0, 5, out=(out, out[:2]), stream=S),
                 lambda: paged.gather(p, 0, t, 0, 5, out=(out, out.half()), stream=S)):
        refused(E, call)
    k, v = paged.gather(p, 0, t, 3, 0, stream=S)
    assert k.shape == v.shape == (3, 0, 2, 128)


def test_packed_lse_refusals(aatc, monkeypatch):
    monkeypatch.setattr(aatc, "_DEVICE_TYPE", "cpu")
    plan = types.SimpleNamespace(dims=aatc.dims(1, 2, 8), handle=None, cache_bytes=lambda b, m: 4 * b * m,
                                 workspace_bytes=lambda b, n: 1024)
    q, cache = torch.zeros((1, 8, 128), dtype=bf16), torch.zeros(100, dtype=i32)
    for lse in (torch.zeros((1, 4)), torch.zeros((1, 8), dtype=bf16), torch.zeros(8)):
        refused(aatc.AatcError, lambda: aatc.decode_attention_sw(plan, 0, q, cache, 0, 5, 9, lse=lse, stream=S), what="lse")
    refused(aatc.AatcError, lambda: aatc.decode_attention_sw(plan, 0, q, cache, 0, 5, 9, lse=torch.zeros((1, 8)), stream=S))
    lib = aatc.load()
    assert lib.aatc_decode_attention_lse(None, 0, 16, 16, 1, 0, 1, 1, None, None, 0, 0, 16, None, 16, 1 << 20, None) == 1


def test_places_past_31_bits_are_refused(paged, aatc):
    """Tables wide enough for more than 2^31 - 1 tokens: a gather past that and a decode are refused before anything is read."""
    lib, d = aatc.load(), paged._Desc(0, 1, 256, 1 << 20)
    at, wide = ctypes.c_void_p(4096), 1 << 24
    gather = lambda first, n, pages: lib.aatc_paged_gather(ctypes.byref(d), at, at, 1, pages, pages, first, n, None, at, at, None, None)  # noqa: E731
    assert gather(2**31 - 1, 1, wide) == 3 and gather(2**31 - 10, 2**31 - 1, wide) == 3
    assert gather(100, 157, 1) == 3 and gather(100, 0, 1) == 0
    how, q = paged._Decode(1.0, 0.0, 0), paged._Heads(4096, 128, 128)
    assert lib.aatc_paged_decode_attention(ctypes.byref(d), at, at, wide, wide, at, 1, ctypes.byref(q), 1, ctypes.byref(how), at, None, at,
                                           1 << 30, None, None) == 1
    p, t, n = pool(paged), torch.zeros((3, 4), dtype=i32), torch.ones(3, dtype=i32)
    for first in (2**31, 2**32 + 1):
        refused(aatc.AatcError, lambda: paged.gather(p, 0, t, first, 1, stream=S))
    refused(aatc.AatcError, lambda: paged.decode_attention(p, 0, torch.zeros((3, 2, 128), dtype=bf16), t, n, window=2**32 + 5,
                                                           workspace=torch.zeros(1 << 20), stream=S))


def test_copy_ids_are_not_wrapped(paged, aatc):
    """Ids that int32 does not hold, and fractions, are refused, not turned into another page's id."""
    p = pool(paged)
    for pairs in (np.array([[2**32 + 3, 1]]), np.array([[1, 2**32 + 3]]), np.array([[-2**32 + 3, 1]]), np.array([[1.7, 3]]),
                  np.array([[3, math.nan]]), np.array([[math.inf, 3]]), np.array([[2**31 + 2**31 + 1, 3]], np.uint64),
                  np.array([[2**63 + 3, 1]], np.uint64), [(2**70, 1)], [("1", "2")], torch.tensor([[2**32 + 3, 1]])):
        refused(aatc.AatcError, lambda: paged.copy_pages(p, pairs, stream=S), what="pairs")
    # equal whole numbers of other types are taken: only the library refuses these, for page 4, which is written twice
    for pairs in (np.array([[1.0, 4.0], [2.0, 4.0]]), np.array([[1, 4], [2, 4]], np.uint8), torch.tensor([[1, 4], [2, 4]])):
        with pytest.raises(aatc.AatcError) as e:
            paged.copy_pages(p, pairs, stream=S)
        assert e.value.status == 1 and "pairs" not in str(e.value)


def test_overlapping_results_are_refused(paged, aatc):
    """Results whose heads overlap, among them a broadcast tensor turned in place; strides that only cross are taken (the launch
    itself then fails here)."""
    rope, p = paged.Rotary(64, device="cpu"), torch.zeros(6, dtype=i32)
    x, flat = torch.zeros((6, 4, 128), dtype=bf16), torch.zeros(1 << 16, dtype=bf16)
    one = x[:1].expand(6, 4, 128)
    bad = [one, x[:, :1].expand(6, 4, 128)] + [flat.as_strided((6, 4, 128), s + (1,)) for s in (
        (128, 128), (512, 64), (64, 1024), (256, 384), (384, 128), (128, 640), (1000, 504))]
    for out in bad:
        refused(aatc.AatcError, lambda: paged.rotate(rope, x, p, out=out, stream=S))
        refused(aatc.AatcError, lambda: paged.rotate(rope, out, p, out=out, stream=S))
    pages, t = pool(paged), torch.zeros((6, 4), dtype=i32)
    for q in bad:
        refused(aatc.AatcError, lambda: paged.append(pages, 0, x[:, :2], x[:, :2], t, p, rope=rope, q=q, q_out=q, stream=S))
    good = [(x.clone(), one), (x.clone(), x[:, :1].expand(6, 4, 128)), (x[:1].expand(1, 4, 128), x[:1])]
    good += [(y, y) for y in (flat.as_strided(n + (128,), s + (1,)) for n, s in (
        ((6, 4), (512, 128)), ((6, 4), (128, 768)), ((2, 3), (384, 256)), ((3, 2), (256, 384)), ((2, 1), (128, 0)), ((1, 4), (0, 136))))]
    for out, src in good:
        with pytest.raises(aatc.AatcError) as e:
            paged.rotate(rope, src, p[:len(src)], out=out, stream=S)
        assert e.value.status != 1
