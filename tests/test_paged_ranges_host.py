"""Paged calls without a GPU: what the sources promise, and calls of the bookkeeping that change nothing when they fail."""
import glob
import os
import re

import numpy as np
import pytest
import torch
from test_paged_shorter import lists  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_no_read_only_loads():
    """The paged kernels begin while the one before may still write tables, lengths and lists, which loads that assume constant
    memory do not allow for."""
    found = glob.glob(os.path.join(ROOT, "paper_2608_14191_gb300", "csrc", "paged*.cu*"))
    assert len(found) >= 4
    for path in found:
        with open(path) as f:
            assert not re.search(r"__ldg\b|ld\.global\.nc|ldu\.global", f.read()), path


@pytest.mark.parametrize("call", ["accept", "evict"])
@pytest.mark.parametrize("bad", ["type", "rows", "heads", "stride", "dims", "width", "device", "none", "list"])
def test_weights_that_do_not_fit_change_nothing(lists, call, bad):
    """A later layer's weights of another type, shape or stride: refused before the first layer's tokens move."""
    b = lists(20, 3, 64, 8)
    b.s.pages = b.s.pages.__class__.of(torch.zeros((2, 20, 2, 1, 8, 128), dtype=torch.bfloat16))
    for r, n in ((0, 40), (1, 9)):
        b.s.add()
        b.s.grow({r: n})
    good = torch.rand((3, 1, 64))
    second = {"type": good.double(), "rows": good[:2].clone(), "heads": torch.zeros((3, 2, 64)), "stride": torch.zeros((3, 1, 128))[:, :, ::2],
              "dims": good[0].clone(), "width": torch.zeros((3, 1, 39)), "device": torch.zeros((3, 1, 64), device="meta"), "none": None,
              "list": good.tolist()}[bad]
    b.s.pages.data.copy_(torch.rand(b.s.pages.data.shape))
    state = lambda: (b.s.pages.data.clone(), good.clone(), b.s._table.copy(), b.s._lens.copy(), b.s.refs.copy(), list(b.s._free))  # noqa: E731
    before = state()
    for weights in ([good, second], (good, second)):
        with pytest.raises(ValueError, match="weights"):
            if call == "evict":
                b.s.evict(weights, 16, 2, 4)
            else:
                b.s.accept({0: 9, 1: 3}, {0: [1, 5], 1: [2]}, weights)
        for x, y in zip(before, state()):
            assert torch.equal(x, y) if isinstance(x, torch.Tensor) else np.array_equal(x, y)
    if call == "evict":
        b.s.evict([good, torch.rand((3, 1, 70))], 16, 2, 4)
    else:
        b.s.accept({0: 9, 1: 3}, {0: [1, 5], 1: [2]}, [good, torch.rand((3, 1, 70))])
    assert list(b.s._lens) == ([16, 9, 0] if call == "evict" else [33, 7, 0])


def test_evictions_with_numbers_that_are_not_whole(lists):
    b = lists(20, 3, 64, 8)
    b.s.add()
    b.s.grow({0: 40})
    fork = b.s.fork(0)
    before = b.s._table.copy()
    for numbers in ((16, 2, 4.0), (16.0, 2, 4), (16, 2.0, 4)):
        with pytest.raises(TypeError):
            b.s.evict([torch.rand((3, 1, 64))], *numbers)
        assert np.array_equal(b.s._table, before) and b.s.length(fork) == 40


@pytest.mark.parametrize("call", ["accept", "evict"])
def test_layers_that_share_weights_are_refused(lists, call):
    """Weights of two layers in one tensor, or in tensors that overlap, would be moved twice."""
    b = lists(20, 3, 64, 8)
    b.s.pages = b.s.pages.__class__.of(torch.zeros((2, 20, 2, 1, 8, 128), dtype=torch.bfloat16))
    b.s.add()
    b.s.grow({0: 40})
    run = (lambda w: b.s.evict(w, 16, 2, 4)) if call == "evict" else (lambda w: b.s.accept({0: 9}, {0: [1, 5]}, w))
    room = torch.rand(6 * 64)
    one, end, apart = room[:192].view(3, 1, 64), room[191:383].view(3, 1, 64), room[192:].view(3, 1, 64)
    before = room.clone()
    for weights in ([one, one], [one, end], [end, one], one[None].expand(2, 3, 1, 64)):
        with pytest.raises(ValueError, match="weights"):
            run(weights)
        assert torch.equal(room, before) and b.s.length(0) == 40
    run([one, apart])
    assert b.s.length(0) == (16 if call == "evict" else 33)
