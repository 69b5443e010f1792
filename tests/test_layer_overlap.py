"""Which strided tensors share memory: the host arithmetic behind the refusal of results that lie over an input or over one another."""
import itertools

import numpy as np
import pytest

from paper_2609_21594_b200 import binding as mb


def places(base, shape, strides, elem):
    """Byte addresses of the elements, one by one."""
    at = [base + elem * (b * strides[0] + t * strides[1] + h * strides[2] + d)
          for b, t, h, d in itertools.product(*(range(n) for n in shape))]
    return at


def heads(base, strides):
    return mb.Heads(base, *strides)


def test_against_every_byte():
    rng = np.random.default_rng(0)
    yes = no = 0
    for _ in range(4000):
        elem = int(rng.choice([2, 4]))
        shape = [int(rng.integers(1, 5)) for _ in range(3)] + [int(rng.integers(1, 7))]
        other = shape[:2] + [int(rng.integers(1, 4)), int(rng.integers(1, 7))] if rng.random() < 0.5 else [int(rng.integers(0, 4)) for _ in range(4)]
        strides = [int(rng.integers(0, 60)) for _ in range(3)]
        theirs = strides if rng.random() < 0.5 else [int(rng.integers(0, 60)) for _ in range(3)]
        a, b = 4096, 4096 + int(rng.integers(-200, 200))
        pa, pb = places(a, shape, strides, elem), places(b, other, theirs, elem)
        both = {x + i for x in pa for i in range(elem)} & {x + i for x in pb for i in range(elem)}
        assert mb.muon_heads_overlap(heads(a, strides), shape, heads(b, theirs), other, elem) == bool(both)
        assert mb.muon_heads_overlap(heads(a, strides), shape, None, (), elem) == (len(set(pa)) < len(pa))
        yes, no = yes + bool(both), no + (not both)
    assert min(yes, no) > 500


def test_layouts_of_programs():
    q, k = (8, 8192, 32, 128), (8, 8192, 8, 128)
    row = 48 * 128
    fused = lambda first: heads(1 << 20 | (first * 128 * 2), (8192 * row, row, 128))  # noqa: E731
    assert not mb.muon_heads_overlap(fused(0), q, fused(32), k, 2)                       # views of one projection interleave
    assert not mb.muon_heads_overlap(fused(40), k, fused(32), k, 2)
    assert mb.muon_heads_overlap(fused(0), q, fused(31), k, 2)
    by_head = heads(1 << 20, (32 * 8192 * 128, 128, 8192 * 128))
    assert not mb.muon_heads_overlap(by_head, q, None, (), 2) and not mb.muon_heads_overlap(fused(0), q, None, (), 2)
    assert mb.muon_heads_overlap(by_head, q, fused(0), q, 2)
    assert mb.muon_heads_overlap(heads(1 << 20, (0, 4096, 128)), q, None, (), 2)         # a stride of zero
    assert mb.muon_heads_overlap(heads(1 << 20, (1 << 25, 4096, 64)), q, None, (), 2)    # heads that lie half over one another
    assert not mb.muon_heads_overlap(fused(0), (8, 0, 32, 128), fused(0), q, 2)          # no elements
    assert not mb.muon_heads_overlap(heads(None, (1, 1, 1)), q, fused(0), q, 2)
    assert not mb.muon_heads_overlap(heads(1 << 20, (1 << 62, 1 << 62, 128)), (1, 1, 4, 128), heads(1 << 30, (1, 1, 128)), (1, 1, 4, 128), 2)


def test_refusals():
    t, shape = heads(64, (64, 64, 64)), (1, 1, 1, 64)
    for call in (lambda: mb.muon_heads_overlap(t, shape, t, shape, 0), lambda: mb.muon_heads_overlap(heads(64, (-1, 1, 1)), shape, t, shape, 2),
                 lambda: mb.muon_heads_overlap(t, shape, heads(64, (1, -1, 1)), shape, 2)):
        with pytest.raises(mb.MuonError) as e:
            call()
        assert e.value.code == mb.ERR_INVALID_ARG
