"""Host logic of the layer operators that needs no GPU: descriptors, scratch sizes, frequencies, refusals."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2609_21594_b200 import binding as mb


def test_struct_sizes_match_the_header():
    assert C.sizeof(mb.NormDesc) == 32
    assert C.sizeof(mb.Heads) == 32
    assert C.sizeof(mb.RotaryDesc) == 56
    assert C.sizeof(mb.RotaryItem) == 72
    assert C.sizeof(mb.AttentionDesc) == 80


def test_frequencies():
    f = mb.muon_rotary_frequencies(10000.0, 64)
    assert f.shape == (32,) and f[0] == 1.0
    assert np.allclose(f, [10000.0 ** (-2 * i / 64) for i in range(32)], rtol=1e-15, atol=0)
    assert np.allclose(mb.muon_rotary_frequencies(10000.0, 64, mb.ROTARY_LINEAR, 4.0), f / 4, rtol=1e-15, atol=0)
    g = mb.muon_rotary_frequencies(500000.0, 128, mb.ROTARY_BY_PARTS, 8.0, 8192, 1.0, 4.0)
    for i in range(64):
        p = 500000.0 ** (-2 * i / 128)
        turns = 8192 * p / (2 * math.pi)
        k = min(1.0, max(0.0, (turns - 1) / 3))
        assert g[i] == pytest.approx(k * p + (1 - k) * p / 8, rel=1e-14)
    assert g[0] == 1.0 and g[63] == pytest.approx(500000.0 ** (-126 / 128) / 8, rel=1e-14)
    for bad in (dict(base=0.0), dict(base=float("nan")), dict(rotary_dim=3), dict(rotary_dim=0), dict(scaling=5), dict(scaling=1, factor=0.0),
                dict(scaling=2, factor=2.0, original_length=0.0), dict(scaling=2, factor=2.0, original_length=10.0, low=4.0, high=4.0)):
        with pytest.raises(mb.MuonError) as e:
            mb.muon_rotary_frequencies(**{"base": 10000.0, "rotary_dim": 64, **bad})
        assert e.value.code == mb.ERR_INVALID_ARG


def norm(**kw):
    d = mb.NormDesc(0, 1, 1, 256, 100, 1e-5, 0)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def test_norm_scratch_and_refusals():
    assert mb.muon_layer_norm_workspace_bytes(norm(rows=0)) == 0
    assert mb.muon_layer_norm_workspace_bytes(norm(rows=128)) == 0             # few narrow rows: one cluster adds its sums itself
    one = mb.muon_layer_norm_workspace_bytes(norm(rows=1, cols=600))
    assert one == 2 * 600 * 4
    many = mb.muon_layer_norm_workspace_bytes(norm(rows=1 << 40))
    assert many == mb.muon_layer_norm_workspace_bytes(norm(rows=1 << 20)) > one
    for kw, code in ((dict(dtype=2), -1), (dict(param_dtype=-1), -1), (dict(center=2), -1), (dict(cols=0), -1), (dict(rows=-1), -1), (dict(eps=-1.0), -1),
                     (dict(eps=math.nan), -1), (dict(reserved=1), -1), (dict(cols=16385), -3)):
        with pytest.raises(mb.MuonError) as e:
            mb.muon_layer_norm_workspace_bytes(norm(**kw))
        assert e.value.code == code


def attention(**kw):
    d = mb.AttentionDesc(0, 2, 300, 300, 8, 2, 64, 1, 0, 0.125, 0, 0, None, None, None, None)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def test_attention_scratch_and_refusals():
    assert mb.muon_attention_workspace_bytes(attention()) == 2 * 8 * 3 * 1024                # two rows, eight heads, three blocks of 128
    assert mb.muon_attention_workspace_bytes(attention(batch=0)) == 0
    packed = dict(batch=1, num_seqs=5, q_offsets=64, k_offsets=64)                            # an address: only checked for alignment here
    assert mb.muon_attention_workspace_bytes(attention(**packed)) == 8 * (300 // 128 + 5 + 2) * 1024
    for kw, code in ((dict(dtype=3), -1), (dict(batch=-1), -1), (dict(q_heads=7), -1), (dict(kv_heads=0), -1), (dict(head_dim=0), -1), (dict(head_dim=257), -3),
                     (dict(causal=2), -1), (dict(window=-1), -1), (dict(causal=0, window=3), -1), (dict(scale=0.0), -1), (dict(scale=math.inf), -1),
                     (dict(reserved=1), -1), (dict(num_seqs=3), -1), (dict(q_offsets=64), -1), (dict(packed, batch=2), -1), (dict(packed, q_lens=64), -1),
                     (dict(q_lens=65), -1), (dict(batch=1 << 16, q_tokens=1 << 20), -3)):
        with pytest.raises(mb.MuonError) as e:
            mb.muon_attention_workspace_bytes(attention(**kw))
        assert e.value.code == code, kw


def test_packed_blocks_never_collide():
    """Sequence s keeps its 128-row blocks from q0 / 128 + s on: by brute force over ragged lengths, disjoint and inside the scratch."""
    rng = np.random.default_rng(0)
    for _ in range(200):
        lens = rng.choice([0, 1, 127, 128, 129, 255, 256, 300], size=rng.integers(1, 12))
        total = int(lens.sum()) + int(rng.integers(0, 300))
        off = np.concatenate([[0], np.cumsum(lens), [total]])
        used = set()
        for s in range(len(lens) + 1):
            for blk in range(-(-(off[s + 1] - off[s]) // 128)):
                at = off[s] // 128 + s + blk
                assert at not in used and at < total // 128 + len(lens) + 2
                used.add(at)


def test_cpu_tensors_are_refused():
    from paper_2609_21594_b200 import functional as F

    x = torch.zeros((2, 4, 2, 64))
    with pytest.raises(ValueError):
        F.layer_norm_forward(x)
    with pytest.raises(ValueError):
        F.rotary_forward([x], np.ones(4))
    with pytest.raises(ValueError):
        F.attention_forward(x, x, x)
