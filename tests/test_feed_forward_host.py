"""Host logic of the feed-forward block, the 8-bit blocks and the 8-bit linear layer that needs no GPU: descriptors, scratch sizes, refusals; and the
tests' own reference against values worked out by hand."""
import ctypes as C
import math

import pytest
import torch

import feed_forward_reference as ref
from paper_2609_21594_b200 import binding as mb


def test_struct_sizes_match_the_header():
    assert C.sizeof(mb.Rows) == 16
    assert C.sizeof(mb.Blocks) == 40
    assert C.sizeof(mb.FeedForwardDesc) == 24
    assert C.sizeof(mb.FeedForwardKept) == 152
    assert C.sizeof(mb.LinearBlocksDesc) == 16


def desc(**kw):
    d = mb.FeedForwardDesc(mb.DTYPE_BF16, mb.ACTIVATION_SILU, mb.KEEP_FULL, 100, 64, 130)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def test_scratch_and_refusals():
    up = lambda n: -(-n // 256) * 256  # noqa: E731
    assert mb.muon_feed_forward_workspace_bytes(desc(), False) == up(100 * 136 * 2)                       # h, rows of 136
    assert mb.muon_feed_forward_workspace_bytes(desc(), True) == 3 * up(100 * 136 * 2)                    # dg, du, h
    assert mb.muon_feed_forward_workspace_bytes(desc(keep=mb.KEEP_8BIT), True) == 3 * up(100 * 136 * 2) + up(100 * 64 * 2)      # and x
    assert mb.muon_feed_forward_workspace_bytes(desc(keep=mb.KEEP_8BIT), False) == up(100 * 136 * 2) + 2 * up(100 * 130 * 4)
    assert mb.muon_feed_forward_workspace_bytes(desc(tokens=0), True) == 0
    long = [mb.muon_feed_forward_workspace_bytes(desc(keep=mb.KEEP_8BIT, tokens=t, hidden=136), False) - up(t * 136 * 2) for t in (512, 5000)]
    assert long[0] == long[1]                                                                             # the fp32 rows are those of 512 tokens at most
    assert mb.muon_feed_forward_workspace_bytes(desc(dtype=mb.DTYPE_FP32), False) == up(100 * 136 * 4)
    for kw, code in ((dict(dtype=2), -1), (dict(activation=2), -1), (dict(keep=3), -1), (dict(tokens=-1), -1), (dict(dim=0), -1), (dict(hidden=0), -1),
                     (dict(tokens=2**31 - 1), -3), (dict(hidden=2**31 - 1), -3)):
        with pytest.raises(mb.MuonError) as e:
            mb.muon_feed_forward_workspace_bytes(desc(**kw), True)
        assert e.value.code == code, kw
    lin = mb.LinearBlocksDesc(100, 64, 130, 0)
    assert mb.muon_linear_blocks_workspace_bytes(lin, False) == 0
    assert mb.muon_linear_blocks_workspace_bytes(lin, True) == up(100 * 144) + up(100 * 16) + up(100 * 64 * 2)
    # rows that TMA cannot address have room for copies where the products are large: 4096 * 64 * 130 and 4096 * 65 * 130 are more than 2^21, 100 * 64 * 130 is not
    t, big = 4096, mb.LinearBlocksDesc(4096, 64, 130, 0)
    assert mb.muon_linear_blocks_workspace_bytes(big, False) == up(t * 136 * 2)                                          # y
    big.dim = 65
    assert mb.muon_linear_blocks_workspace_bytes(big, False) == up(t * 136 * 2) + up(130 * 80)                           # and w8
    assert mb.muon_linear_blocks_workspace_bytes(big, True) == (up(130 * 80) + up(t * 136 * 2) + up(t * 72 * 2) + up(130 * 72 * 2)       # w8, dy, dx, dw
                                                                + up(t * 144) + up(t * 16) + up(t * 72 * 2))             # dy in 8 bits, x
    odd = desc(tokens=t)                                                                                                 # hidden = 130: w_down, gate, up
    assert mb.muon_feed_forward_workspace_bytes(odd, False) == up(t * 136 * 2) + up(64 * 136 * 2) + 2 * up(t * 136 * 2)
    assert mb.muon_feed_forward_workspace_bytes(odd, True) == 3 * up(t * 136 * 2) + 2 * up(64 * 136 * 2) + 2 * up(t * 136 * 2)
    odd.dtype = mb.DTYPE_FP32
    assert mb.muon_feed_forward_workspace_bytes(odd, False) == up(t * 136 * 4)
    for fields, code in (((-1, 64, 130, 0), -1), ((1, 0, 130, 0), -1), ((1, 64, 0, 0), -1), ((1, 64, 130, 1), -1), ((2**31 - 1, 64, 130, 0), -3)):
        with pytest.raises(mb.MuonError) as e:
            mb.muon_linear_blocks_workspace_bytes(mb.LinearBlocksDesc(*fields), True)
        assert e.value.code == code, fields


def test_cpu_tensors_are_refused():
    from paper_2609_21594_b200 import functional as F

    x, w = torch.zeros((4, 8), dtype=torch.bfloat16), torch.zeros((8, 8), dtype=torch.bfloat16)
    codes, scales = torch.zeros((4, 8), dtype=torch.float8_e4m3fn), torch.zeros((4, 1), dtype=torch.uint8)
    for call in (lambda: F.quantize(x), lambda: F.dequantize(codes, scales, torch.bfloat16), lambda: F.feed_forward_forward(x, w, w, w),
                 lambda: F.feed_forward(x, w, w, w), lambda: F.feed_forward_backward(x, x, w, w, w, (x, x)), lambda: F.linear_8bit(x, w),
                 lambda: F.linear_8bit_forward(x, codes, scales), lambda: F.linear_8bit_backward(x, codes, scales, codes, scales)):
        with pytest.raises(ValueError):
            call()


def test_the_reference_by_hand():
    x = torch.zeros((2, 130), dtype=torch.float64)
    x[0, :4] = torch.tensor([448.0, 17.0, 19.0, 2.0 ** -10])       # 17 and 19 lie between codes 2 apart: to the even one
    x[0, 129], x[1, 0] = 449.0, 1.75 * 2.0 ** -130
    codes, e = ref.pack(x, 1)
    assert e.tolist() == [[127, 128], [0, 0]]
    assert codes[0, :4].tolist() == [448.0, 16.0, 20.0, 0.0] and codes[0, 129] == 224.0 and codes[1, 0] == 1.75 * 2.0 ** -3
    assert ref.unpack(codes, e, 1)[0, 129] == 448.0
    codes, e = ref.pack(x, 128)
    assert e.tolist() == [[127, 128]] and codes[1, 0] == 0
    x[0, 1], x[0, 2] = math.inf, math.nan
    codes, e = ref.pack(x, 1)
    assert e[0, 0] == 127 and torch.isnan(codes[0, 1:3]).all() and codes[0, 0] == 448.0
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    assert torch.equal(torch.nan_to_num(ref.nearest_e4m3(every)), torch.nan_to_num(every))
    middle = (every[:126] + every[1:127]) / 2                      # ties: to the code whose last bit is 0
    assert torch.equal(ref.nearest_e4m3(middle), every[1:127][0::1].where(torch.arange(126) % 2 == 1, every[:126]))
    a, slope = ref.act_and_slope(torch.tensor([0.0, 1.0], dtype=torch.float64), "silu")
    s = 1 / (1 + math.exp(-1))
    assert a[1] == pytest.approx(s) and slope.tolist() == pytest.approx([0.5, s + s * (1 - s)])
    a, slope = ref.act_and_slope(torch.tensor([0.0, 2.0], dtype=torch.float64), "gelu")
    assert a[1] == pytest.approx(1.954597694087775) and slope[0] == pytest.approx(0.5)
