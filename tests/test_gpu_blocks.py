"""Blocks in 8 bits: codes and scales bit for bit against the definition in 64 bits, and back."""
import math

import pytest
import torch

import feed_forward_reference as ref

pytestmark = pytest.mark.gpu

SIZES = [(1, 1), (1, 128), (3, 127), (5, 129), (128, 256), (129, 1000), (300, 5633), (64, 16), (257, 72), (2, 14336)]


def make(rows, cols, dtype, seed=0):
    """Blocks of very unequal size, some of them zeros, and elements far below their block's largest."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((rows, cols), generator=g, device="cuda") * torch.exp2(torch.randint(-40, 40, (rows, 1), generator=g, device="cuda").float())
    x = x * torch.exp2(torch.randint(-12, 1, (rows, cols), generator=g, device="cuda").float())
    x[:, ::7] = 0
    if rows > 2:
        x[1] = 0
    return x.to(dtype)


def same(a, b):
    return torch.equal(torch.nan_to_num(a.double(), nan=12345.0), torch.nan_to_num(b.double(), nan=12345.0))


@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_against_the_definition(rows, cols, dtype, block):
    from paper_2609_21594_b200 import functional as F

    x = make(rows, cols, dtype)
    codes, scales = F.quantize(x, block)
    want, e = ref.pack(x, block)
    assert codes.dtype == torch.float8_e4m3fn and scales.dtype == torch.uint8 and codes.shape == x.shape and scales.shape == e.shape
    assert torch.equal(scales.long(), e) and same(codes.float(), want)
    for out in (torch.bfloat16, torch.float32):
        assert same(F.dequantize(codes, scales, out), ref.unpack(want, e, block).to(out))


@pytest.mark.parametrize("block", [1, 128])
def test_borders(block):
    """The least scale at and around its borders, subnormals, the largest values, ties, zeros, NaN and infinities."""
    from paper_2609_21594_b200 import functional as F

    tops = [448.0, 448.0 * (1 + 2 ** -23), 448.0 * (1 - 2 ** -24), 1.75, 1.7500001, 2.0 ** -118, 1.75 * 2.0 ** -119, 1.76 * 2.0 ** -119, 1e-40, 2.0 ** -149,
            3.4028234663852886e38, 0.0, -0.0, -448.0, 240.0, math.nan, math.inf, -math.inf]
    for k, top in enumerate(tops):
        x = torch.zeros((3, 300), device="cuda")
        x[0, 5] = top
        x[0, 6:40] = torch.arange(34, device="cuda") * 0.0625 * (top if math.isfinite(top) else 1.0) / 34
        x[2, 130:150] = torch.tensor([17.0, 19.0, 21.0, 23.0, 1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -9, 448.0] * 2, device="cuda")
        codes, scales = F.quantize(x, block)
        want, e = ref.pack(x, block)
        assert torch.equal(scales.long(), e), (k, top)
        assert same(codes.float(), want), (k, top)
        assert torch.isfinite(codes.float()[2]).all() and (block == 128 or math.isfinite(top) or torch.isfinite(codes.float()[0, 6:]).all())
        back = F.dequantize(codes, scales, torch.float32)
        assert same(back, ref.unpack(want, e, block).float()), (k, top)


def test_every_code_and_scale_comes_back():
    from paper_2609_21594_b200 import functional as F

    codes = torch.arange(256, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn).repeat(255, 1)
    scales = torch.arange(255, device="cuda", dtype=torch.uint8)[:, None].repeat(1, 2)
    for dtype in (torch.bfloat16, torch.float32):
        assert same(F.dequantize(codes, scales, dtype), ref.unpack(codes.float(), scales, 1).to(dtype))
    assert torch.isnan(F.dequantize(codes[:1], scales[:1] * 0 + 255, torch.float32)).all()


@pytest.mark.parametrize("block", [1, 128])
def test_views_and_shapes(block):
    """Rows that are part of wider ones, transposed input, codes of a slice; more than two dimensions, none of the elements."""
    from paper_2609_21594_b200 import functional as F

    wide = make(140, 700, torch.bfloat16)
    for x in (wide[:, 3:260], wide[:, 8:264], wide[::2, :129], wide.T):
        codes, scales = F.quantize(x, block)
        want, e = ref.pack(x, block)
        assert torch.equal(scales.long(), e) and same(codes.float(), want)
        assert same(F.dequantize(codes, scales, torch.bfloat16), ref.unpack(want, e, block).bfloat16())
    if block == 1:
        x = make(24, 100, torch.float32)
        codes, scales = F.quantize(x.view(2, 3, 4, 100))
        assert codes.shape == (2, 3, 4, 100) and scales.shape == (2, 3, 4, 1)
        want, e = ref.pack(x, 1)
        assert same(codes.float().view(24, 100), want) and torch.equal(scales.view(24, 1).long(), e)
        assert same(F.dequantize(codes, scales, torch.float32).view(24, 100), ref.unpack(want, e, 1).float())
        part = F.dequantize(codes[:, 1:, 2:], scales[:, 1:, 2:], torch.float32)
        assert same(part.reshape(-1, 100), ref.unpack(want, e, 1).view(2, 3, 4, 100)[:, 1:, 2:].reshape(-1, 100).float())
    codes, scales = F.quantize(wide[:0], block)
    assert codes.shape == (0, 700) and scales.shape == (0, 6) and F.dequantize(codes, scales, torch.float32).shape == (0, 700)


def test_what_lies_behind_the_columns_is_left_alone():
    from paper_2609_21594_b200 import binding as mb, functional as F

    x = make(7, 100, torch.float32)
    codes, scales = torch.full((7, 144), 99, dtype=torch.uint8, device="cuda"), torch.full((7, 3), 99, dtype=torch.uint8, device="cuda")
    back = torch.full((7, 120), -5.0, device="cuda")
    blocks = mb.Blocks(codes.data_ptr(), 144, scales.data_ptr(), 3, 1, 0)
    F.context().muon_quantize(mb.DTYPE_FP32, 7, 100, mb.Rows(x.data_ptr(), 100), blocks)
    F.context().muon_dequantize(mb.DTYPE_FP32, 7, 100, blocks, mb.Rows(back.data_ptr(), 120))
    want, e = ref.pack(x, 1)
    assert same(codes[:, :100].view(torch.float8_e4m3fn).float(), want) and (codes[:, 100:] == 99).all()
    assert torch.equal(scales[:, :1].long(), e) and (scales[:, 1:] == 99).all()
    assert same(back[:, :100], ref.unpack(want, e, 1).float()) and (back[:, 100:] == -5).all()


def test_refusals():
    from paper_2609_21594_b200 import binding as mb, functional as F

    x = torch.zeros((4, 256), device="cuda")
    codes, scales = F.quantize(x)
    for call in (lambda: F.quantize(x.half()), lambda: F.quantize(x, 64), lambda: F.quantize(x.view(2, 2, 256), 128), lambda: F.quantize(x[:, :0]),
                 lambda: F.quantize(x[0, 0]), lambda: F.dequantize(codes, scales[:, :1], torch.float32), lambda: F.dequantize(codes, scales, torch.float16),
                 lambda: F.dequantize(x, scales, torch.float32), lambda: F.dequantize(codes, scales.int(), torch.float32),
                 lambda: F.dequantize(codes, scales.cpu(), torch.float32), lambda: F.dequantize(codes, scales[:3], torch.float32)):
        with pytest.raises(ValueError):
            call()
    c = F.context()
    good = mb.Blocks(codes.data_ptr(), 256, scales.data_ptr(), 2, 1, 0)
    for blocks, rows in ((mb.Blocks(codes.data_ptr(), 255, scales.data_ptr(), 2, 1, 0), mb.Rows(x.data_ptr(), 256)),
                         (mb.Blocks(codes.data_ptr(), 256, scales.data_ptr(), 1, 1, 0), mb.Rows(x.data_ptr(), 256)),
                         (mb.Blocks(codes.data_ptr(), 256, scales.data_ptr(), 2, 2, 0), mb.Rows(x.data_ptr(), 256)),
                         (mb.Blocks(codes.data_ptr(), 256, scales.data_ptr(), 2, 1, 1), mb.Rows(x.data_ptr(), 256)),
                         (mb.Blocks(None, 256, scales.data_ptr(), 2, 1, 0), mb.Rows(x.data_ptr(), 256)),
                         (mb.Blocks(x.data_ptr(), 256, scales.data_ptr(), 2, 1, 0), mb.Rows(x.data_ptr(), 256)),        # over the input
                         (mb.Blocks(codes.data_ptr(), 256, codes.data_ptr() + 100, 2, 1, 0), mb.Rows(x.data_ptr(), 256)),
                         (good, mb.Rows(x.data_ptr(), 255)), (good, mb.Rows(x.data_ptr() + 2, 256)), (good, None), (None, mb.Rows(x.data_ptr(), 256))):
        with pytest.raises(mb.MuonError) as e:
            c.muon_quantize(mb.DTYPE_FP32, 4, 256, rows, blocks)
        assert e.value.code == mb.ERR_INVALID_ARG
        if blocks is None or blocks.codes != x.data_ptr():
            if blocks is None or blocks.scales != codes.data_ptr() + 100:
                with pytest.raises(mb.MuonError):
                    c.muon_dequantize(mb.DTYPE_FP32, 4, 256, blocks, rows)
