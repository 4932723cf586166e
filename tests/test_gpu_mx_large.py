"""Conversions of matrices into and out of blocks at the sizes that the kernels of large calls serve: wide tiles, and past the caches.

A conversion has one right result.  That of a matrix is compared with the oracle where it is small enough, and else with those of its
pieces, each of a size whose kernel the oracle pins (tests of small sizes), and with the oracle at rows of both ends and of the middle."""
import numpy as np
import pytest
import torch

from mx_helpers import FORMATS, TYPES, Room, f64
from oracle import mx
from paper_2210_09603_amd import binding as hb

pytestmark = pytest.mark.gpu


def _numbers_of_many_sizes(rows, cols, dtype, seed, before, after):
    """A view whose rows lie apart, of numbers of many sizes with some zeros, a NaN and an infinity."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = torch.full((rows, before + cols + after), 7.0, dtype=TYPES[dtype], device="cuda")
    x = wide[:, before:before + cols]
    for r in range(0, rows, 4096):
        part = x[r:r + 4096]
        n = part.shape
        v = torch.randn(n, generator=g, device="cuda") * torch.exp2(torch.randint(-12, 6, (n[0], 1), generator=g, device="cuda").float())
        v *= torch.exp2(torch.randint(-3, 3, n, generator=g, device="cuda").float())
        part.copy_(v * (torch.rand(n, generator=g, device="cuda") > 0.05))
    x[rows // 2, cols // 3], x[rows - 1, cols - 1] = float("nan"), float("inf")
    x[rows // 3, :] = 0.0
    return wide, x


def _same(room, m):
    codes, scales = room.read()
    ocodes, oscales = mx.quantize(m, room.fmt)
    assert np.array_equal(scales, oscales) and np.array_equal(codes, ocodes)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_rows_in_wide_tiles(dtype, fmt):
    """1026 tiles of 16 x 512 (2052 of 8 x 512 in fp32), the last ones cut on both sides; rows at element alignment."""
    rows, cols = 5471, 1030
    for before, after in ((0, 2), (1, 2)):
        _, x = _numbers_of_many_sizes(rows, cols, dtype, fmt, before, after)
        r = Room(rows, cols, fmt)
        hb.hidet_mx_quantize(x, by_rows=r.m)
        _same(r, f64(x))


def _part(room, r0, r1, cols):
    """Rows r0 .. r1 of a matrix in blocks, as a matrix of its own."""
    return hb.make_mx(r1 - r0, cols, room.fmt, room.values[r0:r1, :room.width], room.scales[:room.blocks, r0:r1])


LARGE = {"f32": (8203, 4099), "f16": (16391, 4099), "bf16": (16391, 4099)}  # 128 MiB and more: past the caches


@pytest.mark.parametrize("dtype,fmt", [("f32", 0), ("f32", 1), ("f32", 2), ("f16", 1), ("f16", 2), ("bf16", 0), ("bf16", 1), ("bf16", 2)])
def test_conversions_past_the_caches(dtype, fmt):
    rows, cols = LARGE[dtype]
    before = (fmt + (dtype == "bf16")) % 2
    wide, x = _numbers_of_many_sizes(rows, cols, dtype, 10 + fmt, before, 1)
    assert x.numel() * x.element_size() >= 128 << 20
    one, both_r = Room(rows, cols, fmt), Room(rows, cols, FORMATS[(fmt + 1) % 3])
    columns, both_c = Room(cols, rows, FORMATS[(fmt + 2) % 3]), Room(cols, rows, fmt)
    hb.hidet_mx_quantize(x, by_rows=one.m)
    hb.hidet_mx_quantize(x, by_columns=columns.m)
    hb.hidet_mx_quantize(x, by_rows=both_r.m, by_columns=both_c.m)
    ends = np.r_[0:5, rows // 2 - 2:rows // 2 + 3, rows // 3, rows - 20:rows]
    some = f64(x[torch.from_numpy(ends).cuda()])
    for room in (one, both_r):
        codes, scales = room.read()
        ocodes, oscales = mx.quantize(some, room.fmt)
        assert np.array_equal(scales[:, ends], oscales) and np.array_equal(codes[ends], ocodes)
    ends = np.r_[0:5, cols // 3 - 2:cols // 3 + 3, cols - 20:cols]
    some = f64(x[:, torch.from_numpy(ends).cuda()]).T
    for room in (columns, both_c):
        codes, scales = room.read()
        ocodes, oscales = mx.quantize(some, room.fmt)
        assert np.array_equal(scales[:, ends], oscales) and np.array_equal(codes[ends], ocodes)
    # 1024 rows a piece (whole blocks of columns): neither many tiles nor many bytes
    for r0 in range(0, rows, 1024):
        r1 = min(r0 + 1024, rows)
        for room in (one, both_r):
            piece = hb.make_mx(r1 - r0, cols, room.fmt, device="cuda")
            hb.hidet_mx_quantize(x[r0:r1], by_rows=piece)
            values, scales = piece.tensors
            assert torch.equal(room.values[r0:r1, :room.width], values) and torch.equal(room.scales[:room.blocks, r0:r1], scales)
        for room in (columns, both_c):
            piece = hb.make_mx(cols, r1 - r0, room.fmt, device="cuda")
            hb.hidet_mx_quantize(x[r0:r1], by_columns=piece)
            values, scales = piece.tensors
            b = room.width // room.blocks  # (bytes of a block)
            assert torch.equal(room.values[:cols, r0 // 32 * b:(r1 + 31) // 32 * b], values)
            assert torch.equal(room.scales[r0 // 32:(r1 + 31) // 32, :cols], scales)
    # and back: the whole, and in pieces
    for i, room in enumerate((one, both_r)):
        wide.fill_(7.0)
        hb.hidet_mx_dequantize(room.m, x)
        assert bool((wide[:, :before] == 7).all()) and bool((wide[:, before + cols:] == 7).all())
        for r0 in range(0, rows, 1024):
            r1 = min(r0 + 1024, rows)
            y = torch.empty((r1 - r0, cols), dtype=TYPES[dtype], device="cuda")
            hb.hidet_mx_dequantize(_part(room, r0, r1, cols), y)
            bits = torch.int32 if dtype == "f32" else torch.int16
            same = x[r0:r1].contiguous().view(bits) == y.view(bits)
            assert bool((same | (y.isnan() & x[r0:r1].isnan())).all())
        some = np.r_[0:4, rows // 2, rows - 4:rows]
        codes, scales = room.read()
        want = torch.from_numpy(mx.numbers(codes[some], scales[:, some], room.fmt)[:, :cols].astype(np.float32)).to(TYPES[dtype])
        assert np.array_equal(f64(x[torch.from_numpy(some).cuda()]), f64(want), equal_nan=True)
