"""What products lose where an operand has 8 bits, against sums whose eights are cut as the header says.

With one block of 8 elements that are not 0 the result is one such sum: equal, but for the rounding to fp32, which it needs none of (fewer than
24 bits).  Longer ones: these sums are added in fp32, a step of 2^-24 of sum |a b| for each of K / 128 + 16 additions."""
import numpy as np
import pytest
import torch

from mx_helpers import FORMATS, f64, matrix, rng
from oracle import mx
from paper_2210_09603_amd import binding as hb

pytestmark = pytest.mark.gpu

PAIRS = [(a, b) for a in FORMATS for b in FORMATS]


def _elements(g, rows, k, fmt, zeros):
    """Any code but NaN and infinity."""
    codes = g.integers(0, {mx.E4M3: 0x7F, mx.E5M2: 0x7C, mx.E2M1: 8}[fmt], (rows, mx.blocks(k) * 32)).astype(np.uint8)
    codes = np.where(g.random(codes.shape) < 0.5, codes, codes + mx.sign_bit(fmt)).astype(np.uint8)
    codes[g.random(codes.shape) < zeros] = 0
    codes[:, k:] = 0
    return codes, g.integers(125, 130, (mx.blocks(k), rows)).astype(np.uint8)


# (workgroups of 16 x 16, of 16 x 64, in slices of K too, 64 x 64 tiles, and 128 x 128)
@pytest.mark.parametrize("formats", PAIRS, ids=str)
@pytest.mark.parametrize("size", [(5, 48, 8), (40, 48, 8), (1000, 130, 8), (5, 48, 400), (40, 130, 256), (300, 260, 256), (70, 66, 9000), (517, 1030, 40), (1030, 2050, 8)], ids=str)
def test_eights_are_cut_and_no_more(size, formats):
    m, n, k = size
    for zeros in (0.0, 0.5):
        g = rng(m, n, k, *formats, int(2 * zeros))
        a, b = _elements(g, m, k, formats[0], zeros), _elements(g, n, k, formats[1], zeros)
        ma, mb = matrix(*a, k, formats[0]), matrix(*b, k, formats[1])
        c = torch.full((m, n), 7.0, device="cuda")
        ws = torch.empty(max(4, hb.hidet_mx_gemm_workspace_bytes(ma, mb)), dtype=torch.uint8, device="cuda")
        hb.hidet_mx_gemm(ma, mb, c, workspace=ws)
        want, size_of = mx.product_of_cut_eights(a, formats[0], b, formats[1])
        error = np.abs(f64(c) - want)
        assert (error <= (0 if k == 8 else (mx.blocks(k) / 4 + 16) * 2.0 ** -24) * size_of).all()


@pytest.mark.parametrize("formats", PAIRS, ids=str)
def test_scales_of_all_sizes(formats):
    """1 * 2^(i - 127) times 1 * 2^(j - 127) for all finite scales: numbers below the normal range among the results, infinities above."""
    one = {mx.E4M3: 0x38, mx.E5M2: 0x3C, mx.E2M1: 2}
    scales = np.arange(255, dtype=np.uint8)[None]

    def ones(fmt):
        codes = np.zeros((255, 32), dtype=np.uint8)
        codes[:, 5] = one[fmt]
        return matrix(codes, scales, 32, fmt)

    a, b = ones(formats[0]), ones(formats[1])
    c = torch.empty((255, 255), device="cuda")
    hb.hidet_mx_gemm(a, b, c)
    with np.errstate(over="ignore"):
        want = np.ldexp(1.0, np.arange(255)[:, None] + np.arange(255)[None] - 254).astype(np.float32)
    assert np.array_equal(c.cpu().numpy(), want)


@pytest.mark.parametrize("size", [(7, 40, 200), (40, 70, 200), (600, 1030, 200)], ids=str)
@pytest.mark.parametrize("formats", [p for p in PAIRS if p != (mx.E2M1, mx.E2M1)], ids=str)
def test_elements_that_are_not_finite(size, formats):
    """They make of their rows and columns what they make of sums of numbers, and nothing of others."""
    m, n, k = size
    g = rng(m, n, *formats)
    a, b = _elements(g, m, k, formats[0], 0.2), _elements(g, n, k, formats[1], 0.2)
    for side, fmt, rows in ((a, formats[0], m), (b, formats[1], n)):
        if fmt == mx.E2M1:
            continue
        for row, code in ((1, 0x7F), (3, 0xFF)) + (((rows - 1, 0x7C), (rows - 2, 0xFC), (4, 0x7E)) if fmt == mx.E5M2 else ()):
            side[0][row, int(g.integers(0, k))] = code
    c = torch.full((m, n), 7.0, device="cuda")
    hb.hidet_mx_gemm(matrix(*a, k, formats[0]), matrix(*b, k, formats[1]), c)
    got = f64(c)
    with np.errstate(invalid="ignore"):
        want = mx.numbers(*a, formats[0]) @ mx.numbers(*b, formats[1]).T
    for f in (np.isnan, np.isposinf, np.isneginf):
        assert np.array_equal(f(got), f(want)), f
