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
