"""Block-scaled products on every tile and in slices of K, for every pair of formats."""
import numpy as np
import pytest
import torch

from mx_helpers import FLOOR, FORMATS, TYPES, U, f64, matrix, on_gpu, rng
from oracle import mx
from paper_2210_09603_amd import binding as hb
from test_gpu_mx import _exact_case, _powers

pytestmark = pytest.mark.gpu

PAIRS = [(a, b) for a in FORMATS for b in FORMATS]
# (64 x 64 tiles, in two slices of K too, 64 x 128, 128 x 128, 256 x 256)
TILES = [(1000, 1020, 1060), (500, 1000, 8200), (1030, 1020, 2500), (1030, 2050, 700), (4000, 4090, 300)]


@pytest.mark.parametrize("formats", PAIRS, ids=str)
@pytest.mark.parametrize("size", TILES + [(1024, 1024, 1024)], ids=str)
def test_products_of_every_pair_on_tiles(size, formats):
    _exact_case(*size, *formats, ("f32", "bf16", "f16")[(sum(size) + sum(formats)) % 3], 7, odd=bool(sum(formats) % 2))


@pytest.mark.parametrize("formats", PAIRS, ids=str)
@pytest.mark.parametrize("size", TILES, ids=str)
def test_products_of_elements_of_all_sizes_on_tiles(size, formats):
    """Every element code but NaN and infinity, and scales apart by 2^8, against sums of eights as the matrix cores cut them, for 40 rows and 40 columns,
    both ends and the middle among them: a step of fp32 for every one of K / 128 + 16 additions, and half a step of the output's type."""
    m, n, k = size
    g = rng(m, n, k, *formats)

    def operand(rows, fmt):
        top = {mx.E4M3: 0x7F, mx.E5M2: 0x7C, mx.E2M1: 8}[fmt]
        width = mx.blocks(k) * 32
        codes = g.integers(0, top, (rows, width)).astype(np.uint8)
        codes = np.where(g.random((rows, width)) < 0.5, codes, codes + mx.sign_bit(fmt)).astype(np.uint8)
        codes[:, k:] = 0
        middle = 127 - mx.POWER[fmt]
        return codes, g.integers(middle - 4, middle + 5, (mx.blocks(k), rows)).astype(np.uint8)

    a, b = operand(m, formats[0]), operand(n, formats[1])
    ma, mb = matrix(*a, k, formats[0]), matrix(*b, k, formats[1])

    def some(count):
        return np.unique(np.r_[0:3, count // 2:count // 2 + 2, count - 3:count, g.integers(0, count, 32)])

    rows, cols = some(m), some(n)
    want, size_of = mx.product_of_cut_eights((a[0][rows], a[1][:, rows]), formats[0], (b[0][cols], b[1][:, cols]), formats[1])
    bound = (mx.blocks(k) / 4 + 16) * 2.0 ** -24 * size_of
    for out in ("f32", "bf16"):
        c = torch.empty((m, n), dtype=TYPES[out], device="cuda")
        ws = torch.empty(max(4, hb.hidet_mx_gemm_workspace_bytes(ma, mb)), dtype=torch.uint8, device="cuda")
        hb.hidet_mx_gemm(ma, mb, c, workspace=ws)
        first = c.clone()
        got = f64(c)[np.ix_(rows, cols)]
        ratio = (np.abs(got - want) / (bound + U[out] * (np.abs(want) + bound) + FLOOR[out])).max()
        assert ratio <= 1, ratio
        for _ in range(3):  # the same bits again
            c.fill_(7.0)
            hb.hidet_mx_gemm(ma, mb, c, workspace=ws)
            assert torch.equal(first, c)


# (slices of 16 x 16, 16 x 64 and 64 x 64, whose sums another kernel adds and finishes)
@pytest.mark.parametrize("size,formats", [((3, 41, 20000), (0, 2)), ((16, 100, 20000), (2, 2)), ((20, 66, 12001), (2, 1)), ((70, 66, 9000), (0, 2)), ((70, 67, 9000), (0, 0)),
                                          ((129, 202, 9000), (1, 0)), ((500, 1001, 8200), (2, 2))], ids=str)
@pytest.mark.parametrize("out", ["f32", "f16", "bf16"])
def test_epilogues_behind_slices(size, formats, out):
    m, n, k = size
    assert hb.lib().hidet_mx_gemm_workspace_bytes(m, n, k, *formats) > 0
    for i, e in enumerate((dict(bias="col"), dict(bias="row", relu=True), dict(residual=True), dict(residual=True, apart=3, odd=True),
                           dict(alpha=0.5, bias="col", residual=True, relu=True, odd=True))):
        _exact_case(m, n, k, *formats, out, 20 + i, **e)


@pytest.mark.parametrize("size", [(3, 41, 20000), (70, 67, 9000)], ids=str)
def test_a_residual_in_place_behind_slices(size):
    m, n, k = size
    g = rng(m, n, k, 6)
    a, b = _powers(g, m, k, 0), _powers(g, n, k, 0)
    r = g.integers(-8, 8, (m, n)).astype(np.float64)
    c = on_gpu(r, "f32")
    ma, mb = matrix(*a, k, 0), matrix(*b, k, 0)
    ws = torch.full((hb.hidet_mx_gemm_workspace_bytes(ma, mb),), 0xFF, dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0
    hb.hidet_mx_gemm(ma, mb, c, epilogue=hb.make_epilogue(residual=c), workspace=ws)
    assert np.array_equal(f64(c), mx.numbers(*a, 0) @ mx.numbers(*b, 0).T + r)


def test_parts_of_k_are_products_of_their_own():
    """Columns from a multiple of 32 on: views of the values, whole rows of scales."""
    g = rng(12)
    for m, n in ((5, 40), (40, 130), (1000, 1020)):
        k, k0, k1 = 1060, 160, 800
        a, b = _powers(g, m, k, 0), _powers(g, n, k, 2)
        va, sa = matrix(*a, k, 0).tensors
        vb, sb = matrix(*b, k, 2).tensors
        pa = hb.make_mx(m, k1 - k0, 0, va[:, k0:k1], sa[k0 // 32:k1 // 32])
        pb = hb.make_mx(n, k1 - k0, 2, vb[:, k0 // 2:k1 // 2], sb[k0 // 32:k1 // 32])
        c = torch.empty((m, n), device="cuda")
        ws = torch.empty(max(4, hb.hidet_mx_gemm_workspace_bytes(pa, pb)), dtype=torch.uint8, device="cuda")
        hb.hidet_mx_gemm(pa, pb, c, workspace=ws)
        assert np.array_equal(f64(c), mx.numbers(*a, 0)[:, k0:k1] @ mx.numbers(*b, 2)[:, k0:k1].T)
