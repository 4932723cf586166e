"""Pins of the float64 oracle of block-scaled matrices and norms."""
import numpy as np
import pytest
import torch

from oracle import mx

FORMATS = [mx.E4M3, mx.E5M2, mx.E2M1]
TORCH = {mx.E4M3: torch.float8_e4m3fn, mx.E5M2: torch.float8_e5m2}


def test_the_grids_are_those_of_the_formats():
    assert list(mx.grid(mx.E2M1)) == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    for fmt, dtype in TORCH.items():
        codes = np.arange(256, dtype=np.uint8)
        want = torch.from_numpy(codes).view(dtype).double().numpy()
        assert np.array_equal(mx.values(codes, fmt), want, equal_nan=True)
        assert mx.grid(fmt)[-1] == mx.LARGEST[fmt] == torch.finfo(dtype).max and 2.0 ** mx.POWER[fmt] in mx.grid(fmt)


@pytest.mark.parametrize("fmt", FORMATS)
def test_nearest_is_nearest_and_even(fmt):
    g = mx.grid(fmt)
    for i in range(len(g) - 1):
        middle = (g[i] + g[i + 1]) / 2
        even = i if i % 2 == 0 else i + 1
        assert mx.nearest(np.array([middle]), fmt)[0] == even
        assert mx.nearest(np.array([np.nextafter(middle, 0)]), fmt)[0] == i
        assert mx.nearest(np.array([-np.nextafter(middle, 9e9)]), fmt)[0] == i + 1 + mx.sign_bit(fmt)
    assert mx.nearest(np.array([1e30]), fmt)[0] == len(g) - 1
    if fmt in TORCH:
        q = np.random.default_rng(0).standard_normal(4000) * g[-1] / 5
        q = q[np.abs(q) <= g[-1]].astype(np.float32)
        want = torch.from_numpy(q).to(TORCH[fmt]).view(torch.uint8).numpy()
        assert np.array_equal(mx.nearest(q.astype(np.float64), fmt), want)


@pytest.mark.parametrize("fmt", FORMATS)
def test_scales(fmt):
    p = mx.POWER[fmt]
    x = np.zeros((4, 33))
    x[0, 5], x[1, 32], x[2, 0], x[3, 1] = 2.0 ** p, -1.999, 2.0 ** -140, np.inf
    codes, scales = mx.quantize(x, fmt)
    assert scales.shape == (2, 4) and codes.shape == (4, 64)
    assert list(scales[0]) == [127, 0, 0, 255] and list(scales[1]) == [0, 127 - p, 0, 0]
    n = mx.numbers(codes, scales, fmt)
    assert n[0, 5] == 2.0 ** p and np.isnan(n[3, :32]).all() and not n[3, 32:].any()
    assert n[1, 32] == -mx.LARGEST[fmt] * 2.0 ** -p
    # numbers of the format come back as they are
    again, s = mx.quantize(n[:3], fmt)
    assert np.array_equal(mx.numbers(again, s, fmt), n[:3])


def test_four_bits_lie_low_half_first():
    codes = np.arange(16, dtype=np.uint8)[None].repeat(2, 0)
    data = mx.pack(codes, mx.E2M1)
    assert data[0, 0] == 0x10 and data[0, 7] == 0xFE and np.array_equal(mx.unpack(data, mx.E2M1), codes)


def test_norm_and_its_gradient():
    g = np.random.default_rng(1)
    h, w, gy = g.standard_normal((5, 11)), g.standard_normal(11), g.standard_normal((5, 11))
    t = torch.from_numpy(h).requires_grad_()
    tw = torch.from_numpy(w).requires_grad_()
    out = torch.nn.functional.rms_norm(t, (11,), eps=1e-3) * (tw + 0.5)
    out.backward(torch.from_numpy(gy))
    y, rstd = mx.rms_norm(h, w, 1e-3, 0.5)
    gh, gw = mx.rms_norm_grad(gy, h, rstd, w, 0.5)
    assert np.allclose(y, out.detach().numpy(), rtol=1e-12) and np.allclose(gh, t.grad.numpy(), rtol=1e-10)
    assert np.allclose(gw, tw.grad.numpy(), rtol=1e-12)
    step = 1e-6  # and against differences
    for i, j in ((0, 0), (3, 7)):
        a, b = h.copy(), h.copy()
        a[i, j] += step
        b[i, j] -= step
        d = ((mx.rms_norm(a, w, 1e-3, 0.5)[0] - mx.rms_norm(b, w, 1e-3, 0.5)[0]) * gy).sum() / (2 * step)
        assert abs(d - gh[i, j]) < 1e-7


def test_products_whose_eights_are_cut():
    """By hand: e4m3, 2^8 * 2^8 beside 2^k; 4 by 4 bits and eights of one size lose nothing."""
    def row(*codes):
        c = np.zeros((1, 32), dtype=np.uint8)
        c[0, :len(codes)] = codes
        return c, np.full((1, 1), 127, dtype=np.uint8)

    def power(e):
        return (e + 7) << 3

    for small, want in ((3, 2.0 ** 16 + 2.0 ** 3), (2, 2.0 ** 16)):
        total, size = mx.product_of_cut_eights(row(power(8), power(small)), 0, row(power(8), power(0)), 0)
        assert total[0, 0] == want and size[0, 0] == 2.0 ** 16 + 2.0 ** small
    # the small one in another eight; 2^-9 counts as 2^-6: 2^-9 * 2^8 keeps 2^-11, and cuts 2^-12 towards zero
    assert mx.product_of_cut_eights(row(power(8), 0, 0, 0, 0, 0, 0, 0, power(2)), 0, row(power(8), 0, 0, 0, 0, 0, 0, 0, power(0)), 0)[0][0, 0] == 2.0 ** 16 + 4
    for small, want in ((-5, 0.5 + 2.0 ** -11), (-6, 0.5)):
        assert mx.product_of_cut_eights(row(1, power(small)), 0, row(power(8), power(-6)), 0)[0][0, 0] == want
        assert mx.product_of_cut_eights(row(1, power(small) | 128), 0, row(power(8), power(-6)), 0)[0][0, 0] == 1.0 - want
    # elements that meet a 0 do not count
    assert mx.product_of_cut_eights(row(0, power(-6), power(8)), 0, row(power(8), power(-6), 0), 0)[0][0, 0] == 2.0 ** -12
    g = np.random.default_rng(2)
    a, b = (g.integers(0, 16, (5, 64)).astype(np.uint8) for _ in range(2))
    s = g.integers(120, 130, (2, 5)).astype(np.uint8)
    assert np.array_equal(mx.product_of_cut_eights((a, s), 2, (b, s), 2)[0], mx.numbers(a, s, 2) @ mx.numbers(b, s, 2).T)
