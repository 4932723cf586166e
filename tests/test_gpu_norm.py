"""Root-mean-square norms against the float64 oracle.

y: half a step of its type, and 2^-24 each for rstd, the weight's offset and two products.  In blocks: what the rounding of y (1 - d) or y (1 + d)
gives, d = 2^-21 for the same.  Gradients: half a step; 8 roundings of fp32 of every term, and (8 + rows of a workgroup + 64 + 16) * 2^-24 of the sum
of magnitudes for the sums."""
import numpy as np
import pytest
import torch

from mx_helpers import FLOOR, FORMATS, TYPES, U, Room, f64, on_gpu, padded, rng
from oracle import mx
from paper_2210_09603_amd import binding as hb

pytestmark = pytest.mark.gpu

PAIRS = [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f32")]
SMALL = [(1, 1), (3, 7), (5, 32), (2, 64), (33, 128), (4, 129), (17, 1000), (9, 1024), (6, 2048), (3, 4096), (5, 5121), (2, 8192)]
WIDE = [(3, 12000), (3, 16384), (2, 32768), (1030, 520), (1025, 1029), (1024, 1500), (1027, 2040), (1025, 3000), (1026, 4096), (1024, 5120),
        (1024, 100)]
CASES = [(size, types) for size in SMALL for types in PAIRS] + [(size, PAIRS[(sum(size) + i) % 5]) for size in WIDE for i in (0, 2)]


def _check_blocks(room, y, what):
    codes, scales = room.read()
    d = 2.0 ** -21
    low, high = (mx.quantize(y * f, room.fmt) for f in (1 - d, 1 + d))
    assert ((scales == low[1]) | (scales == high[1])).all(), what
    one, two = (mx.quantize(y * f, room.fmt, scales)[0] for f in (1 - d, 1 + d))
    assert ((codes == one) | (codes == two)).all(), what


def _bound(y, dtype):
    return np.abs(y) * (U[dtype] + 5 * 2.0 ** -24) + FLOOR[dtype]


@pytest.mark.parametrize("size,types", CASES + [((1024, 8192), PAIRS[2])], ids=str)
def test_norm(size, types):
    rows, cols = size
    dtype, wtype = types
    g = rng(rows, cols)
    x, r = g.standard_normal((rows, cols)) * 2.0 ** g.integers(-3, 8, (rows, 1)), g.standard_normal((rows, cols))
    w = on_gpu(0.3 * g.standard_normal(cols) + 1, wtype)
    for i, (before, after) in enumerate(((0, 0), (1, 4))):
        _, tx = padded(x, dtype, before, after)
        _, tr = padded(r, dtype, before, after + 1)
        wide, y = padded(np.zeros((rows, cols)), dtype, 2, 1)
        wides, s = padded(np.zeros((rows, cols)), dtype, 0, 3)
        rstd = torch.full((rows + 1,), 7.0, device="cuda")
        room = Room(rows, cols, FORMATS[(rows + cols + i) % 3])
        offset, eps = (0.0, 1e-5) if i else (1.0, 1e-3)
        # without the residual
        hb.hidet_rms_norm(tx, w, y=y, rstd=rstd[:rows], eps=eps, offset=offset)
        want, orstd = mx.rms_norm(f64(tx), f64(w), eps, offset)
        assert (np.abs(f64(y) - want) <= _bound(want, dtype)).all()
        assert (np.abs(f64(rstd)[:rows] - orstd) <= 2.0 ** -23 * orstd).all() and float(rstd[rows]) == 7.0
        # with it, all outputs
        hb.hidet_rms_norm(tx, w, y=y, residual=tr, sum=s, quantized=room.m, eps=eps, offset=offset)
        h = (tx.float() + tr.float()).to(TYPES[dtype])
        assert bool((s == h).all())
        want, _ = mx.rms_norm(f64(h), f64(w), eps, offset)
        assert (np.abs(f64(y) - want) <= _bound(want, dtype)).all()
        _check_blocks(room, want, (size, types))
        # blocks alone, the stream in place of the residual, then y in place of x
        room = Room(rows, cols, FORMATS[(rows + i) % 3], wide=False)
        hb.hidet_rms_norm(tx, w, residual=tr, sum=tr, quantized=room.m, eps=eps, offset=offset)
        assert bool((tr == h).all())
        _check_blocks(room, want, (size, types))
        hb.hidet_rms_norm(tx, w, y=tx, eps=eps, offset=offset)
        want, _ = mx.rms_norm(f64(padded(x, dtype, 0, 0)[1]), f64(w), eps, offset)
        assert (np.abs(f64(tx) - want) <= _bound(want, dtype)).all()
        for t, a, b in ((wide, 2, 1), (wides, 0, 3)):
            assert bool((t[:, :a] == 7).all()) and bool((t[:, t.shape[1] - b:] == 7).all())


@pytest.mark.parametrize("size,types", CASES + [((4000, 72), PAIRS[2]), ((2500, 300), PAIRS[1]), ((1030, 800), PAIRS[3])], ids=str)
def test_backward(size, types):
    rows, cols = size
    dtype, wtype = types
    g = rng(rows, cols, 1)
    w = on_gpu(0.3 * g.standard_normal(cols), wtype)
    offset = float(rows % 2)
    for before, after in ((0, 0), (3, 2)):
        _, h = padded(g.standard_normal((rows, cols)) * 2.0 ** g.integers(-3, 4, (rows, 1)), dtype, before, after)
        _, gy = padded(g.standard_normal((rows, cols)), dtype, before, after + 1)
        _, gs = padded(g.standard_normal((rows, cols)), dtype, before, after + 2)
        _, orstd = mx.rms_norm(f64(h), f64(w), 1e-5, offset)
        rstd = torch.from_numpy(orstd.astype(np.float32)).cuda()
        n = hb.hidet_rms_norm_backward_workspace_bytes(rows, cols)
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        r64, w64, g64, h64 = f64(rstd)[:, None], f64(w) + offset, f64(gy), f64(h)
        terms = np.abs(r64 * g64 * w64) + np.abs(r64 * h64 * r64) * np.abs(g64 * w64 * h64 * r64).mean(1, keepdims=True)
        gh0, gw0 = mx.rms_norm_grad(g64, h64, f64(rstd), f64(w), offset)
        parts = -(-rows // 256)  # (more rows of a workgroup than any cut has)
        b_gw = U[wtype] * np.abs(gw0) + (8 + parts + 80) * 2.0 ** -24 * np.abs(g64 * h64 * r64).sum(0) + FLOOR[wtype]
        for stream in (None, gs):
            wide, gh = padded(np.zeros((rows, cols)), dtype, 1, 1)
            gw = torch.full((cols + 1,), 7.0, dtype=TYPES[wtype], device="cuda")
            hb.hidet_rms_norm_backward(gy, h, rstd, w, gh, gw[:cols], ws, grad_sum=stream, offset=offset)
            want = gh0 + (0 if stream is None else f64(gs))
            bound = U[dtype] * np.abs(want) + 17 * 2.0 ** -24 * (terms + (0 if stream is None else np.abs(f64(gs)))) + FLOOR[dtype]
            assert (np.abs(f64(gh) - want) <= bound).all()
            assert (np.abs(f64(gw)[:cols] - gw0) <= b_gw).all() and float(gw[cols]) == 7.0
            assert bool((wide[:, :1] == 7).all()) and bool((wide[:, -1:] == 7).all())
        first = gw.clone()
        hb.hidet_rms_norm_backward(gy, h, rstd, w, gs, None, None, grad_sum=gs, offset=offset)  # in place, without the weight's
        assert (np.abs(f64(gs) - want) <= bound).all()
        hb.hidet_rms_norm_backward(gy, h, rstd, w, gy, gw[:cols], ws, offset=offset)
        assert bool((first == gw).all())  # (the same bits)


def test_rows_that_are_not_finite_or_zero_stay_alone():
    g = rng(7)
    x = g.standard_normal((6, 200))
    x[1, 3], x[2, 199], x[3] = np.nan, np.inf, 0.0
    x[4] *= 1e30
    t, w = on_gpu(x, "f32"), torch.ones(200, device="cuda")
    y, room = torch.empty_like(t), Room(6, 200, hb.HIDET_MX_E4M3)
    hb.hidet_rms_norm(t, w, y=y, quantized=room.m, eps=1e-5)
    got = f64(y)
    want, _ = mx.rms_norm(f64(t)[[0, 4, 5]], np.ones(200), 1e-5, 0.0)
    assert (np.abs(got[[0, 4, 5]] - want) <= _bound(want, "f32")).all() and not got[3].any()
    assert np.isnan(got[1]).all() and np.isnan(got[2, 199]) and not got[2, :199].any()
    _, scales = room.read()
    assert (scales[:, 1] == 255).all() and (scales[:6, 2] == 0).all() and scales[6, 2] == 255 and not scales[:, 3].any()


@pytest.mark.parametrize("size,types", [(s, t) for s in ((260, 4000), (300, 5999), (515, 8192), (513, 2041)) for t in PAIRS], ids=str)
def test_backward_of_rows_that_fill_a_workgroup(size, types):
    test_backward(size, types)


def test_no_rows_have_no_gradient():
    w = torch.ones(50, device="cuda")
    gw = torch.full((50,), 7.0, device="cuda")
    e = torch.empty((0, 50), device="cuda")
    hb.hidet_rms_norm_backward(e, e, torch.empty(0, device="cuda"), w, e, gw, None)
    assert bool((gw == 0).all())
