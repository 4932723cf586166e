"""Norms and their gradients at the sizes that the kernels of large calls serve: past the caches, and long rows of which a workgroup
takes several, against float64.

Bounds.  y: half a step of its type and 2^-24 for each of five roundings.  Blocks: what y (1 - d) or y (1 + d) gives, d = 2^-21.
grad_h: half a step; 8 roundings of fp32 of its own terms; the mean's terms have 4 roundings each and are added one after the
other up to 128 times in a lane, 6 times over lanes and 16 times over wavefronts, and the product with them has 4 more: 160.
grad_weight: 8 roundings of a term, one addition for each row of a lane (fewer than rows / 256 + 1), 16 over the rows of a workgroup, 32 and 16 over workgroups: rows / 256 + 80."""
import numpy as np
import pytest
import torch

import norm_reference
from mx_helpers import FLOOR, FORMATS, TYPES, U, Room, f64
from oracle import mx
from paper_2210_09603_amd import binding as hb

pytestmark = pytest.mark.gpu

ES = {"f32": 4, "f16": 2, "bf16": 2}
FAR = 256 << 20  # bytes of rows that a call reads and writes: more pass the caches by
PIECE = 1 << 22  # elements of float64 at a time


def _view(rows, cols, dtype, g, size, before, after):
    """Normally distributed numbers times sizes of rows, as a view whose rows lie apart."""
    wide = torch.full((rows, before + cols + after), 7.0, dtype=TYPES[dtype], device="cuda")
    view = wide[:, before:before + cols]
    if size is not None:
        view.copy_(torch.randn((rows, cols), generator=g, device="cuda") * torch.exp2(torch.randint(-size, size + 1, (rows, 1), generator=g, device="cuda").float()))
    return wide, view


def _pieces(rows, cols):
    step = max(1, PIECE // cols)
    return [slice(r, min(r + step, rows)) for r in range(0, rows, step)]


def _kept(wide, before, after):
    assert bool((wide[:, :before] == 7).all()) and bool((wide[:, wide.shape[1] - after:] == 7).all())


def _check_y(y, h, w, eps, offset, dtype, rstd=None):
    for p in _pieces(*h.shape):
        want, r = norm_reference.norm(h[p], w, eps, offset)
        assert bool(((y[p].double() - want).abs() <= want.abs() * (U[dtype] + 5 * 2.0 ** -24) + FLOOR[dtype]).all())
        if rstd is not None:
            assert bool(((rstd[p].double() - r).abs() <= 2.0 ** -23 * r).all())


def _check_blocks(room, h, w, eps, offset):
    """At rows of both ends and between."""
    rows = h.shape[0]
    some = np.unique(np.r_[0:18, rows // 2:rows // 2 + 9, rows - 18:rows, np.arange(0, rows, max(1, rows // 40))])
    want = f64(norm_reference.norm(h[torch.from_numpy(some).cuda()], w, eps, offset)[0])
    codes, scales = room.read()
    codes, scales = codes[some], scales[:, some]
    low, high = (mx.quantize(want * f, room.fmt) for f in (1 - 2.0 ** -21, 1 + 2.0 ** -21))
    assert ((scales == low[1]) | (scales == high[1])).all()
    one, two = (mx.quantize(want * f, room.fmt, scales)[0] for f in (1 - 2.0 ** -21, 1 + 2.0 ** -21))
    assert ((codes == one) | (codes == two)).all()


HALF = [("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f32")]
# a column count for every number of lanes and chunks a row is cut into
FORWARD = [(c, HALF[(i + j) % 4], i + j) for i, c in enumerate((100, 501, 1003, 1500, 2040, 2999, 4090, 6001, 8190, 12007, 16380, 30011)) for j in (0, 1)] + [
    (c, ("f32", "f32"), i) for i, c in enumerate((60, 251, 500, 751, 1003, 1500, 2040, 2999, 4090, 6001, 8190, 16379, 30011))]


@pytest.mark.parametrize("cols,types,turn", FORWARD, ids=str)
def test_norm_past_the_caches(cols, types, turn):
    dtype, wtype = types
    rows = FAR // (2 * ES[dtype] * cols) + 7
    g = torch.Generator(device="cuda").manual_seed(cols + turn)
    before, after = turn % 2, 2 - turn % 2
    widex, x = _view(rows, cols, dtype, g, 3, before, after)
    _, r = _view(rows, cols, dtype, g, 2, before, after + 1)
    w = (0.3 * torch.randn(cols, generator=g, device="cuda") + 1).to(TYPES[wtype])
    widey, y = _view(rows, cols, dtype, g, None, 1, 1)
    wides, s = _view(rows, cols, dtype, g, None, 0, 3)
    rstd = torch.full((rows + 1,), 7.0, device="cuda")
    offset, eps = float(turn % 2), 1e-5
    hb.hidet_rms_norm(x, w, y=y, rstd=rstd[:rows], eps=eps, offset=offset)
    _check_y(y, x, w, eps, offset, dtype, rstd)
    assert float(rstd[rows]) == 7.0
    h = (x.float() + r.float()).to(TYPES[dtype])
    room = Room(rows, cols, FORMATS[turn % 3])
    hb.hidet_rms_norm(x, w, y=y, residual=r, sum=s, quantized=room.m, eps=eps, offset=offset)
    assert torch.equal(s, h)
    _check_y(y, h, w, eps, offset, dtype)
    _check_blocks(room, h, w, eps, offset)
    _kept(widey, 1, 1)
    _kept(wides, 0, 3)
    # blocks alone, the stream in place of the residual; y in place of x
    room = Room(rows, cols, FORMATS[(turn + 1) % 3], wide=False)
    hb.hidet_rms_norm(x, w, residual=r, sum=r, quantized=room.m, eps=eps, offset=offset)
    assert torch.equal(r, h)
    _check_blocks(room, h, w, eps, offset)
    h = (x.float() + s.float()).to(TYPES[dtype])
    hb.hidet_rms_norm(x, w, y=x, residual=s, eps=eps, offset=offset)
    _check_y(x, h, w, eps, offset, dtype)
    _kept(widex, before, after)


def _check_backward(rows, cols, types, before, after):
    dtype, wtype = types
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    _, h = _view(rows, cols, dtype, g, 3, before, after)
    widey, gy = _view(rows, cols, dtype, g, 0, before, after + 1)
    wides, gs = _view(rows, cols, dtype, g, 0, before, after + 2)
    wideh, gh = _view(rows, cols, dtype, g, None, 1, 1)
    w = (0.3 * torch.randn(cols, generator=g, device="cuda")).to(TYPES[wtype])
    offset = float(rows % 2)
    rstd = torch.cat([norm_reference.norm(h[p], w, 1e-5, offset)[1] for p in _pieces(rows, cols)]).float()
    ws = torch.full((hb.hidet_rms_norm_backward_workspace_bytes(rows, cols),), 0xFF, dtype=torch.uint8, device="cuda")
    gw = torch.full((cols + 1,), 7.0, dtype=TYPES[wtype], device="cuda")

    def check(got, stream):
        total = size = 0.0
        for p in _pieces(rows, cols):
            want, near, far, part, part_size = norm_reference.gradients(gy0[p], h[p], rstd[p], w, offset)
            total, size = total + part, size + part_size
            if stream is not None:
                s = stream[p].double()
                want, near = want + s, near + s.abs()
            bound = U[dtype] * want.abs() + 2.0 ** -24 * (8 * near + 160 * far) + FLOOR[dtype]
            assert bool(((got[p].double() - want).abs() <= bound).all())
        bound = U[wtype] * total.abs() + (8 + -(-rows // 256) + 80) * 2.0 ** -24 * size + FLOOR[wtype]
        assert bool(((gw[:cols].double() - total).abs() <= bound).all()) and float(gw[cols]) == 7.0

    gy0 = gy.clone()
    hb.hidet_rms_norm_backward(gy, h, rstd, w, gh, gw[:cols], ws, offset=offset)
    check(gh, None)
    alone, first = gh.clone(), gw.clone()
    hb.hidet_rms_norm_backward(gy, h, rstd, w, gh, gw[:cols], ws, grad_sum=gs, offset=offset)
    check(gh, gs)
    assert torch.equal(first, gw)
    _kept(wideh, 1, 1)
    # in place of the stream's, without the weight's; in place of grad_y, the same bits as apart
    hb.hidet_rms_norm_backward(gy, h, rstd, w, gs, None, None, grad_sum=gs, offset=offset)
    assert torch.equal(gs, gh)
    _kept(wides, before, after + 2)
    ws.fill_(0xFF)
    hb.hidet_rms_norm_backward(gy, h, rstd, w, gy, gw[:cols], ws, offset=offset)
    assert torch.equal(gy, alone) and torch.equal(first, gw)
    _kept(widey, before, after + 1)


BACKWARD = [(c, HALF[(i + j) % 4]) for i, c in enumerate((100, 501, 1003, 2040, 4090, 6001, 8190, 12007, 16380, 30011)) for j in (0, 1)] + [
    (c, ("f32", "f32")) for c in (60, 251, 500, 1003, 2040, 2999, 4090, 6001, 8190, 16379, 30011)]


@pytest.mark.parametrize("cols,types", BACKWARD, ids=str)
def test_backward_past_the_caches(cols, types):
    _check_backward(FAR // (3 * ES[types[0]] * cols) + 7, cols, types, cols % 2, 1)


@pytest.mark.parametrize("size,types", [(s, t) for s in ((515, 20001), (515, 32768), (771, 16390)) for t in HALF] + [
    (s, ("f32", "f32")) for s in ((515, 12003), (515, 16384), (300, 32768), (771, 20001), (515, 8200))], ids=str)
def test_backward_of_several_long_rows_a_workgroup(size, types):
    _check_backward(*size, types, 0, 0)
    _check_backward(*size, types, 1, 2)
