"""Refusals of the norms and the block-scaled matrices, before anything is launched: all device addresses are made up."""
import ctypes
import math

import pytest
import torch

from paper_2210_09603_amd import binding as hb

OK, INVALID, UNSUPPORTED, ALIGN = 0, 1, 2, 3


def blocks(**kw):
    m = hb.hidet_mx_t()
    m.struct_size = ctypes.sizeof(m)
    m.format, m.values, m.scales, m.stride_values, m.stride_scales = hb.HIDET_MX_E4M3, 0x1000, 0x2000, 128, 64
    for n, v in kw.items():
        setattr(m, n, v)
    return m


def quantize(**kw):
    a = dict(dtype=hb.HIDET_F16, rows=40, cols=100, x=0x10000, ldx=100, by_rows=blocks(), by_columns=None)
    a.update(kw)
    return hb.lib().hidet_mx_quantize(a["dtype"], a["rows"], a["cols"], a["x"], a["ldx"], a["by_rows"], a["by_columns"], None)


def dequantize(**kw):
    a = dict(dtype=hb.HIDET_F16, rows=40, cols=100, x=0x10000, ldx=100, by_rows=blocks())
    a.update(kw)
    return hb.lib().hidet_mx_dequantize(a["rows"], a["cols"], a["by_rows"], a["dtype"], a["x"], a["ldx"], None)


def gemm(**kw):
    a = dict(out=hb.HIDET_F16, M=40, N=50, K=100, A=blocks(), B=blocks(), C=0x10000, ldc=50, e=None, ws=None, wb=0)
    a.update(kw)
    return hb.lib().hidet_mx_gemm(a["out"], a["M"], a["N"], a["K"], a["A"], a["B"], a["C"], a["ldc"], a["e"], a["ws"], a["wb"], None)


def norm(**kw):
    a = dict(dtype=hb.HIDET_F16, wtype=hb.HIDET_F32, rows=40, cols=100, x=0x10000, ldx=100, r=0x20000, ldr=100, w=0x1000, eps=1e-5, offset=0.0,
             s=0x30000, lds=100, y=0x40000, ldy=100, q=blocks(), rstd=0x2000)
    a.update(kw)
    return hb.lib().hidet_rms_norm(a["dtype"], a["wtype"], a["rows"], a["cols"], a["x"], a["ldx"], a["r"], a["ldr"], a["w"], a["eps"], a["offset"],
                                   a["s"], a["lds"], a["y"], a["ldy"], a["q"], a["rstd"], None)


def backward(**kw):
    a = dict(dtype=hb.HIDET_F16, wtype=hb.HIDET_F32, rows=40, cols=100, x=0x10000, ldx=100, h=0x20000, ldh=100, rstd=0x2000, w=0x1000, offset=0.0,
             s=0x30000, lds=100, y=0x40000, ldy=100, gw=0x3000, ws=0x50000, wb=1 << 20)
    a.update(kw)
    return hb.lib().hidet_rms_norm_backward(a["dtype"], a["wtype"], a["rows"], a["cols"], a["x"], a["ldx"], a["h"], a["ldh"], a["rstd"], a["w"],
                                            a["offset"], a["s"], a["lds"], a["y"], a["ldy"], a["gw"], a["ws"], a["wb"], None)


@pytest.mark.parametrize("call", [quantize, dequantize, norm, backward])
def test_rows(call):
    assert call(dtype=3) == INVALID and call(dtype=-1) == INVALID and call(rows=-1) == INVALID and call(cols=-1) == INVALID
    assert call(rows=1 << 29) == UNSUPPORTED and call(cols=1 << 29) == UNSUPPORTED
    assert call(x=None) == INVALID and call(ldx=99) == INVALID and call(x=0x10001) == ALIGN
    assert call(ldx=1 << 43) == UNSUPPORTED


@pytest.mark.parametrize("call", [quantize, dequantize, norm])
def test_blocks(call):
    q = "q" if call is norm else "by_rows"
    for bad, status in ((dict(struct_size=8), INVALID), (dict(format=3), INVALID), (dict(format=-1), INVALID), (dict(values=None), INVALID),
                        (dict(scales=None), INVALID), (dict(values=0x1008), ALIGN), (dict(scales=0x2002), ALIGN), (dict(stride_values=136), ALIGN),
                        (dict(stride_scales=66), ALIGN), (dict(stride_values=112), INVALID), (dict(stride_scales=36), INVALID),
                        (dict(stride_values=-128), INVALID), (dict(stride_values=1 << 23), UNSUPPORTED), (dict(stride_scales=1 << 29), UNSUPPORTED)):
        assert call(**{q: blocks(**bad)}) == status, bad


def test_quantize_needs_a_destination():
    assert quantize(by_rows=None) == INVALID
    assert quantize(by_rows=None, by_columns=blocks(stride_values=48, stride_scales=100)) == INVALID  # (a row of 64 bytes)
    assert quantize(by_rows=None, by_columns=blocks(stride_values=64, stride_scales=96)) == INVALID
    assert dequantize(by_rows=None) == INVALID
    assert quantize(rows=0) == OK and quantize(cols=0) == OK and dequantize(rows=0, x=None) == OK


def test_quantize_needs_two_destinations_for_two():
    one = blocks(stride_values=1 << 10, stride_scales=1 << 10)
    assert quantize(by_rows=one, by_columns=one) == INVALID
    assert quantize(by_rows=one, by_columns=blocks(values=0x8000, stride_scales=1 << 10)) == INVALID
    assert quantize(by_rows=one, by_columns=blocks(scales=0x8000, stride_scales=1 << 10)) == INVALID


def test_more_tiles_than_a_launch_has():
    # 2^29 - 32 rows: a launch has fewer than 2^32 threads (nothing is launched)
    rows = (1 << 29) - 32
    wide = blocks(stride_values=32, stride_scales=rows)
    assert quantize(rows=rows, cols=32, by_rows=wide) == UNSUPPORTED and dequantize(rows=rows, cols=32, by_rows=wide) == UNSUPPORTED
    assert norm(rows=rows, cols=1024, ldx=1024, ldr=1024, lds=1024, ldy=1024, q=None) == UNSUPPORTED
    assert gemm(M=16, N=rows, K=32, A=wide, B=wide, ldc=rows) == UNSUPPORTED


def test_more_tiles_along_columns_than_a_launch_has():
    # 512 threads to a tile of 128 x 128: 2^23 tiles are 2^32 threads (nothing is launched)
    long = (1 << 29) - 32
    one = blocks(stride_values=160, stride_scales=long)
    assert quantize(rows=129, cols=long, ldx=long, by_rows=None, by_columns=one) == UNSUPPORTED
    rows, cols = 1 << 19, 1 << 18
    by_rows = blocks(format=hb.HIDET_MX_E2M1, stride_values=cols // 2, stride_scales=rows)
    by_columns = blocks(format=hb.HIDET_MX_E2M1, values=0x8000, scales=0x9000, stride_values=rows // 2, stride_scales=cols)
    assert quantize(rows=rows, cols=cols, ldx=cols, by_rows=by_rows, by_columns=by_columns) == UNSUPPORTED
    assert quantize(rows=rows, cols=cols, ldx=cols, by_rows=None, by_columns=by_columns) == UNSUPPORTED


def test_gemm():
    assert gemm(out=3) == INVALID and gemm(M=-1) == INVALID and gemm(K=-1) == INVALID and gemm(wb=-1) == INVALID
    for n in ("M", "N", "K"):
        assert gemm(**{n: 1 << 29}) == UNSUPPORTED
    assert gemm(A=None) == INVALID and gemm(B=blocks(format=7)) == INVALID and gemm(A=blocks(values=0x1008)) == ALIGN
    assert gemm(K=200) == INVALID  # (rows of 224 bytes)
    assert gemm(C=None) == INVALID and gemm(ldc=49) == INVALID and gemm(C=0x10001) == ALIGN and gemm(ldc=1 << 32) == UNSUPPORTED
    assert gemm(ws=0x1008, wb=1 << 20) == ALIGN
    assert gemm(M=0) == OK and gemm(N=0) == OK


def test_gemm_epilogue():
    def e(**kw):
        d = hb.hidet_epilogue_t()
        d.struct_size, d.alpha = ctypes.sizeof(d), 1.0
        for n, v in kw.items():
            setattr(d, n, v)
        return d

    assert gemm(e=e(struct_size=4)) == INVALID and gemm(e=e(alpha=math.nan)) == INVALID and gemm(e=e(bias_axis=3)) == INVALID
    assert gemm(e=e(bias_axis=1)) == INVALID and gemm(e=e(bias_axis=1, bias=0x1001)) == ALIGN and gemm(e=e(act=2)) == INVALID
    assert gemm(e=e(out_map=1, map_seq=40, map_head_dim=50)) == UNSUPPORTED and gemm(e=e(prologue=1)) == UNSUPPORTED
    assert gemm(e=e(residual=0x20000, ld_residual=49)) == INVALID and gemm(e=e(residual=0x20001, ld_residual=50)) == ALIGN
    assert gemm(e=e(residual=0x20000, ld_residual=1 << 32)) == UNSUPPORTED
    assert gemm(e=e(residual=0x10000, ld_residual=52)) == INVALID  # (C itself with another distance)


def test_norm():
    assert norm(wtype=hb.HIDET_BF16) == UNSUPPORTED and norm(wtype=5) == INVALID and norm(cols=32769) == UNSUPPORTED
    assert norm(eps=-1.0) == INVALID and norm(eps=math.nan) == INVALID and norm(eps=math.inf) == INVALID and norm(offset=math.nan) == INVALID
    assert norm(w=None) == INVALID and norm(w=0x1002) == ALIGN and norm(rstd=0x2002) == ALIGN and norm(y=None, q=None) == INVALID
    for p, ld in (("r", "ldr"), ("s", "lds"), ("y", "ldy")):
        assert norm(**{ld: 99}) == INVALID and norm(**{p: 0x60001}) == ALIGN
    assert norm(s=0x10000, lds=104) == INVALID and norm(y=0x20000, ldy=104) == INVALID and norm(s=0x40000) == INVALID
    assert norm(rows=0) == OK and norm(cols=0) == OK


def test_backward():
    assert backward(wtype=hb.HIDET_BF16) == UNSUPPORTED and backward(cols=32769) == UNSUPPORTED and backward(offset=math.inf) == INVALID
    for n in ("h", "rstd", "w", "y", "ws"):
        assert backward(**{n: None}) == INVALID, n
    assert backward(gw=0x3002) == ALIGN and backward(ws=0x50008) == ALIGN and backward(rstd=0x2001) == ALIGN
    assert backward(ldh=99) == INVALID and backward(lds=99) == INVALID and backward(ldy=99) == INVALID
    assert backward(y=0x20000) == INVALID and backward(y=0x10000, ldy=104) == INVALID
    n = hb.hidet_rms_norm_backward_workspace_bytes(40, 100)
    assert n > 0 and backward(wb=n - 1) == INVALID and backward(wb=-1) == INVALID
    assert hb.hidet_rms_norm_backward_workspace_bytes(0, 100) == 0 and hb.hidet_rms_norm_backward_workspace_bytes(4, 40000) == 0
    assert backward(cols=0) == OK and backward(rows=0, gw=None) == OK


def test_workspaces_are_whole_numbers_of_a_size():
    for m, n, k in ((0, 4, 4), (4, 4, 0), (1 << 29, 4, 4)):
        assert hb.lib().hidet_mx_gemm_workspace_bytes(m, n, k, 0, 0) == 0


def test_the_binding_refuses_what_does_not_fit():
    v, s = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(2, 4, dtype=torch.uint8)
    m = hb.make_mx(4, 50, hb.HIDET_MX_E4M3, v, s)
    assert m.tensors[0] is v and (m.stride_values, m.stride_scales) == (64, 4)
    for args in ((5, 50, 0, v, s), (4, 70, 0, v, s), (4, 50, 0, v, s[:1]), (4, 50, 0, v.float(), s), (4, 50, 0, v, None), (4, 50, 0, v.t(), s),
                 (4, 50, 0, v, torch.zeros(2, 3, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            hb.make_mx(*args)
    with pytest.raises(ValueError, match="up to a multiple of 4"):
        hb.make_mx(3, 50, 0, v[:3], torch.zeros(7, dtype=torch.uint8).as_strided((2, 3), (4, 1)))
    x = torch.zeros(4, 50)
    for call in (lambda: hb.hidet_mx_quantize(x, by_rows=hb.make_mx(4, 51, 0, device="cpu")), lambda: hb.hidet_mx_quantize(x, by_columns=m),
                 lambda: hb.hidet_mx_quantize(x, by_rows=m), lambda: hb.hidet_mx_dequantize(m, torch.zeros(4, 49)),
                 lambda: hb.hidet_mx_gemm(m, m, torch.zeros(4, 5)), lambda: hb.hidet_rms_norm(x, torch.ones(49), y=x),
                 lambda: hb.hidet_rms_norm(x, torch.ones(50), y=x[:3]), lambda: hb.hidet_rms_norm(x, torch.ones(50), y=x.half()),
                 lambda: hb.hidet_rms_norm(x, torch.ones(50), y=x)):  # (the last: not on the GPU)
        with pytest.raises(ValueError):
            call()
