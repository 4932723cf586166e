"""Norms, block-scaled matrices and products run together, as a layer and a training step run them: on streams, captured, at the ends of memory."""
import threading

import numpy as np
import pytest
import torch

from mx_helpers import TYPES, f64, matrix, on_gpu, rng
from oracle import mx
from paper_2210_09603_amd import binding as hb

pytestmark = pytest.mark.gpu


def _product(a, b, dtype, **kw):
    c = torch.empty((a.shape[0], b.shape[0]), dtype=dtype, device="cuda")
    ws = torch.empty(max(4, hb.hidet_mx_gemm_workspace_bytes(a, b)), dtype=torch.uint8, device="cuda")
    hb.hidet_mx_gemm(a, b, c, workspace=ws, **kw)
    return c


def _read(m):
    """(element codes, scale codes) of a matrix in blocks."""
    v, s = (x.cpu().numpy() for x in m.tensors)
    return mx.unpack(v, m.format), s


def _numbers(m):
    return mx.numbers(*_read(m), m.format)


@pytest.mark.parametrize("rows", [1, 5, 40, 130])
def test_a_layer(rows):
    """x, residual -> norm into 8 bits -> product with 4-bit weights, the stream added to its output.  The product's bound is that of its test: for 8-bit
    operands 2^-12 of the largest of 8 products each, here below 8 * 2^-12 sum |a b| / 8, and 2^-24 for each addition."""
    g = rng(rows, 11)
    n, k = 96, 300
    x, r = on_gpu(g.standard_normal((rows, k)), "bf16"), on_gpu(g.standard_normal((rows, k)), "bf16")
    w = on_gpu(0.1 * g.standard_normal(k) + 1, "bf16")
    weights = on_gpu(g.standard_normal((n, k)) * k ** -0.5, "bf16")
    b, q = hb.make_mx(n, k, hb.HIDET_MX_E2M1, device="cuda"), hb.make_mx(rows, k, hb.HIDET_MX_E4M3, device="cuda")
    hb.hidet_mx_quantize(weights, by_rows=b)
    stream = torch.empty_like(x)
    hb.hidet_rms_norm(x, w, quantized=q, residual=r, sum=stream, eps=1e-5)
    out = torch.full((rows, n), 0.5, dtype=torch.bfloat16, device="cuda")
    hb.hidet_mx_gemm(q, b, out, epilogue=hb.make_epilogue(residual=out))  # (C is its own residual)
    h = f64(stream)
    assert np.array_equal(h, f64((x.float() + r.float()).bfloat16()))
    y, _ = mx.rms_norm(h, f64(w), 1e-5, 0.0)
    codes, scales = mx.quantize(f64(weights), mx.E2M1)
    assert np.array_equal(_read(b)[0], codes) and np.array_equal(_read(b)[1], scales)
    # elements on a border may fall to either side: the product is that of what the norm wrote, and what it wrote is near y
    a = _numbers(q)
    _, scale = _read(q)
    assert (np.abs(a[:, :k] - y) <= np.maximum(np.abs(y) / 16, np.repeat(np.ldexp(1.0, scale.T.astype(int) - 127), 32, axis=1)[:, :k] * 2.0 ** -9)
            * (1 + 2.0 ** -20) + (np.abs(y) >= 448 * np.repeat(np.ldexp(1.0, scale.T.astype(int) - 127), 32, axis=1)[:, :k]) * np.abs(y) / 8).all()
    nb = mx.numbers(codes, scales, mx.E2M1)
    want, size = a @ nb.T + 0.5, np.abs(a) @ np.abs(nb).T
    assert (np.abs(f64(out) - want) <= 2.0 ** -8 * np.abs(want) * 1.01 + (8 * 2.0 ** -12 + 40 * 2.0 ** -24) * size).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_training_step(dtype):
    """y = x w^T and both gradients from operands quantised along both axes, against float64 products of the same blocks."""
    g = rng(3)
    m, n, k = 70, 130, 200
    x, w, gy = on_gpu(g.standard_normal((m, k)), dtype), on_gpu(g.standard_normal((n, k)) * 0.1, dtype), on_gpu(g.standard_normal((m, n)) * 0.01, dtype)
    sides = {}
    for name, t, fmt in (("x", x, mx.E4M3), ("w", w, mx.E2M1), ("g", gy, mx.E5M2)):
        by_rows, by_columns = hb.make_mx(*t.shape, fmt, device="cuda"), hb.make_mx(t.shape[1], t.shape[0], fmt, device="cuda")
        hb.hidet_mx_quantize(t, by_rows=by_rows, by_columns=by_columns)
        for side, q, v in (("r", by_rows, f64(t)), ("c", by_columns, f64(t).T)):
            codes, scales = mx.quantize(v, fmt)
            assert np.array_equal(_read(q)[0], codes) and np.array_equal(_read(q)[1], scales)
            sides[name + side] = (q, mx.numbers(codes, scales, fmt))
    for a, b in (("xr", "wr"), ("gr", "wc"), ("gc", "xc")):
        c = _product(sides[a][0], sides[b][0], torch.float32)
        na, nb = sides[a][1], sides[b][1]
        want, size = na @ nb.T, np.abs(na) @ np.abs(nb).T
        assert (np.abs(f64(c) - want) <= (8 * 2.0 ** -12 + 40 * 2.0 ** -24) * size).all()


def _exact_operands(g, m, n, k, fa, fb):
    table = {mx.E4M3: [0, 0x38, 0x40], mx.E5M2: [0, 0x3C, 0x40], mx.E2M1: [0, 2, 4]}

    def one(rows, fmt):
        codes = np.array(table[fmt], dtype=np.uint8)[g.integers(0, 3, (rows, mx.blocks(k) * 32))]
        codes[:, k:] = 0
        return codes, g.integers(126, 129, (mx.blocks(k), rows)).astype(np.uint8)

    a, b = one(m, fa), one(n, fb)
    return a, b, mx.numbers(*a, fa) @ mx.numbers(*b, fb).T


@pytest.mark.parametrize("size", [(3, 40, 20000), (70, 66, 9000), (300, 200, 500)], ids=str)
def test_any_workspace_gives_the_sum(size):
    m, n, k = size
    a, b, want = _exact_operands(rng(*size), m, n, k, mx.E4M3, mx.E2M1)
    ma, mb = matrix(*a, k, mx.E4M3), matrix(*b, k, mx.E2M1)
    most = hb.hidet_mx_gemm_workspace_bytes(ma, mb)
    assert (most > 0) == (k > 1000)
    for size_of in (None, 0, 4 * m * n, 2 * 4 * m * n, 3 * 4 * m * n + 5, most):
        ws = None if size_of is None else torch.full((size_of + 64,), 0xFF, dtype=torch.uint8, device="cuda")
        c = torch.full((m, n), 7.0, device="cuda")
        hb.hidet_mx_gemm(ma, mb, c, workspace=None if ws is None else ws[:size_of])
        assert np.array_equal(f64(c), want)
        assert ws is None or bool((ws[size_of:] == 0xFF).all())
        first = c.clone()
        hb.hidet_mx_gemm(ma, mb, c, workspace=None if ws is None else ws[:size_of])
        assert bool((first == c).all())


def test_captured_and_replayed_with_new_inputs():
    g = rng(5)
    m, n, k = 20, 64, 12000  # (a product in slices)
    x, r, w = (on_gpu(g.standard_normal(s), "bf16") for s in ((m, k), (m, k), (k,)))
    weights = on_gpu(g.standard_normal((n, k)), "bf16")
    q, b = hb.make_mx(m, k, hb.HIDET_MX_E4M3, device="cuda"), hb.make_mx(n, k, hb.HIDET_MX_E4M3, device="cuda")
    s, c, rstd, y = torch.empty_like(x), torch.empty((m, n), device="cuda"), torch.empty(m, device="cuda"), torch.empty_like(x)
    gh, gw = torch.empty_like(x), torch.empty_like(w)
    ws = torch.empty(hb.hidet_mx_gemm_workspace_bytes(q, b), dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0
    ws2 = torch.empty(hb.hidet_rms_norm_backward_workspace_bytes(m, k), dtype=torch.uint8, device="cuda")

    def run():
        hb.hidet_rms_norm(x, w, y=y, residual=r, sum=s, quantized=q, rstd=rstd)
        hb.hidet_mx_quantize(weights, by_rows=b)
        hb.hidet_mx_gemm(q, b, c, workspace=ws)
        hb.hidet_rms_norm_backward(y, s, rstd, w, gh, gw, ws2, grad_sum=r)
        return [t.clone() for t in (s, y, c, gh, gw, rstd) + q.tensors]

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hb.hidet_rms_norm(x, w, y=y, residual=r, sum=s, quantized=q, rstd=rstd)
        hb.hidet_mx_quantize(weights, by_rows=b)
        hb.hidet_mx_gemm(q, b, c, workspace=ws)
        hb.hidet_rms_norm_backward(y, s, rstd, w, gh, gw, ws2, grad_sum=r)
    for i in range(4):
        x.copy_(on_gpu(g.standard_normal((m, k)), "bf16"))
        weights.copy_(on_gpu(g.standard_normal((n, k)), "bf16"))
        want = run()
        for t in (s, y, c, gh, gw, rstd) + q.tensors:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b2 in zip(want, (s, y, c, gh, gw, rstd) + q.tensors):
            assert torch.equal(a, b2)


def test_two_threads_on_two_streams():
    results, errors = {}, []

    def work(i):
        try:
            g = rng(i, 21)
            m, n, k = (4, 500, 4000) if i else (150, 200, 700)
            a, b, want = _exact_operands(g, m, n, k, mx.E4M3, mx.E2M1)
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                ma, mb = matrix(*a, k, mx.E4M3), matrix(*b, k, mx.E2M1)
                x = on_gpu(g.standard_normal((m, k)), "bf16")
                w = torch.ones(k, dtype=torch.bfloat16, device="cuda")
                outs = []
                for _ in range(20):
                    c, y = torch.zeros((m, n), device="cuda"), torch.empty_like(x)
                    ws = torch.empty(max(4, hb.hidet_mx_gemm_workspace_bytes(ma, mb)), dtype=torch.uint8, device="cuda")
                    hb.hidet_mx_gemm(ma, mb, c, workspace=ws)
                    hb.hidet_rms_norm(x, w, y=y)
                    outs.append((c, y))
                stream.synchronize()
                assert all(np.array_equal(f64(c), want) for c, _ in outs) and all(torch.equal(outs[0][1], y) for _, y in outs)
                results[i] = True
        except Exception as e:  # (of the thread)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not errors and len(results) == 2


def test_on_a_stream_that_is_given():
    g = rng(6)
    x = on_gpu(g.standard_normal((300, 1000)), "f16")
    q, y = hb.make_mx(300, 1000, hb.HIDET_MX_E4M3, device="cuda"), torch.zeros_like(x)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    hb.hidet_mx_quantize(x, by_rows=q, stream=stream)
    hb.hidet_mx_dequantize(q, y, stream=stream)
    stream.synchronize()
    want = mx.numbers(*mx.quantize(f64(x), mx.E4M3), mx.E4M3)[:, :1000]
    assert np.array_equal(f64(y), want)


@pytest.mark.parametrize("m", [10, 40, 600])
def test_rows_and_blocks_far_apart(m):
    """Distances that take rows of values past 2^32 bytes, and blocks of scales likewise."""
    n, k = 70, 352
    fa, fb = mx.E4M3, mx.E2M1
    a, b, want = _exact_operands(rng(m, 31), m, n, k, fa, fb)
    stride, apart = (1 << 23) - 16, (1 << 29) - 4
    values = torch.empty(m * stride, dtype=torch.uint8, device="cuda").as_strided((m, mx.blocks(k) * 32), (stride, 1))
    scales = torch.empty(mx.blocks(k) * apart, dtype=torch.uint8, device="cuda").as_strided((mx.blocks(k), m), (apart, 1))
    values.copy_(torch.from_numpy(a[0]))
    scales.copy_(torch.from_numpy(a[1]))
    far = hb.make_mx(m, k, fa, values, scales)
    c = _product(far, matrix(*b, k, fb), torch.float32)
    assert np.array_equal(f64(c), want)
    c = _product(matrix(*b, k, fb), far, torch.float32)
    assert np.array_equal(f64(c), want.T)
    # and as what conversions write and read
    x = torch.empty((m, k), device="cuda")
    hb.hidet_mx_dequantize(far, x)
    assert np.array_equal(f64(x), mx.numbers(*a, fa)[:, :k])
    values.zero_()
    scales.zero_()
    hb.hidet_mx_quantize(x, by_rows=far)
    codes, codes_of_scales = mx.quantize(f64(x), fa)
    assert np.array_equal(values.cpu().numpy(), codes) and np.array_equal(scales.cpu().numpy(), codes_of_scales)
    wide = torch.empty((m - 1) * (1 << 24) + k, dtype=torch.bfloat16, device="cuda").as_strided((m, k), (1 << 24, 1))
    wide.copy_(x)
    y = torch.empty((m, k), dtype=torch.bfloat16, device="cuda")
    hb.hidet_rms_norm(wide, torch.ones(k, dtype=torch.bfloat16, device="cuda"), y=y, quantized=far, eps=1e-5)
    near = hb.make_mx(m, k, fa, device="cuda")
    y2 = torch.empty_like(y)
    hb.hidet_rms_norm(wide.contiguous(), torch.ones(k, dtype=torch.bfloat16, device="cuda"), y=y2, quantized=near, eps=1e-5)
    assert torch.equal(y, y2) and torch.equal(values, near.tensors[0]) and torch.equal(scales, near.tensors[1])


def test_rows_of_a_larger_matrix():
    """Parts that begin at a multiple of 4 rows are matrices of their own: what lies behind them stays."""
    g = rng(8)
    whole = hb.make_mx(16, 100, hb.HIDET_MX_E4M3, device="cuda")
    values, scales = whole.tensors
    values.fill_(0x55)
    scales.fill_(0x55)
    x = on_gpu(g.standard_normal((5, 100)), "bf16")
    part = hb.make_mx(5, 100, hb.HIDET_MX_E4M3, values[4:9], scales[:, 4:9])
    for call in (lambda: hb.hidet_mx_quantize(x, by_rows=part),
                 lambda: hb.hidet_rms_norm(x, torch.ones(100, dtype=torch.bfloat16, device="cuda"), quantized=part)):
        call()
        for t, axis in ((values, 0), (scales, 1)):
            rest = torch.cat((t.narrow(axis, 0, 4), t.narrow(axis, 9, 7)), axis)
            assert bool((rest == 0x55).all())
            assert not bool((t.narrow(axis, 4, 5) == 0x55).all())
