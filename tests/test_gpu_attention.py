"""Fused attention and its backward pass against the float64 oracle: sizes, head layouts, masks, strides, values that must not matter,
splits, streams, graphs."""
import threading

import numpy as np
import pytest
import torch

from attention_helpers import TYPES, assert_within, bounds, f64
from oracle import attention as oa
from paper_2210_09603_amd import binding as hb

pytestmark = pytest.mark.gpu


def _draw(g, shape, dtype, layout):
    """A [batch, heads, rows, dim] tensor: dense, seen through [batch, rows, heads, dim], or a slice of a wider odd-sized buffer."""
    b, h, n, d = shape
    x = torch.from_numpy(g.standard_normal(shape).astype(np.float32)).to(TYPES[dtype]).cuda()
    if layout == "dense":
        return x
    if layout == "tokens":
        return x.transpose(1, 2).contiguous().transpose(1, 2)
    buf = torch.zeros(b * n * (h + 2) * (d + 3) + 5, dtype=TYPES[dtype], device="cuda")
    view = buf[5:5 + b * n * (h + 2) * (d + 3)].view(b, n, h + 2, d + 3)[:, :, 1:h + 1, 1:d + 1].transpose(1, 2)
    view.copy_(x)
    return view


def _surrounded(shape, dtype, layout):
    """A tensor to write to, in a buffer of sevens: (view, function that checks that nothing beside it changed)."""
    b, h, n, d = shape
    if layout == "odd":
        buf = torch.full((b * n * (h + 2) * (d + 3) + 5,), 7.0, dtype=TYPES[dtype], device="cuda")
        view = buf[5:].view(b, n, h + 2, d + 3)[:, :, 1:h + 1, 1:d + 1].transpose(1, 2)
    else:
        buf = torch.full((16 + b * h * n * d + 16,), 7.0, dtype=TYPES[dtype], device="cuda")
        view = buf[16:-16].view(b, h, n, d) if layout == "dense" else buf[16:-16].view(b, n, h, d).transpose(1, 2)

    def check(what):
        keep = view.clone()
        view.fill_(7.0)
        assert bool((buf == 7.0).all()), what + ": wrote beside its output"
        view.copy_(keep)

    return view, check


def _run(seed, dtype, b, h, hk, n, m, d, layout="dense", causal=False, window=0, softcap=0.0, slopes=False, ranges=None, scale=None,
         poison=None, split=False, back=True):
    g = np.random.Generator(np.random.PCG64(seed))
    q, k, v = _draw(g, (b, h, n, d), dtype, layout), _draw(g, (b, hk, m, d), dtype, layout), _draw(g, (b, hk, m, d), dtype, layout)
    dout = _draw(g, (b, h, n, d), dtype, layout)
    sl = torch.tensor([2.0 ** (-8.0 * (i + 1) / h) for i in range(h)], device="cuda") if slopes else None
    rg = None
    if ranges is not None:
        rg = torch.from_numpy(ranges.astype(np.int32)).cuda()
        see = np.stack([oa.in_ranges(r, m) for r in ranges])
    else:
        see = np.stack([oa.sees(n, m, causal, window)] * b)
    if poison is not None:
        poison(q, k, v, dout, see)
    out, check_out = _surrounded((b, h, n, d), dtype, layout)
    out.fill_(float("nan"))
    lse = torch.full((b, h, n), float("nan"), device="cuda")
    opts = dict(scale=scale, causal=causal, window=window, softcap=softcap, slopes=sl, ranges=rg)
    ws = None
    if split:
        size = hb.hidet_attention_workspace_bytes(q, k)
        assert size > 0, "this size is not split"
        ws = torch.full((size // 4,), float("nan"), device="cuda")
    hb.hidet_attention(q, k, v, out, lse=lse, workspace=ws, **opts)
    torch.cuda.synchronize()
    what = "%s %s" % (dtype, (b, h, hk, n, m, d))
    sc = d ** -0.5 if scale is None else scale
    args = (f64(q), f64(k), f64(v), see, sc, softcap, None if sl is None else f64(sl))
    if not back:
        want, bound = bounds(dtype, *args)
    else:
        grads = []
        for shape in ((b, h, n, d), (b, hk, m, d), (b, hk, m, d)):
            t, check = _surrounded(shape, dtype, layout)
            t.fill_(float("nan"))
            grads.append((t, check))
        size = hb.hidet_attention_backward_workspace_bytes(q, k)
        ws2 = torch.full((max(size, 4) // 4,), float("nan"), device="cuda")
        hb.hidet_attention_backward(dout, q, k, v, out, lse, *(t for t, _ in grads), ws2, **opts)
        torch.cuda.synchronize()
        want, bound = bounds(dtype, *args, grad_out=f64(dout))
        for name, (t, check), w, e in zip(("dq", "dk", "dv"), grads, want[2:], bound[2:]):
            assert_within(t, w, e, what + " " + name)
            check(what + " " + name)
    assert_within(out, want[0], bound[0], what + " out")
    assert_within(lse, want[1], bound[1], what + " lse")
    check_out(what)
    return out, lse


SIZES = [  # batch, heads, kv heads, queries, keys, dim
    (1, 1, 1, 1, 1, 64), (2, 3, 1, 1, 7, 64), (1, 2, 2, 2, 1, 8), (1, 2, 1, 31, 33, 40), (2, 4, 2, 65, 64, 64), (1, 4, 4, 64, 65, 72),
    (1, 2, 1, 127, 129, 128), (1, 7, 1, 50, 50, 128), (1, 3, 3, 200, 300, 96), (2, 2, 1, 300, 200, 64), (1, 1, 1, 129, 517, 120),
]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_full_and_causal(size, dtype):
    for i, causal in enumerate((False, True)):  # (fewer keys than queries: the first queries see nothing)
        _run(1000 + 10 * SIZES.index(size) + i, dtype, *size, causal=causal, layout=("dense", "tokens", "odd")[SIZES.index(size) % 3])


# (512 tiles of 128 rows: a wavefront for 32 rows, where fewer take two)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("size", [(128, 4, 4, 40, 150, 64), (86, 12, 6, 19, 193, 112)], ids=str)
def test_many_tiles(size, dtype):
    _run(22, dtype, *size)
    _run(22, dtype, *size, causal=True, window=40, softcap=10.0, slopes=True, layout="tokens")


def test_many_tiles_under_ranges_with_values_that_must_not_matter():
    g = np.random.Generator(np.random.PCG64(23))
    b, n, m = 128, 40, 150
    ranges = np.sort(g.integers(-20, m + 20, size=(b, n, 2)), axis=2)
    ranges[::3, ::5] = 7  # (empty)
    ranges[5] = 0

    def poison(q, k, v, dout, see):
        for i in range(b):
            hidden = torch.from_numpy(~see[i].any(0)).cuda()
            k[i][:, hidden] = float("nan")
            v[i][:, hidden] = float("inf")

    _run(23, "bf16", b, 4, 4, n, m, 64, ranges=ranges, poison=poison)


# (more blocks of 64 keys than begin at once: the longest first, 256 of an entry at a time)
@pytest.mark.parametrize("size", [(2, 4, 2, 90, 4500, 64), (1, 2, 1, 33, 17000, 128)], ids=str)
def test_ranges_over_many_blocks_of_keys(size):
    b, h, hk, n, m, d = size
    g = np.random.Generator(np.random.PCG64(24))
    lo = g.integers(-20, m, size=(b, n, 1))
    ranges = np.concatenate([lo, lo + g.integers(-5, m // 2, size=(b, n, 1))], axis=2)
    ranges[0, 3] = (0, m)
    ranges[-1, 32:64] = 0
    _run(24, "bf16", b, h, hk, n, m, d, ranges=ranges)


@pytest.mark.parametrize("window", [1, 2, 33, 64, 150, 1 << 40])
@pytest.mark.parametrize("causal", [False, True])
def test_window(window, causal):
    _run(2000 + window % 997, "bf16", 1, 4, 2, 90, 190, 64, causal=causal, window=window)
    _run(2100 + window % 997, "f16", 1, 2, 2, 190, 90, 128, causal=causal, window=window, layout="odd")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 24])
def test_cap_and_slopes(dtype, dim):
    for i, (softcap, slopes) in enumerate(((0.7, False), (30.0, False), (0.0, True), (5.0, True))):
        _run(3000 + 7 * i + dim, dtype, 1, 6, 2, 70, 100, dim, causal=i % 2 == 0, softcap=softcap, slopes=slopes)


@pytest.mark.parametrize("softcap", [2.0, 20.0, 50.0, 64.0, 65.0, 300.0, 1e4, 1e6, 1e12, 3e38])
@pytest.mark.parametrize("scale", [0.35, -0.35, 40.0])
def test_a_capped_score_is_as_good_as_an_uncapped_one(softcap, scale):
    """The log-sum of a query's only key is its score.  Off by at most: 16 * 2^-24 of the products' sum of absolute values (8 exact
    products, added in fp32, times scale), 16 * 2^-23 of itself (tanh, 4 * 2^-22 where the cap is no more than 4 of it, and steps of
    fp32 on the way), and up to a cap of 64 2^-22 of the cap (1.5e-5 at most, whatever the score)."""
    g = np.random.Generator(np.random.PCG64(61))
    n, d = 3000, 8
    q, k, v = (torch.from_numpy(g.standard_normal((1, 1, n, d)).astype(np.float32)).half().cuda() for _ in range(3))
    q.mul_(torch.from_numpy(np.exp2(g.integers(-8, 5, (1, 1, n, 1))).astype(np.float32)).cuda())
    out, lse = torch.empty_like(q), torch.empty(1, 1, n, device="cuda")
    hb.hidet_attention(q, k, v, out, lse=lse, scale=scale, softcap=softcap, window=1)
    products = f64(q)[0, 0] * f64(k)[0, 0]
    scale, softcap = float(np.float32(scale)), float(np.float32(softcap))
    x = softcap * np.tanh(scale * products.sum(1) / softcap)
    bound = 16 * 2.0 ** -24 * abs(scale) * np.abs(products).sum(1) + 16 * 2.0 ** -23 * np.abs(x) + (2.0 ** -22 * softcap if softcap <= 64 else 0.0)
    assert_within(f64(lse)[0, 0], x, bound, "cap %g scale %g" % (softcap, scale))
    assert torch.equal(out, v)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 24])
@pytest.mark.parametrize("softcap", [100.0, 1e4, 1e7, 1e30])
def test_large_caps(softcap, dim, dtype):
    _run(3500 + dim, dtype, 2, 6, 2, 140, 190, dim, softcap=softcap, causal=True)
    _run(3510 + dim, dtype, 1, 4, 4, 200, 260, dim, softcap=softcap, slopes=True, layout="tokens")
    _run(3520 + dim, dtype, 1, 8, 2, 3, 70, dim, softcap=softcap, scale=0.9)
    _run(3530 + dim, dtype, 1, 2, 1, 2, 9000, dim, softcap=softcap, split=True, back=False)


def test_scales_of_any_sign():
    for i, scale in enumerate((0.0, -0.2, 1.0)):
        _run(3100 + i, "f16", 1, 2, 1, 40, 70, 64, scale=scale)


def _random_ranges(g, b, n, m):
    lo, hi = g.integers(-5, m, (b, n)), g.integers(-5, m + 9, (b, n))
    r = np.stack([lo, hi], -1)
    r[:, ::7] = (0, m)
    r[:, 3::11] = (5, 5)
    return r


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("size", [(2, 4, 2, 70, 130, 64), (1, 3, 1, 150, 150, 128), (3, 1, 1, 33, 5, 16)], ids=str)
def test_ranges(size, dtype):
    g = np.random.Generator(np.random.PCG64(size[3]))
    r = _random_ranges(g, size[0], size[3], size[4])
    _run(4000 + size[3], dtype, *size, ranges=r, slopes=True)
    r[:] = 0  # nobody sees anything
    out, lse = _run(4100 + size[3], dtype, *size, ranges=r)
    assert bool((out == 0).all()) and bool((lse == -np.inf).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [40, 128])
@pytest.mark.parametrize("softcap", [0.0, 3.0])
def test_the_only_key_of_a_query_has_no_gradient_of_its_score(dtype, dim, softcap):
    """Windows of one key, sequences and documents of one token, one key in a longer range: dQ and dK are zeros, not roundings."""
    g = np.random.Generator(np.random.PCG64(25))
    for b, h, hk, n, m, window in ((2, 4, 2, 70, 70, 1), (1, 2, 2, 1, 1, 0), (2, 3, 1, 9, 1, 0), (1, 2, 1, 600, 600, 0)):
        q, dout, out = (_draw(g, (b, h, n, dim), dtype, "dense") for _ in range(3))
        k, v = (_draw(g, (b, hk, m, dim), dtype, "dense") for _ in range(2))
        ranges = None
        if n == 600:
            at = torch.arange(n, dtype=torch.int32)
            ranges = torch.stack([(at * 7) % m, (at * 7) % m + 1], dim=1)[None].contiguous().cuda()
        opts = dict(window=window, softcap=softcap, ranges=ranges)
        lse = torch.empty(b, h, n, device="cuda")
        hb.hidet_attention(q, k, v, out, lse=lse, **opts)
        dq, dk, dv = (torch.full_like(t, 3.0) for t in (q, k, v))
        ws = torch.empty(hb.hidet_attention_backward_workspace_bytes(q, k) // 4, device="cuda")
        hb.hidet_attention_backward(dout, q, k, v, out, lse, dq, dk, dv, ws, **opts)
        assert not dq.any() and not dk.any(), (b, h, hk, n, m)
        assert bool((dv != 3.0).any())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim,h,hk,softcap", [(64, 4, 2, 0.0), (128, 2, 1, 0.0), (40, 3, 3, 20.0)])
def test_gradients_of_few_keys_do_not_carry_the_rounding_of_the_output(dtype, dim, h, hk, softcap):
    """Large scores of which one key has nearly all the weight: dS is far smaller than dP and D, whose difference it is."""
    g = np.random.Generator(np.random.PCG64(27))
    documents = np.array([[i // 6 if i < 90 else i // 3 for i in range(200)]] * 2)
    for n, window in ((5, 0), (32, 0), (300, 3), (200, None), (70, 32)):
        q, dout = (_draw(g, (2, h, n, dim), dtype, "dense") for _ in range(2))
        k, v = (_draw(g, (2, hk, n, dim), dtype, "dense") for _ in range(2))
        q.mul_(4.0)
        if window is None:
            see = np.stack([(x[:, None] == x[None]) & np.tril(np.ones((n, n), bool)) for x in documents])
            ranges = torch.empty(2, n, 2, dtype=torch.int32, device="cuda")
            hb.hidet_attention_ranges(ranges, documents=torch.from_numpy(documents.astype(np.int32)).cuda(), causal=True)
            opts = dict(softcap=softcap, ranges=ranges)
        else:
            see = np.stack([oa.sees(n, n, True, window)] * 2)
            opts = dict(softcap=softcap, causal=True, window=window)
        out, dq, dk, dv = (torch.empty_like(t) for t in (q, q, k, v))
        lse = torch.empty(2, h, n, device="cuda")
        hb.hidet_attention(q, k, v, out, lse=lse, **opts)
        ws = torch.empty(hb.hidet_attention_backward_workspace_bytes(q, k) // 4, device="cuda")
        hb.hidet_attention_backward(dout, q, k, v, out, lse, dq, dk, dv, ws, **opts)
        want, bound = bounds(dtype, f64(q), f64(k), f64(v), see, dim ** -0.5, softcap, None, grad_out=f64(dout), few=True)
        for name, t, x, e in zip(("dq", "dk", "dv"), (dq, dk, dv), want[2:], bound[2:]):
            assert_within(t, x, e, "%s %d keys %s" % (dtype, n, name))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim,h,hk,softcap", [(64, 4, 2, 0.0), (128, 2, 1, 0.0), (40, 3, 3, 20.0)])
@pytest.mark.parametrize("mask", ["causal", "documents", "alternating", "alternating in splits"])
def test_gradients_of_few_keys_beside_queries_that_see_many(mask, dtype, dim, h, hk, softcap):
    """The first rows of a causal sequence, short documents beside long ones, every other row: the same bounds as where all see few.
    Gradients of rows that see more than 32 keys are zeros, so that dK and dV are those of the others alone."""
    g = np.random.Generator(np.random.PCG64(28))
    n, m = (200, 200) if mask != "alternating in splits" else (90, 3000)
    q, dout = (_draw(g, (2, h, n, dim), dtype, "dense") for _ in range(2))
    k, v = (_draw(g, (2, hk, m, dim), dtype, "dense") for _ in range(2))
    q.mul_(4.0)
    at = np.arange(n)
    if mask == "causal":
        r = np.stack([0 * at, at + 1], 1)
    elif mask == "documents":  # 5, 60, 7, 100 and 28 tokens, causal
        first = np.repeat([0, 5, 65, 72, 172], [5, 60, 7, 100, 28])
        r = np.stack([first, at + 1], 1)
    else:
        few = (at * 37) % (m - 32)
        r = np.where((at % 2 == 0)[:, None], np.stack([few, few + 2 + at % 31], 1), np.stack([0 * at, 0 * at + m], 1))
    ranges = torch.from_numpy(np.stack([r, r]).astype(np.int32)).cuda()
    see = np.stack([oa.in_ranges(r, m)] * 2)
    opts = dict(softcap=softcap, causal=True) if mask == "causal" else dict(softcap=softcap, ranges=ranges)
    dout[:, :, torch.from_numpy(r[:, 1] - r[:, 0] > 32).cuda()] = 0.0
    out, dq, dk, dv = (torch.empty_like(t) for t in (q, q, k, v))
    lse = torch.empty(2, h, n, device="cuda")
    hb.hidet_attention(q, k, v, out, lse=lse, **opts)
    ws = torch.empty(hb.hidet_attention_backward_workspace_bytes(q, k) // 4, device="cuda")
    hb.hidet_attention_backward(dout, q, k, v, out, lse, dq, dk, dv, ws, **opts)
    want, bound = bounds(dtype, f64(q), f64(k), f64(v), see, dim ** -0.5, softcap, None, grad_out=f64(dout), few=True)
    for name, t, x, e in zip(("dq", "dk", "dv"), (dq, dk, dv), want[2:], bound[2:]):
        assert_within(t, x, e, "%s %s %s" % (mask, dtype, name))


@pytest.mark.parametrize("size", [(1, 2, 1, 300, 4096, 64), (1, 2, 2, 130, 4096, 128), (2, 4, 2, 70, 900, 40), (1, 2, 1, 3, 12, 64)], ids=str)
@pytest.mark.parametrize("twos,opts", [(-10, dict()), (-10, dict(causal=True, softcap=20.0)), (11, dict(causal=True)), (-16, dict(window=40))], ids=str)
def test_fp16_gradients_of_any_size(size, twos, opts):
    """Gradients are linear in that of the output, and powers of two are exact: dQ, dK and dV of 2^twos times the gradient are 2^twos times
    dQ, dK and dV, but for the two roundings of what is stored -- 2^-11 of each, or 2^-25 where fp16 is subnormal -- as dS keeps its bits
    whatever its size.  (Elements of the gradient are at least 2^-4, or multiples of 2^-8, so that fp16 holds what they are scaled to.)"""
    b, h, hk, n, m, d = size
    g = np.random.Generator(np.random.PCG64(71))
    q, dout, out = (_draw(g, (b, h, n, d), "f16", "dense") for _ in range(3))
    k, v = (_draw(g, (b, hk, m, d), "f16", "dense") for _ in range(2))
    dout = torch.where(dout.abs() < 2.0 ** -4, torch.zeros_like(dout), dout)
    if twos < -10:  # (multiples of 2^-8)
        dout = (dout * 256).round() / 256
    lse = torch.empty(b, h, n, device="cuda")
    hb.hidet_attention(q, k, v, out, lse=lse, **opts)
    ws = torch.empty(hb.hidet_attention_backward_workspace_bytes(q, k) // 4, device="cuda")
    got = []
    for factor in (1.0, 2.0 ** twos):
        scaled = dout * factor
        assert torch.equal(scaled.double(), dout.double() * factor)
        grads = [torch.empty_like(t) for t in (q, k, v)]
        hb.hidet_attention_backward(scaled, q, k, v, out, lse, *grads, ws, **opts)
        got.append([f64(t) for t in grads])
    u, small = 2.0 ** -11, 2.0 ** -25
    for name, one, other in zip(("dq", "dk", "dv"), *got):
        value = (np.abs(one) + small) / (1 - u)
        assert_within(other * 2.0 ** -twos, one, 2 * u * value + small + small * 2.0 ** -twos, "%s %s" % (size, name))


@pytest.mark.parametrize("size", [(1, 2, 1, 300, 4096, 64), (1, 2, 2, 130, 1500, 128), (2, 4, 2, 70, 900, 40)], ids=str)
@pytest.mark.parametrize("twos", [-8, 7, 12])
def test_fp16_gradients_under_values_of_any_size(size, twos):
    """dQ and dK are linear in the values (and the output with them) as well, and dV has nothing to do with them."""
    b, h, hk, n, m, d = size
    g = np.random.Generator(np.random.PCG64(72))
    q, dout, out = (_draw(g, (b, h, n, d), "f16", "dense") for _ in range(3))
    k, v = (_draw(g, (b, hk, m, d), "f16", "dense") for _ in range(2))
    v = torch.where(v.abs() < 2.0 ** -4, torch.zeros_like(v), v)
    lse = torch.empty(b, h, n, device="cuda")
    hb.hidet_attention(q, k, v, out, lse=lse)
    out = (out.float() * 2048).round().half() / 2048
    ws = torch.empty(hb.hidet_attention_backward_workspace_bytes(q, k) // 4, device="cuda")
    got = []
    for factor in (1.0, 2.0 ** twos):
        values, result = v * factor, out * factor
        assert torch.equal(values.double(), v.double() * factor) and torch.equal(result.double(), out.double() * factor)
        grads = [torch.empty_like(t) for t in (q, k, v)]
        hb.hidet_attention_backward(dout, q, k, values, result, lse, *grads, ws)
        assert all(bool(torch.isfinite(t).all()) for t in grads)
        got.append([f64(t) for t in grads])
    u, small = 2.0 ** -11, 2.0 ** -25
    for name, one, other in zip(("dq", "dk"), *got):
        value = (np.abs(one) + small) / (1 - u)
        assert_within(other * 2.0 ** -twos, one, 2 * u * value + small + small * 2.0 ** -twos, "%s %s" % (size, name))
    assert np.array_equal(got[0][2], got[1][2])


def test_no_keys_and_no_queries():
    q = torch.randn(2, 4, 5, 64, device="cuda").half()
    k = torch.empty(2, 2, 0, 64, device="cuda", dtype=torch.float16)
    out, lse, dq = torch.full_like(q, 3.0), torch.zeros(2, 4, 5, device="cuda"), torch.full_like(q, 3.0)
    hb.hidet_attention(q, k, k, out, lse=lse)
    ws = torch.empty(hb.hidet_attention_backward_workspace_bytes(q, k), dtype=torch.uint8, device="cuda")
    hb.hidet_attention_backward(q, q, k, k, out, lse, dq, torch.empty_like(k), torch.empty_like(k), ws)
    assert bool((out == 0).all()) and bool((lse == -np.inf).all()) and bool((dq == 0).all())
    none = torch.empty(2, 4, 0, 64, device="cuda", dtype=torch.float16)
    kv = torch.randn(2, 2, 9, 64, device="cuda").half()
    dk, dv = torch.full_like(kv, 3.0), torch.full_like(kv, 3.0)
    hb.hidet_attention(none, kv, kv, none)
    hb.hidet_attention_backward(none, none, kv, kv, none, torch.empty(2, 4, 0, device="cuda"), none, dk, dv, None)
    assert bool((dk == 0).all()) and bool((dv == 0).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [24, 64, 128])
@pytest.mark.parametrize("form", [dict(), dict(causal=True), dict(softcap=20.0), dict(slopes=True), dict(softcap=5.0, slopes=True, window=3)], ids=str)
def test_keys_without_queries_have_gradients_of_zero(form, dim, dtype):
    """There is nothing then that says which rows see a key: no list of them is read."""
    form = dict(form)
    none = torch.empty(2, 4, 0, dim, device="cuda", dtype=TYPES[dtype])
    k = torch.randn(2, 2, 150, dim, device="cuda").to(TYPES[dtype])
    dk, dv = torch.full_like(k, 3.0), torch.full_like(k, 3.0)
    if form.pop("slopes", False):
        form["slopes"] = torch.ones(4, device="cuda")
    hb.hidet_attention_backward(none, none, k, k, none, torch.empty(2, 4, 0, device="cuda"), none, dk, dv, None, **form)
    assert not dk.any() and not dv.any()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 104])
def test_what_nobody_sees_and_what_others_see_has_no_influence(dtype, dim):
    def padding(q, k, v, g, see):  # keys and queries that take no part, and the gradients of the latter
        for b in range(len(see)):
            none = torch.from_numpy(~see[b].any(0)).cuda()
            k[b][:, none] = float("nan")
            v[b][:, none] = float("inf")
            alone = torch.from_numpy(~see[b].any(1)).cuda()
            q[b][:, alone] = float("nan")
            g[b][:, alone] = float("inf")

    lens = np.array([90, 0, 41])
    r = np.zeros((3, 100, 2), dtype=int)
    for b, length in enumerate(lens):
        r[b, :length, 1] = np.arange(1, length + 1)
    _run(5000 + dim, dtype, 3, 2, 1, 100, 100, dim, ranges=r, poison=padding)


def test_a_poisoned_key_reaches_only_the_queries_that_see_it():
    g = np.random.Generator(np.random.PCG64(5))
    for dtype in ("f16", "bf16"):
        q, k, v, dout = (_draw(g, (1, 4, 100, 64), dtype, "dense") for _ in range(4))
        k, v = k[:, :2].contiguous(), v[:, :2].contiguous()
        clean = [t.clone() for t in (k, v)]
        v[0, 0, 60, 3] = float("inf")
        k[0, 1, 70, 5] = float("nan")
        outs = []
        for kk, vv in ((k, v), clean):
            out, lse = torch.empty_like(q), torch.empty(1, 4, 100, device="cuda")
            dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(k)
            ws = torch.empty(hb.hidet_attention_backward_workspace_bytes(q, k), dtype=torch.uint8, device="cuda")
            hb.hidet_attention(q, kk, vv, out, lse=lse, causal=True)
            hb.hidet_attention_backward(dout, q, kk, vv, out, lse, dq, dk, dv, ws, causal=True)
            outs.append([out, lse, dq, dk, dv])
        (out, lse, dq, dk, dv), want = outs
        u = 4 * {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}[dtype]

        def same(a, b):  # (computed another way: a few roundings apart)
            assert float((a.float() - b.float()).abs().max()) <= u * max(1.0, float(b.float().abs().max()))

        same(out[:, :2, :60], want[0][:, :2, :60])
        same(out[:, 2:, :70], want[0][:, 2:, :70])
        same(dq[:, :2, :60], want[2][:, :2, :60])
        same(dq[:, 2:, :70], want[2][:, 2:, :70])
        assert bool(torch.isinf(out[:, :2, 60:, 3]).all()) and bool(torch.isnan(out[:, 2:, 70:]).all())
        same(out[:, :2, :, :3], want[0][:, :2, :, :3])  # (an infinite value spoils its own dimension only)
        assert bool(torch.isnan(lse[:, 2:, 70:]).all())
        same(lse[:, :2], want[1][:, :2])
        # every query of these heads that sees the key is spoilt, and with it the keys that such a query sees: all of them
        assert bool(torch.isnan(dk[:, 1]).all()) and bool(torch.isnan(dv[:, 1]).all())


def _scatter(g, shape, count):
    """`count` places of a tensor of that shape with an infinity of either sign or NaN for each."""
    return [(tuple(int(g.integers(n)) for n in shape), (np.inf, -np.inf, np.nan)[int(g.integers(3))]) for _ in range(count)]


def _sums_of_odd(see, places, shape):
    """What sums over the seen keys come to in the dimensions where a key holds something that is not finite: 0 where none does.
    see [batch, n, m], places of [batch, heads, m, dim] -> [batch, heads, n, dim]."""
    out = np.zeros((shape[0], shape[1], see.shape[1], shape[3]))
    with np.errstate(invalid="ignore"):
        for (b, h, j, d), x in dict(places).items():
            out[b, h, see[b, :, j], d] += x
    return out


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("size", [(1, 4, 2, 300, 300, 64), (2, 2, 1, 200, 260, 128), (86, 12, 6, 19, 193, 112), (1, 2, 1, 3, 700, 40), (1, 4, 2, 1, 9000, 128),
                                  (1, 4, 2, 90, 3000, 64), (2, 3, 3, 130, 130, 24), (1, 4, 2, 1500, 1500, 64), (1, 2, 1, 1300, 2100, 128), (1, 9, 9, 2000, 1100, 104),
                                  (1, 40, 40, 1000, 1000, 64)], ids=str)
@pytest.mark.parametrize("mask", ["causal", "window", "ranges"])
def test_values_that_are_not_finite_reach_the_queries_that_see_them_alone(mask, size, dtype):
    """In every kernel and cut: a dimension in which a query sees infinities or a NaN is their sum, and every other result has the bits
    that it has without them."""
    b, h, hk, n, m, d = size
    g = np.random.Generator(np.random.PCG64(81))
    q, k, v = _draw(g, (b, h, n, d), dtype, "dense"), _draw(g, (b, hk, m, d), dtype, "tokens"), _draw(g, (b, hk, m, d), dtype, "tokens")
    if mask == "ranges":
        lo = g.integers(0, m, (b, n))
        r = np.stack([lo, np.minimum(m, lo + g.integers(0, m, (b, n)))], 2).astype(np.int32)
        see, opts = np.stack([oa.in_ranges(x, m) for x in r]), dict(ranges=torch.from_numpy(r).cuda())
    else:
        opts = dict(causal=True, window=60 if mask == "window" else 0)
        see = np.stack([oa.sees(n, m, **opts)] * b)
    size = hb.hidet_attention_workspace_bytes(q, k)
    for count in (1, 7, 60):
        places = _scatter(g, v.shape, count)
        # (one in the last key that is seen, which stands for those behind it in its tile)
        places.append(((0, 0, m - 1, d - 1), np.inf))
        odd = v.clone()
        for at, x in places:
            odd[at] = x
        for ws in ([None, torch.empty(size // 4, device="cuda")] if size else [None]):
            results = []
            for values in (v, odd):
                out, lse = torch.full_like(q, 7.0), torch.empty(b, h, n, device="cuda")
                hb.hidet_attention(q, k, values, out, lse=lse, workspace=ws, **opts)
                results.append((out, lse))
            (clean, lse_clean), (out, lse) = results
            sums = np.repeat(_sums_of_odd(see, places, tuple(v.shape)), h // hk, 1)
            reached = torch.from_numpy(sums != 0.0).cuda()
            want = torch.where(reached, torch.from_numpy(sums).cuda().to(out.dtype), clean)
            assert torch.equal(lse, lse_clean)
            assert torch.equal(torch.nan_to_num(out, 11.0, 12.0, 13.0), torch.nan_to_num(want, 11.0, 12.0, 13.0)), (count, ws is None)


@pytest.mark.parametrize("size", [(1, 4, 2, 1500, 1500, 64), (1, 2, 1, 1300, 2100, 128), (1, 40, 40, 1000, 1000, 64), (1, 2, 1, 2, 9000, 64)], ids=str)
def test_queries_that_are_not_finite_are_so_alone(size):
    b, h, hk, n, m, d = size
    for dtype in ("f16", "bf16"):
        g = np.random.Generator(np.random.PCG64(86))
        q, k, v = _draw(g, (b, h, n, d), dtype, "dense"), _draw(g, (b, hk, m, d), dtype, "dense"), _draw(g, (b, hk, m, d), dtype, "dense")
        odd, rows = q.clone(), torch.zeros(b, h, n, dtype=torch.bool, device="cuda")
        for (bb, hh, i, dd), _ in _scatter(g, q.shape, 9):
            odd[bb, hh, i, dd] = np.nan
            rows[bb, hh, i] = True
        size = hb.hidet_attention_workspace_bytes(q, k)
        for ws in (None, torch.full((size // 4 + 4,), float("nan"), device="cuda")):
            results = []
            for queries in (q, odd):
                out, lse = torch.full_like(q, 7.0), torch.empty(b, h, n, device="cuda")
                hb.hidet_attention(queries, k, v, out, lse=lse, workspace=ws)
                results.append((out, lse))
            (clean, lse_clean), (out, lse) = results
            assert bool((torch.isnan(lse) == rows).all()) and bool((torch.isnan(out) == rows[..., None]).all())
            # (maxima are replaced for 32 rows at a time, which moves the others' last bits: two roundings of weights and of the result)
            u = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}[dtype]
            off = torch.where(rows[..., None], torch.zeros_like(out), (out - clean).abs()).float()
            assert float(off.max()) <= 4 * u * float(v.abs().max()) and float(torch.where(rows, 0.0, lse - lse_clean).abs().max()) <= 1e-5


def test_scores_that_are_not_finite_and_values_beside_them():
    """A row of which a score is NaN or +inf is NaN, one whose scores are all -inf is 0, whatever values are beside; keys of score -inf
    count as masked, and so do their values."""
    for dtype in ("f16", "bf16"):
        for n in (1, 70, 200):
            g = np.random.Generator(np.random.PCG64(82))
            q, k, v = (_draw(g, (1, 2, 200, 64), dtype, "dense") for _ in range(3))
            q = q[:, :, :n].abs() + 0.1
            k[0, 0, 5:9] = -np.inf  # (scores of -inf, and values that nobody sees for it)
            v[0, 0, 5:9] = np.nan
            k[0, 1, 150, 3] = np.nan
            v[0, 1, 20, 7] = np.inf
            plain = [t.clone() for t in (k, v)]
            see = np.ones((1, n, 200), bool)
            see[0, :, 5:9] = False
            out, lse = torch.empty_like(q), torch.empty(1, 2, n, device="cuda")
            hb.hidet_attention(q, k, v, out, lse=lse)
            assert bool(torch.isnan(out[0, 1]).all()) and bool(torch.isnan(lse[0, 1]).all())
            plain[0][0, 0, 5:9] = 0.0
            plain[1][0, 0, 5:9] = 0.0
            want, bound = bounds(dtype, f64(q)[:, :1], f64(plain[0])[:, :1], f64(plain[1])[:, :1], see, 64 ** -0.5)
            assert_within(out[:, :1], want[0], bound[0], "%s %d out" % (dtype, n))
            assert_within(lse[:, :1], want[1], bound[1], "%s %d lse" % (dtype, n))
            k[0, 0] = -np.inf
            hb.hidet_attention(q, k, v, out, lse=lse)
            assert not out[0, 0].any() and bool((lse[0, 0] == -np.inf).all())
            q[0, 1, n // 2] = np.nan  # (all scores NaN, none of which makes a maximum)
            k[0, 1] = plain[0][0, 0]
            hb.hidet_attention(q, k, v, out, lse=lse)
            assert bool(torch.isnan(out[0, 1, n // 2]).all()) and bool(torch.isnan(lse[0, 1, n // 2]))
            assert bool(torch.isfinite(lse[0, 1, torch.arange(n) != n // 2]).all())
            k[0, 1] = k[0, 1].abs() + 0.1
            q[0, 1, n // 2] = -np.inf  # (all scores -inf, beside an infinite value that the others see)
            hb.hidet_attention(q, k, v, out, lse=lse)
            others = torch.arange(n) != n // 2
            assert not out[0, 1, n // 2].any() and float(lse[0, 1, n // 2]) == -np.inf
            assert bool((out[0, 1, others, 7] == np.inf).all()) and bool(torch.isfinite(out[0, 1, others, :7]).all())


BACK_SIZES = [(1, 4, 2, 300, 300, 64), (2, 2, 1, 200, 260, 128), (1, 3, 1, 70, 700, 40), (1, 2, 1, 90, 3000, 128), (1, 4, 2, 900, 70, 64), (86, 12, 6, 19, 193, 112)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("size", BACK_SIZES, ids=str)
@pytest.mark.parametrize("mask", ["causal", "window", "ranges"])
def test_gradients_of_what_is_not_finite_spoil_what_it_reaches_alone(mask, size, dtype):
    """Infinities and NaN in the gradient of the output, queries, keys, values: a query that has or sees one has a gradient that is not finite,
    and so have the keys that it sees; dV where the gradient of the output has it is the sum of those (NaN where a weight is).  All
    else has the bits that it has without them (dK in fp16 two roundings, as the scale of dS in a block of keys may be another)."""
    b, h, hk, n, m, d = size
    g = np.random.Generator(np.random.PCG64(83))
    q, dout = (_draw(g, (b, h, n, d), dtype, "dense") for _ in range(2))
    k, v = (_draw(g, (b, hk, m, d), dtype, "tokens") for _ in range(2))
    if mask == "ranges":
        lo = g.integers(0, m, (b, n))
        r = np.stack([lo, np.minimum(m, lo + g.integers(0, m, (b, n)))], 2).astype(np.int32)
        see, opts = np.stack([oa.in_ranges(x, m) for x in r]), dict(ranges=torch.from_numpy(r).cuda())
    else:
        opts = dict(causal=True, window=60 if mask == "window" else 0)
        see = np.stack([oa.sees(n, m, **opts)] * b)
    see = np.repeat(see[:, None], h, 1)  # [b, h, n, m]
    group = h // hk

    def forward(q, k, v):
        out, lse = torch.full_like(q, 7.0), torch.empty(b, h, n, device="cuda")
        hb.hidet_attention(q, k, v, out, lse=lse, **opts)
        return out, lse

    def run(q, k, v, dout, out, lse):
        dq, dk, dv = (torch.full_like(t, 7.0) for t in (q, k, v))
        ws = torch.full((hb.hidet_attention_backward_workspace_bytes(q, k) // 4,), float("nan"), device="cuda")
        hb.hidet_attention_backward(dout, q, k, v, out, lse, dq, dk, dv, ws, **opts)
        return dq, dk, dv

    out, lse = forward(q, k, v)
    clean = run(q, k, v, dout, out, lse)
    for which in range(4):
        for count in (1, 5):
            x = [t.clone() for t in (q, k, v, dout)]
            places = _scatter(g, x[which].shape, count)
            if which < 2:  # (an infinite query or key may leave scores of -inf, and no weight)
                places = [(at, np.nan) for at, _ in places]
            for at, value in places:
                x[which][at] = value
            row = np.zeros((b, h, n), bool)  # (rows of which the log-sum or D is not finite)
            for (bb, hh, i, _), _ in places:
                if which in (0, 3):
                    row[bb, hh, i] |= see[bb, hh, i].any()
                else:
                    row[bb, hh * group:(hh + 1) * group] |= see[bb, hh * group:(hh + 1) * group, :, i]
            key = np.einsum("bhn,bhnm->bhm", row, see).reshape(b, hk, group, m).any(2)
            row, key = (torch.from_numpy(t).cuda()[..., None] for t in (row, key))
            # (outputs of the other rows as they are without: maxima are replaced for 32 rows at a time, which moves their last bits)
            odd_out, odd_lse = forward(*x[:3])
            dq, dk, dv = run(*x, torch.where(row, odd_out, out), torch.where(row[..., 0], odd_lse, lse))
            bits = lambda t: torch.nan_to_num(t, 11.0, 12.0, 13.0)
            what = "%s %s" % (("q", "k", "v", "grad_out")[which], count)
            assert not bool((torch.isfinite(dq) & row).any()) and not bool((torch.isfinite(dk) & key).any()), what
            assert torch.equal(torch.where(row, clean[0], dq), clean[0]), what + " dq"
            rest = torch.where(key, clean[1], dk)
            if dtype == "bf16":
                assert torch.equal(rest, clean[1]), what + " dk"
            else:
                assert_within(rest, f64(clean[1]), 2.0 ** -10 * np.abs(f64(clean[1])) * 1.01 + 2.0 ** -24, what + " dk")
            if which < 2:
                assert bool((torch.isnan(dv) | ~key).all()) and torch.equal(torch.where(key, clean[2], dv), clean[2]), what + " dv"
            elif which == 2:
                assert torch.equal(dv, clean[2]), what + " dv"
            else:
                sums = np.zeros((b, hk, m, d))
                with np.errstate(invalid="ignore"):
                    for (bb, hh, i, dd), value in dict(places).items():
                        sums[bb, hh // group, see[bb, hh, i], dd] += value
                want = torch.where(torch.from_numpy(sums != 0.0).cuda(), torch.from_numpy(sums).cuda().to(dv.dtype), clean[2])
                assert torch.equal(bits(dv), bits(want)), what + " dv"


def test_gradients_of_keys_of_score_minus_infinity():
    """Keys of -inf under queries that are positive have no weight, and neither they nor their values reach a gradient; their own are 0."""
    for dtype in ("f16", "bf16"):
        for n, d, level in ((70, 64, 0.0), (200, 128, 0.0), (40, 24, 0.0), (90, 64, -30.0), (700, 128, -30.0)):  # (scores of -200)
            g = np.random.Generator(np.random.PCG64(84))
            q, dout = (_draw(g, (1, 2, n, d), dtype, "dense") for _ in range(2))
            k, v = (_draw(g, (1, 1, 3 * n, d), dtype, "dense") for _ in range(2))
            q = q.abs() + 0.1
            k = k + level
            masked = torch.zeros(3 * n, dtype=torch.bool)
            masked[::7] = True
            kk = k.clone()
            kk[:, :, masked.cuda()] = -np.inf
            out, dq, dk, dv = (torch.full_like(t, 7.0) for t in (q, q, k, v))
            lse = torch.empty(1, 2, n, device="cuda")
            hb.hidet_attention(q, kk, v, out, lse=lse, causal=True)
            ws = torch.empty(hb.hidet_attention_backward_workspace_bytes(q, k) // 4, device="cuda")
            hb.hidet_attention_backward(dout, q, kk, v, out, lse, dq, dk, dv, ws, causal=True)
            see = (oa.sees(n, 3 * n, True) & ~masked.numpy()[None])[None]
            want, bound = bounds(dtype, f64(q), f64(k), f64(v), see, d ** -0.5, grad_out=f64(dout))
            for name, t, x, e in zip(("out", "lse", "dq", "dk", "dv"), (out, lse, dq, dk, dv), want, bound):
                assert_within(t, x, e, "%s %d %s" % (dtype, n, name))
            assert not dk[:, :, masked.cuda()].any() and not dv[:, :, masked.cuda()].any()


@pytest.mark.parametrize("dim", [64, 128, 40])
@pytest.mark.parametrize("h,n,m", [(2, 40, 40), (4, 300, 300), (2, 70, 2000)])
def test_fp16_gradients_of_values_that_cancel_in_the_output(h, n, m, dim):
    """Large values of either sign, with nearly equal weights: the output says nothing of how large dS is, which passes fp16 (some 1e6)."""
    g = np.random.Generator(np.random.PCG64(85))
    q, dout = (_draw(g, (1, h, n, dim), "f16", "dense") for _ in range(2))
    k, v = (_draw(g, (1, h // 2, m, dim), "f16", "dense") for _ in range(2))
    q.mul_(0.01)
    dout.mul_(100.0)
    v = (30000.0 + 0 * v) * torch.where(torch.arange(m, device="cuda") % 2 == 0, 1.0, -1.0).half()[None, None, :, None]
    ranges = torch.tensor([[2 * (i % (m // 2)), 2 * (i % (m // 2)) + 2] for i in range(n)], dtype=torch.int32, device="cuda")[None]
    out, dq, dk, dv = (torch.full_like(t, 7.0) for t in (q, q, k, v))
    lse = torch.empty(1, h, n, device="cuda")
    hb.hidet_attention(q, k, v, out, lse=lse, ranges=ranges)
    ws = torch.empty(hb.hidet_attention_backward_workspace_bytes(q, k) // 4, device="cuda")
    hb.hidet_attention_backward(dout, q, k, v, out, lse, dq, dk, dv, ws, ranges=ranges, scale=None)
    see = np.stack([oa.in_ranges(ranges[0].cpu().numpy(), m)])
    want, bound = bounds("f16", f64(q), f64(k), f64(v), see, dim ** -0.5, grad_out=f64(dout), few=True)
    for name, t, x, e in zip(("dq", "dk", "dv"), (dq, dk, dv), want[2:], bound[2:]):
        fits = np.abs(x) < 60000.0
        got = f64(t)
        assert np.all(np.isinf(got[np.abs(x) > 66000.0]))
        assert_within(np.where(fits, got, 0.0), np.where(fits, x, 0.0), e + 1e-30, name)


@pytest.mark.parametrize("n,m,splits", [(3, 600, 2), (90, 3000, 2), (1, 9000, 17)])
def test_an_infinite_value_of_a_key_of_little_weight(n, m, splits):
    """Its weight, 2^-288, is not a number of fp32 beside the others', nor is that of its split; times infinity it is infinite all the same."""
    for dtype in ("f16", "bf16"):
        q = torch.ones(1, 2, n, 64, device="cuda").to(TYPES[dtype])
        k, v = (torch.ones(1, 1, m, 64, device="cuda").to(TYPES[dtype]) for _ in range(2))
        k[:, :, :m // 2] = -24.0  # (scores of -192 and 8)
        for at in (5, m // 2 - 1):
            v[0, 0, at, 9] = np.inf
        out, lse = torch.empty_like(q), torch.empty(1, 2, n, device="cuda")
        size = hb.hidet_attention_workspace_bytes(q, k)
        rows, width = (n * 2), 66
        assert size // (rows * width * 4) >= splits, "this size is not split enough"
        want = torch.ones_like(q)
        want[..., 9] = np.inf
        for ws in (None, torch.full((size // 4,), float("nan"), device="cuda")):
            hb.hidet_attention(q, k, v, out, lse=lse, workspace=ws)
            assert torch.equal(out, want), (dtype, ws is None)
            assert float((lse - 8.0 - np.log(m - m // 2)).abs().max()) <= 1e-4


def _time(f):
    f()
    times = []
    for _ in range(5):
        e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        e[0].record()
        f()
        e[1].record()
        torch.cuda.synchronize()
        times.append(e[0].elapsed_time(e[1]))
    return sorted(times)[2]


@pytest.mark.parametrize("dtype,dim", [("f16", 64), ("bf16", 128)])
def test_what_is_not_finite_costs_a_few_times_the_time(dtype, dim):
    """Of a causal prompt of 2048: one value, the last, one in every key, all of them; measured 2 to 12 times the time, here up to 40."""
    q = torch.randn(1, 8, 2048, dim, device="cuda").to(TYPES[dtype])
    k, v = (torch.randn(1, 4, 2048, dim, device="cuda").to(TYPES[dtype]) for _ in range(2))
    out, lse = torch.empty_like(q), torch.empty(1, 8, 2048, device="cuda")
    clean = _time(lambda: hb.hidet_attention(q, k, v, out, lse=lse, causal=True))
    for name, at in (("one", (0, 1, 100, 5)), ("the last", (0, 1, 2047, 5)), ("in every key", (slice(None), slice(None), slice(None), 5)), ("all", Ellipsis)):
        for x in (np.inf, np.nan):
            odd = v.clone()
            odd[at] = x
            took = _time(lambda: hb.hidet_attention(q, k, odd, out, lse=lse, causal=True))
            print("%s %s: %.1f times" % (name, x, took / clean), flush=True)
            assert took <= 40 * clean, name


@pytest.mark.parametrize("dtype,dim", [("f16", 64), ("bf16", 128)])
def test_gradients_of_what_is_not_finite_cost_a_few_times_the_time(dtype, dim):
    """Of a causal prompt of 2048: one element of a tensor, one in every vector, all of them; measured 1 to 6 times the time, here up to 30."""
    n = 2048
    x = [torch.randn(1, heads, n, dim, device="cuda").to(TYPES[dtype]) for heads in (8, 4, 4, 8)]
    out, dq, dk, dv = (torch.empty_like(x[i]) for i in (0, 0, 1, 2))
    lse = torch.empty(1, 8, n, device="cuda")
    ws = torch.empty(hb.hidet_attention_backward_workspace_bytes(x[0], x[1]) // 4, device="cuda")

    def run(q, k, v, dout):
        hb.hidet_attention(q, k, v, out, lse=lse, causal=True)
        return _time(lambda: hb.hidet_attention_backward(dout, q, k, v, out, lse, dq, dk, dv, ws, causal=True))

    clean = run(*x)
    for i, name in enumerate(("q", "k", "v", "grad_out")):
        for at in ((0, 1, 100, 5), (0, 1, n - 1, 5), (slice(None), slice(None), slice(None), 5), Ellipsis):
            odd = [t.clone() for t in x]
            odd[i][at] = np.inf
            took = run(*odd)
            print("%s %s: %.1f times" % (name, at, took / clean), flush=True)
            assert took <= 30 * clean, name


def test_large_scores_and_flat_ones():
    def grow(q, k, v, g, see):  # maxima that grow from tile to tile by far more than the slack before a rescale
        q.copy_(torch.ones_like(q))
        k.copy_((torch.arange(k.shape[2], device="cuda") / 8.0).to(k.dtype)[None, None, :, None].expand_as(k))

    def shrink(q, k, v, g, see):
        grow(q, k, v, g, see)
        k.copy_(-k)

    def flat(q, k, v, g, see):
        q.zero_()

    for i, poison in enumerate((grow, shrink, flat)):
        _run(6000 + i, "f16", 1, 1, 1, 40, 400, 64, poison=poison)
        _run(6010 + i, "bf16", 1, 2, 1, 140, 300, 128, poison=poison, causal=True)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("size", [(1, 2, 1, 1, 9000, 64), (1, 8, 1, 3, 5000, 128), (1, 4, 2, 90, 3000, 128), (1, 2, 2, 200, 2500, 80)], ids=str)
def test_splits(size, dtype):
    a, la = _run(7000 + size[3], dtype, *size, causal=True, split=True, back=False)
    b, lb = _run(7000 + size[3], dtype, *size, causal=True, split=True, back=False)
    assert torch.equal(a, b) and torch.equal(la, lb)
    _run(7000 + size[3], dtype, *size, causal=True, split=False, back=False)
    g = np.random.Generator(np.random.PCG64(1))
    r = _random_ranges(g, size[0], size[3], size[4])  # (some rows see little or nothing: empty splits)
    r[:, 0] = (17, 40)
    _run(7100 + size[3], dtype, *size, ranges=r, split=True, back=False, softcap=3.0)


def test_a_workspace_that_is_too_small_for_all_splits_serves_fewer():
    g = np.random.Generator(np.random.PCG64(8))
    q, k, v = (_draw(g, (1, 2, n, 64), "f16", "dense") for n in (1, 8192, 8192))
    size = hb.hidet_attention_workspace_bytes(q, k)
    outs = []
    for part in (0, 100, size // 3 // 16 * 16, size):
        guard = torch.full((part + 64,), 0x5A, dtype=torch.uint8, device="cuda")
        out = torch.empty_like(q)
        hb.hidet_attention(q, k, v, out, workspace=guard[:part] if part else None)
        assert bool((guard[part:] == 0x5A).all())
        outs.append(out)
    for o in outs[1:]:
        assert float((o.float() - outs[0].float()).abs().max()) <= 2e-3  # (outputs below 1/4: two roundings to fp16 are 2.4e-4)


def test_shared_inputs_with_stride_zero():
    g = np.random.Generator(np.random.PCG64(9))
    q = _draw(g, (3, 4, 20, 64), "bf16", "tokens")
    k, v = (_draw(g, (1, 1, 50, 64), "bf16", "dense").expand(3, 2, 50, 64) for _ in range(2))
    see = np.ones((3, 20, 50), bool)
    out, lse = torch.empty_like(q), torch.empty(3, 4, 20, device="cuda")
    hb.hidet_attention(q, k, v, out, lse=lse)
    want, bound = bounds("bf16", f64(q), f64(k), f64(v), see, 0.125)
    assert_within(out, want[0], bound[0], "out")
    assert_within(lse, want[1], bound[1], "lse")


@pytest.mark.parametrize("n,m", [(5, 5), (1500, 1500), (40, 2100), (300, 100), (4097, 4097)])
def test_attention_ranges(n, m):
    g = np.random.Generator(np.random.PCG64(n + m))
    docs = np.repeat(g.integers(-1, 4, m), g.integers(1, 1 + max(2, m // 6), m))[:m].astype(np.int32)
    prefix = np.array([int(g.integers(0, m + 3)), 2], dtype=np.int32)
    documents = np.stack([docs, np.roll(docs, 3)])
    for use_docs, use_prefix, causal, window in ((1, 0, 1, 0), (1, 0, 0, 0), (1, 1, 1, 0), (0, 1, 1, 0), (1, 0, 1, 3), (1, 0, 0, 4), (0, 0, 1, 0), (0, 0, 0, 2)):
        r = torch.full((2, n, 2), -99, dtype=torch.int32, device="cuda")
        hb.hidet_attention_ranges(r, keys=m, documents=torch.from_numpy(documents).cuda() if use_docs else None,
                                  prefix=torch.from_numpy(prefix).cuda() if use_prefix else None, causal=bool(causal), window=window)
        got = r.cpu().numpy()
        rows = sorted({0, 1, n // 2, n - 1} | set(g.integers(0, n, 40).tolist())) if n > 200 else range(n)
        for b in range(2):
            at = np.arange(n) + m - n
            lo, hi = got[b, :, 0], got[b, :, 1]
            d = documents[b] if use_docs else np.zeros(m, dtype=int)
            for i in rows:
                want = np.zeros(m, dtype=bool)
                if at[i] >= 0 and d[at[i]] >= 0:  # (a query before the first key is in no document)
                    s = at[i]
                    while s > 0 and d[s - 1] == d[at[i]]:
                        s -= 1
                    e = at[i] + 1
                    while e < m and d[e] == d[at[i]]:
                        e += 1
                    j = np.arange(m)
                    want = (j >= s) & (j < e)
                    if window:
                        want &= (np.abs(j - at[i]) < window)
                    if causal:
                        want &= (j <= at[i]) | (j < s + (prefix[b] if use_prefix else 0))
                    want &= (j >= s) & (j < e)
                have = np.zeros(m, dtype=bool)
                have[max(lo[i], 0):max(hi[i], 0)] = True
                assert np.array_equal(have, want), (use_docs, use_prefix, causal, window, b, i)


def test_documents_and_prefixes_through_the_kernels():
    docs = np.array([[0] * 30 + [1] * 70 + [-1] * 20, [5] * 120], dtype=np.int32)
    prefix = np.array([10, 50], dtype=np.int32)
    for causal, pre in ((True, False), (True, True), (False, False)):
        see = np.stack([oa.sees(120, 120, causal, 0, docs[b], prefix[b] if pre else 0) for b in range(2)])
        r = torch.empty(2, 120, 2, dtype=torch.int32, device="cuda")
        hb.hidet_attention_ranges(r, documents=torch.from_numpy(docs).cuda(), prefix=torch.from_numpy(prefix).cuda() if pre else None, causal=causal)
        ranges = r.cpu().numpy()
        assert np.array_equal(np.stack([oa.in_ranges(x, 120) for x in ranges]), see)
        _run(8000 + causal + 2 * pre, "bf16", 2, 4, 2, 120, 120, 64, ranges=ranges)


def test_gradients_against_differences():
    """The forward kernel itself, differenced: a step that fp16 inputs hold exactly, in a direction of ones and minus ones."""
    g = np.random.Generator(np.random.PCG64(17))
    shape_q, shape_k = (1, 2, 24, 64), (1, 1, 40, 64)
    q, k, v = (torch.from_numpy(np.round(g.standard_normal(s) * 16) / 16).cuda() for s in (shape_q, shape_k, shape_k))
    dout = torch.from_numpy(np.round(g.standard_normal(shape_q) * 16) / 16).cuda()
    opts = dict(causal=True, softcap=4.0, slopes=torch.tensor([0.1, 0.3], device="cuda"))

    def loss(q, k, v):  # (differences of an output rounded to fp16: its oracle has the same definition in 64 bits)
        see = np.ones((1, 24, 40), bool) & oa.sees(24, 40, causal=True)[None]
        return float((oa.attention(f64(q), f64(k), f64(v), see, 0.125, 4.0, [float(np.float32(0.1)), float(np.float32(0.3))])[0] * f64(dout)).sum())

    h = torch.float16
    out, lse = torch.empty(shape_q, dtype=h, device="cuda"), torch.empty(1, 2, 24, device="cuda")
    grads = [torch.empty(s, dtype=h, device="cuda") for s in (shape_q, shape_k, shape_k)]
    args = [t.to(h) for t in (q, k, v)]
    hb.hidet_attention(*args, out, lse=lse, **opts)
    ws = torch.empty(hb.hidet_attention_backward_workspace_bytes(args[0], args[1]), dtype=torch.uint8, device="cuda")
    hb.hidet_attention_backward(dout.to(h), *args, out, lse, *grads, ws, **opts)
    for which in range(3):
        t = [q, k, v]
        direction = torch.from_numpy(g.choice([-1.0, 1.0], t[which].shape)).cuda()
        ends = []
        for step in (1e-4, -1e-4):
            moved = list(t)
            moved[which] = t[which] + step * direction
            ends.append(loss(*moved))
        want = (ends[0] - ends[1]) / 2e-4
        got = float((f64(grads[which]) * f64(direction)).sum())
        # a sum of n gradients of random sign, each off by 2^-10 of itself and of its terms: sqrt(n) of the largest, generously
        n = grads[which].numel()
        assert abs(got - want) <= 2.0 ** -9 * n ** 0.5 * float(grads[which].float().abs().max()) + 1e-5, which


def _chain(q, k, v, dout, bufs, stream=None):
    out, lse, dq, dk, dv, ws, r, docs = bufs
    hb.hidet_attention_ranges(r, documents=docs, causal=True, stream=stream)
    hb.hidet_attention(q, k, v, out, lse=lse, ranges=r, workspace=ws, stream=stream)
    hb.hidet_attention_backward(dout, q, k, v, out, lse, dq, dk, dv, ws, ranges=r, stream=stream)


def _chain_state(seed=3):
    g = np.random.Generator(np.random.PCG64(seed))
    q, dout = (_draw(g, (2, 4, 150, 64), "bf16", "tokens") for _ in range(2))
    k, v = (_draw(g, (2, 2, 150, 64), "bf16", "tokens") for _ in range(2))
    docs = torch.tensor([[0] * 70 + [1] * 80, [2] * 149 + [-1]], dtype=torch.int32, device="cuda")
    size = max(hb.hidet_attention_workspace_bytes(q, k), hb.hidet_attention_backward_workspace_bytes(q, k))

    def bufs():
        return (torch.empty_like(q), torch.empty(2, 4, 150, device="cuda"), torch.empty_like(q), torch.empty_like(k), torch.empty_like(k),
                torch.empty(size, dtype=torch.uint8, device="cuda"), torch.empty(2, 150, 2, dtype=torch.int32, device="cuda"), docs)

    return q, k, v, dout, bufs


def test_graph_replays_match_eager_calls():
    q, k, v, dout, make = _chain_state()
    eager, captured = make(), make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _chain(q, k, v, dout, captured)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _chain(q, k, v, dout, captured)
    for step in range(4):
        q.add_(0.25)
        v.mul_(-1.0)
        for t in captured[:6]:
            t.zero_()
        graph.replay()
        _chain(q, k, v, dout, eager)
        torch.cuda.synchronize()
        for a, b in zip(eager[:5], captured[:5]):
            assert torch.equal(a, b), step


def test_on_another_stream():
    q, k, v, dout, make = _chain_state(4)
    a, b = make(), make()
    _chain(q, k, v, dout, a)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    _chain(q, k, v, dout, b, stream=side)
    side.synchronize()
    for x, y in zip(a[:5], b[:5]):
        assert torch.equal(x, y)


def test_two_threads_on_two_streams():
    """Calls from several threads at once, each on its own stream with its own buffers."""
    states = [_chain_state(), _chain_state()]
    states[1][0].mul_(-0.5)
    want = []
    for q, k, v, dout, make in states:
        want.append(make())
        _chain(q, k, v, dout, want[-1])
    torch.cuda.synchronize()
    got, errors = [make() for *_, make in states], []

    def work(i):
        try:
            q, k, v, dout, _ = states[i]
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    _chain(q, k, v, dout, got[i])
                torch.cuda.current_stream().synchronize()
        except Exception as e:
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for a, b in zip(want, got):
        for x, y in zip(a[:5], b[:5]):
            assert torch.equal(x, y)


@pytest.mark.parametrize("group", [1, 3])
def test_strides_beyond_32_bits(group):
    """All tensors in one buffer, every position 2^23 - 8 elements behind the last."""
    n, d, h, stride = 290, 64, 2 * group, (1 << 23) - 8
    buf = torch.empty(n * stride, dtype=torch.bfloat16, device="cuda")
    view = lambda at, heads: buf.as_strided((1, heads, n, d), (d, d, stride, 1), at * 8 * d)
    g = np.random.Generator(np.random.PCG64(26))
    dense = [torch.from_numpy(g.standard_normal((1, heads, n, d)).astype(np.float32)).to(torch.bfloat16).cuda() for heads in (h, 2, 2, h)]
    far = [view(i, t.shape[1]) for i, t in enumerate(dense)] + [view(4 + i, heads) for i, heads in enumerate((h, h, 2, 2))]
    for a, b in zip(far, dense):
        a.copy_(b)
    near = dense + [torch.empty_like(t) for t in (dense[0], dense[0], dense[1], dense[2])]
    for q, k, v, dout, out, dq, dk, dv in (near, far):
        lse = torch.empty(1, h, n, device="cuda")
        hb.hidet_attention(q, k, v, out, lse=lse, causal=True, workspace=torch.empty(1 << 22, device="cuda"))
        ws = torch.empty(hb.hidet_attention_backward_workspace_bytes(q, k) // 4, device="cuda")
        hb.hidet_attention_backward(dout, q, k, v, out, lse, dq, dk, dv, ws, causal=True)
    for a, b in zip(near[4:], far[4:]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim,softcap", [(64, 0.0), (128, 0.0), (40, 8.0)])
def test_gradients_under_slopes_at_positions_beyond_2_to_24(dtype, dim, softcap):
    """The distance of a query to a key is exact wherever both are: one query, and windows of several, at the end of 2^25 + 2^24 keys."""
    g = np.random.Generator(np.random.PCG64(31))
    m, h, hk = 2 ** 25 + 2 ** 24, 4, 2
    slopes = torch.tensor([0.5, 0.25, 1.0, 0.125], device="cuda")
    for n, width in ((1, 7), (40, 33), (200, 90)):
        q, dout = (_draw(g, (1, h, n, dim), dtype, "dense") for _ in range(2))
        near = n + width - 1  # keys that a query sees one of
        k, v = (_draw(g, (1, hk, near, dim), dtype, "dense") for _ in range(2))
        lo = torch.arange(n, dtype=torch.int32) + (m - near)
        ranges = torch.stack([lo, lo + width], 1)[None].contiguous().cuda()
        keys, values = (torch.zeros(1, hk, m, dim, dtype=TYPES[dtype], device="cuda") for _ in range(2))
        keys[:, :, m - near:], values[:, :, m - near:] = k, v
        out, dq = torch.empty_like(q), torch.empty_like(q)
        lse = torch.empty(1, h, n, device="cuda")
        dk, dv = (torch.full_like(keys, 3.0) for _ in range(2))
        opts = dict(slopes=slopes, ranges=ranges, softcap=softcap)
        hb.hidet_attention(q, keys, values, out, lse=lse, **opts)
        ws = torch.empty(hb.hidet_attention_backward_workspace_bytes(q, keys) // 4, device="cuda")
        hb.hidet_attention_backward(dout, q, keys, values, out, lse, dq, dk, dv, ws, **opts)
        see = np.stack([oa.in_ranges(ranges[0].cpu().numpy() - (m - near), near)])
        want, bound = bounds(dtype, f64(q), f64(k), f64(v), see, dim ** -0.5, softcap, f64(slopes), grad_out=f64(dout))
        got = (out, lse, dq, dk[:, :, m - near:], dv[:, :, m - near:])
        for name, t, w, e in zip(("out", "lse", "dq", "dk", "dv"), got, want, bound):
            assert_within(t, w, e, "%s %d %s" % (dtype, n, name))
        assert not dk[:, :, :m - near].any() and not dv[:, :, :m - near].any()


def test_a_training_step_from_tokens_to_gradients():
    """rope -> attention -> backward -> rope backward, as a step runs them, against the oracle's chain of the same."""
    g = np.random.Generator(np.random.PCG64(23))
    x, kx, v, dout = (_draw(g, s, "bf16", "tokens") for s in ((2, 4, 90, 64), (2, 2, 90, 64), (2, 2, 90, 64), (2, 4, 90, 64)))
    f = hb.hidet_rope_frequencies(64).cuda()
    pos = torch.arange(90, dtype=torch.int32, device="cuda").expand(2, 90).contiguous() + 1000
    q, k = torch.empty_like(x), torch.empty_like(kx)
    hb.hidet_rope(x, q, f, positions=pos)
    hb.hidet_rope(kx, k, f, positions=pos)
    out, lse = torch.empty_like(q), torch.empty(2, 4, 90, device="cuda")
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    ws = torch.empty(hb.hidet_attention_backward_workspace_bytes(q, k), dtype=torch.uint8, device="cuda")
    hb.hidet_attention(q, k, v, out, lse=lse, causal=True)
    hb.hidet_attention_backward(dout, q, k, v, out, lse, dq, dk, dv, ws, causal=True)
    hb.hidet_rope(dq, dq, f, positions=pos, inverse=True)
    hb.hidet_rope(dk, dk, f, positions=pos, inverse=True)
    p, ff = pos.cpu().numpy(), f.cpu().numpy()
    see = np.stack([oa.sees(90, 90, causal=True)] * 2)
    q64, k64 = oa.rope(f64(x), p, ff), oa.rope(f64(kx), p, ff)
    wq, wk, wv = oa.attention_grad(f64(dout), q64, k64, f64(v), see, 0.125)
    wq, wk = oa.rope(wq, p, ff, inverse=True), oa.rope(wk, p, ff, inverse=True)
    for got, want, name in ((dq, wq, "dq"), (dk, wk, "dk"), (dv, wv, "dv")):
        # seven roundings of 2^-8 / sqrt(3) in a row at most (inputs, weights, dS, gradient, turned gradient), relative to the whole
        assert np.linalg.norm(f64(got) - want) <= 7 * 2.0 ** -8 / 3 ** 0.5 * np.linalg.norm(want), name
