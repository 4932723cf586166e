"""Rotary positions against the float64 oracle.

Bound of an element: u |y| for the rounding of the result (u half a step of the type), and 1e-6 amplitude (|a| + |b|) for fp32 sine and
cosine (2^-23 each), the angle's own rounding to fp32 (pi 2^-24) and two products and a sum (3 * 2^-24)."""
import numpy as np
import pytest
import torch

from attention_helpers import TYPES, U, assert_within, f64
from oracle import attention as oa
from paper_2210_09603_amd import binding as hb

pytestmark = pytest.mark.gpu


def _bound(dtype, x, want, half, interleaved, amplitude):
    size = np.abs(x)
    pair = size.copy()
    first = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    second = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    pair[..., first] += size[..., second]
    pair[..., second] += size[..., first]
    b = U[dtype] * np.abs(want) + 1e-6 * amplitude * pair + 2.0 ** -25 * (dtype == "f16")
    b[..., 2 * half:] = 1e-30  # (copied)
    return b


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("size", [(1, 1, 1, 2, 2), (2, 3, 5, 64, 64), (1, 40, 1, 128, 128), (3, 2, 70, 80, 50), (1, 5, 33, 96, 2),
                                  (2, 1, 300, 20, 14), (1, 2, 9, 7, 6), (1, 70, 1100, 8, 8), (1, 1, 2500, 256, 130)], ids=str)
def test_rope(size, interleaved, dtype):
    b, h, n, d, r = size
    g = np.random.Generator(np.random.PCG64(n + d + r))
    f = 10000.0 ** (-2.0 * np.arange(r // 2) / r)
    for i, layout in enumerate(("dense", "tokens", "odd")):
        x = torch.from_numpy(g.standard_normal((b, h, n, d)).astype(np.float32)).to(TYPES[dtype]).cuda()
        y = torch.full((b, h, n, d), 7.0, dtype=TYPES[dtype], device="cuda")
        if layout == "tokens":
            x, y = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (x, y))
        if layout == "odd":
            wide = torch.full((b, n, h + 1, d + 3), 7.0, dtype=TYPES[dtype], device="cuda")
            y = wide[:, :, 1:, 1:d + 1].transpose(1, 2)
        pos = torch.from_numpy(g.integers(-50, 1 << 20, (b, n)).astype(np.int32)).cuda()
        inverse, amplitude = i == 1, (1.0, 1.25, 0.5)[i]
        hb.hidet_rope(x, y, torch.from_numpy(f).cuda(), positions=pos, interleaved=interleaved, inverse=inverse, amplitude=amplitude)
        torch.cuda.synchronize()
        want = oa.rope(f64(x), pos.cpu().numpy(), f, interleaved, inverse, amplitude)
        assert_within(y, want, _bound(dtype, f64(x), want, r // 2, interleaved, amplitude), "%s %s" % (size, layout))
        if layout == "odd":
            y.fill_(7.0)
            assert bool((wide == 7.0).all())
        # in place, the rest of the vector left alone
        before = f64(x)
        hb.hidet_rope(x, x, torch.from_numpy(f).cuda(), positions=pos, interleaved=interleaved, inverse=inverse, amplitude=amplitude)
        assert_within(x, want, _bound(dtype, before, want, r // 2, interleaved, amplitude), "in place")


def test_positions_that_are_shared_counted_or_far():
    g = np.random.Generator(np.random.PCG64(2))
    x = torch.from_numpy(g.standard_normal((2, 3, 10, 64)).astype(np.float32)).cuda()
    f = hb.hidet_rope_frequencies(64)
    y, z = torch.empty_like(x), torch.empty_like(x)
    for first in (0, 77, 2 ** 31 - 10, -5):
        pos = np.arange(10) + first
        hb.hidet_rope(x, y, f.cuda(), first_position=first)
        want = oa.rope(f64(x), np.stack([pos, pos]), f.numpy())
        # (2^31 positions keep 2^-22 of a turn: 2^-22 * 2 pi = 1.5e-6 of the pair)
        assert_within(y, want, _bound("f32", f64(x), want, 32, False, 3.0), "first %d" % first)
        shared = torch.from_numpy(pos.astype(np.int32)).cuda()
        hb.hidet_rope(x, z, f.cuda(), positions=shared)
        assert torch.equal(y, z)
        hb.hidet_rope(x, z, f.cuda(), positions=shared.expand(2, 10))
        assert torch.equal(y, z)


def test_the_gradient_is_the_transpose():
    """<rope(x), g> = <x, rope_inverse(g)> for the kernel's own results in fp32."""
    g = np.random.Generator(np.random.PCG64(4))
    x, grad = (torch.from_numpy(g.standard_normal((1, 2, 40, 48)).astype(np.float32)).cuda() for _ in range(2))
    f = hb.hidet_rope_frequencies(32, scaling=hb.HIDET_ROPE_BANDS, factor=8.0).cuda()
    for interleaved in (False, True):
        y, dx = torch.empty_like(x), torch.empty_like(x)
        hb.hidet_rope(x, y, f, first_position=5000, interleaved=interleaved, amplitude=1.2)
        hb.hidet_rope(grad, dx, f, first_position=5000, interleaved=interleaved, amplitude=1.2, inverse=True)
        a, b = (f64(y) * f64(grad)).sum(), (f64(x) * f64(dx)).sum()
        assert abs(a - b) <= 1e-6 * (np.abs(f64(y)) * np.abs(f64(grad))).sum()
        # copied elements take no amplitude
        assert torch.equal(y[..., 32:], x[..., 32:])


def test_graph_replays_and_another_stream():
    x = torch.randn(1, 4, 30, 64, device="cuda").bfloat16()
    f = hb.hidet_rope_frequencies(64).cuda()
    pos = torch.arange(30, dtype=torch.int32, device="cuda")
    y, z = torch.empty_like(x), torch.empty_like(x)
    hb.hidet_rope(x, y, f, positions=pos)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hb.hidet_rope(x, y, f, positions=pos)
    for _ in range(3):
        x.mul_(-0.5)
        pos.add_(11)
        graph.replay()
        hb.hidet_rope(x, z, f, positions=pos)
        torch.cuda.synchronize()
        assert torch.equal(y, z)
    side = torch.cuda.Stream()
    z.zero_()
    hb.hidet_rope(x, z, f, positions=pos, stream=side)
    side.synchronize()
    assert torch.equal(y, z)
