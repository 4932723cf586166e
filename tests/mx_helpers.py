"""Shared by the tests of norms and block-scaled matrices: types, and matrices in memory with room around them."""
import numpy as np
import torch

from oracle import mx
from paper_2210_09603_amd import binding as hb

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # half a step, relative
FLOOR = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134, "f32": 2.0 ** -150}  # half a step of the smallest numbers
FORMATS = [hb.HIDET_MX_E4M3, hb.HIDET_MX_E5M2, hb.HIDET_MX_E2M1]
FILL = 0x55  # of memory that is not to be written


def rng(*seed):
    return np.random.Generator(np.random.PCG64(list(seed)))


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def on_gpu(x, dtype):
    """float64 -> tensor of dtype on the GPU (rounded once, from fp32)."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(TYPES[dtype]).cuda()


def padded(x, dtype, before, after):
    """The same as a view whose rows lie apart, its first element `before` elements behind an aligned address."""
    rows, cols = x.shape
    wide = torch.full((rows, before + cols + after), 7.0, dtype=TYPES[dtype], device="cuda")
    view = wide[:, before:before + cols]
    view.copy_(on_gpu(x, dtype))
    return wide, view


class Room:
    """An empty matrix in blocks, with room around it that has to stay as it is."""

    def __init__(self, rows, cols, fmt, wide=True):
        blocks, self.rows, self.width = mx.blocks(cols), rows, mx.blocks(cols) * (16 if fmt == mx.E2M1 else 32)
        extra = 32 if wide else 0
        self.values = torch.full((rows + 1, self.width + extra), FILL, dtype=torch.uint8, device="cuda")
        self.scales = torch.full((blocks + 1, (rows + 3) // 4 * 4 + (8 if wide else 0)), FILL, dtype=torch.uint8, device="cuda")
        self.blocks = blocks
        self.m = hb.make_mx(rows, cols, fmt, values=self.values[:rows, :self.width] if rows else self.values[:0],
                            scales=self.scales[:blocks, :rows] if blocks else self.scales[:0, :rows])
        self.fmt = fmt

    def read(self):
        """(element codes, scale codes), and that nothing around them was written."""
        v, s = self.values.cpu().numpy(), self.scales.cpu().numpy()
        assert (v[self.rows:] == FILL).all() and (v[:, self.width:] == FILL).all()
        assert (s[self.blocks:] == FILL).all() and (s[:, self.rows:] == FILL).all()
        return mx.unpack(v[:self.rows, :self.width], self.fmt), s[:self.blocks, :self.rows]


def matrix(codes, scales, cols, fmt, wide=True):
    """A matrix in blocks on the GPU from its codes."""
    rows = codes.shape[0]
    r = Room(rows, cols, fmt, wide)
    r.values[:rows, :r.width] = torch.from_numpy(np.ascontiguousarray(mx.pack(codes, fmt))).cuda()
    r.scales[:r.blocks, :rows] = torch.from_numpy(np.ascontiguousarray(scales)).cuda()
    return r.m
