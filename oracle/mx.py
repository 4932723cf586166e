"""Matrices in blocks of 32 that share a power of two, and root-mean-square norms, in float64 from their definitions."""
import numpy as np

# bits of exponent and of mantissa, bias; exponents that are used, largest mantissa of the highest one
E4M3, E5M2, E2M1 = 0, 1, 2
_BITS = {E4M3: (4, 3), E5M2: (5, 2), E2M1: (2, 1)}
_BIAS = {E4M3: 7, E5M2: 15, E2M1: 1}
LARGEST = {E4M3: 448.0, E5M2: 57344.0, E2M1: 6.0}
POWER = {E4M3: 8, E5M2: 15, E2M1: 2}  # of the largest power of two


def grid(fmt):
    """The finite values of a format that are not negative; an index is the code."""
    e_bits, m_bits = _BITS[fmt]
    out = []
    for code in range(2 ** (e_bits + m_bits)):
        e, m = code >> m_bits, code & (2 ** m_bits - 1)
        v = m * 2.0 ** (1 - _BIAS[fmt] - m_bits) if e == 0 else (1 + m / 2 ** m_bits) * 2.0 ** (e - _BIAS[fmt])
        if v > LARGEST[fmt]:
            break
        out.append(v)
    return np.array(out)


def sign_bit(fmt):
    return 8 if fmt == E2M1 else 128


def values(codes, fmt):
    """What element codes stand for (NaN and infinities of the 8-bit formats included)."""
    g, sign = grid(fmt), sign_bit(fmt)
    size = np.asarray(codes).astype(np.int64) & (sign - 1)
    table = np.full(sign, np.nan)
    table[:len(g)] = g
    if fmt == E5M2:
        table[0x7C] = np.inf
    out = table[size]
    return np.where((np.asarray(codes).astype(np.int64) & sign) != 0, -out, out)


def nearest(q, fmt):
    """Codes of numbers: the nearest value, of two as near the even code, beyond the largest the largest."""
    g = grid(fmt)
    size = np.minimum(np.abs(q), g[-1])
    below = np.clip(np.searchsorted(g, size, side="right") - 1, 0, len(g) - 2)
    down, up = size - g[below], g[below + 1] - size
    code = np.where((up < down) | ((up == down) & (below % 2 == 1)), below + 1, below)
    return (code + np.where(np.signbit(q), sign_bit(fmt), 0)).astype(np.uint8)


def blocks(n):
    return (n + 31) // 32


def quantize(x, fmt, scales=None):
    """x [rows, cols] -> (element codes [rows, whole blocks], scale codes [blocks, rows]); `scales`: those to use."""
    rows, cols = x.shape
    filled = np.zeros((rows, blocks(cols) * 32))
    filled[:, :cols] = x
    filled = filled.reshape(rows, -1, 32)
    top = np.abs(filled).max(2, initial=0.0)  # (NaN where there is one)
    finite = np.isfinite(top)
    if scales is None:
        _, e = np.frexp(np.where(finite & (top > 0), top, 1.0))
        code = np.where(top > 0, np.maximum(e - 1 - POWER[fmt], -127) + 127, 0)
        code = np.where(finite, code, 255).astype(np.uint8)
    else:
        code = scales.T
    factor = np.ldexp(1.0, 127 - code.astype(np.int64))
    with np.errstate(invalid="ignore"):
        q = np.where((code != 255)[..., None], filled * factor[..., None], 0.0)
    return nearest(q, fmt).reshape(rows, -1), np.ascontiguousarray(code.T)


def numbers(codes, scales, fmt):
    """What codes [rows, whole blocks] and scale codes [blocks, rows] stand for."""
    scale = np.where(scales.T == 255, np.nan, np.ldexp(1.0, scales.T.astype(np.int64) - 127))
    return values(codes, fmt) * np.repeat(scale, 32, axis=1)


def pack(codes, fmt):
    """Element codes as bytes in memory."""
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8) if fmt == E2M1 else codes


def unpack(data, fmt):
    return np.stack((data & 15, data >> 4), 2).reshape(data.shape[0], -1) if fmt == E2M1 else data


def rms_norm(h, weight, eps, offset):
    """(y, rstd)"""
    rstd = 1.0 / np.sqrt((h * h).mean(1) + eps)
    return h * rstd[:, None] * (offset + weight), rstd


def rms_norm_grad(grad_y, h, rstd, weight, offset):
    """(grad_h, grad_weight) for a given rstd"""
    g, xhat = grad_y * (offset + weight), h * rstd[:, None]
    return rstd[:, None] * (g - xhat * (g * xhat).mean(1, keepdims=True)), (grad_y * xhat).sum(0)


def exponents(codes, fmt):
    """Powers of two of elements; below the normal numbers, that of the smallest one."""
    field = (np.asarray(codes).astype(np.int64) & (sign_bit(fmt) - 1)) >> _BITS[fmt][1]
    return np.maximum(field, 1) - _BIAS[fmt]


def product_of_cut_eights(a, a_fmt, b, b_fmt):
    """A . B^T of (codes [rows, whole blocks], scale codes) whose products of 8 neighbouring k are cut to multiples of 2^(e - 13), e the largest sum
    of the exponents of two elements that are not 0 -> (sums, sums of the magnitudes of uncut products)."""
    va, vb, ea, eb = values(a[0], a_fmt), values(b[0], b_fmt), exponents(a[0], a_fmt), exponents(b[0], b_fmt)
    sa, sb = (np.ldexp(1.0, s.astype(np.int64) - 127) for s in (a[1], b[1]))
    total, size = np.zeros((len(va), len(vb))), np.zeros((len(va), len(vb)))
    for k in range(0, va.shape[1], 8):
        if not va[:, k:k + 8].any():
            continue
        p = va[:, None, k:k + 8] * vb[None, :, k:k + 8]
        e = np.where(p == 0, -1000, ea[:, None, k:k + 8] + eb[None, :, k:k + 8]).max(2, keepdims=True)
        step = np.where(e > -1000, np.ldexp(1.0, np.maximum(e, -100) - 13), 1.0)
        scale = sa[k // 32][:, None] * sb[k // 32][None, :]
        total += (np.trunc(p / step) * step).sum(2) * scale
        size += np.abs(p).sum(2) * scale
    return total, size
