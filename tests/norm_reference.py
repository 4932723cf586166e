"""Root-mean-square norms and their gradients in float64 from their definitions, as elementary tensor operations: on the GPU for sizes
that the numpy oracle takes long for, and compared with it on the CPU."""
import torch


def norm(h, weight, eps, offset):
    """(y, rstd), float64"""
    h = h.double()
    rstd = 1.0 / torch.sqrt((h * h).sum(1) / h.shape[1] + eps)
    return h * rstd[:, None] * (offset + weight.double()), rstd


def gradients(grad_y, h, rstd, weight, offset):
    """float64: grad_h; its terms' magnitudes, those of the mean apart; grad_weight, and the sum of its terms' magnitudes"""
    g, h, r = grad_y.double(), h.double(), rstd.double()[:, None]
    xhat, gw = h * r, g * (offset + weight.double())
    grad_h = r * (gw - xhat * (gw * xhat).sum(1, keepdim=True) / h.shape[1])
    near, far = (r * gw).abs(), (r * xhat).abs() * (gw * xhat).abs().sum(1, keepdim=True) / h.shape[1]
    return grad_h, near, far, (g * xhat).sum(0), (g * xhat).abs().sum(0)
