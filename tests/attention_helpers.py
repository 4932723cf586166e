"""Bounds of the attention tests, element by element, from the roundings that the operators make.

u is half a step of the storage type (2^-11 fp16, 2^-8 bf16).  Everything else is fp32: a score of |x| is off by E = 1e-5 (1 + |x|)
at most -- a dot product of up to 128 terms whose absolute values add up to some 10 |x| (1e-6 of those), the cap's tanh
(2^-22 of the cap, which bounds |x|), and a step of fp32 in each of scale, slope, maximum and log-sum -- and so is its weight,
relatively.  fp16 operands below 2^-14 are rounded on a grid of 2^-24, 2^-25 off at most.

  out   u |out| (its rounding) + (u + E) sum_j p |v|  (weights rounded for the product) + 2^-25 sum_j |v| (fp16; weights are at least
        relative to a maximum of 1)
  D     sum_d |g| (error of out) + 1e-6 sum_d |g out|
        where no query of 128 rows sees more than 32 keys (`few`) it is sum_j p dP instead: 2 E sum_j p |dP| + 1e-6 sum_j p sum_d |g v|
  dS    |dS| (u + E) + p (error of D + 1e-6 sum_d |g v| + 2e-5 |dP - D| (1 + |x|) for the cap's derivative) + 2^-25 (fp16)
  dQ    u |dQ| + scale sum_j (error of dS) |k|;  dK the same with q, summed over the heads that share a key
  dV    u |dV| + sum_i (u + E) p |g| + 2^-35 sum_i |g| (fp16; weights are lifted by 2^10)
"""
import numpy as np
import torch

from oracle import attention as oa

U = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def bounds(dtype, q, k, v, see, scale, softcap=0.0, slopes=None, grad_out=None, few=False):
    """(out, lse, their bounds) and, with grad_out, (dq, dk, dv) and theirs; everything float64."""
    u, small = U[dtype], (2.0 ** -25 if dtype == "f16" else 0.0)
    batch, heads, n, d = q.shape
    group = heads // k.shape[1]
    out, lse = oa.attention(q, k, v, see, scale, softcap, slopes)
    b_out, b_lse = np.zeros_like(out), np.zeros_like(lse)
    b_dq, b_dk, b_dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    grads = oa.attention_grad(grad_out, q, k, v, see, scale, softcap, slopes) if grad_out is not None else None
    for b in range(batch):
        m = see[b]
        for h in range(heads):
            kh, vh = (np.where(m.any(0)[:, None], t[b, h // group], 0.0) for t in (k, v))
            x, derivative = oa.scores(q[b, h], kh, scale, softcap, 0.0 if slopes is None else float(slopes[h]))
            x = np.where(m, x, 0.0)
            p, _ = oa.probabilities(np.where(m, x, -np.inf), m)
            top = np.abs(x).max(initial=0.0)
            e = 1e-5 * (1.0 + top)
            b_out[b, h] = u * np.abs(out[b, h]) + (u + e) * (p @ np.abs(vh)) + small * (m @ np.abs(vh)) + 1e-30
            b_lse[b, h] = e
            if grads is None:
                continue
            g = grad_out[b, h]
            g = np.where(m.any(1)[:, None], g, 0.0)
            dp, delta = g @ vh.T, (g * out[b, h]).sum(1, keepdims=True)
            ds = np.abs(p * (dp - delta) * derivative)
            d_delta = (np.abs(g) * b_out[b, h]).sum(1, keepdims=True) + 1e-6 * np.abs(g * out[b, h]).sum(1, keepdims=True)
            if few:
                d_delta = 2 * e * (p * np.abs(dp)).sum(1, keepdims=True) + 1e-6 * (p * (np.abs(g) @ np.abs(vh).T)).sum(1, keepdims=True)
            d_ds = ds * (u + 2 * e) + p * (d_delta + 1e-6 * (np.abs(g) @ np.abs(vh).T) + 2e-5 * (1 + top) * np.abs(dp - delta) * (softcap > 0))
            d_ds = np.where(m, d_ds + small, 0.0)
            b_dq[b, h] = u * np.abs(grads[0][b, h]) + abs(scale) * (d_ds @ np.abs(kh)) + small
            b_dk[b, h // group] += abs(scale) * (d_ds.T @ np.abs(np.where(m.any(1)[:, None], q[b, h], 0.0)))
            b_dv[b, h // group] += (u + e) * (p.T @ np.abs(g)) + small / 1024 * (m.T @ np.abs(g))
    if grads is None:
        return (out, lse), (b_out, b_lse)
    b_dk += u * np.abs(grads[1]) + small
    b_dv += u * np.abs(grads[2]) + small
    return (out, lse) + grads, (b_out, b_lse, b_dq + 1e-30, b_dk + 1e-30, b_dv + 1e-30)


def assert_within(got, want, bound, what):
    got = f64(got) if isinstance(got, torch.Tensor) else got
    off = np.isfinite(want)
    assert np.array_equal(got[~off], want[~off], equal_nan=True), what  # (log-sums of -inf)
    ratio = np.abs(got - want)[off] / np.broadcast_to(bound, want.shape)[off]
    worst = float(ratio.max(initial=0.0)) if not np.isnan(ratio).any() else float("nan")
    print("%s: worst error %.3f of its bound" % (what, worst), flush=True)
    assert worst <= 1.0, "%s: %.2f of the bound" % (what, worst)
