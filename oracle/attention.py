"""CPU oracle for fused attention, its rotary positions and its paged cache: plain definitions in float64 (numpy).

TEST INFRASTRUCTURE ONLY, like the rest of this package.

* ``rope``: every pair (a, b) as the complex number a + ib times amplitude * exp(i * position * frequency).
* ``sees``: which keys a query sees, as a boolean matrix, from the words of the definition (causal, window, document, prefix), key
  by key; ``in_ranges``: from begin and end.
* ``attention``: scores with cap and slope, softmax over the keys that a query sees, product with the values; a query that
  sees nothing gives 0 and a log-sum of -inf.  Keys that a query does not see are left out, not multiplied by zero.
* ``attention_grad``: the gradients of sum(grad_out * out), written out from the softmax's derivative.
* ``cache_rows``: the keys and values of a sequence, gathered from its pages.
"""
import numpy as np


def rope(x, positions, frequencies, interleaved=False, inverse=False, amplitude=1.0):
    """x [batch, heads, seq, dim], positions [batch, seq] -> the same shape."""
    x = np.asarray(x, dtype=np.float64)
    half = len(frequencies)
    y = x.copy()
    angle = np.asarray(positions, dtype=np.float64)[:, None, :, None] * np.asarray(frequencies, dtype=np.float64)
    turn = amplitude * np.exp((-1j if inverse else 1j) * angle)
    first = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    second = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    z = (x[..., first] + 1j * x[..., second]) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def sees(seq_q, seq_k, causal=False, window=0, documents=None, prefix=0):
    """Boolean [seq_q, seq_k].  documents: [seq_k] (runs of equal numbers, negative: padding); prefix: positions from the start of
    a document that all its queries see."""
    out = np.zeros((seq_q, seq_k), dtype=bool)
    run = np.zeros(seq_k, dtype=int)
    start = np.zeros(seq_k, dtype=int)
    for j in range(1, seq_k):
        new = documents is not None and documents[j] != documents[j - 1]
        run[j] = run[j - 1] + (1 if new else 0)
        start[j] = j if new else start[j - 1]
    for i in range(seq_q):
        at = i + seq_k - seq_q
        if documents is not None and (at < 0 or documents[at] < 0):
            continue
        for j in range(seq_k):
            ok = (j <= at) if causal else True
            if documents is not None and run[j] != run[at]:
                continue
            if window and not (at - j < window and j - at < window):
                ok = False
            if causal and prefix and at >= 0 and j - start[j] < prefix:
                ok = True
            out[i, j] = ok
    return out


def in_ranges(ranges, seq_k):
    """Boolean [seq_q, seq_k] of ranges [seq_q, 2]."""
    j = np.arange(seq_k)[None, :]
    return (j >= ranges[:, :1]) & (j < ranges[:, 1:])


def scores(q, k, scale, softcap=0.0, slope=0.0):
    """(x, dx / d(scale q.k)) of one head: q [n, d], k [m, d]."""
    n, m = len(q), len(k)
    x = scale * (q @ k.T)
    derivative = np.ones_like(x)
    if softcap:
        t = np.tanh(x / softcap)
        x, derivative = softcap * t, 1.0 - t * t
    if slope:
        x = x - slope * np.abs(np.arange(n)[:, None] + (m - n) - np.arange(m)[None, :])
    return x, derivative


def probabilities(x, see):
    """(P, lse) of scores x [n, m] over the keys that each query sees."""
    p, lse = np.zeros_like(x), np.full(len(x), -np.inf)
    for i in range(len(x)):
        keys = np.flatnonzero(see[i])
        if len(keys) == 0:
            continue
        top = x[i, keys].max()
        if top == -np.inf:
            continue
        e = np.exp(x[i, keys] - top)
        p[i, keys] = e / e.sum()
        lse[i] = top + np.log(e.sum())
    return p, lse


def weighted(p, v, see):
    """sum over the seen keys of p v; the others are left out."""
    out = np.zeros((len(p), v.shape[1]))
    for i in range(len(p)):
        keys = np.flatnonzero(see[i])
        if len(keys):
            out[i] = p[i, keys] @ v[keys]
    return out


def attention(q, k, v, see, scale, softcap=0.0, slopes=None):
    """q [batch, heads, n, d], k, v [batch, kv_heads, m, d], see [batch, n, m] -> out, lse."""
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    batch, heads, n, _ = q.shape
    group = heads // k.shape[1]
    out, lse = np.zeros_like(q), np.zeros((batch, heads, n))
    for b in range(batch):
        for h in range(heads):
            x, _ = scores(q[b, h], k[b, h // group], scale, softcap, 0.0 if slopes is None else float(slopes[h]))
            p, lse[b, h] = probabilities(x, see[b])
            out[b, h] = weighted(p, v[b, h // group], see[b])
    return out, lse


def attention_grad(grad_out, q, k, v, see, scale, softcap=0.0, slopes=None):
    """Gradients of q, k, v; the group's heads add up in those of k and v."""
    g, q, k, v = (np.asarray(t, dtype=np.float64) for t in (grad_out, q, k, v))
    batch, heads, _, _ = q.shape
    group = heads // k.shape[1]
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for b in range(batch):
        for h in range(heads):
            kh, vh = k[b, h // group], v[b, h // group]
            x, derivative = scores(q[b, h], kh, scale, softcap, 0.0 if slopes is None else float(slopes[h]))
            p, _ = probabilities(x, see[b])
            out = weighted(p, vh, see[b])
            dp = np.where(see[b], g[b, h] @ vh.T, 0.0)
            ds = np.where(see[b], p * (dp - (g[b, h] * out).sum(1, keepdims=True)) * np.where(see[b], derivative, 0.0), 0.0)
            dq[b, h] = scale * weighted(ds, kh, see[b])
            dk[b, h // group] += scale * weighted(ds.T, q[b, h], see[b].T)
            dv[b, h // group] += weighted(p.T, g[b, h], see[b].T)
    return dq, dk, dv


def cache_rows(pages, table, length):
    """The first `length` rows of a sequence: pages [pages, size, heads, d], table of page numbers -> [heads, length, d] and which of
    them are on a page at all."""
    size = pages.shape[1]
    out = np.zeros((pages.shape[2], length, pages.shape[3]))
    there = np.zeros(length, dtype=bool)
    for t in range(length):
        page = int(table[t // size])
        if 0 <= page < len(pages):
            out[:, t] = pages[page, t % size]
            there[t] = True
    return out, there
