"""Pins of the attention oracle: closed forms, differences, other ways to say the same."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from oracle import reduction as red

RNG = np.random.Generator(np.random.PCG64(31))


def _qkv(b, h, hk, n, m, d):
    return RNG.standard_normal((b, h, n, d)), RNG.standard_normal((b, hk, m, d)), RNG.standard_normal((b, hk, m, d))


def test_without_a_mask_it_is_the_three_step_attention():
    q, k, v = _qkv(1, 3, 3, 5, 7, 4)
    out, lse = oa.attention(q, k, v, np.ones((1, 5, 7), bool), 0.5)
    assert np.allclose(out[0], red.attention(q[0], k[0], v[0], 0.5), rtol=0, atol=1e-13)
    assert np.allclose(lse[0], torch.logsumexp(0.5 * torch.from_numpy(q[0] @ k[0].transpose(0, 2, 1)), -1).numpy())


def test_a_query_that_sees_nothing_is_zero_and_what_is_not_seen_does_not_matter():
    q, k, v = _qkv(1, 1, 1, 3, 4, 2)
    see = np.array([[[True, False, False, True], [False] * 4, [False, True, False, False]]])
    a, la = oa.attention(q, k, v, see, 1.0)
    k[0, 0, 2], v[0, 0, 2] = np.nan, np.inf
    b, lb = oa.attention(q, k, v, see, 1.0)
    assert np.array_equal(a, b) and np.array_equal(la, lb)
    assert np.all(a[0, 0, 1] == 0) and la[0, 0, 1] == -np.inf
    assert np.array_equal(a[0, 0, 2], v[0, 0, 1])  # one key: its value


@pytest.mark.parametrize("softcap,slopes", [(0.0, None), (2.0, None), (0.0, [0.3, 0.1]), (1.5, [0.2, 0.4])])
def test_gradients_against_differences(softcap, slopes):
    q, k, v = _qkv(2, 2, 1, 4, 5, 3)
    g = RNG.standard_normal(q.shape)
    see = np.stack([oa.sees(4, 5, causal=True), oa.in_ranges(np.array([[0, 2], [3, 3], [1, 5], [4, 5]]), 5)])
    grads = oa.attention_grad(g, q, k, v, see, 0.7, softcap, slopes)
    for which, grad in enumerate(grads):
        for at in np.ndindex(grad.shape):
            ends = []
            for step in (1e-5, -1e-5):
                t = [x.copy() for x in (q, k, v)]
                t[which][at] += step
                ends.append((oa.attention(*t, see, 0.7, softcap, slopes)[0] * g).sum())
            assert abs((ends[0] - ends[1]) / 2e-5 - grad[at]) < 1e-8


def test_shared_heads_are_the_same_as_repeated_ones():
    q, k, v = _qkv(1, 6, 2, 3, 4, 2)
    see = np.ones((1, 3, 4), bool)
    a, _ = oa.attention(q, k, v, see, 1.0)
    b, _ = oa.attention(q, np.repeat(k, 3, 1), np.repeat(v, 3, 1), see, 1.0)
    assert np.array_equal(a, b)


def test_masks_by_hand():
    assert oa.sees(2, 4, causal=True).tolist() == [[1, 1, 1, 0], [1, 1, 1, 1]]
    assert oa.sees(3, 2, causal=True).tolist() == [[0, 0], [1, 0], [1, 1]]
    assert oa.sees(4, 4, causal=True, window=2).tolist() == [[1, 0, 0, 0], [1, 1, 0, 0], [0, 1, 1, 0], [0, 0, 1, 1]]
    assert oa.sees(3, 3, window=2).tolist() == [[1, 1, 0], [1, 1, 1], [0, 1, 1]]
    assert oa.sees(4, 4, causal=True, prefix=2).tolist() == [[1, 1, 0, 0], [1, 1, 0, 0], [1, 1, 1, 0], [1, 1, 1, 1]]
    assert oa.sees(5, 5, causal=True, documents=[4, 4, -1, 4, 4]).tolist() == [
        [1, 0, 0, 0, 0], [1, 1, 0, 0, 0], [0] * 5, [0, 0, 0, 1, 0], [0, 0, 0, 1, 1]]
    assert oa.sees(4, 4, causal=True, documents=[0, 0, 1, 1], prefix=2).tolist() == [[1, 1, 0, 0], [1, 1, 0, 0], [0, 0, 1, 1], [0, 0, 1, 1]]


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_turns_pairs_keeps_norms_and_depends_on_distances(interleaved):
    f = 10000.0 ** (-np.arange(3) / 3.0)
    q, k = RNG.standard_normal((1, 1, 1, 8)), RNG.standard_normal((1, 1, 1, 8))

    def dot(a, b):
        return (oa.rope(q, [[a]], f, interleaved) * oa.rope(k, [[b]], f, interleaved)).sum()

    assert abs(dot(7, 3) - dot(1007, 1003)) < 1e-9
    y = oa.rope(q, [[11]], f, interleaved)
    assert abs((y * y).sum() - (q * q).sum()) < 1e-12 and np.array_equal(y[..., 6:], q[..., 6:])
    back = oa.rope(oa.rope(q, [[11]], f, interleaved, amplitude=2.0), [[11]], f, interleaved, inverse=True, amplitude=0.5)
    assert np.allclose(back, q, atol=1e-13)
    one = np.zeros((1, 1, 1, 2))
    one[..., 0] = 1.0
    assert np.allclose(oa.rope(one, [[1]], [np.pi / 2], interleaved)[0, 0, 0], [0.0, 1.0])


def test_cache_rows_follow_the_table():
    pages = RNG.standard_normal((4, 2, 1, 3))
    rows, there = oa.cache_rows(pages, [3, -1, 0], 5)
    assert np.array_equal(rows[0, 0], pages[3, 0, 0]) and np.array_equal(rows[0, 4], pages[0, 0, 0])
    assert there.tolist() == [True, True, False, False, True]
